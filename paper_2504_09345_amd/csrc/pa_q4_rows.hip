// The 4-bit cache's write and read of rows (format in pagedattn_q4.h).
//
// A (row, KV head) vector of D elements is D / 8 lanes of 8 consecutive ones, four
// lanes to a block of 32.  Writing: the block's largest magnitude over its lanes
// (DPP), the scale from that value's bits, v_cvt_scalef32_pk_fp4_f32 to codes (its
// rounding is the format's).  A lane's four bytes are one word of the K tile and
// four bytes, one in every fourth word, of the V tile.  Reading mirrors it.
#include "pa_device.h"
#include "pa_q4_tile.h"

namespace pa {

namespace {

constexpr int kRowsWaves = 4;

// The place of a row in the cache: its slot's token and page, or why it has none.
struct Place {
  bool skip, bad;  // a row of no sequence; a row that the contract does not allow
  int page, token;
};
__device__ __forceinline__ Place place_of(const Q4RowsArgs& a, int row, int lane) {
  Place p{true, false, 0, 0};
  int b = row, L = 1, j = 0;
  const int32_t* qsl = a.query_start_loc;
  if (qsl != nullptr) {
    b = q4::wave_search(a.B, row, lane, [&](int i) { return qsl[i]; });
    L = qsl[b + 1] - qsl[b];
    j = row - qsl[b];
    if (j < 0 || j >= L) return p;
  }
  const int C = a.context_lens[b];
  if (qsl == nullptr && C == 0) return p;
  p.skip = false;
  const int pos = C - L + j;
  p.bad = C < 0 || L > C || C > a.max_context_len || pos / kPage >= a.bt_stride;
  if (p.bad) return p;
  p.page = a.block_table[(int64_t)b * a.bt_stride + pos / kPage];
  p.token = pos % kPage;
  p.bad = p.page < 0 || p.page >= a.num_pages;
  return p;
}

template <typename T>
__device__ __forceinline__ void load_eight(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    widen(*reinterpret_cast<const u32x4*>(p), x, uint16_t());
  } else {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p), b = *reinterpret_cast<const u32x4*>(p + 4);
    widen(a, x, 0.0f);
    widen(b, x + 4, 0.0f);
  }
}

// Codes (a byte per pair) of a lane's eight elements and their block's scale byte.
__device__ __forceinline__ uint32_t quantise(const float (&x)[8], uint32_t& scale) {
  float a = 0.0f;
  bool odd = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    a = fmaxf(a, fabsf(x[e]));
    odd |= !(fabsf(x[e]) <= __FLT_MAX__);
  }
  a = fmaxf(a, dpp_xor1(a));
  a = fmaxf(a, dpp_xor2(a));
  float o = odd ? 1.0f : 0.0f;
  o = fmaxf(o, dpp_xor1(o));
  o = fmaxf(o, dpp_xor2(o));
  // the exponent's byte less 2, or 1 above 1.75 (a carry out of the mantissa)
  const int e = min(max((int)((__float_as_uint(a) + 0x1fffffu) >> 23) - 2, 2), 252);
  scale = a == 0.0f ? 127u : (uint32_t)e;
  const float s = __uint_as_float(scale << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  if (o != 0.0f) {
    scale = 255u;
    w = 0;
  }
  return w;
}

template <int D>
struct Where {  // a lane's place in a tile: chunk c of eight dims of a token
  static __device__ __forceinline__ int k(int token, int c) {
    return (c * 4 / (D / 8) * kPage + token) * (D / 8) + c * 4 % (D / 8);
  }
  // of pair i (of four): 16 i bytes further per pair of D = 128
  static __device__ __forceinline__ int v(int token, int c, int i) {
    return ((token >> 2) * 16 + (c & 3) * 4 + i) * (D / 8) + 4 * (c >> 2) + (token & 3);
  }
  static __device__ __forceinline__ int scale(int token, int c) { return q4::kScales<D> + token * (D / 32) + (c >> 2); }
};

template <typename T, int D>
__global__ __launch_bounds__(64 * kRowsWaves) void q4_append_kernel(Q4RowsArgs a) {
  constexpr int CH = D / 8;
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * kRowsWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.rows) return;
  const Place p = place_of(a, row, lane);
  if (p.skip || p.bad) return;
  for (int i = lane; i < a.H_kv * CH; i += 64) {
    const int g = i / CH, c = i % CH;
    const int64_t from = ((int64_t)row * a.H_kv + g) * D + c * 8;
    const int64_t tile = ((int64_t)p.page * a.H_kv + g) * q4_tile_bytes(D);
    float x[8];
    uint32_t scale;
    load_eight(reinterpret_cast<const T*>(a.k_rows) + from, x);
    const uint32_t k = quantise(x, scale);
    *reinterpret_cast<uint32_t*>(a.k_pages + tile + Where<D>::k(p.token, c)) = k;
    if ((c & 3) == 0) a.k_pages[tile + Where<D>::scale(p.token, c)] = (uint8_t)scale;
    load_eight(reinterpret_cast<const T*>(a.v_rows) + from, x);
    const uint32_t v = quantise(x, scale);
#pragma unroll
    for (int m = 0; m < 4; ++m) a.v_pages[tile + Where<D>::v(p.token, c, m)] = (uint8_t)(v >> (8 * m));
    if ((c & 3) == 0) a.v_pages[tile + Where<D>::scale(p.token, c)] = (uint8_t)scale;
  }
}

// Eight values of a word of codes.
template <typename T>
__device__ __forceinline__ void put_eight(T* p, uint32_t w, uint32_t scale) {
  const float s = __uint_as_float(scale << 23);
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x4*>(p) = q4::eight_of(w, s);
  } else {
    const q4::f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
    const q4::f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
    *reinterpret_cast<q4::f32x4_t*>(p) = q4::f32x4_t{a[0], a[1], b[0], b[1]};
    *reinterpret_cast<q4::f32x4_t*>(p + 4) = q4::f32x4_t{c[0], c[1], d[0], d[1]};
  }
}

template <typename T, int D>
__global__ __launch_bounds__(64 * kRowsWaves) void q4_read_kernel(Q4RowsArgs a) {
  constexpr int CH = D / 8;
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * kRowsWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.rows) return;
  const Place p = place_of(a, row, lane);
  if (p.skip) return;
  T* k_out = reinterpret_cast<T*>(const_cast<void*>(a.k_rows));
  T* v_out = reinterpret_cast<T*>(const_cast<void*>(a.v_rows));
  for (int i = lane; i < a.H_kv * CH; i += 64) {
    const int g = i / CH, c = i % CH;
    const int64_t to = ((int64_t)row * a.H_kv + g) * D + c * 8;
    uint32_t k = 0, v = 0, ks = 255, vs = 255;
    if (!p.bad) {
      const int64_t tile = ((int64_t)p.page * a.H_kv + g) * q4_tile_bytes(D);
      k = *reinterpret_cast<const uint32_t*>(a.k_pages + tile + Where<D>::k(p.token, c));
      ks = a.k_pages[tile + Where<D>::scale(p.token, c)];
#pragma unroll
      for (int m = 0; m < 4; ++m) v |= (uint32_t)a.v_pages[tile + Where<D>::v(p.token, c, m)] << (8 * m);
      vs = a.v_pages[tile + Where<D>::scale(p.token, c)];
    }
    put_eight(k_out + to, k, ks);
    put_eight(v_out + to, v, vs);
  }
}

template <typename Fn>
hipError_t by_type(int dtype, int D, const Q4RowsArgs& a, Fn fn) {
  if (a.rows == 0) return hipSuccess;
  const int grid = (a.rows + kRowsWaves - 1) / kRowsWaves;
  if (dtype == 0 && D == 128) fn(uint16_t(), std::integral_constant<int, 128>{}, grid);
  else if (dtype == 0 && D == 64) fn(uint16_t(), std::integral_constant<int, 64>{}, grid);
  else if (dtype == 1 && D == 128) fn(float(), std::integral_constant<int, 128>{}, grid);
  else if (dtype == 1 && D == 64) fn(float(), std::integral_constant<int, 64>{}, grid);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_q4_append(int dtype, int D, const Q4RowsArgs& a, hipStream_t st) {
  return by_type(dtype, D, a, [&](auto t, auto d, int grid) {
    q4_append_kernel<decltype(t), decltype(d)::value><<<grid, 64 * kRowsWaves, 0, st>>>(a);
  });
}

hipError_t launch_q4_read(int dtype, int D, const Q4RowsArgs& a, hipStream_t st) {
  return by_type(dtype, D, a, [&](auto t, auto d, int grid) {
    q4_read_kernel<decltype(t), decltype(d)::value><<<grid, 64 * kRowsWaves, 0, st>>>(a);
  });
}

}  // namespace pa
