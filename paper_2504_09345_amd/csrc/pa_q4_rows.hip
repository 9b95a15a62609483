// The 4-bit cache's write and read of rows (format in pagedattn_q4.h).
//
// A (row, KV head) vector of D elements is D / 8 lanes of 8 consecutive ones, four
// lanes to a block of 32.  Writing: the block's largest magnitude over its lanes
// (DPP), the scale from that value's bits, v_cvt_scalef32_pk_fp4_f32 to codes (its
// rounding is the format's).  A lane's four bytes are one word of the K tile and four
// bytes of the V tile, each in a word with those of three neighbouring tokens: a wave
// takes four tokens and swaps the bytes in registers.  Reading mirrors it.
#include "pa_q4_tile.h"
#include "pa_q_rows.h"

namespace pa {

namespace {

constexpr int kGroup = kQRowsGroup;

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
__global__ __launch_bounds__(64 * kRowsWaves) void q4_append_kernel(QRowsArgs a, int slots) {
  constexpr int CH = D / 8;
  const int lane = threadIdx.x & 63;
  const int slot = blockIdx.x * kRowsWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (slot >= slots) return;
  const Group p = group_of<kGroup>(a, slot, lane);
  if (p.n <= 0 || p.bad) return;
  const int i = blockIdx.y * 64 + lane;
  if (i >= a.H_kv * CH) return;
  const int g = i / CH, c = i % CH;
  const int64_t from = ((int64_t)p.row * a.H_kv + g) * D + c * 8, step = (int64_t)a.H_kv * D;
  const int64_t tile = ((int64_t)p.page * a.H_kv + g) * q4_tile_bytes(D);
  uint8_t* kt = a.k_pages + tile;
  uint8_t* vt = a.v_pages + tile;
  auto k_row = [&](int t, const float (&x)[8]) {
    uint32_t scale;
    const uint32_t k = quantise(x, scale);
    *reinterpret_cast<uint32_t*>(kt + Where<D>::k(p.token + t, c)) = k;
    if ((c & 3) == 0) kt[Where<D>::scale(p.token + t, c)] = (uint8_t)scale;
  };
  auto v_row = [&](int t, const float (&x)[8]) {
    uint32_t scale;
    const uint32_t v = quantise(x, scale);
    if ((c & 3) == 0) vt[Where<D>::scale(p.token + t, c)] = (uint8_t)scale;
    return v;
  };
  if (p.n == kGroup) {
    float x[kGroup][8], y[kGroup][8];
#pragma unroll
    for (int t = 0; t < kGroup; ++t) {
      load_eight(reinterpret_cast<const T*>(a.k_rows) + from + t * step, x[t]);
      load_eight(reinterpret_cast<const T*>(a.v_rows) + from + t * step, y[t]);
    }
    uint32_t v[4];
#pragma unroll
    for (int t = 0; t < kGroup; ++t) {
      k_row(t, x[t]);
      v[t] = v_row(t, y[t]);
    }
    transpose4(v);
#pragma unroll
    for (int m = 0; m < 4; ++m) *reinterpret_cast<uint32_t*>(vt + Where<D>::v(p.token, c, m)) = v[m];
  } else {
#pragma unroll 1
    for (int t = 0; t < p.n; ++t) {
      float x[8], y[8];
      load_eight(reinterpret_cast<const T*>(a.k_rows) + from + t * step, x);
      load_eight(reinterpret_cast<const T*>(a.v_rows) + from + t * step, y);
      k_row(t, x);
      const uint32_t v = v_row(t, y);
#pragma unroll
      for (int m = 0; m < 4; ++m) vt[Where<D>::v(p.token + t, c, m)] = (uint8_t)(v >> (8 * m));
    }
  }
}

// The values of a lane's codes, 16 bytes of them: a word's eight or a half's four.
template <bool kPast, typename T>
__device__ __forceinline__ void put(T* p, uint32_t w, uint32_t scale) {
  const float s = __uint_as_float(scale << 23);
  if constexpr (sizeof(T) == 2) {
    store_row<kPast>(p, q4::eight_of(w, s));
  } else {
    const q4::f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
    store_row<kPast>(p, q4::f32x4_t{a[0], a[1], b[0], b[1]});
  }
}

// A wave reads a group's tokens for 64 (KV head, 16 bytes of the output): its stores are
// a KiB in a row each.  (Eight dims of fp32 a lane, in two stores that alternate by 16
// bytes, take 104 us instead of 88 for 64 contexts of 512-2,048 tokens, 8 heads of 64
// dims, through the caches.)
template <typename T, int D, bool kPast>
__global__ __launch_bounds__(64 * kRowsWaves) void q4_read_kernel(QRowsArgs a, int slots) {
  constexpr int kHalf = sizeof(T) == 4;  // four dims a lane, half a word's codes
  constexpr int CH = D / 8 << kHalf, kV = kGroup >> kHalf;
  const int lane = threadIdx.x & 63;
  const int slot = blockIdx.x * kRowsWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = blockIdx.y * 64 + lane;
  if (slot >= slots) return;
  const Group p = group_of<kGroup>(a, slot, lane);
  if (p.n <= 0 || i >= a.H_kv * CH) return;
  const int g = i / CH, c = i % CH >> kHalf, half = kHalf ? i & 1 : 0, first = p.token & ~(kGroup - 1);
  // (all four tokens of the group, whichever are asked for)
  uint32_t k[kGroup] = {}, v[kGroup] = {}, ks[kGroup], vs[kGroup];
  if (!p.bad) {
    const int64_t tile = ((int64_t)p.page * a.H_kv + g) * q4_tile_bytes(D);
#pragma unroll
    for (int t = 0; t < kGroup; ++t) {
      k[t] = *reinterpret_cast<const uint32_t*>(a.k_pages + tile + Where<D>::k(first + t, c));
      ks[t] = a.k_pages[tile + Where<D>::scale(first + t, c)];
      vs[t] = a.v_pages[tile + Where<D>::scale(first + t, c)];
    }
#pragma unroll
    for (int m = 0; m < kV; ++m) v[m] = *reinterpret_cast<const uint32_t*>(a.v_pages + tile + Where<D>::v(first, c, half * kV + m));
  } else {
#pragma unroll
    for (int t = 0; t < kGroup; ++t) ks[t] = vs[t] = 255;
  }
  transpose4(v);
  const int64_t to = (int64_t)p.row * a.H_kv * D + (int64_t)i * (16 / sizeof(T)), step = (int64_t)a.H_kv * D;
  T* k_out = reinterpret_cast<T*>(const_cast<void*>(a.k_rows)) + to;
  T* v_out = reinterpret_cast<T*>(const_cast<void*>(a.v_rows)) + to;
#pragma unroll
  for (int t = 0; t < kGroup; ++t) {
    const int r = first + t - p.token;  // (wave-uniform)
    if (r < 0 || r >= p.n) continue;
    put<kPast>(k_out + r * step, k[t] >> (16 * half), ks[t]);
    put<kPast>(v_out + r * step, v[t], vs[t]);
  }
}

// Slots of a call (group_of; checked to be 32-bit).
int slots_of(const QRowsArgs& a) { return (int)q_row_slots(a.query_start_loc != nullptr, a.rows, a.B); }

}  // namespace

hipError_t launch_q4_append(int dtype, int D, const QRowsArgs& a, hipStream_t st) {
  return by_type(dtype, D, a, [&](auto t, auto d) {
    constexpr int D = decltype(d)::value;
    const int slots = slots_of(a);
    const dim3 grid((slots + kRowsWaves - 1) / kRowsWaves, (a.H_kv * (D / 8) + 63) / 64);
    q4_append_kernel<decltype(t), D><<<grid, 64 * kRowsWaves, 0, st>>>(a, slots);
  });
}

hipError_t launch_q4_read(int dtype, int D, const QRowsArgs& a, hipStream_t st) {
  return by_type(dtype, D, a, [&](auto t, auto d) {
    const int slots = slots_of(a);
    const dim3 grid((slots + kRowsWaves - 1) / kRowsWaves, (a.H_kv * D * (int)sizeof(t) / 16 + 63) / 64);
    const bool past = (int64_t)2 * a.rows * a.H_kv * D * sizeof(t) > kCached;
    constexpr int D = decltype(d)::value;
    const auto fn = past ? &q4_read_kernel<decltype(t), D, true> : &q4_read_kernel<decltype(t), D, false>;
    fn<<<grid, 64 * kRowsWaves, 0, st>>>(a, slots);
  });
}

}  // namespace pa
