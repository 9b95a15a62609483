// The 8-bit cache's write and read of rows (format in pagedattn_q8.h).
//
// Writing: a page's scale is that of its largest value, so a wave takes a page's new rows
// whole, for one KV head (two at head_dim 64), of which a lane has 8 dims of four tokens.
// (Lanes of 8 dims of all 16 tokens, for four heads, 8 heads of 128: 8 prompts of 500 rows
// 8.4 us instead of 7.8, of 2,048 24.1 instead of 20.3; fp32 10.6 and 9.3, 29.6 and 26.1;
// but 256 of 20 rows 9.3 instead of 9.9, 8 of 512 beside 512 single ones 11.9 instead of
// 12.6, with fewer waves that find no rows.  A decode call's one row a page it does take
// so, for as many heads as it has lanes: 256 rows 3.8 us.)  What bounds it is a wave's
// chain of loads (its sequence, the page's entry, the scale) and the rows' load beside it:
// those 16,384 rows, 67 MB read and 34 written, stream at 5 TB/s.  The largest
// magnitude over the rows and then the lanes, the exponent from its bits, the scaled
// conversions to codes (their rounding is the format's).  Where the page holds earlier tokens and their
// scale is too small, the same lanes round those again: a power of two apart, their values
// are exact in fp32.  K and V are waves of their own.
// A lane's eight bytes of a token are eight in a row of the K tile; in the V tile they lie
// in eight words, each with the bytes of four tokens, swapped in registers where all four
// are new.  Reading mirrors it, four tokens a wave.
#include "pa_q_rows.h"
#include "pa_q8_tile.h"

namespace pa {
namespace {

constexpr int kLow = 17, kHigh = 246;  // scale bytes

template <int D>
struct Place {  // of a lane's chunk c of eight dims
  static __device__ __forceinline__ int k(int token, int c) { return ((c >> 1) * kPage + token) * 16 + (c & 1) * 8; }
  // of the words of dims 8 c + 2 m and + 1, tokens 4 t ..
  static __device__ __forceinline__ int v(int t, int c, int m) {
    return (c >> 3) * 1024 + (t * 16 + (c & 3) * 4 + m) * 16 + (c >> 2 & 1) * 8;
  }
};

__device__ __forceinline__ float power(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// Two codes (a half of w) from values that e4m3 holds or rounds to at most 448.
template <bool HIGH>
__device__ __forceinline__ uint32_t codes_of(uint32_t w, float a, float b) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)w, HIGH);
}
// Eight elements as they lie in memory.
template <typename T>
struct Raw {
  u32x4 w[sizeof(T) / 2];
};
__device__ __forceinline__ void widen_raw(const Raw<uint16_t>& r, float (&x)[8]) { widen(r.w[0], x, uint16_t()); }
__device__ __forceinline__ void widen_raw(const Raw<float>& r, float (&x)[8]) {
  widen(r.w[0], x, 0.0f);
  widen(r.w[1], x + 4, 0.0f);
}
// The codes of x times inv, whatever x is.
template <typename T>
__device__ __forceinline__ u32x2_t encode_any(const Raw<T>& r, float inv) {
  float x[8], y[8];
  widen_raw(r, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // (infinities too are held as NaN)
    y[e] = fabsf(x[e]) <= __FLT_MAX__ ? __builtin_amdgcn_fmed3f(x[e] * inv, -448.0f, 448.0f) : NAN;
  }
  u32x2_t w = {0, 0};
  w.x = codes_of<false>(w.x, y[0], y[1]);
  w.x = codes_of<true>(w.x, y[2], y[3]);
  w.y = codes_of<false>(w.y, y[4], y[5]);
  w.y = codes_of<true>(w.y, y[6], y[7]);
  return w;
}
// The same of finite x of at most 448 scale, in four instructions.
template <typename T>
__device__ __forceinline__ u32x2_t encode(const Raw<T>& r, float scale) {
  typedef short s16x2_t __attribute__((ext_vector_type(2)));
  u32x2_t w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    s16x2_t c = {0, 0};
    if constexpr (sizeof(T) == 2) {
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, as_bf16x2(r.w[0][2 * h]), scale, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, as_bf16x2(r.w[0][2 * h + 1]), scale, true);
    } else {
      const u32x4 x = r.w[h];
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, __uint_as_float(x[0]), __uint_as_float(x[1]), scale, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, __uint_as_float(x[2]), __uint_as_float(x[3]), scale, true);
    }
    w[h] = __builtin_bit_cast(uint32_t, c);
  }
  return w;
}
// Four codes rounded again, f (a power of two below 1) times their values.
__device__ __forceinline__ uint32_t again(uint32_t w, float f) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return codes_of<true>(codes_of<false>(0, a[0] * f, a[1] * f), b[0] * f, b[1] * f);
}

// The largest magnitude of m and the elements, an infinity or (bf16) a NaN where there is
// one; and the largest finite one.
__device__ __forceinline__ float most_of(float m, const Raw<uint16_t>& r) {
  typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
  u16x2_t x = {0, 0};  // (bits of magnitudes compare as they do)
#pragma unroll
  for (int i = 0; i < 4; ++i) x = __builtin_elementwise_max(x, __builtin_bit_cast(u16x2_t, r.w[0][i] & 0x7fff7fffu));
  return __uint_as_float(max(__float_as_uint(m), (uint32_t)max(x[0], x[1]) << 16));
}
__device__ __forceinline__ float most_of(float m, const Raw<float>& r) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = r.w[h][i] & 0x7fffffffu;  // (NaN too)
      m = __uint_as_float(max(__float_as_uint(m), u));
    }
  return m;
}
template <typename T>
__device__ __forceinline__ float finite_most_of(float m, const Raw<T>& r) {
  float x[8];
  widen_raw(r, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fabsf(x[e]) <= __FLT_MAX__ ? fmaxf(m, fabsf(x[e])) : m;
  return m;
}

// Scale byte of a page whose largest new value is m: the exponent's byte less 8, or 7
// above 1.75 (a carry out of the mantissa).
__device__ __forceinline__ int scale_byte(float m) {
  return min(max((int)((__float_as_uint(m) + 0x1fffffu) >> 23) - 8, kLow), kHigh);
}
// The page's tokens from .. to - 1 (from: a multiple of four) brought from scale byte
// `held` to e.
template <int D>
__device__ __forceinline__ void rescale(uint8_t* tile, bool k, int c, int from, int to, int held, int e) {
  const float f = power(127 + max(held - e, -64));  // (2^-64 of any code is 0)
  if (k) {
    for (int t = from; t < to; ++t) {
      u32x2_t* at = reinterpret_cast<u32x2_t*>(tile + Place<D>::k(t, c));
      const u32x2_t w = *at;
      *at = u32x2_t{again(w.x, f), again(w.y, f)};
    }
  } else {
    for (int t = from; t < to; t += 4) {
      const uint32_t early = to - t >= 4 ? ~0u : (1u << 8 * (to - t)) - 1;  // bytes
#pragma unroll
      for (int m4 = 0; m4 < 4; ++m4) {
        u32x2_t* at = reinterpret_cast<u32x2_t*>(tile + Place<D>::v(t >> 2, c, m4));
        const u32x2_t w = *at;
        *at = u32x2_t{(again(w.x, f) & early) | (w.x & ~early), (again(w.y, f) & early) | (w.y & ~early)};
      }
    }
  }
}
// A token's codes alone.
template <int D>
__device__ __forceinline__ void put_token(uint8_t* tile, bool k, int c, int t, u32x2_t w) {
  if (k) {
    *reinterpret_cast<u32x2_t*>(tile + Place<D>::k(t, c)) = w;
    return;
  }
#pragma unroll
  for (int m4 = 0; m4 < 4; ++m4) {
    uint8_t* at = tile + Place<D>::v(t >> 2, c, m4) + (t & 3);
    const uint32_t pair = (m4 < 2 ? w.x : w.y) >> 16 * (m4 & 1);
    at[0] = (uint8_t)pair;
    at[4] = (uint8_t)(pair >> 8);
  }
}

// PAGES: lanes of four tokens of a head each; otherwise every sequence has one row, and a
// wave takes it for as many heads as it has lanes.
template <typename T, int D, bool PAGES>
__global__ __launch_bounds__(64 * kRowsWaves) void q8_append_kernel(QRowsArgs a, int slots) {
  constexpr int CH = D / 8, N = PAGES ? 4 : 1, kLanes = PAGES ? 4 * CH : CH;  // tokens of a lane, lanes of a head
  const int lane = threadIdx.x & 63;
  const int slot = blockIdx.x * kRowsWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (slot >= slots) return;
  Group p = group_of<kPage, false>(a, slot, lane);
  if (p.n <= 0 || p.bad) return;
  const int i = blockIdx.y * 64 + lane;
  const bool is_k = blockIdx.z == 0;
  const int g = i / kLanes, c = i % CH;
  if (g >= a.H_kv) return;  // (whole heads)
  const int t0 = PAGES ? i / CH % 4 * 4 : p.token;  // the lane's first token
  const int64_t step = (int64_t)a.H_kv * D;
  const T* from = reinterpret_cast<const T*>(is_k ? a.k_rows : a.v_rows) + (int64_t)p.row * step + (int64_t)g * D + c * 8;
  // loaded while the page's entry is; a token that is not new: a new row again, unused
  Raw<T> raw[N];
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const int row = PAGES ? min(max(t0 + t - p.token, 0), p.n - 1) : 0;
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) raw[t].w[h] = *reinterpret_cast<const u32x4*>(from + row * step + h * (16 / (int)sizeof(T)));
  }
  checked_page(a, p);
  if (p.bad) return;
  const int64_t head = (int64_t)p.page * a.H_kv + g;
  uint8_t* tile = (is_k ? a.k_pages : a.v_pages) + head * q8_tile_bytes(D);
  uint8_t* scale = a.scales + head * 2 + blockIdx.z;
  const int held = p.token > 0 ? *scale : 0;  // (no earlier tokens: none that bounds it)

  float most = 0.0f;
#pragma unroll
  for (int t = 0; t < N; ++t) most = most_of(most, raw[t]);
  // (rare: values that are not finite are left out of the scale, and those beyond the
  // largest scale's are cut)
  bool plain = most <= __FLT_MAX__;
  if (__builtin_amdgcn_ballot_w64(!plain) != 0) {
    plain = false;
    most = 0.0f;
#pragma unroll
    for (int t = 0; t < N; ++t) most = finite_most_of(most, raw[t]);
  }
  most = fmaxf(most, dpp_xor1(most));
  most = fmaxf(most, dpp_xor2(most));
  most = fmaxf(most, dpp_half_mirror(most));
  if constexpr (kLanes >= 16) most = fmaxf(most, dpp_mirror(most));
  if constexpr (kLanes >= 32) most = fmaxf(most, swz_xor16(most));
  if constexpr (kLanes >= 64) most = fmaxf(most, xor32(most));
  const int e = max(scale_byte(most), held);
  if (p.token > 0 && e > held) {
    if constexpr (PAGES) rescale<D>(tile, is_k, c, t0, min(p.token, t0 + 4), held, e);
    else rescale<D>(tile, is_k, c, 0, p.token, held, e);
  }
  if (i % kLanes == 0 && (p.token == 0 || e > held)) *scale = (uint8_t)e;
  plain = __builtin_amdgcn_ballot_w64(!plain || e >= kHigh) == 0;
  const float size = power(e), inv = power(254 - e);
  u32x2_t w[N];
#pragma unroll
  for (int t = 0; t < N; ++t) w[t] = plain ? encode(raw[t], size) : encode_any(raw[t], inv);

  if constexpr (PAGES) {
    const int end = p.token + p.n;
    if (!is_k && t0 >= p.token && t0 + 4 <= end) {  // words of new tokens alone
      uint32_t lo[4] = {w[0].x, w[1].x, w[2].x, w[3].x}, hi[4] = {w[0].y, w[1].y, w[2].y, w[3].y};
      transpose4(lo);
      transpose4(hi);
#pragma unroll
      for (int m4 = 0; m4 < 4; ++m4) {
        const int o = m4 % 2 * 2;
        *reinterpret_cast<u32x2_t*>(tile + Place<D>::v(t0 >> 2, c, m4)) = m4 < 2 ? u32x2_t{lo[o], lo[o + 1]} : u32x2_t{hi[o], hi[o + 1]};
      }
      return;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (t0 + t >= p.token && t0 + t < end) put_token<D>(tile, is_k, c, t0 + t, w[t]);
  } else {
    put_token<D>(tile, is_k, c, t0, w[0]);
  }
}

// The values of a lane's codes, 16 bytes of them: eight codes or (fp32) w.x's four.
template <bool kPast, typename T>
__device__ __forceinline__ void put(T* p, u32x2_t w, float scale) {
  if constexpr (sizeof(T) == 2) {
    store_row<kPast>(p, q8::eight_of(w.x, w.y, scale));
  } else {
    const q::f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, scale, true);
    store_row<kPast>(p, q::f32x4_t{a[0], a[1], b[0], b[1]});
  }
}

// A wave reads a group's tokens for 64 (KV head, 16 bytes of the output): its stores are
// a KiB in a row each.
template <typename T, int D, bool kPast>
__global__ __launch_bounds__(64 * kRowsWaves) void q8_read_kernel(QRowsArgs a, int slots) {
  constexpr int kGroup = kQRowsGroup;
  constexpr int kHalf = sizeof(T) == 4;  // four dims a lane
  constexpr int CH = D / 8 << kHalf;
  const int lane = threadIdx.x & 63;
  const int slot = blockIdx.x * kRowsWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = blockIdx.y * 64 + lane;
  if (slot >= slots) return;
  const Group p = group_of<kGroup>(a, slot, lane);
  if (p.n <= 0 || i >= a.H_kv * CH) return;
  const int g = i / CH, c = i % CH >> kHalf, half = kHalf ? i & 1 : 0, first = p.token & ~(kGroup - 1);
  // (all four tokens of the group, whichever are asked for)
  u32x2_t k[kGroup], v[kGroup];
  float ks = 1.0f, vs = 1.0f;
  if (!p.bad) {
    const int64_t head = (int64_t)p.page * a.H_kv + g, tile = head * q8_tile_bytes(D);
    const uint32_t sc = *reinterpret_cast<const uint16_t*>(a.scales + head * 2);
    ks = q::scale_of<0>(sc);
    vs = q::scale_of<1>(sc);
    uint32_t lo[4], hi[4] = {};
#pragma unroll
    for (int t = 0; t < kGroup; ++t) {
      const uint8_t* at = a.k_pages + tile + Place<D>::k(first + t, c);
      if constexpr (kHalf) k[t] = u32x2_t{*reinterpret_cast<const uint32_t*>(at + 4 * half), 0};
      else k[t] = *reinterpret_cast<const u32x2_t*>(at);
    }
#pragma unroll
    for (int m = 0; m < (kHalf ? 2 : 4); ++m) {
      const u32x2_t w = *reinterpret_cast<const u32x2_t*>(a.v_pages + tile + Place<D>::v(first >> 2, c, 2 * half + m));
      (m < 2 ? lo : hi)[m % 2 * 2] = w.x;
      (m < 2 ? lo : hi)[m % 2 * 2 + 1] = w.y;
    }
    transpose4(lo);
    if constexpr (!kHalf) transpose4(hi);
#pragma unroll
    for (int t = 0; t < kGroup; ++t) v[t] = u32x2_t{lo[t], hi[t]};
  } else {
#pragma unroll
    for (int t = 0; t < kGroup; ++t) k[t] = v[t] = u32x2_t{0x7f7f7f7fu, 0x7f7f7f7fu};
  }
  const int64_t to = (int64_t)p.row * a.H_kv * D + (int64_t)i * (16 / sizeof(T)), step = (int64_t)a.H_kv * D;
  T* k_out = reinterpret_cast<T*>(const_cast<void*>(a.k_rows)) + to;
  T* v_out = reinterpret_cast<T*>(const_cast<void*>(a.v_rows)) + to;
#pragma unroll
  for (int t = 0; t < kGroup; ++t) {
    const int r = first + t - p.token;  // (wave-uniform)
    if (r < 0 || r >= p.n) continue;
    put<kPast>(k_out + r * step, k[t], ks);
    put<kPast>(v_out + r * step, v[t], vs);
  }
}

// Slots of a call (group_of; checked to be 32-bit).
int slots_of(const QRowsArgs& a, int group) { return (int)q_row_slots(a.query_start_loc != nullptr, a.rows, a.B, group); }

}  // namespace

hipError_t launch_q8_append(int dtype, int D, const QRowsArgs& a, hipStream_t st) {
  return by_type(dtype, D, a, [&](auto t, auto d) {
    constexpr int D = decltype(d)::value;
    const bool pages = a.query_start_loc != nullptr;
    const int slots = slots_of(a, kPage);
    const dim3 grid((slots + kRowsWaves - 1) / kRowsWaves, (a.H_kv * (D / (pages ? 2 : 8)) + 63) / 64, 2);
    const auto fn = pages ? &q8_append_kernel<decltype(t), D, true> : &q8_append_kernel<decltype(t), D, false>;
    fn<<<grid, 64 * kRowsWaves, 0, st>>>(a, slots);
  });
}

hipError_t launch_q8_read(int dtype, int D, const QRowsArgs& a, hipStream_t st) {
  return by_type(dtype, D, a, [&](auto t, auto d) {
    const int slots = slots_of(a, kQRowsGroup);
    const dim3 grid((slots + kRowsWaves - 1) / kRowsWaves, (a.H_kv * D * (int)sizeof(t) / 16 + 63) / 64);
    const bool past = (int64_t)2 * a.rows * a.H_kv * D * sizeof(t) > kCached;
    constexpr int D = decltype(d)::value;
    const auto fn = past ? &q8_read_kernel<decltype(t), D, true> : &q8_read_kernel<decltype(t), D, false>;
    fn<<<grid, 64 * kRowsWaves, 0, st>>>(a, slots);
  });
}

}  // namespace pa
