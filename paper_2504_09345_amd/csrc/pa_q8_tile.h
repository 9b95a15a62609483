// The 8-bit cache's format (pagedattn_q8.h): a wave's share of two pages, its values as
// matrix-core operands, and the products of 32 tokens.
#pragma once

#include "pa_q_tile.h"

namespace pa {
namespace q8 {

using namespace q;

template <int D> constexpr int kWords = D / 16;  // 4-byte words of codes of a lane and page

// Codes 2 H and 2 H + 1 of w times scale, as two bf16 (exact for scale bytes 17 .. 246)
// or two fp16 (exact for 112 .. 134).
template <int H, bool F16>
__device__ __forceinline__ uint32_t pair_of(uint32_t w, float scale) {
  if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, H != 0));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, H != 0));
}

// Eight codes times scale, as bf16.
__device__ __forceinline__ u32x4 eight_of(uint32_t lo, uint32_t hi, float scale) {
  return u32x4{pair_of<0, false>(lo, scale), pair_of<1, false>(lo, scale), pair_of<0, false>(hi, scale), pair_of<1, false>(hi, scale)};
}

// A lane's part of a unit (two pages of one KV head).
template <int D>
struct Unit {
  uint32_t k[2][kWords<D>];  // token lane % 16: dims 16 (lane / 16) .. +15, then (D = 128) 64 more
  uint32_t ks[2];            // the pages' scale bytes: K's, V's above it
  uint32_t v[2][kWords<D>];  // word 2 j + h: tokens 4 (lane / 16) .. +3, dim 32 j + 2 (lane % 16) + h
  uint32_t vs[2];            // the scale bytes that V is multiplied by (keep_scales)
};

// The lane's 16 bytes of each KiB of a tile.
template <int D, int Policy>
__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t r, int lane, uint32_t (&x)[kWords<D>]) {
#pragma unroll
  for (int h = 0; h < D / 64; ++h) {
    const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(r, h * 1024 + lane * 16, 0, Policy);
    x[4 * h] = w.x; x[4 * h + 1] = w.y; x[4 * h + 2] = w.z; x[4 * h + 3] = w.w;
  }
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_at(const uint8_t* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), (short)0, bytes, 0x00020000);
}
// The scale bytes (two) of the tile `at` (a multiple of 16 D) bytes into the pool.  (Two bytes per tile of 2 KiB, so
// they stay in the caches.)
template <int D>
__device__ __forceinline__ uint32_t scale_bytes(const uint8_t* scales, int64_t at) {
  return *reinterpret_cast<const uint16_t*>(scales + ((uint64_t)at / (8 * D)));
}

// Scores S^T[token][column] = K . Q^T of the unit's tokens, K as bf16, exactly.  (e4m3
// operands need no conversion of K, 16 instructions a page at head_dim 128, and take as long
// with the queries in two parts; but such a product adds the dims in eights of which it keeps
// the bits down to 2^-13 of the largest of the eight alone, and a channel of K that
// is larger than its neighbours, as some are, costs those their last bits.)
template <typename T, int D, int NB, bool C>
__device__ __forceinline__ void fold_qk(const State<T, D, NB, C>& st, const Unit<D>& u, f32x4_t (&s)[NB][2]) {
  static_assert(!C, "K in bf16");
#pragma unroll
  for (int p = 0; p < 2; ++p) {
#pragma unroll
    for (int c = 0; c < NB; ++c) s[c][p] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const float ks = scale_of<0>(u.ks[p]);
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
      const bf16x8_t a = __builtin_bit_cast(bf16x8_t, eight_of(u.k[p][2 * w], u.k[p][2 * w + 1], ks));
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int i = 0; i < kQParts<T>; ++i)
          s[c][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, st.q[c].x[w][i]), s[c][p], 0, 0, 0);
    }
  }
}

// V of keys past all_last, which no column sees: their weights are 0, but an unused
// slot may hold anything, and 0 times a NaN is NaN.  Their codes become 0, and the scale of
// a page of none else 1.
__device__ __forceinline__ uint32_t live_bytes(int key0, int all_last) {  // of a word whose first token is key0
  const int n = all_last - key0 + 1;
  return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << 8 * n) - 1;
}
constexpr uint32_t kScaleOne = 127u << 8;  // (V's)
template <int D>
__device__ __forceinline__ void clear_dead(Unit<D>& u, int key0, int all_last, int lane) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const uint32_t live = live_bytes(key0 + 16 * p + 4 * (lane >> 4), all_last);
#pragma unroll
    for (int w = 0; w < kWords<D>; ++w) u.v[p][w] &= live;
    if (key0 + 16 * p > all_last) u.vs[p] = kScaleOne;
  }
}

// Whether fp16 does not hold a page's V exactly: a scale of 2^-15 .. 2^7 puts 2^-9 at
// 2^-24 or more, and 448 below 2^16.
__device__ __forceinline__ bool beyond_fp16(uint32_t vs) { return (vs >> 8) - 112u > 22u; }
// Whether a page may have a V of 2^64 or more: scale bytes from 2^56 on.
constexpr uint32_t kLargeScale = 183;
__device__ __forceinline__ bool is_large(uint32_t vs) { return (vs >> 8) >= kLargeScale; }

// O^T += V^T . P^T, in fp16 or in bf16 parts.  k slots 8 G + 4 p + i are token 4 G + i of
// page p, and a word's bytes the four tokens of a dim, so two conversions make a word half
// of an operand.
template <bool F16, typename T, int D, int NB, bool C>
__device__ __forceinline__ void fold_pv(State<T, D, NB, C>& st, const Unit<D>& u, const float (&x)[NB][8]) {
  constexpr int N = F16 ? 1 : kPParts<T>;
  u32x4 pt[NB][N];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    if constexpr (F16) {
#pragma unroll
      for (int h = 0; h < 4; ++h)
        pt[c][0][h] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{x[c][2 * h], x[c][2 * h + 1]}), f16x2_t));
    } else {
      split8(x[c], pt[c]);
    }
  }
  const float s0 = scale_of<1>(u.vs[0]), s1 = scale_of<1>(u.vs[1]);
#pragma unroll
  for (int mb = 0; mb < D / 16; ++mb) {
    const u32x4 a = {pair_of<0, F16>(u.v[0][mb], s0), pair_of<1, F16>(u.v[0][mb], s0), pair_of<0, F16>(u.v[1][mb], s1),
                     pair_of<1, F16>(u.v[1][mb], s1)};
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      f32x4_t& acc = st.acc[c][mb];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (F16)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, pt[c][i]), acc, 0, 0, 0);
        else
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, pt[c][i]), acc, 0, 0, 0);
      }
    }
  }
}

// The bytes of w that are NaN's codes, as 0x80 each.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// The same (in bf16) for a unit of which some columns see a part: a NaN of V reaches the
// columns that see its key, and no other (a weight of 0 times NaN would be NaN).  It
// becomes 0, and where there are any, a product of their places with the keys that each
// column sees says which outputs are NaN.  (Keys that no column sees are cleared.)
template <typename T, int D, int NB, bool C>
__device__ __forceinline__ void fold_pv_edge(State<T, D, NB, C>& st, Unit<D>& u, const float (&x)[NB][8], int key0, int lane) {
  uint32_t any = 0;
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int w = 0; w < kWords<D>; ++w) any |= nan_bytes(u.v[p][w]);
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(any != 0) != 0, 0)) {
    u32x4 seen[NB];
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int key = key0 + 16 * (h >> 1) + 4 * (lane >> 4) + 2 * (h & 1);
        seen[c][h] = (key <= st.last[c] ? 0x3f80u : 0u) | (key + 1 <= st.last[c] ? 0x3f800000u : 0u);
      }
#pragma unroll
    for (int mb = 0; mb < D / 16; ++mb) {
      __builtin_amdgcn_sched_barrier(0);
      u32x4 a;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const uint32_t n = nan_bytes(u.v[p][mb]);
        const uint32_t ones = (n >> 1) - (n >> 4);  // 0x40 - 0x08 = 0x38: 1 in e4m3
        u.v[p][mb] &= ~(n | (n - (n >> 7)));
        a[2 * p] = pair_of<0, false>(ones, 1.0f);
        a[2 * p + 1] = pair_of<1, false>(ones, 1.0f);
      }
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const f32x4_t count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, seen[c]),
                                                                      f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (count[i] > 0.0f) st.acc[c][mb][i] = NAN;
      }
    }
  }
  fold_pv<false>(st, u, x);
}

// What the kernels ask of a format (pa_q4_tile.h).
struct Format {
  template <int D> using Unit = q8::Unit<D>;
  template <typename T, int D> static constexpr bool kCodes = false;
  template <typename T> static constexpr bool kWide = sizeof(T) == 2;  // waves of 32 columns too
  static constexpr bool kSliced = true;  // K operands in bf16: 16 dims in a row of each 64
  static constexpr bool kSums = true;  // a base moves by sums of weights (not by the largest)
  static constexpr int tile_bytes(int D) { return q8_tile_bytes(D); }
  static __device__ __forceinline__ const uint8_t* scales_of_head(const uint8_t* scales, int g) { return scales + 2 * g; }

  template <int Policy, int D>
  static __device__ __forceinline__ void load_k(Unit<D>& u, int p, const uint8_t* pool, int64_t at, const uint8_t* scales, int bytes, int lane) {
    u.ks[p] = scale_bytes<D>(scales, at);
    load_words<D, Policy>(tile_at(pool + at, bytes), lane, u.k[p]);
  }
  template <int Policy, int D>
  static __device__ __forceinline__ void load_v(Unit<D>& u, int p, const uint8_t* pool, int64_t at, const uint8_t*, int bytes, int lane) {
    load_words<D, Policy>(tile_at(pool + at, bytes), lane, u.v[p]);
  }
  template <int D> static __device__ __forceinline__ void keep_scales(Unit<D>& u) {
#pragma unroll
    for (int p = 0; p < 2; ++p) u.vs[p] = u.ks[p];
  }
  template <int D> static __device__ __forceinline__ int shift(int) { return 0; }
  template <bool F16, int D>
  static __device__ __forceinline__ bool odd(const Unit<D>& u) {
    return F16 ? beyond_fp16(u.vs[0]) || beyond_fp16(u.vs[1]) : has_large(u);
  }
  template <int D> static __device__ __forceinline__ bool has_large(const Unit<D>& u) { return is_large(u.vs[0]) || is_large(u.vs[1]); }
  // (a page's first key: any of its tokens may be the large one)
  template <int D>
  static __device__ __forceinline__ int first_large(const Unit<D>& u, int key0, int) {
    return __builtin_amdgcn_readfirstlane(is_large(u.vs[0]) ? key0 : is_large(u.vs[1]) ? key0 + kPage : INT32_MAX);
  }
  template <int D>
  static __device__ __forceinline__ void clear_dead(Unit<D>& u, int key0, int all_last, int lane) { q8::clear_dead(u, key0, all_last, lane); }
  template <typename T, int D, int NB, bool C>
  static __device__ __forceinline__ void fold_qk(const State<T, D, NB, C>& st, const Unit<D>& u, int, f32x4_t (&s)[NB][2]) {
    q8::fold_qk(st, u, s);
  }
  template <bool F16, typename T, int D, int NB, bool C>
  static __device__ __forceinline__ void fold_pv(State<T, D, NB, C>& st, const Unit<D>& u, const float (&x)[NB][8]) {
    q8::fold_pv<F16>(st, u, x);
  }
  template <typename T, int D, int NB, bool C>
  static __device__ __forceinline__ void fold_pv_edge(State<T, D, NB, C>& st, Unit<D>& u, const float (&x)[NB][8], int key0, int lane) {
    q8::fold_pv_edge(st, u, x, key0, lane);
  }
};

}  // namespace q8
}  // namespace pa
