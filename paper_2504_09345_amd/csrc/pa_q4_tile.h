// The 4-bit cache's format (pagedattn_q4.h): a wave's share of two pages, its values as
// matrix-core operands, and the products of 32 tokens.
#pragma once

#include "pa_q_tile.h"

namespace pa {

namespace q4 {

using namespace q;

template <int D> constexpr int kWords = D / 32;  // 4-byte words of codes of a lane and page, and scales of a token
template <int D> constexpr int kScales = 8 * D;  // offset of a tile's scales

// Byte B of w (two codes) times scale, as two bf16: exact for scale bytes 0 ..
// 252, NaN for 255 (v_cvt_scalef32_pk_bf16_fp4); or as two fp16, exact for 104 .. 140.
template <int B, bool F16 = false>
__device__ __forceinline__ uint32_t pair_of(uint32_t w, float scale) {
  if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, B));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}
__device__ __forceinline__ u32x4 eight_of(uint32_t w, float scale) {
  return u32x4{pair_of<0>(w, scale), pair_of<1>(w, scale), pair_of<2>(w, scale), pair_of<3>(w, scale)};
}

// A lane's part of a unit (two pages of one KV head).
template <int D>
struct Unit {
  uint32_t k[2][kWords<D>];  // codes of token lane % 16, dims D/4 (lane / 16) .. +D/4
  uint32_t ks[2];            // the word that holds the scale byte of those dims (k_shift)
  uint32_t v[2][kWords<D>];  // word j: tokens 4 (lane / 16) .. +3, dims 32 j + 2 (lane % 16), +1
  uint32_t vs[2][kWords<D>];  // scales of those four tokens, token-major
};

// Loads of a unit are non-temporal in the decode kernel (as its 16-bit sibling's:
// each byte is read once), and cached where other workgroups read them again.
template <int D, int Policy>
__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t r, int off, uint32_t (&x)[kWords<D>]) {
  if constexpr (D == 128) {
    const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, Policy);
    x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
  } else {
    const u32x2_t w = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, Policy);
    x[0] = w.x; x[1] = w.y;
  }
}
// Loads of page p (0 or 1) of a unit from the tiles at k and v; with bytes = 0 instead
// of the tile's nothing is read, and every code and scale is 0.
template <int D, int Policy>
__device__ __forceinline__ void load_k(Unit<D>& u, int p, const uint8_t* k, int bytes, int lane) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(k), (short)0, bytes, 0x00020000);
  load_words<D, Policy>(r, lane * (D / 8), u.k[p]);
  u.ks[p] = __builtin_amdgcn_raw_buffer_load_b32(r, kScales<D> + ((lane & 15) * (D / 32) & ~3), 0, Policy);
}
// The shift that brings the scale byte of the lane's K codes down, with others above it.
// (A load of the byte alone is extended where it is loaded, which waits for it there.)
template <int D>
__device__ __forceinline__ int k_shift(int lane) {
  return D == 128 ? (lane >> 4) * 8 : (lane & 1) * 16 + (lane >> 5) * 8;
}
template <int D, int Policy>
__device__ __forceinline__ void load_v(Unit<D>& u, int p, const uint8_t* v, int bytes, int lane) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(v), (short)0, bytes, 0x00020000);
  load_words<D, Policy>(r, lane * (D / 8), u.v[p]);
  load_words<D, Policy>(r, kScales<D> + (lane >> 4) * (D / 8), u.vs[p]);
}

// Scale of block j of the lane's token i (of four).
template <int D, int J, int I>
__device__ __forceinline__ float v_scale(const uint32_t (&vs)[kWords<D>]) {
  if constexpr (D == 128) return scale_of<J>(vs[I]);
  else return scale_of<(I & 1) * 2 + J>(vs[I >> 1]);
}

// V^T operands of block J: rows are its even dims 32 J + 2 r (a[0]) or odd ones
// (a[1]), k slots 8 G + 4 p + i the token 4 G + i of page p.  A byte holds the two
// dims of a token, so each pair of tokens is two conversions and two byte
// permutations.
template <int D, int J, bool F16>
__device__ __forceinline__ void v_operands(const Unit<D>& u, u32x4 (&a)[2]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const uint32_t w = u.v[p][J];
    const uint32_t t0 = pair_of<0, F16>(w, v_scale<D, J, 0>(u.vs[p])), t1 = pair_of<1, F16>(w, v_scale<D, J, 1>(u.vs[p]));
    const uint32_t t2 = pair_of<2, F16>(w, v_scale<D, J, 2>(u.vs[p])), t3 = pair_of<3, F16>(w, v_scale<D, J, 3>(u.vs[p]));
    a[0][2 * p] = __builtin_amdgcn_perm(t1, t0, 0x05040100u);
    a[0][2 * p + 1] = __builtin_amdgcn_perm(t3, t2, 0x05040100u);
    a[1][2 * p] = __builtin_amdgcn_perm(t1, t0, 0x07060302u);
    a[1][2 * p + 1] = __builtin_amdgcn_perm(t3, t2, 0x07060302u);
  }
}

// Fold of the unit of keys key0 .. key0 + 31, in three steps, so that K's registers
// and then V's are free for the next unit's loads as soon as they are read.
//
// Scores S^T[token][column] = K . Q^T, the K operand shared by the columns.  shift: of
// the scale words.
template <typename T, int D, int NB, bool C>
__device__ __forceinline__ void fold_qk(const State<T, D, NB, C>& st, const Unit<D>& u, int shift, f32x4_t (&s)[NB][2]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
#pragma unroll
    for (int c = 0; c < NB; ++c) s[c][p] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if constexpr (C) {
      const int ks = (int)(u.ks[p] >> shift);  // (the product reads the lowest byte)
      const i32x8_t a = {(int)u.k[p][0], (int)u.k[p][1], (int)u.k[p][2], (int)u.k[p][3], 0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < NB; ++c)  // (formats: 4 the codes, 0 e4m3)
          s[c][p] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, st.q[c].x[i], s[c][p], 4, 0, 0, ks, 0, (int)st.q[c].s[i]);
    } else {
      const float ks = scale_of<0>(u.ks[p] >> shift);
#pragma unroll
      for (int w = 0; w < D / 32; ++w) {
        const bf16x8_t a = __builtin_bit_cast(bf16x8_t, eight_of(u.k[p][w], ks));
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
          for (int i = 0; i < kQParts<T>; ++i)
            s[c][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, st.q[c].x[w][i]), s[c][p], 0, 0, 0);
      }
    }
  }
}

// V of keys past all_last, which no column sees: their weights are 0, but an unused
// slot may hold anything, and 0 times a NaN is NaN.  Their scales become 1.
template <int D>
__device__ __forceinline__ void clear_dead(Unit<D>& u, int key0, int all_last, int lane) {
  constexpr int n = D / 32;
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (key0 + 16 * p + 4 * (lane >> 4) + i > all_last) {
        uint32_t& w = u.vs[p][n == 4 ? i : i >> 1];
        w = n == 4 ? 0x7f7f7f7fu : (i & 1) != 0 ? (w & 0xffffu) | 0x7f7f0000u : (w & 0xffff0000u) | 0x7f7fu;
      }
}

// Whether fp16 does not hold the unit's V exactly: scale bytes within 104 .. 135 do,
// the 32 from 2^-23 on (a byte below borrows, which leaves high bits set all the
// same), as this lane sees it.
template <int D>
__device__ __forceinline__ bool beyond_fp16(const Unit<D>& u) {
  uint32_t off = 0;
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int w = 0; w < kWords<D>; ++w) off |= u.vs[p][w] - 0x68686868u;
  return (off & 0xe0e0e0e0u) != 0;
}

constexpr int kLargeScale = 192;
// Whether the unit has a V of 2^64 or more (scale bytes from kLargeScale on, that of NaN
// among them: bits 7 and 6), as this lane sees it.
template <int D>
__device__ __forceinline__ bool has_large(const Unit<D>& u) {
  static_assert(kLargeScale == 0xc0);
  uint32_t both = 0;
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int w = 0; w < kWords<D>; ++w) both |= u.vs[p][w] & (u.vs[p][w] << 1);
  return (both & 0x80808080u) != 0;
}

// The first of keys key0 .. key0 + 31 with such a V (those that no column sees are
// cleared), INT32_MAX: none.  (All lanes active; the same in all.)
template <int D>
__device__ __forceinline__ int first_large(const Unit<D>& u, int key0, int lane) {
  int first = INT32_MAX;
  if (__builtin_amdgcn_ballot_w64(has_large(u)) != 0) {
#pragma unroll
    for (int p = 1; p >= 0; --p)
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        const uint32_t w = D == 128 ? u.vs[p][i] : u.vs[p][i >> 1] >> (16 * (i & 1)) & 0xffffu;
        if ((w & w << 1 & 0x80808080u) != 0) first = key0 + 16 * p + 4 * (lane >> 4) + i;
      }
    first = min(first, __shfl_xor(first, 16));
    first = min(first, __shfl_xor(first, 32));
  }
  return __builtin_amdgcn_readfirstlane(first);
}

// O^T += V^T . P^T, in fp16 or in bf16 parts.
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
  auto block = [&](auto j_) {
    constexpr int j = decltype(j_)::value;
    u32x4 a[2];
    v_operands<D, j, F16>(u, a);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        f32x4_t& acc = st.acc[c][2 * j + h];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          if constexpr (F16)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a[h]), __builtin_bit_cast(f16x8_t, pt[c][i]), acc, 0, 0, 0);
          else
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a[h]), __builtin_bit_cast(bf16x8_t, pt[c][i]), acc, 0, 0, 0);
        }
      }
  };
  block(std::integral_constant<int, 0>{});
  block(std::integral_constant<int, 1>{});
  if constexpr (D == 128) {
    block(std::integral_constant<int, 2>{});
    block(std::integral_constant<int, 3>{});
  }
}

// The same (in bf16) for a unit of which some columns see a part: a NaN block of
// V reaches the columns that see its key, and no other (a weight of 0 times NaN
// would be NaN; its codes are 0 already).  Its scale becomes 1, and the columns that see the first such key
// of a block get NaN outright.  (Keys that no column sees are cleared.)
template <typename T, int D, int NB, bool C>
__device__ __forceinline__ void fold_pv_edge(State<T, D, NB, C>& st, Unit<D>& u, const float (&x)[NB][8], int key0, int lane) {
  constexpr int n = D / 32;
  int nan_key[n];
  bool any = false;
#pragma unroll
  for (int j = 0; j < n; ++j) nan_key[j] = INT32_MAX;
#pragma unroll
  for (int p = 1; p >= 0; --p)
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      uint32_t& w = u.vs[p][n == 4 ? i : i >> 1];
#pragma unroll
      for (int j = 0; j < n; ++j) {
        const uint32_t byte = 0xffu << ((n == 4 ? 0 : (i & 1) * 16) + 8 * j);
        if ((w & byte) == byte) {
          w ^= byte & 0x80808080u;  // (255 becomes 127, the scale 1)
          nan_key[j] = key0 + 16 * p + 4 * (lane >> 4) + i;
          any = true;
        }
      }
    }
  const bool nans = __builtin_amdgcn_ballot_w64(any) != 0;
  fold_pv<false>(st, u, x);
  if (nans) {
#pragma unroll
    for (int j = 0; j < n; ++j) {
      int k = nan_key[j];
      k = min(k, __shfl_xor(k, 16));
      k = min(k, __shfl_xor(k, 32));
#pragma unroll
      for (int c = 0; c < NB; ++c)
        if (st.last[c] >= k) st.acc[c][2 * j] = st.acc[c][2 * j + 1] = f32x4_t{NAN, NAN, NAN, NAN};
    }
  }
}

// What the kernels ask of a format.
struct Format {
  template <int D> using Unit = q4::Unit<D>;
  template <typename T, int D> static constexpr bool kCodes = kCodeScores<T, D>;
  template <typename T> static constexpr bool kWide = false;  // waves of 32 columns too
  static constexpr bool kSliced = false;  // K operands in bf16: a lane's dims in a row
  static constexpr bool kSums = false;  // a base moves by sums of weights
  static constexpr int tile_bytes(int D) { return q4_tile_bytes(D); }

  static __device__ __forceinline__ const uint8_t* scales_of_head(const uint8_t*, int) { return nullptr; }  // (in the tile)

  // Page p of a unit from the tile `at` bytes into the pool.
  template <int Policy, int D>
  static __device__ __forceinline__ void load_k(Unit<D>& u, int p, const uint8_t* pool, int64_t at, const uint8_t*, int bytes, int lane) {
    q4::load_k<D, Policy>(u, p, pool + at, bytes, lane);
  }
  template <int Policy, int D>
  static __device__ __forceinline__ void load_v(Unit<D>& u, int p, const uint8_t* pool, int64_t at, const uint8_t*, int bytes, int lane) {
    q4::load_v<D, Policy>(u, p, pool + at, bytes, lane);
  }
  // Whether K's loads bring what V is multiplied by: keep_scales, before K is loaded again.
  template <int D> static __device__ __forceinline__ void keep_scales(Unit<D>&) {}
  template <int D> static __device__ __forceinline__ int shift(int lane) { return k_shift<D>(lane); }
  // Whether the unit's V takes other products than the usual ones, as this lane sees it.
  template <bool F16, int D>
  static __device__ __forceinline__ bool odd(const Unit<D>& u) {
    return F16 ? beyond_fp16<D>(u) : q4::has_large<D>(u);
  }
  template <int D> static __device__ __forceinline__ bool has_large(const Unit<D>& u) { return q4::has_large(u); }
  template <int D>
  static __device__ __forceinline__ int first_large(const Unit<D>& u, int key0, int lane) { return q4::first_large(u, key0, lane); }
  template <int D>
  static __device__ __forceinline__ void clear_dead(Unit<D>& u, int key0, int all_last, int lane) { q4::clear_dead(u, key0, all_last, lane); }
  template <typename T, int D, int NB, bool C>
  static __device__ __forceinline__ void fold_qk(const State<T, D, NB, C>& st, const Unit<D>& u, int shift, f32x4_t (&s)[NB][2]) {
    q4::fold_qk(st, u, shift, s);
  }
  template <bool F16, typename T, int D, int NB, bool C>
  static __device__ __forceinline__ void fold_pv(State<T, D, NB, C>& st, const Unit<D>& u, const float (&x)[NB][8]) {
    q4::fold_pv<F16>(st, u, x);
  }
  template <typename T, int D, int NB, bool C>
  static __device__ __forceinline__ void fold_pv_edge(State<T, D, NB, C>& st, Unit<D>& u, const float (&x)[NB][8], int key0, int lane) {
    q4::fold_pv_edge(st, u, x, key0, lane);
  }
};

}  // namespace q4
}  // namespace pa
