// Device helpers of the 4-bit cache (format in pagedattn_q4.h): the lookup of a
// row's sequence and place, a wave's share of two pages, its values as
// matrix-core operands, and the fold of 32 tokens into a wave's softmax state.
#pragma once

#include "pa_device.h"
#include "pa_q4.h"
#include "pa_tile.h"

namespace pa {
namespace q4 {

using mfma::bf16x8_t;
using mfma::f32x4_t;
typedef float f32x2_t __attribute__((ext_vector_type(2)));

template <int D> constexpr int kWords = D / 32;  // 4-byte words of codes of a lane and page, and scales of a token
template <int D> constexpr int kScales = 8 * D;  // offset of a tile's scales

// The largest b < n with key(b) <= x, key not decreasing and key(0) <= x: the
// wave looks at 64 places at a time.  (All lanes active.)
template <typename Key>
__device__ __forceinline__ int wave_search(int n, int x, int lane, Key key) {
  int lo = 0;
  while (n > 1) {  // the answer is one of lo .. lo + n - 1
    const int step = (n + 63) >> 6;
    const int at = lane * step;
    const bool below = at < n && key(lo + at) <= x;
    const int i = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(below) | 1);
    lo += i * step;
    n = min(step, n - i * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The value 2^(byte - 127) of byte B of w: the byte as a float's exponent, in one
// instruction (the compiler takes two for three of the four bytes).
template <int B>
__device__ __forceinline__ float scale_of(uint32_t w) {
  uint32_t r;
#define Q4_SCALE_OF(BYTE)                                                                                                 \
  asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:" BYTE : "=v"(r) : "v"(23u), "v"(w))
  if constexpr (B == 0) Q4_SCALE_OF("BYTE_0");
  if constexpr (B == 1) Q4_SCALE_OF("BYTE_1");
  if constexpr (B == 2) Q4_SCALE_OF("BYTE_2");
  if constexpr (B == 3) Q4_SCALE_OF("BYTE_3");
#undef Q4_SCALE_OF
  return __uint_as_float(r);
}

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

// How products are formed.
//
// Scores.  bf16 queries at head_dim 128 meet K's codes as they lie in memory: one
// v_mfma_scale_f32_16x16x128_f8f6f4 takes a token's 128 codes and its four scales,
// so K costs no conversion, and the queries as e4m3 in two parts.  With a column's
// queries scaled so that the largest lies in [128, 256), the first part holds four
// significant bits of a value and the second the four that a bf16 has left, times
// 32: exact for values down to 2^-14 of the column's largest, and within 2^-22 of
// that largest below.  (33 cycles per product against four of 19 for bf16 operands
// and 16 conversions of 4.)  At head_dim 64 half of such a product would be zeros,
// and fp32 queries would take six parts: there K becomes bf16, exactly, and the
// queries their own bits or three bf16 parts, which carry the 24 of an fp32.
//
// Outputs.  For bf16 outputs the weights are rounded once, to fp16 (2^-11 of each, as
// the chunk kernel of the 16-bit cache rounds them), and V becomes fp16, exactly where
// its scales lie in 2^-23 .. 2^8; a unit with another scale takes V as bf16 and the
// weights in two bf16 parts.  For fp32 outputs always bf16, in three parts.
template <typename T, int D> constexpr bool kCodeScores = sizeof(T) == 2 && D == 128;
template <typename T> constexpr int kQParts = sizeof(T) == 2 ? 1 : 3;
template <typename T> constexpr int kPParts = sizeof(T) == 2 ? 2 : 3;
template <typename T> constexpr bool kF16 = sizeof(T) == 2;
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));

// A column's queries: the Q^T operands of its lanes.
template <typename T, int D, bool CODES = kCodeScores<T, D>>
struct Query {
  u32x4 x[D / 32][kQParts<T>];  // of step s: dims D/4 (lane / 16) + 8 s .. +8
};
template <typename T, int D>
struct Query<T, D, true> {
  i32x8_t x[2];   // dims 16 (lane / 16) .. +15, then 64 more
  uint32_t s[2];  // the parts' scale bytes
};

// x as a sum of N bf16 parts, each the rest of those before it to nearest even;
// part i of the eight values as one operand.  LIMIT: the first part is the
// largest bf16 where x, from 3.396e38 on, would round up to an infinity (the parts after
// it carry what is left).
template <int N, bool LIMIT = false>
__device__ __forceinline__ void split8(const float (&x)[8], u32x4 (&part)[N]) {
  typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
  constexpr float kMost = 0x1.fep127f;
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    f32x2_t r = f32x2_t{x[2 * h], x[2 * h + 1]};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      f32x2_t t = r;
      if (LIMIT && i == 0) t = f32x2_t{__builtin_amdgcn_fmed3f(r[0], -kMost, kMost), __builtin_amdgcn_fmed3f(r[1], -kMost, kMost)};
      const bf16x2v_t b = __builtin_convertvector(t, bf16x2v_t);
      if (i + 1 < N) r -= __builtin_convertvector(b, f32x2_t);
      part[i][h] = __builtin_bit_cast(uint32_t, b);
    }
  }
}

// Softmax state of a wave's 16 NB columns: column 16 c + lane % 16 in the lanes of
// equal lane % 16.
template <typename T, int D, int NB>
struct State {
  Query<T, D> q[NB];
  f32x4_t acc[NB][D / 16];          // O^T: block 2 j + h, entry i: dim 32 j + 8 (lane / 16) + 2 i + h
  float m[NB], l[NB];               // base (log2 units, one per column), the lane's part of the sum
  int last[NB];                     // last key that the column sees, -1: no column
  bool lifted[NB];                  // the base is that of large V (kLift)
  bool any_lifted;                  // one of the wave's may be
};

template <typename T, int D, int NB>
__device__ __forceinline__ void reset(State<T, D, NB>& st) {
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    st.m[c] = kMInit;
    st.l[c] = 0.0f;
    st.lifted[c] = false;
#pragma unroll
    for (int mb = 0; mb < D / 16; ++mb) st.acc[c][mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  st.any_lifted = false;
}

// row: the column's D elements (nullptr: zeros).  (All lanes active.)
template <typename T, int D>
__device__ __forceinline__ void load_query(Query<T, D>& q, const T* row, int lane) {
  const int G = lane >> 4;
  if constexpr (kCodeScores<T, D>) {
    uint32_t f[16];
#pragma unroll
    for (int h = 0; h < 4; ++h) {  // 16-byte pieces: two of dims 16 G, two of 64 + 16 G
      const u32x4 w = row != nullptr ? *reinterpret_cast<const u32x4*>(row + h / 2 * 64 + G * 16 + h % 2 * 8) : u32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) f[4 * h + i] = w[i];
    }
    // the column's largest magnitude, as bits (those of infinities and NaN are larger)
    typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
    u16x2_t m2 = {0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2_t, f[i] & 0x7fff7fffu));
    const uint32_t most = __float_as_uint(rows4_max(__uint_as_float((uint32_t)max(m2[0], m2[1]) << 16)));
    const bool odd = rows4_max((uint32_t)max(m2[0], m2[1]) >= 0x7f80u ? 1.0f : 0.0f) != 0.0f;
    // 2^E: the largest over it lies in [128, 256).  The first part may be 256, which at
    // the largest E is 2^128: what it leaves is formed of halves.
    const int byte = min(max((int)(most >> 23) - 7, 7), 250);
    const float sc = __uint_as_float((uint32_t)byte << 23), sc_half = __uint_as_float((uint32_t)(byte - 1) << 23);
    const float sc_lo_half = __uint_as_float((uint32_t)(byte - 6) << 23);
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      typedef short s16x2_t __attribute__((ext_vector_type(2)));
      s16x2_t hi = {0, 0}, lo = {0, 0};
      hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_bit_cast(bf16x2_t, f[2 * w]), sc, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_bit_cast(bf16x2_t, f[2 * w + 1]), sc, true);
      const uint32_t hw = __builtin_bit_cast(uint32_t, hi);
      const f32x2_t ab = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hw, sc_half, false), cd = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hw, sc_half, true);
      lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, fmaf(bf16_lo(f[2 * w]), 0.5f, -ab[0]), fmaf(bf16_hi(f[2 * w]), 0.5f, -ab[1]), sc_lo_half, false);
      lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, fmaf(bf16_lo(f[2 * w + 1]), 0.5f, -cd[0]), fmaf(bf16_hi(f[2 * w + 1]), 0.5f, -cd[1]), sc_lo_half, true);
      q.x[0][w] = odd ? 0 : (int)hw;
      q.x[1][w] = odd ? 0 : __builtin_bit_cast(int, lo);
    }
    // (a query that is infinite or NaN: the scale of NaN, which makes every score NaN)
    q.s[0] = odd ? 255u : (uint32_t)byte;
    q.s[1] = (uint32_t)byte - 5u;
  } else {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      if constexpr (sizeof(T) == 2) {
        q.x[s][0] = row != nullptr ? *reinterpret_cast<const u32x4*>(row + G * (D / 4) + 8 * s) : u32x4{0, 0, 0, 0};
      } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = row != nullptr ? row[G * (D / 4) + 8 * s + e] : 0.0f;
        split8<kQParts<T>, true>(x, q.x[s]);
      }
    }
  }
}

// Fold of the unit of keys key0 .. key0 + 31, in three steps, so that K's registers
// and then V's are free for the next unit's loads as soon as they are read.
//
// Scores S^T[token][column] = K . Q^T, the K operand shared by the columns.  shift: of
// the scale words.
template <typename T, int D, int NB>
__device__ __forceinline__ void fold_qk(const State<T, D, NB>& st, const Unit<D>& u, int shift, f32x4_t (&s)[NB][2]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
#pragma unroll
    for (int c = 0; c < NB; ++c) s[c][p] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if constexpr (kCodeScores<T, D>) {
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

// Scores of a unit that some columns see in part, or of which a page's entry lies
// outside the pool (bit p of bad): those of the latter are NaN, and of keys that a
// column does not see -inf.
template <typename T, int D, int NB>
__device__ __forceinline__ void mask_scores(const State<T, D, NB>& st, int key0, int bad, int lane, f32x4_t (&s)[NB][2]) {
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (bad >> (i >> 2) & 1) s[c][i >> 2][i & 3] = NAN;
      if (key0 + 16 * (i >> 2) + 4 * (lane >> 4) + (i & 3) > st.last[c]) s[c][i >> 2][i & 3] = -INFINITY;
    }
}

// The base of a column's weights is kHeadroom log2 units below its largest score:
// weights lie between 2^7 (the largest so far, when the base moves) and the 2^15
// that moves it again, so that in fp16 all from 2^-21 of the largest on are normal
// numbers, and what is rounded of a smaller one is 2^-32 of the largest at most.
constexpr float kHeadroom = 7.0f;
constexpr float kWeightLimit = 32768.0f;
// From the first key with a V of 2^64 or more on (scale byte kLargeScale), the base of
// the columns that see it lies kLift above instead, and their weights stay below 2^-31:
// 2^30 keys of the largest V, 6 2^125, then sum to less than 2^128.  (Below that size
// sums stay under 2^15 2^30 2^67.)  Weights are bf16 parts there, so a power of two
// costs them nothing; what is lost are products below 2^-126, so V below 2^-78 or so
// beside the large ones.
constexpr float kLift = 39.0f;
constexpr float kLiftedLimit = 0x1p-31f;
constexpr int kLargeScale = 192;

// Online softmax: the weights, formed with the base of the units before; whether
// one exceeds the limit (as a column's first does, whose base is kMInit).
template <typename T, int D, int NB>
__device__ __forceinline__ bool form_weights(const State<T, D, NB>& st, const f32x4_t (&s)[NB][2], float scale_log2, float (&x)[NB][8]) {
  float most = 0.0f;
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[c][i] = fast_exp2(fmaf(s[c][i >> 2][i & 3], scale_log2, -st.m[c]));
      most = fmaxf(most, x[c][i]);
    }
  return most > kWeightLimit;
}
template <typename T, int D, int NB>
__device__ __forceinline__ void add_weights(State<T, D, NB>& st, const float (&x)[NB][8]) {
#pragma unroll
  for (int c = 0; c < NB; ++c)
    st.l[c] += ((x[c][0] + x[c][1]) + (x[c][2] + x[c][3])) + ((x[c][4] + x[c][5]) + (x[c][6] + x[c][7]));
}
// Only where one does the bases of the wave move (so a unit needs no maximum across
// lanes); then the columns' sums.  The inner loops of waves alone leave for this: a
// loop that scales the outputs in one of its branches copies them in the others.
// LIFT: first is the unit's first key with large V (INT32_MAX: none); the bases of the
// columns that see it are lifted.  They lie kHeadroom below the largest score so far, or
// up to 8 log2 units more (the limit), so they come to lie kLift to kLift + 8 above.
template <bool LIFT, typename T, int D, int NB>
__device__ __forceinline__ void settle_weights(State<T, D, NB>& st, const f32x4_t (&s)[NB][2], float scale_log2, bool big,
                                               float (&x)[NB][8], int first = INT32_MAX) {
  float up[NB] = {};
  if constexpr (LIFT) {
    if (__builtin_expect(st.any_lifted | (first != INT32_MAX), 0)) {
      big |= first != INT32_MAX;
#pragma unroll
      for (int c = 0; c < NB; ++c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) big |= st.lifted[c] & (x[c][i] > kLiftedLimit);
        const bool now = (st.last[c] >= first) & !st.lifted[c];
        up[c] = now ? kLift + kHeadroom + 8.0f : 0.0f;
        st.lifted[c] |= now;
      }
      st.any_lifted = true;
    }
  }
  if (__builtin_amdgcn_ballot_w64(big) != 0) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) mx = fmaxf(mx, s[c][i >> 2][i & 3]);
      // (scale > 0, so the largest score is the scaled largest)
      float mc = rows4_max(mx) * scale_log2;
      if constexpr (LIFT) mc = fmaxf(st.m[c] + up[c], mc + (st.lifted[c] ? kLift : -kHeadroom));
      else mc = fmaxf(st.m[c], mc - kHeadroom);
      const float alpha = fast_exp2(st.m[c] - mc);
      st.m[c] = mc;
      st.l[c] *= alpha;
#pragma unroll
      for (int mb = 0; mb < D / 16; ++mb) st.acc[c][mb] *= alpha;
    }
    form_weights<T, D, NB>(st, s, scale_log2, x);
  }
  add_weights(st, x);
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
template <bool F16, typename T, int D, int NB>
__device__ __forceinline__ void fold_pv(State<T, D, NB>& st, const Unit<D>& u, const float (&x)[NB][8]) {
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
template <typename T, int D, int NB>
__device__ __forceinline__ void fold_pv_edge(State<T, D, NB>& st, Unit<D>& u, const float (&x)[NB][8], int key0, int lane) {
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
  fold_pv<false, T, D, NB>(st, u, x);
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

// The lane's eight consecutive outputs of block j (dims 32 j + 8 (lane / 16) ..).
template <typename T, int D, int NB>
__device__ __forceinline__ void eight_out(const State<T, D, NB>& st, int c, int j, float (&o)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = st.acc[c][2 * j][i];
    o[2 * i + 1] = st.acc[c][2 * j + 1][i];
  }
}

// Values to the output's type (bf16 to nearest even, v_cvt_pk_bf16_f32).
typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t to_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2v_t));
}
template <typename T>
__device__ __forceinline__ void store_four(T* p, f32x4_t o) {
  if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2_t*>(p) = u32x2_t{to_bf16(o[0], o[1]), to_bf16(o[2], o[3])};
  else *reinterpret_cast<f32x4_t*>(p) = o;
}
template <typename T>
__device__ __forceinline__ void store_eight(T* p, const float (&o)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x4*>(p) = u32x4{to_bf16(o[0], o[1]), to_bf16(o[2], o[3]), to_bf16(o[4], o[5]), to_bf16(o[6], o[7])};
  } else {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{o[0], o[1], o[2], o[3]};
    *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{o[4], o[5], o[6], o[7]};
  }
}

}  // namespace q4
}  // namespace pa
