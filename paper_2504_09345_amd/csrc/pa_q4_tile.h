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

// The value 2^(byte - 127) of byte B of w.
template <int B>
__device__ __forceinline__ float scale_of(uint32_t w) {
  return __uint_as_float(((w >> (8 * B)) & 0xffu) << 23);
}

// Byte B of w (two codes) times scale, as two bf16: exact for scale bytes 0 ..
// 252, NaN for 255 (v_cvt_scalef32_pk_bf16_fp4).
template <int B>
__device__ __forceinline__ uint32_t pair_of(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}
__device__ __forceinline__ u32x4 eight_of(uint32_t w, float scale) {
  return u32x4{pair_of<0>(w, scale), pair_of<1>(w, scale), pair_of<2>(w, scale), pair_of<3>(w, scale)};
}

// A lane's part of a unit (two pages of one KV head).
template <int D>
struct Unit {
  uint32_t k[2][kWords<D>];  // codes of token lane % 16, dims D/4 (lane / 16) .. +D/4
  uint32_t ks[2];            // scale byte of those dims
  uint32_t v[2][kWords<D>];  // word j: tokens 4 (lane / 16) .. +3, dims 32 j + 2 (lane % 16), +1
  uint32_t vs[2][kWords<D>];  // scales of those four tokens, token-major
};

template <int D>
__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t r, int off, uint32_t (&x)[kWords<D>]) {
  if constexpr (D == 128) {
    const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, kKvLoadPolicy);
    x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
  } else {
    const u32x2_t w = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, kKvLoadPolicy);
    x[0] = w.x; x[1] = w.y;
  }
}
// Loads of page p (0 or 1) of a unit from the tiles at k and v; where !there,
// nothing is read and every code and scale is 0.
template <int D>
__device__ __forceinline__ void load_k(Unit<D>& u, int p, const uint8_t* k, bool there, int lane) {
  const __amdgpu_buffer_rsrc_t r =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(k), (short)0, there ? q4_tile_bytes(D) : 0, 0x00020000);
  load_words<D>(r, lane * (D / 8), u.k[p]);
  u.ks[p] = __builtin_amdgcn_raw_buffer_load_b8(r, kScales<D> + (lane & 15) * (D / 32) + (lane >> 4) * D / 128, 0,
                                                kKvLoadPolicy);
}
template <int D>
__device__ __forceinline__ void load_v(Unit<D>& u, int p, const uint8_t* v, bool there, int lane) {
  const __amdgpu_buffer_rsrc_t r =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(v), (short)0, there ? q4_tile_bytes(D) : 0, 0x00020000);
  load_words<D>(r, lane * (D / 8), u.v[p]);
  load_words<D>(r, kScales<D> + (lane >> 4) * (D / 8), u.vs[p]);
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
template <int D, int J>
__device__ __forceinline__ void v_operands(const Unit<D>& u, u32x4 (&a)[2]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const uint32_t w = u.v[p][J];
    const uint32_t t0 = pair_of<0>(w, v_scale<D, J, 0>(u.vs[p])), t1 = pair_of<1>(w, v_scale<D, J, 1>(u.vs[p]));
    const uint32_t t2 = pair_of<2>(w, v_scale<D, J, 2>(u.vs[p])), t3 = pair_of<3>(w, v_scale<D, J, 3>(u.vs[p]));
    a[0][2 * p] = __builtin_amdgcn_perm(t1, t0, 0x05040100u);
    a[0][2 * p + 1] = __builtin_amdgcn_perm(t3, t2, 0x05040100u);
    a[1][2 * p] = __builtin_amdgcn_perm(t1, t0, 0x07060302u);
    a[1][2 * p + 1] = __builtin_amdgcn_perm(t3, t2, 0x07060302u);
  }
}

// bf16 parts of a query (its type's own bits for bf16, three parts for fp32, which
// carry its 24) and of a softmax weight.
template <typename T> constexpr int kQParts = sizeof(T) == 2 ? 1 : 3;
template <typename T> constexpr int kPParts = sizeof(T) == 2 ? 2 : 3;

// x as a sum of N bf16 parts, each the rest of those before it to nearest even;
// part i of the eight values as one operand.
template <int N>
__device__ __forceinline__ void split8(const float (&x)[8], u32x4 (&part)[N]) {
  typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    f32x2_t r = f32x2_t{x[2 * h], x[2 * h + 1]};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bf16x2v_t b = __builtin_convertvector(r, bf16x2v_t);
      if (i + 1 < N) r -= __builtin_convertvector(b, f32x2_t);
      part[i][h] = __builtin_bit_cast(uint32_t, b);
    }
  }
}

// Softmax state of a wave's 16 NB columns: column 16 c + lane % 16 in the lanes of
// equal lane % 16.
template <typename T, int D, int NB>
struct State {
  u32x4 q[NB][D / 32][kQParts<T>];  // Q^T operand of step s: dims D/4 (lane / 16) + 8 s .. +8
  f32x4_t acc[NB][D / 16];          // O^T: block 2 j + h, entry i: dim 32 j + 8 (lane / 16) + 2 i + h
  float m[NB], l[NB];               // base (log2 units, one per column), the lane's part of the sum
  int last[NB];                     // last key that the column sees, -1: no column
};

template <typename T, int D, int NB>
__device__ __forceinline__ void reset(State<T, D, NB>& st) {
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    st.m[c] = kMInit;
    st.l[c] = 0.0f;
#pragma unroll
    for (int mb = 0; mb < D / 16; ++mb) st.acc[c][mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
}

// A column's queries; row: its D elements (nullptr: zeros).
template <typename T, int D>
__device__ __forceinline__ void load_query(u32x4 (&q)[D / 32][kQParts<T>], const T* row, int lane) {
  const int G = lane >> 4;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    if constexpr (sizeof(T) == 2) {
      q[s][0] = row != nullptr ? *reinterpret_cast<const u32x4*>(row + G * (D / 4) + 8 * s) : u32x4{0, 0, 0, 0};
    } else {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = row != nullptr ? row[G * (D / 4) + 8 * s + e] : 0.0f;
      split8(x, q[s]);
    }
  }
}

// Fold of the unit of keys key0 .. key0 + 31, in three steps, so that K's registers
// and then V's are free for the next unit's loads as soon as they are read.
//
// Scores S^T[token][column] = K . Q^T, the K operand shared by the columns.  bad:
// bit p, page p's entry lies outside the pool (its scores are NaN).
template <typename T, int D, int NB>
__device__ __forceinline__ void fold_qk(const State<T, D, NB>& st, const Unit<D>& u, int bad, f32x4_t (&s)[NB][2]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const float ks = __uint_as_float(u.ks[p] << 23);
#pragma unroll
    for (int c = 0; c < NB; ++c) s[c][p] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
      const bf16x8_t a = __builtin_bit_cast(bf16x8_t, eight_of(u.k[p][w], ks));
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int i = 0; i < kQParts<T>; ++i)
          s[c][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, st.q[c][w][i]), s[c][p], 0, 0, 0);
    }
  }
  if (bad != 0) {
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (bad >> p & 1) s[c][p] = f32x4_t{NAN, NAN, NAN, NAN};
  }
}

// Online softmax; the weights' bf16 parts as P^T operands.  edge (wave-uniform):
// some column does not see every key of the unit.  The base moves only past the
// slack.
template <typename T, int D, int NB>
__device__ __forceinline__ void fold_softmax(State<T, D, NB>& st, const f32x4_t (&s)[NB][2], int key0, bool edge,
                                             float scale_log2, int lane, u32x4 (&pt)[NB][kPParts<T>]) {
  const int G = lane >> 4;
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s[c][i >> 2][i & 3];
    if (edge) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = key0 + 16 * (i >> 2) + 4 * G + (i & 3) <= st.last[c] ? x[i] : -INFINITY;
    }
    // (scale > 0, so the largest score is the scaled largest)
    const float mx = rows4_max(fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])))) *
                     scale_log2;
    const float mc = fmaxf(st.m[c], mx);
    if (__builtin_amdgcn_ballot_w64(mc > st.m[c] + kRescaleSlack) != 0) {
      const float alpha = fast_exp2(st.m[c] - mc);
      st.m[c] = mc;
      st.l[c] *= alpha;
#pragma unroll
      for (int mb = 0; mb < D / 16; ++mb) st.acc[c][mb] *= alpha;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fast_exp2(fmaf(x[i], scale_log2, -st.m[c]));
    st.l[c] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    split8(x, pt[c]);
  }
}

// V of keys past all_last, which no column sees: their weights are 0, but an unused
// slot may hold anything, and 0 times a NaN is NaN.  Their scales become 0.
template <int D>
__device__ __forceinline__ void clear_dead(Unit<D>& u, int key0, int all_last, int lane) {
  constexpr int n = D / 32;
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (key0 + 16 * p + 4 * (lane >> 4) + i > all_last) u.vs[p][n == 4 ? i : i >> 1] &= n == 4 ? 0u : 0xffff0000u >> ((i & 1) * 16);
}

// O^T += V^T . P^T
template <typename T, int D, int NB>
__device__ __forceinline__ void fold_pv(State<T, D, NB>& st, const Unit<D>& u, const u32x4 (&pt)[NB][kPParts<T>]) {
  auto block = [&](auto j_) {
    constexpr int j = decltype(j_)::value;
    u32x4 a[2];
    v_operands<D, j>(u, a);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int i = 0; i < kPParts<T>; ++i)
          st.acc[c][2 * j + h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8_t, a[h]), __builtin_bit_cast(bf16x8_t, pt[c][i]), st.acc[c][2 * j + h], 0, 0, 0);
  };
  block(std::integral_constant<int, 0>{});
  block(std::integral_constant<int, 1>{});
  if constexpr (D == 128) {
    block(std::integral_constant<int, 2>{});
    block(std::integral_constant<int, 3>{});
  }
}

// fold_pv for a unit of which some columns see a part of the keys: a NaN block of
// V reaches the columns that see its key, and no other (a weight of 0 times NaN
// would be NaN).  Its scale becomes 0, and the columns that see the first such key
// of a block get NaN outright.
template <typename T, int D, int NB>
__device__ __forceinline__ void fold_pv_edge(State<T, D, NB>& st, Unit<D>& u, const u32x4 (&pt)[NB][kPParts<T>], int key0,
                                             int all_last, int lane) {
  constexpr int n = D / 32;
  clear_dead(u, key0, all_last, lane);
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
          w &= ~byte;
          nan_key[j] = key0 + 16 * p + 4 * (lane >> 4) + i;
          any = true;
        }
      }
    }
  const bool nans = __builtin_amdgcn_ballot_w64(any) != 0;
  fold_pv<T, D, NB>(st, u, pt);
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

template <typename T>
__device__ __forceinline__ void store_eight(T* p, const float (&o)[8]) {
  if constexpr (sizeof(T) == 2) {
    store_vec(reinterpret_cast<uint16_t*>(p), o);
  } else {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{o[0], o[1], o[2], o[3]};
    *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{o[4], o[5], o[6], o[7]};
  }
}

}  // namespace q4
}  // namespace pa
