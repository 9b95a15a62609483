// Chunk rows over the 8-bit paged cache for gfx950, many columns: bf16 queries.
//
// As pa_q4_attn.hip, with K and V shared: the four waves of a workgroup hold 128 columns
// (query row, head of the group) of one sequence and KV head, 32 each, and step through
// the units together.  Each wave loads a quarter of a unit (of one page): of V it makes fp16
// operands and stages those, 8 KiB per unit at head_dim 128, read back with no bank
// conflict; of K bf16 operands, 8 KiB.  (Measured with K's codes as e4m3 operands, eight
// chunks of 2,048 rows on 0-2,048 tokens: loaded by every wave, K takes 16 registers from its
// load on, too many beside 32 columns' queries and outputs, which then move to scratch
// memory, whose loads wait behind K's, 3,480 us; loaded into LDS directly it takes none, but
// every read of LDS then waits for those loads, 750; through the registers of a quarter,
// 690.)  One barrier per unit: unit k is multiplied while V of unit k + 1 and K of unit
// k + 2 are converted and put into the other buffers.
//
// Those eight chunks take 663 us, 850 TFLOP/s of the causal halves' work, 72 % of the rate
// of a large library product.  A unit takes a wave 158 vector, 32 matrix, 67 scalar and 22
// LDS instructions, which two waves of a SIMD overlap little: vector instructions are being
// issued 47 % of the time, the matrix cores are busy 34 %.  (At 690, with e4m3 operands, the
// barrier was 5 % of it, loads and conversions 15, the scores 14.)  Fixed orders of issue
// (sched_group_barrier: products between so many vector instructions each) take 697 to 734.
//
// A unit with a V scale outside fp16's window every wave takes by the general products
// instead, with V of its own; also one with a NaN among keys that some columns do not see
// (flagged by the waves that convert it), and a wave all units after one with large V.
#include "pa_q8_tile.h"
#include "pa_q_attn.h"

namespace pa {
namespace {

constexpr int kChunkNB = 2;                        // column blocks of a wave
constexpr int kColumns = 16 * kChunkNB * kQWaves;  // of a workgroup

// K of a unit in LDS.
template <int D>
struct SharedK {
  u32x4 x[2][D / 32][64];  // a page's operands in bf16, one step's after the other's
  uint32_t scale[2];       // the pages' scale bytes
};

// (Three waves a SIMD at head_dim 64: eight chunks of 2,048 rows on 0-2,030 tokens 401 us
// instead of 482 with two.)
template <int D>
__global__ __launch_bounds__(64 * kQWaves) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2)))
void q8_chunk_kernel(QAttnArgs a) {
  using T = uint16_t;
  constexpr int kNB = kChunkNB;
  // V operands of block j, half h (even or odd dims), page p: 8 bytes per lane
  __shared__ __attribute__((aligned(16))) u32x2_t s_v[2][D / 32][2][2][64];
  __shared__ int32_t s_nan[2][kQWaves];
  __shared__ SharedK<D> s_k[2];
  const int S = a.s;
  const int lane = threadIdx.x & 63, n = lane & 15, G = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % a.n_split, g = blockIdx.x / a.n_split % a.H_kv;
  const QItem it = q_item(a, blockIdx.x / a.n_split / a.H_kv, kColumns / S, lane);
  if (it.n_pos == 0) return;
  T* out = reinterpret_cast<T*>(a.out);
  if (it.bad) {  // (also where there are no pages)
    if (split == 0)
      for (int i = threadIdx.x; i < it.n_pos * S * D; i += 64 * kQWaves)
        store_out<T>(out + ((int64_t)(it.row0 + i / (S * D)) * a.H_q + (int64_t)g * S) * D + i % (S * D), NAN);
    return;
  }
  const int all_last = it.last0 + it.n_pos - 1;
  const int u0 = split * a.split_units, u1 = min(all_last / kQUnit + 1, u0 + a.split_units);
  if (u0 >= u1) return;

  // the wave's columns, and the keys that its first and its last one see
  q::State<T, D, kNB, false> st;
  int64_t at[kNB];
#pragma unroll
  for (int c = 0; c < kNB; ++c) {
    const int col = 16 * (kNB * w + c) + n, pos = col / S;
    const bool there = pos < it.n_pos;
    st.last[c] = there ? it.last0 + pos : -1;
    at[c] = (int64_t)(it.row0 + (there ? pos : 0)) * a.H_q + (int64_t)g * S + col % S;
    q::load_query<true>(st.q[c], there ? reinterpret_cast<const T*>(a.q) + at[c] * D : nullptr, lane);
  }
  q::reset(st);
  const int pos0 = 16 * kNB * w / S, pos1 = min(it.n_pos - 1, (16 * kNB * (w + 1) - 1) / S);
  const int first_last = it.last0 + pos0, wave_last = it.last0 + pos1;
  const int w1 = pos0 < it.n_pos ? min(u1, wave_last / kQUnit + 1) : u0;  // the units that the wave multiplies: u0 .. w1 - 1

  const int edge = (it.last0 + 1) / kQUnit;  // units before are seen whole by every column
  const int n_pages = all_last / kPage + 1;
  const int64_t page_bytes = (int64_t)q8_tile_bytes(D) * a.H_kv;
  const uint8_t* kg = a.k_pages + g * q8_tile_bytes(D);
  const uint8_t* vg = a.v_pages + g * q8_tile_bytes(D);
  const uint8_t* sg = a.scales + 2 * g;
  const int32_t* table = a.block_table + (int64_t)it.b * a.bt_stride;
  // lane i: entries of page 64 (k / 32) + i of the present unit k and of the 64 after
  auto entries = [&](int k) {
    const int p = (k >> 5) * 64 + lane;
    return p < n_pages ? table[p] : 0;
  };
  auto known = [&](int id) { return id >= 0 && id < a.num_pages ? id : -1; };  // (-1: outside the pool)
  int ids = known(entries(u0)), ids_after = entries(u0 + 32);
  struct Pages {
    int a, b, own;  // of the unit; the one of which the wave loads a part
  };
  auto pages = [&](int k) {  // (wave-uniform; k goes up by one from call to call)
    if ((k & 31) == 0 && k != u0) {
      ids = known(ids_after);
      ids_after = entries(k + 32);
    }
    const int i = (2 * k) & 63;
    return Pages{__builtin_amdgcn_readlane(ids, i), __builtin_amdgcn_readlane(ids, i + 1), __builtin_amdgcn_readlane(ids, i + (w & 1))};
  };
  auto at_of = [&](int id) { return max(id, 0) * page_bytes; };  // (of the pool's first tile, where the entry lies outside)

  // The wave's parts: page w mod 2, of V blocks jb .. jb + D / 64 - 1, of K as many steps.
  const int vp = w & 1, jb = (w >> 1) * (D / 64);
  uint32_t vc[D / 32], vs;  // V: words of even and odd dims of each block, and the scale bytes
  uint32_t kc[D / 32], ks;  // K: eight codes of each step
  auto fetch_v = [&](const Pages& t) {
    const int64_t at = at_of(t.own);
    vs = q8::scale_bytes<D>(sg, at);
    if constexpr (D == 128) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(vg + at + (jb * 512 + lane * 16));
      vc[0] = x.x; vc[1] = x.y; vc[2] = x.z; vc[3] = x.w;
    } else {
      const u32x2_t x = *reinterpret_cast<const u32x2_t*>(vg + at + (jb * 8 + lane * 16));
      vc[0] = x.x; vc[1] = x.y;
    }
  };
  auto fetch_k = [&](const Pages& t) {
    const int64_t at = at_of(t.own);
    ks = q8::scale_bytes<D>(sg, at);
    if constexpr (D == 128) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(kg + at + (jb * 512 + lane * 16));
      kc[0] = x.x; kc[1] = x.y; kc[2] = x.z; kc[3] = x.w;
    } else {
      const u32x2_t x = *reinterpret_cast<const u32x2_t*>(kg + at + (jb * 8 + lane * 16));
      kc[0] = x.x; kc[1] = x.y;
    }
  };
  auto put_k = [&](int k) {
    SharedK<D>& to = s_k[k & 1];
    const float s = q::scale_of<0>(ks);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) to.x[vp][jb + i][lane] = q8::eight_of(kc[2 * i], kc[2 * i + 1], s);
    if (lane == 0) to.scale[vp] = ks;  // (two waves write the same)
  };
  auto convert = [&](int k) {
    const int buf = k & 1;
    if (k >= edge) {  // (a NaN may be one that some columns do not see)
      const int key0 = k * kQUnit + 16 * vp;
      if (key0 > all_last) vs = q8::kScaleOne;
      const uint32_t live = q8::live_bytes(key0 + 4 * G, all_last);
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) any |= q8::nan_bytes(vc[i] &= live);
      const bool any_lane = __builtin_amdgcn_ballot_w64(any != 0) != 0;
      if (lane == 0) s_nan[buf][w] = any_lane;
    }
    const float s = q::scale_of<1>(vs);
#pragma unroll
    for (int b = 0; b < D / 64; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        s_v[buf][jb + b][h][vp][lane] = u32x2_t{q8::pair_of<0, true>(vc[2 * b + h], s), q8::pair_of<1, true>(vc[2 * b + h], s)};
  };
  // The scores of unit k, and whether fp16 does not hold its V exactly.  (Known a unit
  // ahead from the scales beside K: a flag of the waves that convert V would be read
  // right after the barrier, 35 us of 687.)
  auto scores = [&](int k, q::f32x4_t (&x)[kNB][2]) -> uint32_t {  // (the same in all lanes)
    const SharedK<D>& from = s_k[k & 1];
    const uint32_t ks0 = from.scale[0], ks1 = from.scale[1];
#pragma unroll
    for (int c = 0; c < kNB; ++c)
#pragma unroll
      for (int p = 0; p < 2; ++p) x[c][p] = q::f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const q::bf16x8_t ka = __builtin_bit_cast(q::bf16x8_t, from.x[p][i][lane]);
#pragma unroll
        for (int c = 0; c < kNB; ++c)
          x[c][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, __builtin_bit_cast(q::bf16x8_t, st.q[c].x[i][0]), x[c][p], 0, 0, 0);
      }
    // (a page past the item's last key may be any)
    const uint32_t second = k * kQUnit + kPage <= all_last ? 1u : 0u;
    return (uint32_t)q8::beyond_fp16(ks0) | ((uint32_t)q8::beyond_fp16(ks1) & second);
  };
  auto has_nan = [&](int k) {  // (k >= edge)
    const int32_t* f = s_nan[k & 1];
    return __builtin_amdgcn_readfirstlane(f[0] | f[1] | f[2] | f[3]) != 0;
  };
  auto fold_staged = [&](int k, const float (&x)[kNB][8]) {
    u32x4 pt[kNB];
#pragma unroll
    for (int c = 0; c < kNB; ++c)
#pragma unroll
      for (int h = 0; h < 4; ++h)
        pt[c][h] = __builtin_bit_cast(uint32_t, __builtin_convertvector((q::f32x2_t{x[c][2 * h], x[c][2 * h + 1]}), q::f16x2_t));
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x2_t lo = s_v[k & 1][j][h][0][lane], hi = s_v[k & 1][j][h][1][lane];
        const q::f16x8_t va = __builtin_bit_cast(q::f16x8_t, u32x4{lo.x, lo.y, hi.x, hi.y});
#pragma unroll
        for (int c = 0; c < kNB; ++c)
          st.acc[c][2 * j + h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, __builtin_bit_cast(q::f16x8_t, pt[c]), st.acc[c][2 * j + h], 0, 0, 0);
      }
  };

  // Pipeline: when unit k starts (after the barrier), its scores are formed, V of k and K
  // of k + 1 are in LDS, and the parts of V of k + 1 and of K of k + 2 on their way.  A unit
  // forms the next one's scores beside its own weights, and converts the next one's V
  // beside its own PV products, so the matrix cores and the vector unit work side
  // by side within a wave.  (Loads of units past the item's are of its last one again.)
  Pages t = pages(u0), t1 = t, t2 = t, t3 = t;  // of units k .. k + 3
  q::f32x4_t s[kNB][2], sn[kNB][2];
  fetch_k(t);
  fetch_v(t);
  if (u0 + 1 < u1) t1 = t2 = t3 = pages(u0 + 1);
  put_k(u0);
  fetch_k(t1);
  if (u0 + 2 < u1) t2 = t3 = pages(u0 + 2);
  put_k(u0 + 1);
  __syncthreads();
  bool odd = __builtin_amdgcn_readfirstlane(scores(u0, s)) != 0;  // V of unit k takes other products
  fetch_k(t2);
  convert(u0);
  fetch_v(t1);
  const int plain = min(w1, (first_last + 1) / kQUnit);  // units before are seen whole by the wave's columns
  for (int k = u0; k < u1;) {
    float x[kNB][8], sum[kNB];
#pragma unroll 1
    for (; k < plain && (t.a | t.b) >= 0 && !odd && !st.any_lifted; ++k) {  // (nothing but the usual unit, so that the sums stay in place)
      __syncthreads();  // unit k is staged, and unit k - 1 is done with
      if (k + 3 < u1) t3 = pages(k + 3);
      const uint32_t odd_next = scores(k + 1, sn);
      const bool big = q::form_weights<true>(st, s, a.scale_log2, x, sum);
      // (the next unit's scores are formed here, between the weights, and not behind the
      // branch where the base moves: used only then, they would sink to the loop's end)
#pragma unroll
      for (int c = 0; c < kNB; ++c)
#pragma unroll
        for (int p = 0; p < 2; ++p) asm volatile("" : "+v"(sn[c][p]));
      q::settle_weights<false, true>(st, s, a.scale_log2, big, x, sum);
      convert(k + 1);
      fetch_v(t2);
      put_k(k + 2);
      fetch_k(t3);
      fold_staged(k, x);
#pragma unroll
      for (int c = 0; c < kNB; ++c)
#pragma unroll
        for (int p = 0; p < 2; ++p) s[c][p] = sn[c][p];
      odd = __builtin_amdgcn_readfirstlane(odd_next) != 0;
      t = t1;
      t1 = t2;
      t2 = t3;
    }
    if (k >= u1) break;
    __syncthreads();
    if (k + 3 < u1) t3 = pages(k + 3);
    uint32_t odd_next = 0;
    if (k + 1 < w1) odd_next = scores(k + 1, sn);
    if (k < w1) {
      q::mask_scores<T, D, kNB>(st, k * kQUnit, (t.a < 0 ? 1 : 0) | (t.b < 0 ? 2 : 0), lane, s);
      q8::Unit<D> whole;
      int first = INT32_MAX;
      if (__builtin_expect(odd, 0)) {  // (the scales alone: all of V would hold registers meanwhile)
        whole.vs[0] = q8::scale_bytes<D>(sg, at_of(t.a));
        whole.vs[1] = k * kQUnit + kPage > all_last ? q8::kScaleOne : q8::scale_bytes<D>(sg, at_of(t.b));
        first = q8::Format::first_large(whole, k * kQUnit, lane);
      }
      const bool big = q::form_weights<true>(st, s, a.scale_log2, x, sum);
      q::settle_weights<true, true>(st, s, a.scale_log2, big, x, sum, first);
      if (__builtin_expect(odd || st.any_lifted || (k >= edge && has_nan(k)), 0)) {
        q8::load_words<D, 0>(q8::tile_at(vg + at_of(t.a), q8_tile_bytes(D)), lane, whole.v[0]);
        q8::load_words<D, 0>(q8::tile_at(vg + at_of(t.b), q8_tile_bytes(D)), lane, whole.v[1]);
        whole.vs[0] = q8::scale_bytes<D>(sg, at_of(t.a));
        whole.vs[1] = q8::scale_bytes<D>(sg, at_of(t.b));
        q8::clear_dead(whole, k * kQUnit, all_last, lane);
        q8::fold_pv_edge(st, whole, x, k * kQUnit, lane);
      } else {
        fold_staged(k, x);
      }
    }
    if (k + 1 < u1) convert(k + 1);
    put_k(k + 2);
    fetch_v(t2);
    fetch_k(t3);
    if (k + 1 < w1) {
#pragma unroll
      for (int c = 0; c < kNB; ++c)
#pragma unroll
        for (int p = 0; p < 2; ++p) s[c][p] = sn[c][p];
    }
    odd = __builtin_amdgcn_readfirstlane(odd_next) != 0;
    t = t1;
    t1 = t2;
    t2 = t3;
    ++k;
  }
  q_finish<T, D, kNB>(a, st, at, split, lane);
}

}  // namespace

template <>
hipError_t launch_q_chunk<q8::Format>(int D, const QAttnArgs& a, hipStream_t st, KernelEvents ev) {
  const void* fn = D == 128 ? reinterpret_cast<const void*>(&q8_chunk_kernel<128>) : reinterpret_cast<const void*>(&q8_chunk_kernel<64>);
  void* args[] = {const_cast<QAttnArgs*>(&a)};
  hipError_t e = hipExtLaunchKernel(fn, dim3((uint32_t)((int64_t)a.n_slots * a.H_kv * a.n_split)), dim3(64 * kQWaves), args, 0, st,
                                    ev.start, ev.stop, 0);
  return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace pa
