// Chunk rows over the caches held in few bits for gfx950, many columns: bf16 queries.
// (Included after the format, as pa_q_attn.h.)
//
// As pa_q4_attn.hip, with V's operands shared: the four waves of a workgroup hold
// 128 columns (query row, head of the group) of one sequence and KV head, 32 each,
// and step through the units together.  Turning a unit's V codes into fp16 operands
// takes 96 vector instructions, nearly as many as the softmax and the rest of a wave's
// unit together (some 110), so each wave converts a quarter (one page, half of the
// blocks) and stages it in LDS, 8 KiB per unit at head_dim 128 and read back as whole operands
// with no bank conflict; K's codes are operands already (head_dim 128) and every
// wave loads its own, out of the L1 after the first.  One barrier per unit: unit k is
// multiplied while unit k + 1 is converted into the other buffer.
//
// A unit with a scale outside fp16's window, or that holds a NaN block, is flagged by
// the wave that converts it, and every wave takes it by the general products instead,
// with V of its own; so does a wave all units after one with large V.
#pragma once

#include "pa_q_attn.h"

namespace pa {

constexpr int kQChunkNB = 2;                               // column blocks of a wave
constexpr int kQChunkColumns = 16 * kQChunkNB * kQWaves;  // of a workgroup

template <class F, int D>
__global__ __launch_bounds__(64 * kQWaves) __attribute__((amdgpu_waves_per_eu(2)))
void q_chunk_kernel(QAttnArgs a) {
  using T = uint16_t;
  constexpr int kNB = kQChunkNB;
  // V operands of block j, half h (even or odd dims), page p: 8 bytes per lane
  __shared__ __attribute__((aligned(16))) u32x2_t s_v[2][D / 32][2][2][64];
  __shared__ int32_t s_odd[2][kQWaves];
  __shared__ typename F::template SharedK<D> s_k[2];
  const int S = a.s;
  const int lane = threadIdx.x & 63, n = lane & 15, G = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % a.n_split, g = blockIdx.x / a.n_split % a.H_kv;
  const QItem it = q_item(a, blockIdx.x / a.n_split / a.H_kv, kQChunkColumns / S, lane);
  if (it.n_pos == 0) return;
  T* out = reinterpret_cast<T*>(a.out);
  if (it.bad) {
    if (split == 0)
      for (int i = threadIdx.x; i < it.n_pos * S * D; i += 64 * kQWaves)
        store_out<T>(out + ((int64_t)(it.row0 + i / (S * D)) * a.H_q + (int64_t)g * S) * D + i % (S * D), NAN);
    return;
  }
  const int all_last = it.last0 + it.n_pos - 1;
  const int u0 = split * a.split_units, u1 = min(all_last / kQUnit + 1, u0 + a.split_units);
  if (u0 >= u1) return;

  // the wave's columns, and the keys that its first and its last one see
  q::State<T, D, kNB> st;
  int64_t at[kNB];
#pragma unroll
  for (int c = 0; c < kNB; ++c) {
    const int col = 16 * (kNB * w + c) + n, pos = col / S;
    const bool there = pos < it.n_pos;
    st.last[c] = there ? it.last0 + pos : -1;
    at[c] = (int64_t)(it.row0 + (there ? pos : 0)) * a.H_q + (int64_t)g * S + col % S;
    q::load_query<F::kSliced, T, D>(st.q[c], there ? reinterpret_cast<const T*>(a.q) + at[c] * D : nullptr, lane);
  }
  q::reset(st);
  const int pos0 = 16 * kNB * w / S, pos1 = min(it.n_pos - 1, (16 * kNB * (w + 1) - 1) / S);
  const int first_last = it.last0 + pos0, wave_last = it.last0 + pos1;
  const int w1 = pos0 < it.n_pos ? min(u1, wave_last / kQUnit + 1) : u0;  // the units that the wave multiplies: u0 .. w1 - 1

  const int edge = (it.last0 + 1) / kQUnit;  // units before are seen whole by every column
  const int n_pages = all_last / kPage + 1;
  const int64_t tile = F::tile_bytes(D), page_bytes = tile * a.H_kv;
  const int tile_size = a.num_pages > 0 ? F::tile_bytes(D) : 0;
  const uint8_t* kg = a.k_pages + g * tile;
  const uint8_t* vg = a.v_pages + g * tile;
  const uint8_t* sg = F::scales_of_head(a.scales, g);
  const int32_t* table = a.block_table + (int64_t)it.b * a.bt_stride;
  // lane i: entries of page 64 (k / 32) + i of the present unit k and of the 64 after
  auto entries = [&](int k) {
    const int p = (k >> 5) * 64 + lane;
    return p < n_pages ? table[p] : 0;
  };
  int ids = entries(u0), ids_after = entries(u0 + 32);
  struct Pages {
    int64_t at[2];
    int bad;  // bit p: page p's entry lies outside the pool
  };
  auto pages = [&](int k) {  // (wave-uniform; k goes up by one from call to call)
    if ((k & 31) == 0 && k != u0) {
      ids = ids_after;
      ids_after = entries(k + 32);
    }
    Pages t{{0, 0}, 0};
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int id = __builtin_amdgcn_readlane(ids, (2 * k + p) & 63);
      const bool ok = id >= 0 && id < a.num_pages;
      t.at[p] = ok ? id * page_bytes : 0;
      t.bad |= (ok ? 0 : 1) << p;
    }
    return t;
  };
  // (chosen between as values: of addresses, the pages would move to memory)
  auto at_of = [](const Pages& t, int p) {
    const int64_t a = t.at[0], b = t.at[1];
    return p == 0 ? +a : +b;
  };
  // This wave's part of a unit's V: page w % 2, blocks jb .. jb + D / 64 - 1.
  const int vp = w & 1, jb = (w >> 1) * (D / 64);
  typename F::template Part<D> part;
  auto fetch_part = [&](const Pages& t, bool any) {
    F::load_part(part, vg, at_of(t, vp), sg, jb, any ? tile_size : 0, lane);
  };
  auto convert = [&](int k) {
    const int buf = k & 1;
    F::convert_part(part, jb, k * kQUnit + 16 * vp + 4 * G, all_last, k >= edge, lane,
                    [&](bool odd) {
                      const bool any_odd = __builtin_amdgcn_ballot_w64(odd) != 0;
                      if (lane == 0) s_odd[buf][w] = any_odd;
                    },
                    [&](int b, u32x2_t even, u32x2_t odd_dims) {
                      s_v[buf][jb + b][0][vp][lane] = even;
                      s_v[buf][jb + b][1][vp][lane] = odd_dims;
                    });
  };
  typename F::template Unit<D> u;  // K of the unit; V only of a flagged one
  // K of a unit: into each wave's registers, or (kSharedK) a part of it, which the wave
  // puts into LDS for all.
  typename F::template KPart<D> kpart;
  auto fetch_k = [&](const Pages& t, bool any) {
    if constexpr (F::kSharedK) {
      F::load_k_part(kpart, w, kg, at_of(t, w & 1), sg, any ? tile_size : 0, lane);
    } else {
#pragma unroll
      for (int p = 0; p < 2; ++p) F::load_k_shared(u, p, kg, t.at[p], sg, any ? tile_size : 0, lane);
    }
  };
  auto put_k = [&](int k) {
    if constexpr (F::kSharedK) F::put_k_part(s_k[k & 1], kpart, w, lane);
  };
  auto scores = [&](int k, q::f32x4_t (&x)[kNB][2]) {
    if constexpr (F::kSharedK) F::take_k(s_k[k & 1], u, lane);
    F::fold_qk(st, u, 0, x);
  };
  auto load_scales = [&](typename F::template Unit<D>& whole, const Pages& t) {  // V's, of a unit
#pragma unroll
    for (int p = 0; p < 2; ++p) F::load_scales(whole, p, vg, t.at[p], sg, tile_size, lane);
  };
  auto flagged = [&](int k) {
    const int32_t* f = s_odd[k & 1];
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

  // Pipeline: when unit k starts, its scores are formed, K of k + 1 and the part of V
  // of k + 1 are on their way, and V of k is staged (after the barrier).  A unit forms
  // the next one's scores beside its own weights, and converts the next one's V
  // beside its own PV products, so the matrix cores and the vector unit work side
  // by side within a wave.  K that goes through LDS is a unit further ahead: that of k + 1
  // is there when unit k starts, and the part of k + 2 on its way.
  Pages t = pages(u0), t1 = t, t2 = t, t3 = t;
  q::f32x4_t s[kNB][2], sn[kNB][2];
  fetch_k(t, true);
  fetch_part(t, true);
  if (u0 + 1 < u1) t1 = t2 = t3 = pages(u0 + 1);
  if constexpr (F::kSharedK) {
    put_k(u0);
    fetch_k(t1, u0 + 1 < u1);
    if (u0 + 2 < u1) t2 = t3 = pages(u0 + 2);
    put_k(u0 + 1);
    __syncthreads();
    scores(u0, s);
    fetch_k(t2, u0 + 2 < u1);
  } else {
    scores(u0, s);
    fetch_k(t1, u0 + 1 < w1);
  }
  convert(u0);
  fetch_part(t1, u0 + 1 < u1);
  // the pages of the units after k, when unit k starts
  auto look_ahead = [&](int k) {
    if constexpr (F::kSharedK) t3 = k + 3 < u1 ? pages(k + 3) : t2;
    else t2 = k + 2 < u1 ? pages(k + 2) : t1;
  };
  auto move_on = [&]() {
    t = t1;
    t1 = t2;
    if constexpr (F::kSharedK) t2 = t3;
  };
  const int plain = min(w1, (first_last + 1) / kQUnit);  // units before are seen whole by the wave's columns
  for (int k = u0; k < u1;) {
    float x[kNB][8];
    bool entered = false;
#pragma unroll 1
    for (; k < plain && t.bad == 0 && !st.any_lifted; ++k) {  // (nothing but the usual unit, so that the sums stay in place)
      __syncthreads();  // unit k is staged, and unit k - 1 is done with
      if (flagged(k)) {
        entered = true;
        break;
      }
      look_ahead(k);
      scores(k + 1, sn);
      const bool big = q::form_weights<T, D, kNB>(st, s, a.scale_log2, x);
      if constexpr (!F::kSharedK) fetch_k(t2, k + 2 < w1);
      q::settle_weights<false, T, D, kNB>(st, s, a.scale_log2, big, x);
      convert(k + 1);
      put_k(k + 2);
      fold_staged(k, x);
      fetch_part(t2, k + 2 < u1);
      if constexpr (F::kSharedK) fetch_k(t3, k + 3 < u1);
#pragma unroll
      for (int c = 0; c < kNB; ++c)
#pragma unroll
        for (int p = 0; p < 2; ++p) s[c][p] = sn[c][p];
      move_on();
    }
    if (k >= u1) break;
    if (!entered) __syncthreads();
    const bool active = k < w1;
    look_ahead(k);
    if (k + 1 < w1) scores(k + 1, sn);
    if constexpr (!F::kSharedK) fetch_k(t2, k + 2 < w1);
    if (active) {
      q::mask_scores<T, D, kNB>(st, k * kQUnit, t.bad, lane, s);
      const bool odd = flagged(k);
      int first = INT32_MAX;
      if (__builtin_expect(odd, 0)) {  // (the scales alone: all of V would hold registers meanwhile)
        typename F::template Unit<D> whole;
        load_scales(whole, t);
        F::clear_dead(whole, k * kQUnit, all_last, lane);
        first = F::first_large(whole, k * kQUnit, lane);
      }
      const bool big = q::form_weights<T, D, kNB>(st, s, a.scale_log2, x);
      q::settle_weights<true, T, D, kNB>(st, s, a.scale_log2, big, x, first);
      if (__builtin_expect(odd | st.any_lifted, 0)) {
        typename F::template Unit<D> whole;
#pragma unroll
        for (int p = 0; p < 2; ++p) F::load_v_whole(whole, p, vg, t.at[p], sg, tile_size, lane);
        F::clear_dead(whole, k * kQUnit, all_last, lane);
        F::fold_pv_edge(st, whole, x, k * kQUnit, lane);
      } else {
        fold_staged(k, x);
      }
    }
    if (k + 1 < u1) convert(k + 1);
    if (k + 2 < u1) put_k(k + 2);
    fetch_part(t2, k + 2 < u1);
    if constexpr (F::kSharedK) fetch_k(t3, k + 3 < u1);
    if (k + 1 < w1) {
#pragma unroll
      for (int c = 0; c < kNB; ++c)
#pragma unroll
        for (int p = 0; p < 2; ++p) s[c][p] = sn[c][p];
    }
    move_on();
    ++k;
  }
  q_finish<T, D, kNB>(a, st, at, split, lane);
}

template <class F>
hipError_t launch_q_chunk(int D, const QAttnArgs& a, hipStream_t st, KernelEvents ev) {
  const void* fn = D == 128 ? reinterpret_cast<const void*>(&q_chunk_kernel<F, 128>) : reinterpret_cast<const void*>(&q_chunk_kernel<F, 64>);
  void* args[] = {const_cast<QAttnArgs*>(&a)};
  hipError_t e = hipExtLaunchKernel(fn, dim3((uint32_t)((int64_t)a.n_slots * a.H_kv * a.n_split)), dim3(64 * kQWaves), args, 0, st,
                                    ev.start, ev.stop, 0);
  return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace pa
