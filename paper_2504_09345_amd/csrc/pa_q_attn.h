// The kernel of chunk rows over the caches held in few bits, its picker and launcher
// (design in pa_q4_attn.hip).  Each (format, element type, head dim) is instantiated in
// one translation unit, which includes the format before this file.
#pragma once

#include "pa_q_tile.h"

namespace pa {

// An item's sequence and rows.
struct QItem {
  int b, row0, n_pos;  // sequence, first query row, query rows (0: none)
  int last0;           // last key of the first row
  bool bad;            // rows are NaN
};

// Item `i` of the call: `positions` query rows of a sequence from a multiple of that on.
// One begins, for each row r of the call that is a multiple of `positions`, within the
// `positions` rows from r on in the sequence that has r (the last rows first: of a
// sequence they see the most keys), and then one for each sequence that begins at no
// such r.  (Sequences of one row, the stream kernel's, are thus looked at last and
// without a search: before every other item, 512 of them beside 8 chunks of 512 rows
// cost 10 us.)
__device__ __forceinline__ QItem q_item(const QAttnArgs& a, int i, int positions, int lane) {
  QItem it{0, 0, 0, 0, false};
  const int32_t* qsl = a.query_start_loc;
  const int blocks = (a.rows + positions - 1) / positions;
  int first = 0, q0;
  if (i < blocks) {
    const int r = (blocks - 1 - i) * positions;
    it.b = q::wave_search(a.B, r, lane, [&](int b) { return qsl[b]; });
    q0 = qsl[it.b];
    if (r < q0) return it;
    first = (r - q0 + positions - 1) / positions * positions;
  } else {
    it.b = i - blocks;
    if (it.b >= a.B) return it;
    q0 = qsl[it.b];
    if (q0 % positions == 0) return it;
  }
  const int L = qsl[it.b + 1] - q0;
  it.row0 = q0 + first;
  if (q0 < 0 || it.row0 >= a.rows || L < a.min_rows) return it;  // (fewer rows: the stream kernel's)
  it.n_pos = max(0, min(positions, min(L - first, a.rows - it.row0)));
  const int C = a.context_lens[it.b];
  it.last0 = C - L + first;
  it.bad = C < 0 || C > a.max_context_len || (C + kPage - 1) / kPage > a.bt_stride || L > C || L > a.max_q_len;
  return it;
}

// The outputs of a wave's columns, or the records of part `split` of them; at: the
// column's (row, head) vector among all.
template <typename T, int D, int NB, bool C>
__device__ __forceinline__ void q_finish(const QAttnArgs& a, const q::State<T, D, NB, C>& st, const int64_t (&at)[NB], int split,
                                          int lane) {
  const int G = lane >> 4;
  T* out = reinterpret_cast<T*>(a.out);
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const float l = rows4_sum(st.l[c]);
    if (st.last[c] < 0) continue;
    const float inv = 1.0f / l;
    const int64_t rec = at[c] * a.n_split + split;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      float o[8];
      q::eight_out(st, c, j, o);
      const int d = 32 * j + 8 * G;
      if (a.n_split == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= inv;
        q::store_eight(out + at[c] * D + d, o);
      } else {
        q::store_eight(a.ws_o + rec * D + d, o);
      }
    }
    if (a.n_split > 1 && G == 0) {
      a.ws_ml[rec * 2] = st.m[c];
      a.ws_ml[rec * 2 + 1] = l;
    }
  }
}

// What a wave hands to the one that joins an item's parts.
template <int D, int NB>
struct QPart {
  q::f32x4_t o[NB][D / 16][64];
  float m[NB][64], l[NB][64];
};

// NB: column blocks of the wave.  (Three waves a SIMD: in fp32 at head_dim 128, whose
// registers would hold two, four chunks of 1,024 rows take 130 us instead of 144.  Two
// blocks there leave room for two.)
template <class F, typename T, int D, int NB>
__global__ __launch_bounds__(64 * kQWaves) __attribute__((amdgpu_waves_per_eu(NB == 2 && D == 128 ? 2 : 3)))
void q_attn_kernel(QAttnArgs a) {
  const int S = a.s;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // row blocks of one head side by side
  const int split = blockIdx.x % a.n_split, g = blockIdx.x / a.n_split % a.H_kv;
  // (a workgroup's waves have items of their own, or 2 or 4 share one)
  const int sharers = a.wave_parts, part = wave & (sharers - 1);
  const QItem it = q_item(a, (int)(blockIdx.x / a.n_split / a.H_kv * kQWaves + wave) / sharers, q_positions(NB, S), lane);

  const int n = lane & 15;
  T* out = reinterpret_cast<T*>(a.out);
  const int all_last = it.last0 + it.n_pos - 1;
  if (it.bad && split == 0 && part == 0) {
    for (int i = lane; i < it.n_pos * S * D; i += 64)
      store_out<T>(out + ((int64_t)(it.row0 + i / (S * D)) * a.H_q + (int64_t)g * S) * D + i % (S * D), NAN);
  }
  // units of the item that the workgroup takes, and the wave's of them
  const int n_units = it.n_pos == 0 || it.bad ? 0 : all_last / kQUnit + 1;
  const int s0 = split * a.split_units, s1 = min(n_units, s0 + a.split_units);
  const int per = (max(s1 - s0, 0) + sharers - 1) / sharers;
  const int u0 = s0 + part * per, u1 = min(s1, u0 + per);
  if (u0 >= u1 && sharers == 1) return;

  q::State<T, D, NB, F::template kCodes<T, D>> st;
  int64_t at[NB];  // of the column's (row, head) vector, among all
  q::reset(st);
  if (u0 < u1) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const int col = 16 * c + n, pos = col / S;
      const bool there = pos < it.n_pos;  // (columns past the item's positions are none)
      st.last[c] = there ? it.last0 + pos : -1;
      at[c] = (int64_t)(it.row0 + (there ? pos : 0)) * a.H_q + (int64_t)g * S + col % S;
      q::load_query<F::kSliced>(st.q[c], there ? reinterpret_cast<const T*>(a.q) + at[c] * D : nullptr, lane);
    }

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
    typename F::template Unit<D> u;
    const int k_shift = F::template shift<D>(lane);
    auto fetch_k = [&](const Pages& t, bool any) {
#pragma unroll
      for (int p = 0; p < 2; ++p) F::template load_k<0>(u, p, kg, t.at[p], sg, any ? tile_size : 0, lane);
    };
    auto fetch_v = [&](const Pages& t, bool any) {
#pragma unroll
      for (int p = 0; p < 2; ++p) F::template load_v<0>(u, p, vg, t.at[p], sg, any ? tile_size : 0, lane);
    };
    Pages t = pages(u0);
    fetch_k(t, true);
    __builtin_amdgcn_sched_barrier(0);  // (K before V, as the loop's waits expect)
    fetch_v(t, true);
    constexpr bool kF16 = q::kF16<T>;
    const int u_full = min(u1, (it.last0 + 1) / kQUnit);  // units before are seen whole by every column
    for (int k = u0; k < u1; ++k) {
      q::f32x4_t s[NB][2];
      float x[NB][8], sum[NB];
      Pages next = t;
      bool big = false, odd = false;  // the base moves; V takes other products
      auto weights = [&](bool usual) {  // the weights of unit k, and the next K; whether it is big or odd
        if (k + 1 < u1) next = pages(k + 1);
        F::fold_qk(st, u, k_shift, s);
        F::keep_scales(u);
        fetch_k(next, k + 1 < u1);
        if (!usual) {
          q::mask_scores<T, D, NB>(st, k * kQUnit, t.bad, lane, s);
          F::clear_dead(u, k * kQUnit, all_last, lane);
        }
        big = q::form_weights<F::kSums>(st, s, a.scale_log2, x, sum);
        __builtin_amdgcn_sched_barrier(0);  // (V is not waited for before the weights are formed)
        odd = F::template odd<kF16>(u);
        return __builtin_amdgcn_ballot_w64(big | odd) != 0;
      };
      bool rare = weights(k < u_full && t.bad == 0) | st.any_lifted;
      if (k < u_full) {
        // (one way out, and nothing but the usual unit: the sums stay in place, and the
        // loads under way are known)
#pragma unroll 1
        while (!rare & (k + 1 < u_full) & (next.bad == 0)) {
          q::add_weights<F::kSums>(st, x, sum);
          F::template fold_pv<kF16>(st, u, x);
          fetch_v(next, true);
          t = next;
          ++k;
          rare = weights(true);
        }
      }
      int first = INT32_MAX;
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, 0)) first = F::first_large(u, k * kQUnit, lane);
      q::settle_weights<true, F::kSums>(st, s, a.scale_log2, big, x, sum, first);
      F::fold_pv_edge(st, u, x, k * kQUnit, lane);
      fetch_v(next, k + 1 < u1);
      t = next;
    }
  }
  if (sharers > 1) {  // join the parts that have units: the first one's wave takes the others'
    __shared__ QPart<D, NB> parts[kQWaves];
    if (part > 0 && u0 < u1) {
#pragma unroll
      for (int c = 0; c < NB; ++c) {
#pragma unroll
        for (int j = 0; j < D / 16; ++j) parts[wave].o[c][j][lane] = st.acc[c][j];
        parts[wave].m[c][lane] = st.m[c];
        parts[wave].l[c][lane] = st.l[c];
      }
    }
    __syncthreads();
    if (part > 0 || u0 >= u1) return;
    const int n_parts = (s1 - s0 + per - 1) / per;
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      float M = st.m[c];
      for (int i = 1; i < n_parts; ++i) M = fmaxf(M, parts[wave + i].m[c][lane]);
      const float c0 = fast_exp2(st.m[c] - M);
      st.m[c] = M;
      st.l[c] *= c0;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) st.acc[c][j] *= c0;
      for (int i = 1; i < n_parts; ++i) {
        const auto& other = parts[wave + i];
        const float ci = fast_exp2(other.m[c][lane] - M);
        st.l[c] = fmaf(other.l[c][lane], ci, st.l[c]);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) st.acc[c][j] = other.o[c][j][lane] * ci + st.acc[c][j];
      }
    }
  }
  q_finish<T, D, NB>(a, st, at, split, lane);
}

// Join the parts of one (query row, head) per wave.
template <typename T, int D>
__global__ __launch_bounds__(256) void q_merge_kernel(QAttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int f = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = f / a.H_q;
  if (row >= a.rows) return;
  const int32_t* qsl = a.query_start_loc;
  const int b = q::wave_search(a.B, row, lane, [&](int i) { return qsl[i]; });
  const int L = qsl[b + 1] - qsl[b], j = row - qsl[b];
  if (j < 0 || j >= L || L < a.min_rows || L > a.max_q_len) return;
  const int C = a.context_lens[b];
  // (rows without keys or with an error are written already)
  if (C < L || C > a.max_context_len || (C + kPage - 1) / kPage > a.bt_stride) return;
  // the parts that have a key of the row: any later ones of its item weigh nothing
  const int n = min(a.n_split, (C - L + j) / kQUnit / a.split_units + 1);
  const int64_t rec = (int64_t)f * a.n_split;
  float m = kMInit, l = 0.0f;
  if (lane < n) {
    m = a.ws_ml[(rec + lane) * 2];
    l = a.ws_ml[(rec + lane) * 2 + 1];
  }
  const float M = across_groups_max<1>(m);  // (every lane takes part)
  const float w = lane < n ? fast_exp2(m - M) : 0.0f;
  const float total = across_groups_sum<1>(l * w);
  constexpr int E = D / 64;
  float o[E] = {};
  for (int i = 0; i < n; ++i) {
    const float wi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), i));
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(a.ws_o[(rec + i) * D + lane * E + e], wi, o[e]);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) store_out<T>(reinterpret_cast<T*>(a.out) + (int64_t)f * D + lane * E + e, o[e] / total);
}

template <class F, typename T, int D>
const void* q_attn_pick(int blocks) {
  if constexpr (F::template kWide<T>)
    if (blocks == 2) return reinterpret_cast<const void*>(&q_attn_kernel<F, T, D, 2>);
  return blocks == 1 ? reinterpret_cast<const void*>(&q_attn_kernel<F, T, D, 1>) : nullptr;
}

template <class F>
const void* q_attn_fn(int dtype, int D, int blocks) {
  if (dtype == 0 && D == 128) return q_attn_pick<F, uint16_t, 128>(blocks);
  if (dtype == 0 && D == 64) return q_attn_pick<F, uint16_t, 64>(blocks);
  if (dtype == 1 && D == 128) return q_attn_pick<F, float, 128>(blocks);
  if (dtype == 1 && D == 64) return q_attn_pick<F, float, 64>(blocks);
  return nullptr;
}

template <class F>
hipError_t launch_q_attn(int dtype, int D, const QAttnArgs& a, hipStream_t st, KernelEvents ev) {
  const void* fn = q_attn_fn<F>(dtype, D, a.blocks);
  if (fn == nullptr) return hipErrorInvalidValue;
  const int64_t parts = (int64_t)a.H_kv * a.n_split;
  const int items = kQWaves / a.wave_parts;  // of a workgroup
  const int64_t grid = (a.n_slots + items - 1) / items * parts;
  void* args[] = {const_cast<QAttnArgs*>(&a)};
  hipError_t e = hipExtLaunchKernel(fn, dim3((uint32_t)grid), dim3(64 * kQWaves), args, 0, st, ev.start, ev.stop, 0);
  return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace pa
