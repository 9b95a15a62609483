// The 4-bit cache's attention kernel and its picker (design in pa_q4_attn.hip).
// Each (element type, head dim) is instantiated in one translation unit.
#pragma once

#include "pa_q4_tile.h"

namespace pa {

// An item's sequence and rows.
struct Q4Item {
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
__device__ __forceinline__ Q4Item q4_item(const Q4AttnArgs& a, int i, int positions, int lane) {
  Q4Item it{0, 0, 0, 0, false};
  const int32_t* qsl = a.query_start_loc;
  const int blocks = (a.rows + positions - 1) / positions;
  int first = 0, q0;
  if (i < blocks) {
    const int r = (blocks - 1 - i) * positions;
    it.b = q4::wave_search(a.B, r, lane, [&](int b) { return qsl[b]; });
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
template <typename T, int D, int NB>
__device__ __forceinline__ void q4_finish(const Q4AttnArgs& a, const q4::State<T, D, NB>& st, const int64_t (&at)[NB], int split,
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
      q4::eight_out(st, c, j, o);
      const int d = 32 * j + 8 * G;
      if (a.n_split == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= inv;
        q4::store_eight(out + at[c] * D + d, o);
      } else {
        q4::store_eight(a.ws_o + rec * D + d, o);
      }
    }
    if (a.n_split > 1 && G == 0) {
      a.ws_ml[rec * 2] = st.m[c];
      a.ws_ml[rec * 2 + 1] = l;
    }
  }
}

// What a wave hands to the one that joins an item's parts.
template <int D>
struct Q4Part {
  q4::f32x4_t o[D / 16][64];
  float m[64], l[64];
};

// (Three waves a SIMD: in fp32 at head_dim 128, whose registers would hold two, four
// chunks of 1,024 rows take 130 us instead of 144.)
template <typename T, int D>
__global__ __launch_bounds__(64 * kQ4Waves) __attribute__((amdgpu_waves_per_eu(3)))
void q4_attn_kernel(Q4AttnArgs a) {
  constexpr int NB = 1;  // column blocks of the wave
  const int S = a.s;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // row blocks of one head side by side
  const int split = blockIdx.x % a.n_split, g = blockIdx.x / a.n_split % a.H_kv;
  // (a workgroup's waves have items of their own, or 2 or 4 share one)
  const int sharers = a.wave_parts, part = wave & (sharers - 1);
  const Q4Item it = q4_item(a, (int)(blockIdx.x / a.n_split / a.H_kv * kQ4Waves + wave) / sharers, q4_positions(NB, S), lane);

  const int n = lane & 15;
  T* out = reinterpret_cast<T*>(a.out);
  const int all_last = it.last0 + it.n_pos - 1;
  if (it.bad && split == 0 && part == 0) {
    for (int i = lane; i < it.n_pos * S * D; i += 64)
      store_out<T>(out + ((int64_t)(it.row0 + i / (S * D)) * a.H_q + (int64_t)g * S) * D + i % (S * D), NAN);
  }
  // units of the item that the workgroup takes, and the wave's of them
  const int n_units = it.n_pos == 0 || it.bad ? 0 : all_last / kQ4Unit + 1;
  const int s0 = split * a.split_units, s1 = min(n_units, s0 + a.split_units);
  const int per = (max(s1 - s0, 0) + sharers - 1) / sharers;
  const int u0 = s0 + part * per, u1 = min(s1, u0 + per);
  if (u0 >= u1 && sharers == 1) return;

  q4::State<T, D, NB> st;
  int64_t at[NB];  // of the column's (row, head) vector, among all
  q4::reset(st);
  if (u0 < u1) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const int col = 16 * c + n, pos = col / S;
      const bool there = pos < it.n_pos;  // (columns past the item's positions are none)
      st.last[c] = there ? it.last0 + pos : -1;
      at[c] = (int64_t)(it.row0 + (there ? pos : 0)) * a.H_q + (int64_t)g * S + col % S;
      q4::load_query<T, D>(st.q[c], there ? reinterpret_cast<const T*>(a.q) + at[c] * D : nullptr, lane);
    }

    const int n_pages = all_last / kPage + 1;
    const int64_t tile = q4_tile_bytes(D), page_bytes = tile * a.H_kv;
    const int tile_size = a.num_pages > 0 ? q4_tile_bytes(D) : 0;
    const uint8_t* kg = a.k_pages + g * tile;
    const uint8_t* vg = a.v_pages + g * tile;
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
    q4::Unit<D> u;
    const int k_shift = q4::k_shift<D>(lane);
    auto fetch_k = [&](const Pages& t, bool any) {
#pragma unroll
      for (int p = 0; p < 2; ++p) q4::load_k<D, 0>(u, p, kg + t.at[p], any ? tile_size : 0, lane);
    };
    auto fetch_v = [&](const Pages& t, bool any) {
#pragma unroll
      for (int p = 0; p < 2; ++p) q4::load_v<D, 0>(u, p, vg + t.at[p], any ? tile_size : 0, lane);
    };
    Pages t = pages(u0);
    fetch_k(t, true);
    __builtin_amdgcn_sched_barrier(0);  // (K before V, as the loop's waits expect)
    fetch_v(t, true);
    constexpr bool kF16 = q4::kF16<T>;
    const int u_full = min(u1, (it.last0 + 1) / kQ4Unit);  // units before are seen whole by every column
    for (int k = u0; k < u1; ++k) {
      q4::f32x4_t s[NB][2];
      float x[NB][8];
      Pages next = t;
      bool big = false, odd = false;  // the base moves; V takes other products
      auto weights = [&](bool usual) {  // the weights of unit k, and the next K; whether it is big or odd
        if (k + 1 < u1) next = pages(k + 1);
        q4::fold_qk<T, D, NB>(st, u, k_shift, s);
        fetch_k(next, k + 1 < u1);
        if (!usual) {
          q4::mask_scores<T, D, NB>(st, k * kQ4Unit, t.bad, lane, s);
          q4::clear_dead(u, k * kQ4Unit, all_last, lane);
        }
        big = q4::form_weights<T, D, NB>(st, s, a.scale_log2, x);
        __builtin_amdgcn_sched_barrier(0);  // (V is not waited for before the weights are formed)
        odd = kF16 ? q4::beyond_fp16<D>(u) : q4::has_large<D>(u);
        return __builtin_amdgcn_ballot_w64(big | odd) != 0;
      };
      bool rare = weights(k < u_full && t.bad == 0) | st.any_lifted;
      if (k < u_full) {
        // (one way out, and nothing but the usual unit: the sums stay in place, and the
        // loads under way are known)
#pragma unroll 1
        while (!rare & (k + 1 < u_full) & (next.bad == 0)) {
          q4::add_weights(st, x);
          q4::fold_pv<kF16, T, D, NB>(st, u, x);
          fetch_v(next, true);
          t = next;
          ++k;
          rare = weights(true);
        }
      }
      int first = INT32_MAX;
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, 0)) first = q4::first_large(u, k * kQ4Unit, lane);
      q4::settle_weights<true, T, D, NB>(st, s, a.scale_log2, big, x, first);
      q4::fold_pv_edge<T, D, NB>(st, u, x, k * kQ4Unit, lane);
      fetch_v(next, k + 1 < u1);
      t = next;
    }
  }
  if (sharers > 1) {  // join the parts that have units: the first one's wave takes the others'
    __shared__ Q4Part<D> parts[kQ4Waves];
    if (part > 0 && u0 < u1) {
#pragma unroll
      for (int j = 0; j < D / 16; ++j) parts[wave].o[j][lane] = st.acc[0][j];
      parts[wave].m[lane] = st.m[0];
      parts[wave].l[lane] = st.l[0];
    }
    __syncthreads();
    if (part > 0 || u0 >= u1) return;
    const int n_parts = (s1 - s0 + per - 1) / per;
    float M = st.m[0];
    for (int i = 1; i < n_parts; ++i) M = fmaxf(M, parts[wave + i].m[lane]);
    const float c0 = fast_exp2(st.m[0] - M);
    st.m[0] = M;
    st.l[0] *= c0;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) st.acc[0][j] *= c0;
    for (int i = 1; i < n_parts; ++i) {
      const auto& other = parts[wave + i];
      const float ci = fast_exp2(other.m[lane] - M);
      st.l[0] = fmaf(other.l[lane], ci, st.l[0]);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) st.acc[0][j] = other.o[j][lane] * ci + st.acc[0][j];
    }
  }
  q4_finish<T, D, NB>(a, st, at, split, lane);
}

// Join the parts of one (query row, head) per wave.
template <typename T, int D>
__global__ __launch_bounds__(256) void q4_merge_kernel(Q4AttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int f = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = f / a.H_q;
  if (row >= a.rows) return;
  const int32_t* qsl = a.query_start_loc;
  const int b = q4::wave_search(a.B, row, lane, [&](int i) { return qsl[i]; });
  const int L = qsl[b + 1] - qsl[b], j = row - qsl[b];
  if (j < 0 || j >= L || L < a.min_rows || L > a.max_q_len) return;
  const int C = a.context_lens[b];
  // (rows without keys or with an error are written already)
  if (C < L || C > a.max_context_len || (C + kPage - 1) / kPage > a.bt_stride) return;
  // the parts that have a key of the row: any later ones of its item weigh nothing
  const int n = min(a.n_split, (C - L + j) / kQ4Unit / a.split_units + 1);
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

template <typename T, int D>
const void* q4_attn_pick() {
  return reinterpret_cast<const void*>(&q4_attn_kernel<T, D>);
}

}  // namespace pa
