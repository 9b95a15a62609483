// The decode kernel of the caches held in few bits, its picker and launcher (design in
// pa_q4_stream.hip).  Each (format, element type, head dim) is instantiated in one
// translation unit, which includes the format before this file.
#pragma once

#include <algorithm>
#include <atomic>

#include "pa_q_tile.h"
#include "pa_stream_body.h"

namespace pa {

// A record's 16-byte chunks: chunk c holds head c / 4 mod S, dims 32 j + 8 (c mod 4)
// + 4 h .. +3 with 2 j + h = c / 4 S (the accumulators' order, a lane's own pairs).
template <int D, int S>
struct QRecord {
  static __device__ __forceinline__ int head(int c) { return c / 4 % S; }
  static __device__ __forceinline__ int dim(int c) { return (c / (8 * S)) * 32 + c % 4 * 8 + c / (4 * S) % 2 * 4; }
  static __device__ __forceinline__ int chunk(int n, int jh, int G) { return (jh * S + n) * 4 + G; }
};

template <int D, int S>
struct QStreamSmem {
  int32_t cum[kQStreamSeqs + 1];  // units of the sequences before, per KV head
  int32_t scan[kQStreamThreads / 64];
  // of each wave, its parts of the items cut by its range's start (0) and end (1)
  struct Part {
    float ml[S][2];
    alignas(16) float o[S * D];
  } part[kQStreamThreads / 64][2];
};

// What the kernel does with sequence b: 1 (its row sees nv > 0 keys), 0 (nothing),
// 2 (zeros), -1 (rows row .. row + n - 1 are NaN).
__device__ __forceinline__ int q_decode_row(const QStreamArgs& a, int b, int& row, int& n, int& nv) {
  nv = a.context_lens[b];
  n = 1;
  row = b;
  if (a.query_start_loc != nullptr) {
    row = a.query_start_loc[b];
    n = a.query_start_loc[b + 1] - row;
    if (n > 1) return a.write_long && n > a.max_q_len ? -1 : 0;
    if (n < 1 || row < 0 || row >= a.rows) return 0;
    if (nv == 0) return -1;
  }
  if (nv < 0 || nv > a.max_context_len || (nv + kPage - 1) / kPage > a.bt_stride) return -1;
  return nv == 0 ? 2 : 1;
}

// Join n <= 64 records of an item, those of workgroups xs, xs + step, .. (record slot
// 1 of the item's first workgroup x0, slot 0 of the others), in order, by one wave;
// lane l takes the records' 16-byte chunks l, l + 64, ..  final: normalise and write
// the output; otherwise the joined record takes the first one's place.  Records
// bypass the L2 (a round trip of 1 to 2 us), so all (m, l), record i by lane i, and
// the first kBatch records' outputs are loaded at once.
template <typename T, int D, int S>
__device__ __forceinline__ void q_join(const QStreamArgs& a, int x0, int xs, int step, int n, bool final, int lane, T* out) {
  using Rec = QRecord<D, S>;
  constexpr int kChunks = S * D / 4, C = (kChunks + 63) / 64;  // chunks per lane
  constexpr int kBatch = 4;  // (8 are no faster)
  asm volatile("" ::: "memory");  // (the loads stay below the arrival)
  auto slot = [&](int i) {
    const int x = xs + i * step;
    return (int64_t)x * 2 + (x == x0 ? 1 : 0);
  };
  f32x4_dev_t v[kBatch][C];
  auto load = [&](int i0) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {  // (past the last record: that one again, unused)
      const __amdgpu_buffer_rsrc_t r = record_rsrc(a.ws_o + slot(min(i0 + b, n - 1)) * S * D, S * D);
#pragma unroll
      for (int u = 0; u < C; ++u) v[b][u] = load_dev4(r, (u * 64 + lane) * 4);
    }
  };
  // lane i: record i's bases and sums, then its weight for each head
  float c[S], l[S], M[S], L[S];
  {
    const float* ml = a.ws_ml + slot(min(lane, n - 1)) * S * 2;
#pragma unroll
    for (int j = 0; j < S; ++j) load_dev2(ml + j * 2, c[j], l[j]);
  }
  load(0);
#pragma unroll
  for (int j = 0; j < S; ++j) {
    M[j] = across_groups_max<1>(c[j]);
    c[j] = fast_exp2(c[j] - M[j]);
    L[j] = 0.0f;
  }
  auto bcast = [](float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); };
  // value of head h among the S wave-uniform ones (chosen between as values: an array
  // indexed at run time would move to memory)
  auto pick = [&](const float (&x)[S], int h) {
    float y = x[0];
#pragma unroll
    for (int j = 1; j < S; ++j) {
      const float xj = x[j];
      y = h == j ? xj : y;
    }
    return y;
  };
  f32x4_dev_t acc[C];
#pragma unroll
  for (int u = 0; u < C; ++u) acc[u] = f32x4_dev_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += kBatch) {
    if (i0 > 0) load(i0);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (i0 + b < n) {  // wave-uniform
        float ci[S];
#pragma unroll
        for (int j = 0; j < S; ++j) {
          ci[j] = bcast(c[j], i0 + b);
          L[j] = fmaf(bcast(l[j], i0 + b), ci[j], L[j]);
        }
#pragma unroll
        for (int u = 0; u < C; ++u) acc[u] = v[b][u] * pick(ci, Rec::head(u * 64 + lane)) + acc[u];
      }
    }
  }
  const __amdgpu_buffer_rsrc_t r = record_rsrc(a.ws_o + slot(0) * S * D, S * D);
#pragma unroll
  for (int u = 0; u < C; ++u) {
    const int ch = u * 64 + lane;
    if (final) {
      const f32x4_dev_t o = acc[u] * (1.0f / pick(L, Rec::head(ch)));
      if (kChunks % 64 == 0 || ch < kChunks) q::store_four(out + Rec::head(ch) * D + Rec::dim(ch), o);
    } else {
      store_dev4(r, ch * 4, acc[u]);  // (a chunk past the record is out of the descriptor's range)
    }
  }
  if (!final && lane == 0) {
#pragma unroll
    for (int j = 0; j < S; ++j) store_dev(a.ws_ml + slot(0) * S * 2 + j * 2, M[j], L[j]);
  }
}

template <class F, typename T, int D, int S>
__global__ __launch_bounds__(kQStreamThreads) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2)))  // (two workgroups a CU at head_dim 64)
void q_stream_kernel(QStreamArgs a) {
  using Rec = QRecord<D, S>;
  constexpr int NT = kQStreamThreads, kWaves = NT / 64;
  __shared__ QStreamSmem<D, S> sm;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wg = blockIdx.x, n_wg = gridDim.x;
  const int bid = wg * kWaves + wave;  // the wave's range
  const int R = a.B, H = a.H_kv;

  // 1. units per sequence and their prefix sums (every workgroup, redundantly);
  // the rows without units are written by the workgroups in turn
  {
    const int per = (R + NT - 1) / NT;
    const int r0 = min(R, tid * per), r1 = min(R, r0 + per);
    int local = 0;
    for (int r = r0; r < r1; ++r) {
      int row, n, nv;
      const int what = q_decode_row(a, r, row, n, nv);
      sm.cum[r] = local;
      local += what == 1 ? (nv + kQUnit - 1) / kQUnit : 0;
    }
    const int off = block_exclusive_scan<NT>(local, sm.scan);
    for (int r = r0; r < r1; ++r) sm.cum[r] += off;
    if (tid == NT - 1) sm.cum[R] = off + local;
    __syncthreads();
  }
  for (int r = wg; r < R; r += n_wg) {
    if (sm.cum[r + 1] != sm.cum[r]) continue;
    int row, n, nv;
    const int what = q_decode_row(a, r, row, n, nv);
    if (what == 0) continue;
    const int64_t from = max(row, 0), to = min((int64_t)row + n, (int64_t)a.rows);
    T* o = reinterpret_cast<T*>(a.out);
    for (int64_t i = from * a.H_q * D + tid; i < to * a.H_q * D; i += NT) store_out<T>(o + i, what == 2 ? 0.0f : NAN);
  }
  const int U = H * sm.cum[R];
  const int busy = min(a.cus, n_wg);  // workgroups, one per CU
  // ranges: one per wave, in a workgroup per CU where more would have few units each
  const int G = max(1, min((U < kQFewUnits * n_wg * kWaves ? busy : n_wg) * kWaves, U));
  if (U == 0) return;
  // Few short items: a workgroup has one of them alone, and nothing is joined through
  // memory (kQAloneUnits).
  bool alone = (int64_t)R * H <= busy;
  if (alone) {
    int most = 0;
    for (int r = lane; r < R; r += 64) most = max(most, sm.cum[r + 1] - sm.cum[r]);
    alone = __builtin_amdgcn_ballot_w64(most > U / busy + kQAloneUnits) == 0;
  }
  if (wg >= (alone ? R * H : (G + kWaves - 1) / kWaves)) return;
  // ranges of each or each + 1 units, the longer ones first
  const int each = U / G, longer = U % G;
  auto begin_of = [&](int x) { return min(x, G) * each + min(x, longer); };
  auto range_of = [&](int e) {
    const int split = longer * (each + 1);
    return e < split ? e / (each + 1) : longer + (e - split) / each;
  };
  int u0, m;  // units of the range
  if (alone) {
    const int r = wg / H, np = sm.cum[r + 1] - sm.cum[r], per = (np + kWaves - 1) / kWaves;
    u0 = H * sm.cum[r] + (wg - r * H) * np + wave * per;
    m = max(0, min(per, np - wave * per));
  } else {
    u0 = begin_of(bid);
    m = begin_of(bid + 1) - u0;
  }

  // 2. The range's units, 64 at a time, one per lane.  (Loading the words that their
  // lengths and pages come from ahead, when the 64 before begin, is no faster.)
  struct Entries {
    int64_t at[2];  // the tiles' first byte (0: outside the pool, or no page)
    int info;       // tokens (6 bits) | page 0, 1 outside the pool | anything but 32 tokens of the pool
    int hb, p, np;  // KV head; unit of the item and the item's units
    int row;
  };
  const int64_t tile = F::tile_bytes(D);
  auto entries = [&](int i0) {
    Entries e;
    const int x = u0 + min(i0 + lane, m - 1);
    const int r = info_row_seq(sm.cum, R, H, x);
    const int rem = x - H * sm.cum[r];
    e.np = sm.cum[r + 1] - sm.cum[r];
    e.hb = rem / e.np;
    e.p = rem - e.hb * e.np;
    e.row = a.query_start_loc != nullptr ? a.query_start_loc[r] : r;
    int page[2], odd = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)  // (past the context's pages: any entry, unused; read without waiting for the length)
      page[h] = a.block_table[(int64_t)r * a.bt_stride + min((int64_t)2 * e.p + h, a.bt_stride - 1)];
    const int left = a.context_lens[r] - e.p * kQUnit;  // tokens from the unit on
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool used = left > kPage * h, ok = used && page[h] >= 0 && page[h] < a.num_pages;
      odd |= (ok || !used ? 0 : 1) << h;
      e.at[h] = ok ? ((int64_t)page[h] * H + e.hb) * tile : 0;
    }
    e.info = min(left, kQUnit) | odd << 6 | (odd != 0 || left < kQUnit) << 8;
    return e;
  };

  q::State<T, D, 1, F::template kCodes<T, D>> st;
  typename F::template Unit<D> u;
  const int k_shift = F::template shift<D>(lane);
  const int n = lane & 15, Gl = lane >> 4;
  T* out = reinterpret_cast<T*>(a.out);
  const int tile_size = a.num_pages > 0 ? F::tile_bytes(D) : 0;
  struct Tiles {
    int64_t at[2];
    int info;
  };
  auto fetch_k = [&](const Tiles& e, bool any) {
#pragma unroll
    for (int p = 0; p < 2; ++p) F::template load_k<kKvLoadPolicy>(u, p, a.k_pages, e.at[p], a.scales, any ? tile_size : 0, lane);
  };
  auto fetch_v = [&](const Tiles& e, bool any) {
#pragma unroll
    for (int p = 0; p < 2; ++p) F::template load_v<kKvLoadPolicy>(u, p, a.v_pages, e.at[p], a.scales, any ? tile_size : 0, lane);
  };
  auto put_part = [&](int which, float l) {
    auto& part = sm.part[wave][which];
    if (n < S) {
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        float o[8];
        q::eight_out(st, 0, j, o);
        *reinterpret_cast<f32x4_dev_t*>(&part.o[Rec::chunk(n, 2 * j, Gl) * 4]) = f32x4_dev_t{o[0], o[1], o[2], o[3]};
        *reinterpret_cast<f32x4_dev_t*>(&part.o[Rec::chunk(n, 2 * j + 1, Gl) * 4]) = f32x4_dev_t{o[4], o[5], o[6], o[7]};
      }
      if (Gl == 0) {
        part.ml[n][0] = st.m[0];
        part.ml[n][1] = l;
      }
    }
  };

  // 3. Stream the units, the next one's K loaded as soon as the scores are formed, its
  // V after the products.
  struct Job {  // an item cut by the range's start (0) or end (1): its first and last unit, row and KV head
    int from = -1, to = -1, row = 0, g = 0;
  } job[2];
  if (m > 0) {
    Entries es = entries(0);
    int i0 = 0;  // unit of es's first lane
    auto of = [&](int x, int i) { return __builtin_amdgcn_readlane(x, i - i0); };
    auto tiles = [&](int i) {  // (wave-uniform)
      Tiles t;
#pragma unroll
      for (int p = 0; p < 2; ++p)
        t.at[p] = (int64_t)((uint64_t)(uint32_t)of((int)(es.at[p] >> 32), i) << 32 | (uint32_t)of((int)es.at[p], i));
      t.info = of(es.info, i);
      return t;
    };
    Tiles t = tiles(0);
    fetch_k(t, true);
    __builtin_amdgcn_sched_barrier(0);  // (K before V, as the loop's waits expect)
    fetch_v(t, true);
    bool open = false, head = false;  // the present item has begun; it began before the range
    int from = 0, to = 0, row = 0, g = 0;
    for (int i = 0; i < m;) {
      const int p = of(es.p, i), left = of(es.np, i) - p;
      if (!open) {
        row = of(es.row, i);
        g = of(es.hb, i);
        head = p > 0;
        from = u0 + i - p;
        to = u0 + i + left - 1;
        const T* q = reinterpret_cast<const T*>(a.q) + ((int64_t)row * a.H_q + (int64_t)g * S + n) * D;
        q::load_query<F::kSliced>(st.q[0], n < S ? q : nullptr, lane);
        q::reset(st);
        st.last[0] = kQUnit - 1;
        open = true;
      }
      // units without anything else to do between them; the last of the 64 is alone: the
      // next one's entry is among the 64 after
      int stop = min(min(m, i + left), i0 + 63);
      if (i + 1 - i0 == 64) {
        stop = i + 1;
        if (stop < m) {
          i0 += 64;
          es = entries(i0);
        }
      }
      const bool ends = stop == i + left;
      for (; i < stop; ++i) {
        constexpr bool kF16 = q::kF16<T>;
        q::f32x4_t s[1][2];
        float x[1][8], sum[1];
        Tiles next;
        bool big;      // the base moves
        uint64_t odd;  // V takes other products (of the lanes)
        auto weights = [&](bool usual) {  // the weights of unit i, and the next K; whether it is big or odd
          const bool more = i + 1 < m;
          next = tiles(more ? i + 1 : i);
          F::fold_qk(st, u, k_shift, s);
          F::keep_scales(u);
          fetch_k(next, more);
          if (!usual) {
            const int tokens = t.info & 63;
            st.last[0] = tokens - 1;  // (of this unit; the item's last, or of pages outside the pool)
            q::mask_scores<T, D, 1>(st, 0, t.info >> 6 & 3, lane, s);
            F::clear_dead(u, 0, tokens - 1, lane);
          }
          big = q::form_weights<F::kSums>(st, s, a.scale_log2, x, sum);
          __builtin_amdgcn_sched_barrier(0);  // (V is not waited for before the weights are formed)
          odd = __builtin_amdgcn_ballot_w64(F::template odd<kF16>(u));
          return (odd | __builtin_amdgcn_ballot_w64(big)) != 0;
        };
        bool rare = weights(!(t.info & 256)) | st.any_lifted;
        // (one way out, and nothing but the usual unit: the sums stay in place, and the
        // loads under way are known)
#pragma unroll 1
        while (!rare & (i + 1 < stop) & !(next.info & 256)) {
          q::add_weights<F::kSums>(st, x, sum);
          F::template fold_pv<kF16>(st, u, x);
          fetch_v(next, true);
          t = next;
          ++i;
          // (of a SIMD's waves the oldest issues first: in turn, so that they end together)
          if ((i ^ (wave >> 2)) & 1) {
            __builtin_amdgcn_s_setprio(1);
          } else {
            __builtin_amdgcn_s_setprio(0);
          }
          rare = weights(true);
        }
        int first = INT32_MAX;  // (every column sees every key of the unit)
        if (__builtin_expect(odd != 0, 0))
          first = __builtin_amdgcn_ballot_w64(F::has_large(u)) != 0 ? 0 : INT32_MAX;
        q::settle_weights<true, F::kSums>(st, s, a.scale_log2, big, x, sum, first);
        F::template fold_pv<false>(st, u, x);
        fetch_v(next, i + 1 < m);
        t = next;
      }
      if (!ends) continue;
      // the item ends: its output, or this range's part of it
      const float l = rows4_sum(st.l[0]);
      if (!head) {
        const float inv = 1.0f / l;
        if (n < S) {
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            float o[8];
            q::eight_out(st, 0, j, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] *= inv;
            q::store_eight(out + ((int64_t)row * a.H_q + (int64_t)g * S + n) * D + 32 * j + 8 * Gl, o);
          }
        }
      } else {
        put_part(0, l);
        job[0] = Job{from, to, row, g};
      }
      open = false;
    }
    if (open) {  // the range ends inside an item
      const float l = rows4_sum(st.l[0]);
      if (head) {
        put_part(0, l);
        job[0] = Job{from, to, row, g};
      } else {
        put_part(1, l);
        job[1] = Job{from, to, row, g};
      }
    }
  }

  // 4. Join the cut items: the parts of the workgroup's waves in LDS, by the wave that
  // has the first.  An item cut by the workgroup's ends too: that wave stores the joined
  // part as the workgroup's record (slot 0: of the item that the workgroup's start cuts,
  // 1: of that which its end cuts) and counts it, and whichever part counts last joins
  // all of them in order; nothing waits on another workgroup.
  __syncthreads();
  auto counter_at = [&](int x) {
    // (global memory for certain: while a generic access is under way, every wait is for all)
    using Global = __attribute__((address_space(1))) unsigned long long;
    Global* p = (Global*)(a.ws_flag + (int64_t)x * kQCounterStride);
    asm("" : "+v"(p));  // (an address of lanes: one atomic, not a wave's reduction)
    return DeviceCounter{(unsigned long long*)p};
  };
#pragma unroll 1
  for (int j = 0; j < 2; ++j) {
    const Job it = j == 0 ? job[0] : job[1];
    if (it.from < 0 || (j == 0 && wave > 0)) continue;  // (else an earlier wave has the item's first part)
    // parts: slot j of this wave, slot 0 of those up to the item's last
    int parts;
    CutItem cut{wg, wg};
    if (alone) {
      parts = (it.to - it.from) / m + 1;
    } else {
      const int to = range_of(it.to);
      parts = min(to - wg * kWaves, kWaves - 1) - wave + 1;
      cut = CutItem{range_of(it.from) / kWaves, to / kWaves};
    }
    const bool whole = cut.x0 == cut.x1;
    T* o = out + ((int64_t)it.row * a.H_q + (int64_t)it.g * S) * D;
    const int64_t slot = (int64_t)wg * 2 + j;
    const __amdgpu_buffer_rsrc_t r = record_rsrc(a.ws_o + slot * S * D, S * D);
#pragma unroll 1
    for (int c = lane; c < S * D / 4; c += 64) {
      const int h = Rec::head(c);
      float M = kMInit, L = 0.0f;
#pragma unroll 4
      for (int i = 0; i < parts; ++i) M = fmaxf(M, sm.part[wave + i][i == 0 ? j : 0].ml[h][0]);
      f32x4_dev_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
      for (int i = 0; i < parts; ++i) {
        const auto& part = sm.part[wave + i][i == 0 ? j : 0];
        const float ci = fast_exp2(part.ml[h][0] - M);
        L = fmaf(part.ml[h][1], ci, L);
        acc = *reinterpret_cast<const f32x4_dev_t*>(&part.o[c * 4]) * ci + acc;
      }
      if (whole) {
        q::store_four(o + h * D + Rec::dim(c), acc * (1.0f / L));
      } else {
        store_dev4(r, c * 4, acc);
        if (Rec::dim(c) == 0) store_dev(a.ws_ml + (slot * S + h) * 2, M, L);
      }
    }
    if (whole) continue;
#pragma unroll 1
    for (int lv = cut.grouped() && !cut.group_of_one(wg) ? 0 : 1; lv < 2; ++lv) {
      const int records = cut.parts(lv, wg);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0);  // the record is stored
      int last = 0;
      if (lane == 0) {
        DeviceCounter ctr = counter_at(cut.counter(lv, wg));
        last = counter_arrive(ctr, a.key, records);
      }
      if (!__builtin_amdgcn_readfirstlane(last)) break;
      // (a group's record counts in the item next)
      q_join<T, D, S>(a, cut.x0, cut.first(lv, wg), cut.step(lv), records, lv == 1, lane, o);
    }
  }
}

template <class F, typename T, int D>
const void* q_stream_pick(int s) {
  switch (s) {
    case 1: return reinterpret_cast<const void*>(&q_stream_kernel<F, T, D, 1>);
    case 2: return reinterpret_cast<const void*>(&q_stream_kernel<F, T, D, 2>);
    case 4: return reinterpret_cast<const void*>(&q_stream_kernel<F, T, D, 4>);
    case 6: return reinterpret_cast<const void*>(&q_stream_kernel<F, T, D, 6>);
    case 8: return reinterpret_cast<const void*>(&q_stream_kernel<F, T, D, 8>);
  }
  return nullptr;
}

template <class F>
const void* q_stream_fn(int dtype, int D, int s) {
  if (dtype == 0 && D == 128) return q_stream_pick<F, uint16_t, 128>(s);
  if (dtype == 0 && D == 64) return q_stream_pick<F, uint16_t, 64>(s);
  if (dtype == 1 && D == 128) return q_stream_pick<F, float, 128>(s);
  if (dtype == 1 && D == 64) return q_stream_pick<F, float, 64>(s);
  return nullptr;
}

// (a property of the kernel and the device, so it is asked for once: the two
// queries take as long as the rest of a small call on the host)
template <class F>
int q_stream_workgroups(int dtype, int D, int s, int* cus) {
  constexpr int kDevices = 64;
  static std::atomic<int64_t> known[kDevices][2][2][9];  // workgroups, and the CUs above them
  int dev = 0, n_cus = 0, per_cu = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 0;
  std::atomic<int64_t>* at = dev >= 0 && dev < kDevices && dtype >= 0 && dtype < 2 && s <= 8 ? &known[dev][dtype][D / 128][s] : nullptr;
  const int64_t have = at != nullptr ? at->load(std::memory_order_relaxed) : 0;
  if (have > 0) {
    *cus = (int)(have >> 32);
    return (int)have;
  }
  const void* fn = q_stream_fn<F>(dtype, D, s);
  if (fn == nullptr || hipDeviceGetAttribute(&n_cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, fn, kQStreamThreads, 0) != hipSuccess)
    return 0;
  const int n = std::min(n_cus * per_cu, kQStreamGroups);
  if (at != nullptr) at->store((int64_t)n_cus << 32 | n, std::memory_order_relaxed);
  *cus = n_cus;
  return n;
}

template <class F>
hipError_t launch_q_stream(int dtype, int D, int s, const QStreamArgs& a, int workgroups, hipStream_t st,
                            KernelEvents ev) {
  const void* fn = q_stream_fn<F>(dtype, D, s);
  if (fn == nullptr || workgroups <= 0) return hipErrorInvalidValue;
  void* args[] = {const_cast<QStreamArgs*>(&a)};
  hipError_t e = hipExtLaunchKernel(fn, dim3(workgroups), dim3(kQStreamThreads), args, 0, st, ev.start, ev.stop, 0);
  return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace pa
