// The 4-bit cache's decode kernel and its picker (design in pa_q4_stream.hip).
// Each (element type, head dim) is instantiated in one translation unit.
#pragma once

#include "pa_q4_tile.h"
#include "pa_stream_body.h"

namespace pa {

// An item cut over ranges x0 .. x1, as CutItem, with groups of 64 for the more
// ranges that this kernel has.
struct Q4Cut {
  int x0, x1;
  __device__ int n() const { return x1 - x0 + 1; }
  __device__ bool grouped() const { return n() > 16; }
  __device__ int shift() const { return n() <= 64 ? 3 : n() <= 256 ? 4 : n() <= 1024 ? 5 : 6; }
  __device__ int group_first(int x) const { return x0 + ((x - x0) >> shift() << shift()); }
  __device__ bool group_of_one(int x) const { return group_first(x) == x1; }
  __device__ int first(int level, int x) const { return level == 0 ? group_first(x) : x0; }
  __device__ int step(int level) const { return level == 1 && grouped() ? 1 << shift() : 1; }
  __device__ int parts(int level, int x) const {
    return level == 0 ? min(1 << shift(), x1 - group_first(x) + 1) : grouped() ? ((n() - 1) >> shift()) + 1 : n();
  }
  __device__ int counter(int level, int x) const { return first(level, x) + (level == 0 && group_first(x) == x0 ? 1 : 0); }
};
static_assert(kQ4StreamWaves <= 64 * 64, "one record per lane at either level");

// A record's 16-byte chunks: chunk c holds head c / 4 mod S, dims 32 j + 8 (c mod 4)
// + 4 h .. +3 with 2 j + h = c / 4 S (the accumulators' order, a lane's own pairs).
template <int D, int S>
struct Q4Record {
  static __device__ __forceinline__ int head(int c) { return c / 4 % S; }
  static __device__ __forceinline__ int dim(int c) { return (c / (8 * S)) * 32 + c % 4 * 8 + c / (4 * S) % 2 * 4; }
  static __device__ __forceinline__ int chunk(int n, int jh, int G) { return (jh * S + n) * 4 + G; }
};

struct Q4UnitEntry {
  int64_t at[2];  // the pages' first byte of the head block (0: outside the pool, or no page)
  int32_t info;   // tokens (6 bits) | page 0, 1 outside the pool | anything but 32 tokens of the pool | head block
  int32_t left;   // units to the item's end, this one included
  int32_t row;
  int32_t first;  // whether it is the item's first
};

template <int W>
struct Q4StreamSmem {
  static constexpr int kTeams = kQ4StreamThreads / 64 / W;
  static constexpr int kUnits = 1024 / kTeams;  // of a table
  int32_t cum[kQ4StreamSeqs + 1];               // units of the sequences before, per head block
  int32_t scan[kQ4StreamThreads / 64];
  struct Team {
    Q4UnitEntry unit[kUnits];
    Q4Cut cut[2];          // the items cut by the range's start and by its end (x0 = -1: none)
    int32_t job[W][2][2];  // their row and KV head
    int32_t last_row, last_hb;  // of the range's last unit
  } team[kTeams];
};

// What the kernel does with sequence b: 1 (its row sees nv > 0 keys), 0 (nothing),
// 2 (zeros), -1 (rows row .. row + n - 1 are NaN).
__device__ __forceinline__ int q4_decode_row(const Q4StreamArgs& a, int b, int& row, int& n, int& nv) {
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

// Join n <= 64 records of an item, those of ranges xs, xs + step, .. (record slot 1
// of the item's first range x0, slot 0 of the others), in range order, by one wave;
// lane l takes the records' 16-byte chunks l, l + 64, ..  final: normalise and write
// the output; otherwise the joined record takes the first one's place.  Records
// bypass the L2 (a round trip of 1 to 2 us), so all (m, l), record i by lane i, and
// the first kBatch records' outputs are loaded at once.
template <typename T, int D, int S, int W>
__device__ __forceinline__ void q4_join(const Q4StreamArgs& a, int x0, int xs, int step, int n, bool final, int w, int lane, T* out) {
  using Rec = Q4Record<D, S>;
  constexpr int kChunks = S * D / 4, C = (kChunks + 63) / 64;  // chunks per lane
  constexpr int kBatch = 4;  // (8 are no faster)
  asm volatile("" ::: "memory");  // (the loads stay below the arrival)
  auto slot = [&](int i) {
    const int x = xs + i * step;
    return ((int64_t)x * 2 + (x == x0 ? 1 : 0)) * W + w;
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
      if (kChunks % 64 == 0 || ch < kChunks) q4::store_four(out + Rec::head(ch) * D + Rec::dim(ch), o);
    } else {
      store_dev4(r, ch * 4, acc[u]);  // (a chunk past the record is out of the descriptor's range)
    }
  }
  if (!final && lane == 0) {
#pragma unroll
    for (int j = 0; j < S; ++j) store_dev(a.ws_ml + slot(0) * S * 2 + j * 2, M[j], L[j]);
  }
}

template <typename T, int D, int S, int W>
__global__ __launch_bounds__(kQ4StreamThreads) __attribute__((amdgpu_waves_per_eu(2)))
void q4_stream_kernel(Q4StreamArgs a) {
  using Sm = Q4StreamSmem<W>;
  using Rec = Q4Record<D, S>;
  constexpr int kTeams = Sm::kTeams, NT = kQ4StreamThreads;
  __shared__ Sm sm;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int team = wave / W, w = wave % W;
  const int wg = blockIdx.x, n_wg = gridDim.x;
  const int bid = team * n_wg + wg;  // the team's range
  auto& tm = sm.team[team];
  const int R = a.B;

  // 1. units per sequence and their prefix sums (every workgroup, redundantly);
  // the rows without units are written by the workgroups in turn
  {
    const int per = (R + NT - 1) / NT;
    const int r0 = min(R, tid * per), r1 = min(R, r0 + per);
    int local = 0;
    for (int r = r0; r < r1; ++r) {
      int row, n, nv;
      const int what = q4_decode_row(a, r, row, n, nv);
      sm.cum[r] = local;
      local += what == 1 ? (nv + kQ4Unit - 1) / kQ4Unit : 0;
    }
    const int off = block_exclusive_scan<NT>(local, sm.scan);
    for (int r = r0; r < r1; ++r) sm.cum[r] += off;
    if (tid == NT - 1) sm.cum[R] = off + local;
    __syncthreads();
  }
  for (int r = wg; r < R; r += n_wg) {
    if (sm.cum[r + 1] != sm.cum[r]) continue;
    int row, n, nv;
    const int what = q4_decode_row(a, r, row, n, nv);
    if (what == 0) continue;
    const int64_t from = max(row, 0), to = min((int64_t)row + n, (int64_t)a.rows);
    T* o = reinterpret_cast<T*>(a.out);
    for (int64_t i = from * a.H_q * D + tid; i < to * a.H_q * D; i += NT) store_out<T>(o + i, what == 2 ? 0.0f : NAN);
  }
  const int U = a.nb * sm.cum[R];
  const int G = max(1, min(n_wg * kTeams, U));  // ranges
  if (wg >= G || U == 0) return;
  // ranges of each or each + 1 units, the longer ones first
  const int each = U / G, longer = U % G;
  auto begin_of = [&](int x) { return min(x, G) * each + min(x, longer); };
  auto range_of = [&](int e) {
    const int split = longer * (each + 1);
    return e < split ? e / (each + 1) : longer + (e - split) / each;
  };
  auto units_of = [&](int x) { return begin_of(x + 1) - begin_of(x); };
  const int u0 = begin_of(bid);
  const int n_units = units_of(bid);
  int n_steps = 0;  // units of the longest range of the workgroup's teams
#pragma unroll
  for (int t = 0; t < kTeams; ++t) n_steps = max(n_steps, units_of(t * n_wg + wg));

  q4::State<T, D, 1> st;
  q4::Unit<D> u;
  const int n = lane & 15, Gl = lane >> 4;
  const int64_t tile = q4_tile_bytes(D);
  T* out = reinterpret_cast<T*>(a.out);
  const uint8_t* kw = a.k_pages + w * tile;
  const uint8_t* vw = a.v_pages + w * tile;
  struct Tiles {
    int64_t at[2];
    int info;
  };
  auto tiles = [&](int i) {  // (wave-uniform)
    const Q4UnitEntry& e = tm.unit[i];
    Tiles t;
#pragma unroll
    for (int p = 0; p < 2; ++p)
      t.at[p] = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(e.at[p] >> 32)) << 32 |
                          (uint32_t)__builtin_amdgcn_readfirstlane((int)e.at[p]));
    t.info = __builtin_amdgcn_readfirstlane(e.info);
    return t;
  };
  const int tile_size = a.num_pages > 0 ? q4_tile_bytes(D) : 0;
  auto fetch_k = [&](const Tiles& e, bool any) {
#pragma unroll
    for (int p = 0; p < 2; ++p) q4::load_k<D, kKvLoadPolicy>(u, p, kw + e.at[p], any ? tile_size : 0, lane);
  };
  auto fetch_v = [&](const Tiles& e, bool any) {
#pragma unroll
    for (int p = 0; p < 2; ++p) q4::load_v<D, kKvLoadPolicy>(u, p, vw + e.at[p], any ? tile_size : 0, lane);
  };

  // Items cut by the range's ends.  Each wave is alone: a part is its record in the
  // workspace and one count of the item's counter for this wave's head.  Whichever
  // part counts last joins all of them in range order; nothing waits on another
  // workgroup.  The item that the start cuts (job 0), its record stored at the end of
  // unit k, counts when unit k + 3 starts: the vector-memory counter retires in issue
  // order, and unit k + 2, whose loads went out after the record, has been folded.
  // It looks at the answer when the range has streamed.  The item that the end cuts
  // (job 1) has usually one other part, which was the first thing of the next range:
  // its count is looked at before the last unit, and if it is there the wave joins
  // its record from registers and stores none of its own.
  auto counter_at = [&](int x) {
    // (global memory for certain: while a generic access is under way, every wait is for all)
    using Global = __attribute__((address_space(1))) unsigned long long;
    Global* p = (Global*)(a.ws_flag + ((int64_t)x * W + w) * kQ4CounterStride);
    asm("" : "+v"(p));  // (an address of lanes: one atomic, not a wave's reduction)
    return DeviceCounter{(unsigned long long*)p};
  };
  auto level_of = [&](const Q4Cut& cut) { return cut.grouped() && !cut.group_of_one(bid) ? 0 : 1; };
  bool stored[2] = {false, false};
  int counted_at = INT32_MAX;  // job 0 counts before this unit
  bool counted = false;
  uint64_t counted_old = 0;    // the counter before
  uint64_t seen = 0;           // the last item's counter
  bool look = false;           // whether it has been read
  bool head_partial = false, open = false;  // of the present item: it began before the range; it has not ended
  auto store_part = [&](int which, float l, int row, int g) {
    const int64_t slot = ((int64_t)bid * 2 + which) * W + w;
    const __amdgpu_buffer_rsrc_t r = record_rsrc(a.ws_o + slot * S * D, S * D);
    if (n < S) {
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        float o[8];
        q4::eight_out(st, 0, j, o);
        store_dev4(r, Rec::chunk(n, 2 * j, Gl) * 4, f32x4_dev_t{o[0], o[1], o[2], o[3]});
        store_dev4(r, Rec::chunk(n, 2 * j + 1, Gl) * 4, f32x4_dev_t{o[4], o[5], o[6], o[7]});
      }
      if (Gl == 0) store_dev(a.ws_ml + (slot * S + n) * 2, st.m[0], l);
    }
    if (lane == 0) {
      tm.job[w][which][0] = row;
      tm.job[w][which][1] = g;
    }
    stored[0] |= which == 0;
    stored[1] |= which == 1;
  };

  for (int base = 0; base < n_steps; base += Sm::kUnits) {
    // 2. unit table of this part of the range, and the items cut by its ends
    const int m = min(n_units - base, Sm::kUnits);
    if (base > 0) __syncthreads();
    for (int i = w * 64 + lane; i < m; i += 64 * W) {
      const int x = u0 + base + i;
      const int r = info_row_seq(sm.cum, R, a.nb, x);
      const int np = sm.cum[r + 1] - sm.cum[r];
      const int rem = x - a.nb * sm.cum[r];
      const int hb = rem / np, p = rem - hb * np;
      int page[2];  // (past the context's pages: any entry, unused; read without waiting for the length)
#pragma unroll
      for (int h = 0; h < 2; ++h) page[h] = a.block_table[(int64_t)r * a.bt_stride + min((int64_t)2 * p + h, a.bt_stride - 1)];
      const int left = a.context_lens[r] - p * kQ4Unit;  // tokens from the unit on
      Q4UnitEntry e;
      int odd = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool used = left > kPage * h, ok = used && page[h] >= 0 && page[h] < a.num_pages;
        odd |= (ok || !used ? 0 : 1) << h;
        e.at[h] = ok ? ((int64_t)page[h] * a.H_kv + hb * W) * tile : 0;
      }
      e.info = min(left, kQ4Unit) | odd << 6 | (odd != 0 || left < kQ4Unit) << 8 | hb << 9;
      e.left = np - p;
      e.row = a.query_start_loc != nullptr ? a.query_start_loc[r] : r;
      e.first = p == 0;
      tm.unit[i] = e;
      if (base + i == 0) tm.cut[0] = p == 0 ? Q4Cut{-1, -1} : Q4Cut{range_of(x - p), range_of(x - p + np - 1)};
      if (base + i == n_units - 1) tm.last_row = e.row, tm.last_hb = hb;
      if (base + i == n_units - 1) tm.cut[1] = p == np - 1 ? Q4Cut{-1, -1} : Q4Cut{range_of(x - p), range_of(x - p + np - 1)};
    }
    __syncthreads();
    if (m <= 0) continue;
    const bool has_next = base + m == n_units && tm.cut[1].x0 == bid && tm.cut[1].x1 == bid + 1;

    // 3. stream the units: wave w handles KV head hb * W + w of every unit, the next
    // unit's K loaded as soon as the scores are formed, its V after the products
    Tiles t = tiles(0);
    fetch_k(t, true);
    __builtin_amdgcn_sched_barrier(0);  // (K before V, as the loop's waits expect)
    fetch_v(t, true);
    for (int i = 0; i < m;) {
      const Q4UnitEntry& e = tm.unit[i];
      const int left = __builtin_amdgcn_readfirstlane(e.left);
      const int g = (__builtin_amdgcn_readfirstlane(e.info) >> 9) * W + w;
      const int row = __builtin_amdgcn_readfirstlane(e.row);
      const int64_t at = ((int64_t)row * a.H_q + (int64_t)g * S + n) * D;
      if (__builtin_amdgcn_readfirstlane(e.first) || base + i == 0) {
        head_partial = !__builtin_amdgcn_readfirstlane(e.first);
        q4::load_query<T, D>(st.q[0], n < S ? reinterpret_cast<const T*>(a.q) + at : nullptr, lane);
        q4::reset(st);
        open = true;
      }
      // units without anything else to do between them
      int stop = min(m, i + left);
      if (base + i == counted_at) {
        asm volatile("" ::: "memory");
        const Q4Cut cut = tm.cut[0];
        if (lane == 0) counted_old = counter_at(cut.counter(level_of(cut), bid)).fetch_add(a.key.step);
        counted = true;
      }
      if (counted_at > base + i) stop = min(stop, counted_at - base);
      if (has_next) {
        if (i < m - 1) stop = min(stop, m - 1);
        else seen = __hip_atomic_load(counter_at(bid).p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), look = true;
      }
      const bool ends = stop == i + left;
      for (; i < stop; ++i) {
        constexpr bool kF16 = q4::kF16<T>;
        q4::f32x4_t s[1][2];
        float x[1][8];
        Tiles next;
        bool big;  // the base moves
        auto weights = [&](bool usual) {  // the weights of unit i, and the next K; whether a base moves or V is beyond fp16
          const bool more = i + 1 < m;
          next = tiles(more ? i + 1 : i);
          q4::fold_qk<T, D, 1>(st, u, lane, s);
          fetch_k(next, more);
          if (!usual) {
            const int tokens = t.info & 63;
            st.last[0] = tokens - 1;
            q4::mask_scores<T, D, 1>(st, 0, t.info >> 6 & 3, lane, s);
            q4::clear_dead(u, 0, tokens - 1, lane);
          }
          big = q4::form_weights<T, D, 1>(st, s, a.scale_log2, x);
          __builtin_amdgcn_sched_barrier(0);  // (V is not waited for before the weights are formed)
          return __builtin_amdgcn_ballot_w64(big | (kF16 && q4::beyond_fp16<D>(u))) != 0;
        };
        bool rare = weights(!(t.info & 256));
        // (one way out, and nothing but the usual unit: the sums stay in place, and the
        // loads under way are known)
#pragma unroll 1
        while (!rare & (i + 1 < stop) & !(next.info & 256)) {
          q4::add_weights(st, x);
          q4::fold_pv<kF16, T, D, 1>(st, u, x);
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
        q4::settle_weights<T, D, 1>(st, s, a.scale_log2, big, x);
        q4::fold_pv<false, T, D, 1>(st, u, x);
        fetch_v(next, i + 1 < m);
        t = next;
      }
      if (!ends) continue;
      // the item ends: its output, or the record of this range's part of it
      const float l = rows4_sum(st.l[0]);
      if (!head_partial) {
        const float inv = 1.0f / l;
        if (n < S) {
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            float o[8];
            q4::eight_out(st, 0, j, o);
#pragma unroll
            for (int x = 0; x < 8; ++x) o[x] *= inv;
            q4::store_eight(out + at + 32 * j + 8 * Gl, o);
          }
        }
      } else {
        store_part(0, l, row, g);
        counted_at = base + i + 2;  // (i: the unit after)
      }
      open = false;
    }
  }
  if (open) {  // the range ends inside an item
    const float l = rows4_sum(st.l[0]);
    const int row = __builtin_amdgcn_readfirstlane(tm.last_row), g = __builtin_amdgcn_readfirstlane(tm.last_hb) * W + w;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)seen), hi = __builtin_amdgcn_readfirstlane((uint32_t)(seen >> 32));
    if (look && ((uint64_t)hi << 32 | lo) == a.key.step) {  // its other part has counted: join it from registers
      asm volatile("" ::: "memory");  // (the record's loads stay below the look at the counter)
      const int64_t slot = ((int64_t)(bid + 1) * 2) * W + w;
      const __amdgpu_buffer_rsrc_t r = record_rsrc(a.ws_o + slot * S * D, S * D);
      const int nn = min(n, S - 1);
      float m1, l1;
      f32x4_dev_t o1[D / 16];
      load_dev2(a.ws_ml + (slot * S + nn) * 2, m1, l1);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) o1[j] = load_dev4(r, Rec::chunk(nn, j, Gl) * 4);
      // (q4_join's operations in its order, so the bits do not depend on who joins)
      const float M = fmaxf(st.m[0], m1);
      const float c0 = fast_exp2(st.m[0] - M), c1 = fast_exp2(m1 - M);
      const float inv = 1.0f / fmaf(l1, c1, l * c0);
      if (n < S) {
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          float o[8];
          q4::eight_out(st, 0, j, o);
#pragma unroll
          for (int x = 0; x < 8; ++x) o[x] = fmaf(o1[2 * j + x / 4][x % 4], c1, o[x] * c0) * inv;
          q4::store_eight(out + ((int64_t)row * a.H_q + (int64_t)g * S + n) * D + 32 * j + 8 * Gl, o);
        }
      }
      if (lane == 0) counter_at(bid).store(0);
    } else {
      store_part(head_partial ? 0 : 1, l, row, g);
    }
  }

  // 4. join the cut items
#pragma unroll 1
  for (int j = 0; j < 2; ++j) {
    if (!(j == 0 ? stored[0] : stored[1])) continue;
    const Q4Cut cut = tm.cut[j];
    const int row = __builtin_amdgcn_readfirstlane(tm.job[w][j][0]), g = __builtin_amdgcn_readfirstlane(tm.job[w][j][1]);
    T* o = out + ((int64_t)row * a.H_q + (int64_t)g * S) * D;
    bool early = j == 0 && counted;
#pragma unroll 1
    for (int lv = level_of(cut); lv < 2; ++lv) {
      const int parts = cut.parts(lv, bid);
      int last = 0;
      if (!early) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0);  // the record is stored
      }
      if (lane == 0) {
        DeviceCounter ctr = counter_at(cut.counter(lv, bid));
        last = early ? counter_answer(ctr, a.key, parts, counted_old) : counter_arrive(ctr, a.key, parts);
      }
      early = false;
      if (!__builtin_amdgcn_readfirstlane(last)) break;
      // (a group's record counts in the item next)
      q4_join<T, D, S, W>(a, cut.x0, cut.first(lv, bid), cut.step(lv), parts, lv == 1, w, lane, o);
    }
  }
}

template <typename T, int D, int S>
const void* q4_stream_pick_w(int W) {
  switch (W) {
    case 1: return reinterpret_cast<const void*>(&q4_stream_kernel<T, D, S, 1>);
    case 2: return reinterpret_cast<const void*>(&q4_stream_kernel<T, D, S, 2>);
    case 4: return reinterpret_cast<const void*>(&q4_stream_kernel<T, D, S, 4>);
    case 8: return reinterpret_cast<const void*>(&q4_stream_kernel<T, D, S, 8>);
  }
  return nullptr;
}
template <typename T, int D>
const void* q4_stream_pick(int s, int W) {
  switch (s) {
    case 1: return q4_stream_pick_w<T, D, 1>(W);
    case 2: return q4_stream_pick_w<T, D, 2>(W);
    case 4: return q4_stream_pick_w<T, D, 4>(W);
    case 6: return q4_stream_pick_w<T, D, 6>(W);
    case 8: return q4_stream_pick_w<T, D, 8>(W);
  }
  return nullptr;
}

}  // namespace pa
