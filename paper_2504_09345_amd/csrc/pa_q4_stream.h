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
  int32_t page[2];  // -1: outside the pool, or no page
  int32_t info;     // tokens (6 bits) | item start | item end | head block
  int32_t row;
};

template <int W>
struct Q4StreamSmem {
  static constexpr int kTeams = kQ4StreamThreads / 64 / W;
  static constexpr int kUnits = 2048 / kTeams;  // of a table
  int32_t cum[kQ4StreamSeqs + 1];               // units of the sequences before, per head block
  int32_t scan[kQ4StreamThreads / 64];
  struct Team {
    Q4UnitEntry unit[kUnits];
    Q4Cut cut[2];
    int32_t last[2];
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

template <typename T, int D, int S, int W>
__global__ __launch_bounds__(kQ4StreamThreads) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 4 : 2)))
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
  auto begin_of = [&](int x) { return (int)((uint64_t)U * (uint32_t)min(x, G) / (uint32_t)G); };
  auto range_of = [&](int e) { return (int)(((uint64_t)(e + 1) * (uint32_t)G - 1) / (uint32_t)U); };
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
  bool head_partial = false;
  bool stored[2] = {false, false};  // this team's part of the item cut by the range's start, by its end
  int job_row[2] = {0, 0}, job_g[2] = {0, 0};
  auto entry = [&](int i) {
    const Q4UnitEntry& e = tm.unit[i];
    return Q4UnitEntry{{__builtin_amdgcn_readfirstlane(e.page[0]), __builtin_amdgcn_readfirstlane(e.page[1])},
                       __builtin_amdgcn_readfirstlane(e.info), __builtin_amdgcn_readfirstlane(e.row)};
  };
  auto tile_at = [&](const Q4UnitEntry& e, int p) {
    return ((int64_t)max(e.page[p], 0) * a.H_kv + (e.info >> 8) * W + w) * tile;
  };
  auto fetch_k = [&](const Q4UnitEntry& e) {
#pragma unroll
    for (int p = 0; p < 2; ++p) q4::load_k<D>(u, p, a.k_pages + tile_at(e, p), e.page[p] >= 0, lane);
  };
  auto fetch_v = [&](const Q4UnitEntry& e) {
#pragma unroll
    for (int p = 0; p < 2; ++p) q4::load_v<D>(u, p, a.v_pages + tile_at(e, p), e.page[p] >= 0, lane);
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
      const int left = a.context_lens[r] - p * kQ4Unit;  // tokens from the unit on
      Q4UnitEntry e;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        e.page[h] = left > kPage * h ? a.block_table[(int64_t)r * a.bt_stride + 2 * p + h] : -1;
        if (e.page[h] < 0 || e.page[h] >= a.num_pages) e.page[h] = -1;
      }
      e.info = min(left, kQ4Unit) | (p == 0) << 6 | (p == np - 1) << 7 | hb << 8;
      e.row = a.query_start_loc != nullptr ? a.query_start_loc[r] : r;
      tm.unit[i] = e;
      const Q4Cut cut{range_of(x - p), range_of(x - p + np - 1)};
      if (base + i == 0) tm.cut[0] = p == 0 ? Q4Cut{-1, -1} : cut;
      if (base + i == n_units - 1) tm.cut[1] = p == np - 1 ? Q4Cut{-1, -1} : cut;
    }
    __syncthreads();
    if (m <= 0) continue;

    // 3. stream the units: wave w handles KV head hb * W + w of every unit
    Q4UnitEntry e = entry(0);
    fetch_k(e);
    fetch_v(e);
    for (int i = 0; i < m; ++i) {
      const int k = base + i, tokens = e.info & 63;
      const int64_t at = (int64_t)e.row * a.H_q + (int64_t)((e.info >> 8) * W + w) * S + n;
      if ((e.info >> 6 & 1) || k == 0) {
        head_partial = !(e.info >> 6 & 1);
        q4::load_query<T, D>(st.q[0], n < S ? reinterpret_cast<const T*>(a.q) + at * D : nullptr, lane);
        q4::reset(st);
      }
      const Q4UnitEntry next = entry(min(i + 1, m - 1));
      const int bad = (e.page[0] < 0 ? 1 : 0) | (e.page[1] < 0 && tokens > kPage ? 2 : 0);
      q4::f32x4_t s[1][2];
      u32x4 pt[1][q4::kPParts<T>];
      q4::fold_qk<T, D, 1>(st, u, bad, s);
      if (i + 1 < m) fetch_k(next);
      st.last[0] = tokens - 1;
      q4::fold_softmax<T, D, 1>(st, s, 0, tokens < kQ4Unit, a.scale_log2, lane, pt);
      if (tokens < kQ4Unit) q4::clear_dead(u, 0, tokens - 1, lane);
      q4::fold_pv<T, D, 1>(st, u, pt);
      if (i + 1 < m) fetch_v(next);
      if ((e.info >> 7 & 1) || k == n_units - 1) {
        const bool tail_partial = !(e.info >> 7 & 1);
        const float l = rows4_sum(st.l[0]);
        if (!head_partial && !tail_partial) {  // the whole item in this range
          const float inv = 1.0f / l;
          if (n < S) {
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
              float o[8];
              q4::eight_out(st, 0, j, o);
#pragma unroll
              for (int x = 0; x < 8; ++x) o[x] *= inv;
              q4::store_eight(out + at * D + 32 * j + 8 * Gl, o);
            }
          }
        } else {
          const int which = head_partial ? 0 : 1;
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
          const int g = (e.info >> 8) * W + w;
          stored[0] |= which == 0;
          stored[1] |= which == 1;
          job_row[0] = which == 0 ? e.row : job_row[0];
          job_row[1] = which == 1 ? e.row : job_row[1];
          job_g[0] = which == 0 ? g : job_g[0];
          job_g[1] = which == 1 ? g : job_g[1];
        }
      }
      e = next;
    }
  }

  // 4. join the cut items: once a part's record is stored it counts its arrival, and
  // the part that arrives last joins all of them in range order (in two levels
  // beyond 16 parts).  Nothing waits on another workgroup.
  int level[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) level[j] = stored[j] && tm.cut[j].grouped() && !tm.cut[j].group_of_one(bid) ? 0 : 1;
  StreamArgs sa{};
  sa.ws_o = a.ws_o;
  sa.ws_ml = a.ws_ml;
#pragma unroll 1
  for (int step = 0; step < 2; ++step) {
    if (kTeams == 1 && !stored[0] && !stored[1]) break;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);  // the records are stored, in every wave
    __syncthreads();
    if (w == 0 && lane < 2 && (lane == 0 ? stored[0] : stored[1])) {
      const Q4Cut cut = tm.cut[lane];
      const int lv = lane == 0 ? level[0] : level[1];
      DeviceCounter ctr{a.ws_flag + cut.counter(lv, bid)};
      tm.last[lane] = counter_arrive(ctr, a.key, cut.parts(lv, bid));
    }
    __syncthreads();
#pragma unroll 1
    for (int j = 0; j < 2; ++j) {
      const bool mine = (j == 0 ? stored[0] : stored[1]) && tm.last[j];
      const int lv = j == 0 ? level[0] : level[1];
      if (mine) {
        const Q4Cut cut = tm.cut[j];
        T* o = out + ((int64_t)(j == 0 ? job_row[0] : job_row[1]) * a.H_q + (int64_t)(j == 0 ? job_g[0] : job_g[1]) * S) * D;
        merge_records<T, D, S, W, Rec>(sa, cut.x0, cut.first(lv, bid), cut.step(lv), cut.parts(lv, bid), lv == 1, w, lane, o);
      }
      // (a group's record counts in the item next)
      if (j == 0) stored[0] = mine && lv == 0, level[0] = 1;
      else stored[1] = mine && lv == 0, level[1] = 1;
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
