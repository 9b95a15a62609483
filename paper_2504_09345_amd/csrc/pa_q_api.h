// Host side of the caches held in few bits (pagedattn_q4.h, pagedattn_q8.h): validation,
// planning and dispatch, by format.  Validation runs before any HIP call; nothing is kept
// between calls but their number (pa_api.hip), which keys the arrival counters.
#pragma once

#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "pa_q.h"
#include "pagedattn.h"

namespace pa {
namespace {

// The arrays of a call's cache.
struct QCache {
  const void* k_pages;
  const void* v_pages;
  const uint8_t* scales;  // nullptr: in the tiles
  const int32_t* block_table;
  const int32_t* context_lens;
  const int32_t* query_start_loc;
};

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// The cache's part of dims.
inline int check_cache(const pa_dims_t* d) {
  if (d == nullptr) return PA_EINVAL;
  if (d->num_seqs < 0 || d->num_kv_heads <= 0 || d->num_pages < 0 || d->max_pages_per_seq < 0 || d->max_context_len < 0 ||
      d->pages_per_split != 0)
    return PA_EINVAL;
  if (d->max_context_len > 1 << 30) return PA_ENOTSUP;  // (page counts are 32-bit)
  if (d->dtype != PA_BF16 && d->dtype != PA_FP32) return PA_ENOTSUP;
  if (d->head_dim != 64 && d->head_dim != 128) return PA_ENOTSUP;
  if (d->page_size != 16) return PA_ENOTSUP;
  if (((int64_t)d->max_context_len + 15) / 16 > d->max_pages_per_seq) return PA_EINVAL;
  return PA_OK;
}

inline bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// group: tokens of a slot.
inline int rows_call(const void* k_rows, const void* v_rows, const QCache& c, bool scaled, int group, const pa_dims_t* d, hipStream_t stream,
              hipError_t (*launch)(int, int, const QRowsArgs&, hipStream_t)) {
  const int rc = check_cache(d);
  if (rc != PA_OK) return rc;
  int rows;
  if (c.query_start_loc != nullptr) {
    if (d->num_q_rows < 0 || (d->num_q_rows > 0 && d->num_seqs == 0)) return PA_EINVAL;
    rows = d->num_q_rows;
  } else {
    if (d->num_q_rows != 0 && d->num_q_rows != d->num_seqs) return PA_EINVAL;
    rows = d->num_seqs;
  }
  if (rows == 0) return PA_OK;
  if ((int64_t)rows + 2 * (int64_t)d->num_seqs > INT32_MAX) return PA_ENOTSUP;  // (32-bit rows and slots)
  if ((q_row_slots(c.query_start_loc != nullptr, rows, d->num_seqs, group) / kQRowsWaves + 1) * 64 * kQRowsWaves > kQMaxThreads)
    return PA_ENOTSUP;
  if (!k_rows || !v_rows || !c.block_table || !c.context_lens || !c.k_pages || !c.v_pages || (scaled && !c.scales)) return PA_EINVAL;
  if (misaligned(k_rows) || misaligned(v_rows) || misaligned(c.k_pages) || misaligned(c.v_pages)) return PA_EINVAL;
  QRowsArgs a;
  a.k_rows = k_rows;
  a.v_rows = v_rows;
  a.k_pages = static_cast<uint8_t*>(const_cast<void*>(c.k_pages));
  a.v_pages = static_cast<uint8_t*>(const_cast<void*>(c.v_pages));
  a.scales = const_cast<uint8_t*>(c.scales);
  a.block_table = c.block_table;
  a.context_lens = c.context_lens;
  a.query_start_loc = c.query_start_loc;
  a.bt_stride = d->max_pages_per_seq;
  a.B = d->num_seqs;
  a.rows = rows;
  a.H_kv = d->num_kv_heads;
  a.num_pages = d->num_pages;
  a.max_context_len = d->max_context_len;
  return launch(d->dtype, d->head_dim, a, stream) == hipSuccess ? PA_OK : PA_EHIP;
}

struct Plan {
  int s = 0, rows = 0;
  bool stream = false, chunks = false;  // which kernels the call needs
  // decode rows
  int per_launch = 0;  // sequences of a launch
  // chunk rows
  bool shared = false;  // V's operands shared by a workgroup
  int blocks = 1, n_slots = 0, n_split = 1, split_units = 1, min_rows = 2, wave_parts = 1;
  size_t st_o = 0, st_ml = 0, st_flag = 0, ch_o = 0, ch_ml = 0;
  size_t stream_bytes() const { return st_o + st_ml + st_flag; }
  size_t chunk_bytes() const { return ch_o + ch_ml; }
  // (the kernels run one after the other and share the workspace)
  size_t bytes() const { return stream_bytes() > chunk_bytes() ? stream_bytes() : chunk_bytes(); }
};

// Waves of a workgroup that share an item's units and join their parts in LDS: 2 or 4
// while the GPU still holds all of them at once (256 CUs of 12 waves).  Shared and
// alone, 32 query heads over 8: a chunk of 16 rows on 200 tokens 7 and 10 us, of 300 9
// and 11, of 64 on 1,500 14 and 18, 4 of 60 on 3,000 34 and 41, 16 of 8 on 2,000 25
// and 31.  (8 bits: 6.4 and 8.5, 7.0 and 10.1, 12.0 and 16.6, 25 and 33 with waves of 16 columns, 17 and 24; four
// times as many waves: one chunk of 1,400 rows 41 us instead of 36, of 700 18 and 15.)
constexpr int kPartWaves = 256 * 12;
// Twice as many waves of 32 columns where each keeps so many units: the longest items end
// sooner.  (Never, from 24 and from 8 on: one chunk of 1,400 rows 36, 36 and 40 us, of 1,700
// 46, 43 and 43, of 2,000 52, 50 and 50, of 2,800 78, 83 and 82; at head_dim 64 of 1,700 34,
// 26 and 26, of 2,600 54, 46 and 46; 8 of 230 on 500 26, 26 and 31.)
constexpr int kLongPart = 24;
// Parts beyond those, through the workspace and a second launch: as many as give the
// GPU 2,048 waves of at least kLeastUnits units, at most 64.  (Parts of 4 units cost one
// chunk of 64 rows on 1,500 tokens 17 us instead of 14; 8 or 16 are one as good as the
// other.  Twice the waves: one chunk of 700 rows 31 us instead of 19.)  (8 bits: units of
// at least 4, 8 or 16 are one as good as the other but for 11.3, 10.0 and 10.0 us of one
// chunk of 64 rows on 1,500 tokens at head_dim 64.)  Of 32 columns, which two fit a SIMD of,
// 2,560, so that a division's rest leaves no half of the GPU idle: with 1,024, 2,048, 2,560
// and 4,096 4 chunks of 64 rows on 16,000 tokens 98, 98, 83 and 88 us, one on 30,000 68, 55,
// 50 and 62, 2 of 120 on 20,000 118, 98, 98 and 106, 4 of 56 on 5,000 37, 35, 35 and 42.
constexpr int kWavesWanted = 2048, kWideWavesWanted = 2560, kLeastUnits = 8, kMaxSplit = 64;
// Bytes of all parts' records, which the host can only reckon for every row of the call:
// it does not know which are of chunks, nor does the grid.  With bounds of 32, 64, 128 and
// 4,096 MiB, 32 query heads over 8: two rows on 65,536 tokens beside 512 decode rows of
// 500 tokens 169, 128, 197 and 624 us, beside 256 87, 109, 180 and 329; on 131,072 beside
// 1,023 of 300 708, 346, 298 and 1,200, beside 4,096 of 100 805, 804, 805 and 4,455; 16
// rows on 32,768 beside 512 of 500 118, 135, 179 and 180.
constexpr int64_t kRecordBytes = 64 << 20;
// Which kernel takes a call's chunks (bf16): waves of 16 columns, each alone, or
// workgroups of 128 columns that share V's operands.  The latter spend a third less
// per column and unit, but need the columns (a chunk of at most 32 leaves three of
// four waves without) and enough work: a wave alone is through its units sooner, and
// there are more of them.  The line is 48 units for each of 2,048 waves, by the
// longest context that the call declares, which is all that the host knows of the
// chunks' own: a bound far above those takes the wrong kernel (below).  Alone and together, 32 query heads over 8:
// one chunk of 700 rows 17 and 32 us, of 1,400 37 and 46, of 2,000 57 and 62, of 2,800
// 98 and 90, of 4,000 171 and 145; 8 of 205-256 rows on 500 tokens 53 and 57; 8 of
// 320-400 on 300 67 and 66; 4 of 240-300 on 1,000 59 and 56; 4 of 48-60 on 3,000 34 and
// 54; 2 of 102-128 on 20,000 153 and 123; 16 of 8 rows on 2,000 24 and 45.  Declared as
// they are and as 4,096, 32,768 and 131,072: one of 16 rows on 200 8.4, 11.0, 11.2 and
// 20.6; one of 700 19.0 and 40.7 with any of them; 4 of 64 on 300 10.7, 10.7, 23.5 and
// 23.6; 16 of 8 on 2,000 17.5 with all; and one of 700 beside a decode row of 32,768
// tokens 62, where the two alone take 19 and 18.  (8 bits: 6.3, 9.1, 11.3 and 11.4; 14.7 and
// 19.5 with any; 9.2 and 19.0 with any; 17.7 with all; one of 2,000 48 with all; 4 of 60 on
// 3,000 38, 44, 57 and 57.)
template <class F> constexpr int64_t kAloneUnits = 0;
template <> inline constexpr int64_t kAloneUnits<q4::Format> = 48 * 2048;
// The 8-bit cache's large calls have waves of 32 columns, each alone: K's and V's
// conversions are paid once for both halves, with no barrier.  (Workgroups of 128 columns
// that share the conversions' results through LDS were slower throughout: 8 chunks of
// 2,048 rows on 0, 290, .. 2,030 tokens 635 us and 583, at head_dim 64 386 and 353; one of
// 4,000 167 and 144.)  The line
// is 15 units for each of 2,048 waves.  Of 16 columns and of 32, 32 query heads over 8,
// head_dim 128: one chunk of 700 rows 15.6 and 20.5 us, of 1,000 24.9 and 22.3, of 1,400
// 36.9 and 36.3, of 2,000 56 and 50, of 2,600 80 and 74; 8 of 300 24.4 and 25.1, of 200 on
// 400 24.8 and 23.4, of 230 on 500 32 and 28; 4 of 128 on 1,000 19.3 and 18.8, of 56 on
// 3,000 25.7 and 29.3, on 5,000 39 and 37; but of 60, of whose items the last are half
// empty, on 3,000 25.3 and 39, on 5,000 39 and 50; 2 of 256 on 8,000 104 and 77; at head_dim 64
// one of 700 10.5 and 11.0, of 1,000 18.3 and 15.5, of 2,000 39 and 31; with 64 query heads
// one of 700 21.5 and 24.4, of 1,400 53 and 50, with 8 of 2,000 22 and 20, with 48 (12 of 16
// columns used, or 30 of 32) 8 of 512 on 1,000 153 and 105.  (fp32 keeps to 16: a third part
// of each query leaves no room; one of 2,000 95 and 100 us, at head_dim 64 64 and 62.)
template <> inline constexpr int64_t kAloneUnits<q8::Format> = 15 * 2048;
template <class F> constexpr bool kWideWaves = false;
template <> inline constexpr bool kWideWaves<q8::Format> = true;
constexpr int kAloneColumns = 32;
// Units of a launch of the stream kernel, at most (its counts are 32-bit).
constexpr int64_t kStreamUnits = 1 << 30;

template <class F>
int plan(const pa_dims_t* d, bool varlen, Plan* p) {
  const int rc = check_cache(d);
  if (rc != PA_OK) return rc;
  if (d->num_q_heads <= 0 || d->num_q_heads % d->num_kv_heads != 0) return PA_EINVAL;
  const int s = p->s = d->num_q_heads / d->num_kv_heads;
  if (s != 1 && s != 2 && s != 4 && s != 6 && s != 8) return PA_ENOTSUP;
  if (varlen) {
    if (d->num_q_rows < 0 || d->max_q_len < 0) return PA_EINVAL;
    if (d->num_q_rows > 0 && (d->max_q_len < 1 || d->num_seqs == 0 || d->max_q_len > d->max_context_len)) return PA_EINVAL;
    p->rows = d->num_q_rows;
  } else {
    if ((d->num_q_rows != 0 && d->num_q_rows != d->num_seqs) || d->max_q_len < 0 || d->max_q_len > 1) return PA_EINVAL;
    p->rows = d->num_seqs;
  }
  if (p->rows == 0) return PA_OK;
  if ((int64_t)p->rows * d->num_q_heads > INT32_MAX) return PA_ENOTSUP;
  const int64_t units = ((int64_t)d->max_context_len + kQUnit - 1) / kQUnit;
  p->chunks = varlen && d->max_q_len > 1;
  // every sequence carrying max_q_len rows leaves no decode row (a single row that
  // is there all the same is then a chunk of one)
  p->stream = !(p->chunks && (int64_t)d->max_q_len * d->num_seqs == d->num_q_rows);
  if (p->stream) {
    const int64_t most = kStreamUnits / ((units > 0 ? units : 1) * d->num_kv_heads);
    if (most < 1) return PA_ENOTSUP;
    p->per_launch = most < kQStreamSeqs ? (int)most : kQStreamSeqs;
    const size_t recs = (size_t)kQStreamGroups * 2 * s;
    p->st_o = align256(recs * d->head_dim * sizeof(float));
    p->st_ml = align256(recs * 2 * sizeof(float));
    p->st_flag = align256((size_t)kQStreamGroups * kQCounterStride * sizeof(unsigned long long));
  }
  if (p->chunks) {
    p->min_rows = p->stream ? 2 : 1;
    // rows of the chunks, as the plan reckons with them: all but a row of each other
    // sequence, and one chunk at least (a batch may hold sequences of no rows)
    const int64_t one = d->max_q_len < p->rows ? d->max_q_len : p->rows;
    int64_t chunk_rows = p->stream ? (int64_t)p->rows - d->num_seqs + 1 : p->rows;
    if (chunk_rows < one) chunk_rows = one;
    const int64_t alone_units = (chunk_rows / q_positions(1, s) + 1) * d->num_kv_heads *
                                ((d->max_context_len - d->max_q_len / 2) / kQUnit + 1);
    const bool large = d->dtype == PA_BF16 && d->max_q_len * (int64_t)s > kAloneColumns && alone_units > kAloneUnits<F>;
    p->shared = large && !kWideWaves<F>;
    p->blocks = p->shared ? kQChunkBlocks : large ? 2 : 1;
    const int64_t slots = p->rows / q_positions(p->blocks, s) + 1 + (int64_t)d->num_seqs;
    const int64_t items = (chunk_rows / q_positions(p->blocks, s) + 1) * d->num_kv_heads;
    if (!p->shared)
      while (p->wave_parts < kQWaves && units >= p->wave_parts * 2 &&
             items * p->wave_parts * 2 <= (p->blocks == 2 && units >= p->wave_parts * 2 * kLongPart ? 2 : 1) * kPartWaves)
        p->wave_parts *= 2;
    const int waves = p->shared ? kQWaves : p->wave_parts;  // of an item
    int64_t split = (p->blocks == 2 ? kWideWavesWanted : kWavesWanted) / (items * waves);
    if (split > units / (kLeastUnits * p->wave_parts)) split = units / (kLeastUnits * p->wave_parts);
    if (split > kMaxSplit) split = kMaxSplit;
    const int64_t record = (int64_t)p->rows * d->num_q_heads * (d->head_dim + 2) * (int64_t)sizeof(float);  // of one part
    if (split > kRecordBytes / record) split = kRecordBytes / record;
    if (split < 1) split = 1;
    p->split_units = (int)((units + split - 1) / split);
    p->n_split = (int)((units + p->split_units - 1) / p->split_units);
    const int64_t groups = (slots / (p->shared ? 1 : kQWaves / p->wave_parts) + 1) * d->num_kv_heads * p->n_split;
    if (groups * 64 * kQWaves > kQMaxThreads) return PA_ENOTSUP;
    p->n_slots = (int)slots;
    if (p->n_split > 1) {
      const size_t recs = (size_t)p->rows * d->num_q_heads * p->n_split;
      p->ch_o = align256(recs * d->head_dim * sizeof(float));
      p->ch_ml = align256(recs * 2 * sizeof(float));
    }
  }
  return PA_OK;
}

template <class F>
int workspace_bytes_of(const pa_dims_t* d, size_t* bytes) {
  if (bytes == nullptr) return PA_EINVAL;
  Plan p;
  const bool varlen = d != nullptr && (d->max_q_len > 1 || (d->num_q_rows != 0 && d->num_q_rows != d->num_seqs));
  const int rc = plan<F>(d, varlen, &p);
  if (rc != PA_OK) return rc;
  *bytes = p.bytes();
  return PA_OK;
}

// scaled: the format has scales beside its tiles.
template <class F>
int attend(const void* q, const QCache& c, bool scaled, float scale, void* out, const pa_dims_t* d, void* workspace,
           size_t workspace_bytes, hipStream_t stream, const pa_timing_t* timing, bool varlen) {
  Plan p;
  const int rc = plan<F>(d, varlen, &p);
  if (rc != PA_OK) return rc;
  if (!isfinite(scale) || !(scale > 0.0f)) return PA_EINVAL;
  if (p.rows > 0) {
    if (!q || !c.k_pages || !c.v_pages || !c.block_table || !c.context_lens || !out || (varlen && !c.query_start_loc) || (scaled && !c.scales))
      return PA_EINVAL;
    if (misaligned(q) || misaligned(c.k_pages) || misaligned(c.v_pages) || misaligned(out) || misaligned(workspace)) return PA_EINVAL;
    if (p.bytes() > 0 && (workspace == nullptr || workspace_bytes < p.bytes())) return PA_ENOSPC;
  }
  const hipEvent_t begin = timing ? timing->attn_begin : nullptr, end = timing ? timing->attn_end : nullptr;
  const hipEvent_t joined = timing ? timing->reduce_end : nullptr;
  if (p.rows == 0) {
    for (hipEvent_t ev : {begin, end, joined})
      if (ev != nullptr) (void)hipEventRecord(ev, stream);
    return PA_OK;
  }
  char* ws = static_cast<char*>(workspace);
  // Without pages nothing of a tile is read, but scales are: the decode kernel's of the
  // first tile (any two bytes), the chunk kernels' none, as a context above the bound.
  const bool no_scales = scaled && d->num_pages == 0;
  const uint8_t* scales = no_scales ? reinterpret_cast<const uint8_t*>(c.context_lens) : c.scales;
  const float scale_log2 = scale * 1.4426950408889634f;
  if (p.chunks) {
    QAttnArgs a{};
    a.q = q;
    a.k_pages = static_cast<const uint8_t*>(c.k_pages);
    a.v_pages = static_cast<const uint8_t*>(c.v_pages);
    a.block_table = c.block_table;
    a.context_lens = c.context_lens;
    a.query_start_loc = c.query_start_loc;
    a.out = out;
    a.ws_o = reinterpret_cast<float*>(ws);
    a.ws_ml = reinterpret_cast<float*>(ws + p.ch_o);
    a.scales = scales;
    a.bt_stride = d->max_pages_per_seq;
    a.scale_log2 = scale_log2;
    a.B = d->num_seqs;
    a.s = p.s;
    a.H_q = d->num_q_heads;
    a.H_kv = d->num_kv_heads;
    a.rows = p.rows;
    a.num_pages = d->num_pages;
    a.max_context_len = no_scales ? -1 : d->max_context_len;
    a.n_slots = p.n_slots;
    a.blocks = p.blocks;
    a.min_rows = p.min_rows;
    a.max_q_len = d->max_q_len;
    a.n_split = p.n_split;
    a.split_units = p.split_units;
    a.wave_parts = p.wave_parts;
    KernelEvents ev;
    ev.start = begin;
    ev.stop = p.stream ? nullptr : end;
    hipError_t e;
    if constexpr (kWideWaves<F>) e = launch_q_attn<F>(d->dtype, d->head_dim, a, stream, ev);
    else e = p.shared ? launch_q_chunk<F>(d->head_dim, a, stream, ev) : launch_q_attn<F>(d->dtype, d->head_dim, a, stream, ev);
    if (e != hipSuccess) return PA_EHIP;
    if (p.n_split > 1 && launch_q_merge(d->dtype, d->head_dim, a, stream) != hipSuccess) return PA_EHIP;
  }
  if (p.stream) {
    QStreamArgs a{};
    const int workgroups = q_stream_workgroups<F>(d->dtype, d->head_dim, p.s, &a.cus);
    if (workgroups <= 0) return PA_EHIP;
    a.k_pages = static_cast<const uint8_t*>(c.k_pages);
    a.v_pages = static_cast<const uint8_t*>(c.v_pages);
    a.ws_o = reinterpret_cast<float*>(ws);
    a.ws_ml = reinterpret_cast<float*>(ws + p.st_o);
    a.ws_flag = reinterpret_cast<unsigned long long*>(ws + p.st_o + p.st_ml);
    a.scales = scales;
    a.bt_stride = d->max_pages_per_seq;
    a.scale_log2 = scale_log2;
    a.H_q = d->num_q_heads;
    a.H_kv = d->num_kv_heads;
    a.num_pages = d->num_pages;
    a.max_context_len = d->max_context_len;
    a.max_q_len = d->max_q_len;
    a.write_long = !p.chunks;
    const size_t row_bytes = (size_t)d->num_q_heads * d->head_dim * (d->dtype == PA_BF16 ? 2 : 4);
    for (int b = 0; b < d->num_seqs; b += p.per_launch) {
      a.B = d->num_seqs - b < p.per_launch ? d->num_seqs - b : p.per_launch;
      a.block_table = c.block_table + (int64_t)b * d->max_pages_per_seq;
      a.context_lens = c.context_lens + b;
      // (query_start_loc counts rows of the call; a decode call's rows are its sequences)
      a.query_start_loc = varlen ? c.query_start_loc + b : nullptr;
      a.rows = varlen ? p.rows : a.B;
      a.q = static_cast<const char*>(q) + (varlen ? 0 : b * row_bytes);
      a.out = static_cast<char*>(out) + (varlen ? 0 : b * row_bytes);
      a.key = new_call_key();
      KernelEvents ev;
      ev.start = b == 0 && !p.chunks ? begin : nullptr;
      ev.stop = b + a.B == d->num_seqs ? end : nullptr;
      if (launch_q_stream<F>(d->dtype, d->head_dim, p.s, a, workgroups, stream, ev) != hipSuccess) return PA_EHIP;
    }
  }
  if (joined != nullptr) (void)hipEventRecord(joined, stream);
  return PA_OK;
}

}  // namespace
}  // namespace pa
