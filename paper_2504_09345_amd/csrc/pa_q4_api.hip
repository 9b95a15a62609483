// C ABI of the 4-bit cache (pagedattn_q4.h): host-side validation, planning and
// dispatch.  Validation runs before any HIP call; nothing is kept between calls but
// their number (pa_api.hip), which keys the arrival counters.
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "pa_q4.h"
#include "pagedattn_q4.h"

namespace {

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// The cache's part of dims.
int check_cache(const pa_dims_t* d) {
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

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

int rows_call(const void* k_rows, const void* v_rows, const int32_t* block_table, const int32_t* context_lens,
              const int32_t* query_start_loc, void* k_pages, void* v_pages, const pa_dims_t* d, hipStream_t stream,
              hipError_t (*launch)(int, int, const pa::Q4RowsArgs&, hipStream_t)) {
  const int rc = check_cache(d);
  if (rc != PA_OK) return rc;
  int rows;
  if (query_start_loc != nullptr) {
    if (d->num_q_rows < 0 || (d->num_q_rows > 0 && d->num_seqs == 0)) return PA_EINVAL;
    rows = d->num_q_rows;
  } else {
    if (d->num_q_rows != 0 && d->num_q_rows != d->num_seqs) return PA_EINVAL;
    rows = d->num_seqs;
  }
  if (rows == 0) return PA_OK;
  if ((int64_t)rows + 2 * (int64_t)d->num_seqs > INT32_MAX) return PA_ENOTSUP;  // (32-bit rows and slots)
  if ((pa::q4_row_slots(query_start_loc != nullptr, rows, d->num_seqs) / pa::kQ4RowsWaves + 1) * 64 * pa::kQ4RowsWaves > pa::kQ4MaxThreads)
    return PA_ENOTSUP;
  if (!k_rows || !v_rows || !block_table || !context_lens || !k_pages || !v_pages) return PA_EINVAL;
  if (misaligned(k_rows) || misaligned(v_rows) || misaligned(k_pages) || misaligned(v_pages)) return PA_EINVAL;
  pa::Q4RowsArgs a;
  a.k_rows = k_rows;
  a.v_rows = v_rows;
  a.k_pages = static_cast<uint8_t*>(k_pages);
  a.v_pages = static_cast<uint8_t*>(v_pages);
  a.block_table = block_table;
  a.context_lens = context_lens;
  a.query_start_loc = query_start_loc;
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
// and 31.
constexpr int kPartWaves = 3072;
// Parts beyond those, through the workspace and a second launch: as many as give the
// GPU 2,048 waves of at least kLeastUnits units, at most 64.  (Parts of 4 units cost one
// chunk of 64 rows on 1,500 tokens 17 us instead of 14; 8 or 16 are one as good as the
// other.  Twice the waves: one chunk of 700 rows 31 us instead of 19.)
constexpr int kWavesWanted = 2048, kLeastUnits = 8, kMaxSplit = 64;
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
// tokens 62, where the two alone take 19 and 18.
constexpr int64_t kAloneUnits = 48 * 2048;
constexpr int kAloneColumns = 32;
// Units of a launch of the stream kernel, at most (its counts are 32-bit).
constexpr int64_t kStreamUnits = 1 << 30;

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
  const int64_t units = ((int64_t)d->max_context_len + pa::kQ4Unit - 1) / pa::kQ4Unit;
  p->chunks = varlen && d->max_q_len > 1;
  // every sequence carrying max_q_len rows leaves no decode row (a single row that
  // is there all the same is then a chunk of one)
  p->stream = !(p->chunks && (int64_t)d->max_q_len * d->num_seqs == d->num_q_rows);
  if (p->stream) {
    const int64_t most = kStreamUnits / ((units > 0 ? units : 1) * d->num_kv_heads);
    if (most < 1) return PA_ENOTSUP;
    p->per_launch = most < pa::kQ4StreamSeqs ? (int)most : pa::kQ4StreamSeqs;
    const size_t recs = (size_t)pa::kQ4StreamGroups * 2 * s;
    p->st_o = align256(recs * d->head_dim * sizeof(float));
    p->st_ml = align256(recs * 2 * sizeof(float));
    p->st_flag = align256((size_t)pa::kQ4StreamGroups * pa::kQ4CounterStride * sizeof(unsigned long long));
  }
  if (p->chunks) {
    p->min_rows = p->stream ? 2 : 1;
    // rows of the chunks, as the plan reckons with them: all but a row of each other
    // sequence, and one chunk at least (a batch may hold sequences of no rows)
    const int64_t one = d->max_q_len < p->rows ? d->max_q_len : p->rows;
    int64_t chunk_rows = p->stream ? (int64_t)p->rows - d->num_seqs + 1 : p->rows;
    if (chunk_rows < one) chunk_rows = one;
    const int64_t alone_units = (chunk_rows / pa::q4_positions(1, s) + 1) * d->num_kv_heads *
                                ((d->max_context_len - d->max_q_len / 2) / pa::kQ4Unit + 1);
    p->shared = d->dtype == PA_BF16 && d->max_q_len * (int64_t)s > kAloneColumns && alone_units > kAloneUnits;
    p->blocks = p->shared ? pa::kQ4ChunkBlocks : 1;
    const int64_t slots = p->rows / pa::q4_positions(p->blocks, s) + 1 + (int64_t)d->num_seqs;
    const int64_t items = (chunk_rows / pa::q4_positions(p->blocks, s) + 1) * d->num_kv_heads;
    if (!p->shared)
      while (p->wave_parts < pa::kQ4Waves && items * p->wave_parts * 2 <= kPartWaves && units >= p->wave_parts * 2) p->wave_parts *= 2;
    const int waves = p->shared ? pa::kQ4Waves : p->wave_parts;  // of an item
    int64_t split = kWavesWanted / (items * waves);
    if (split > units / (kLeastUnits * p->wave_parts)) split = units / (kLeastUnits * p->wave_parts);
    if (split > kMaxSplit) split = kMaxSplit;
    const int64_t record = (int64_t)p->rows * d->num_q_heads * (d->head_dim + 2) * (int64_t)sizeof(float);  // of one part
    if (split > kRecordBytes / record) split = kRecordBytes / record;
    if (split < 1) split = 1;
    p->split_units = (int)((units + split - 1) / split);
    p->n_split = (int)((units + p->split_units - 1) / p->split_units);
    const int64_t groups = (slots / (p->shared ? 1 : pa::kQ4Waves / p->wave_parts) + 1) * d->num_kv_heads * p->n_split;
    if (groups * 64 * pa::kQ4Waves > pa::kQ4MaxThreads) return PA_ENOTSUP;
    p->n_slots = (int)slots;
    if (p->n_split > 1) {
      const size_t recs = (size_t)p->rows * d->num_q_heads * p->n_split;
      p->ch_o = align256(recs * d->head_dim * sizeof(float));
      p->ch_ml = align256(recs * 2 * sizeof(float));
    }
  }
  return PA_OK;
}

int attend(const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table, const int32_t* context_lens,
           const int32_t* query_start_loc, float scale, void* out, const pa_dims_t* d, void* workspace, size_t workspace_bytes,
           hipStream_t stream, const pa_timing_t* timing, bool varlen) {
  Plan p;
  const int rc = plan(d, varlen, &p);
  if (rc != PA_OK) return rc;
  if (!isfinite(scale) || !(scale > 0.0f)) return PA_EINVAL;
  if (p.rows > 0) {
    if (!q || !k_pages || !v_pages || !block_table || !context_lens || !out || (varlen && !query_start_loc)) return PA_EINVAL;
    if (misaligned(q) || misaligned(k_pages) || misaligned(v_pages) || misaligned(out) || misaligned(workspace)) return PA_EINVAL;
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
  const float scale_log2 = scale * 1.4426950408889634f;
  if (p.chunks) {
    pa::Q4AttnArgs a{};
    a.q = q;
    a.k_pages = static_cast<const uint8_t*>(k_pages);
    a.v_pages = static_cast<const uint8_t*>(v_pages);
    a.block_table = block_table;
    a.context_lens = context_lens;
    a.query_start_loc = query_start_loc;
    a.out = out;
    a.ws_o = reinterpret_cast<float*>(ws);
    a.ws_ml = reinterpret_cast<float*>(ws + p.ch_o);
    a.bt_stride = d->max_pages_per_seq;
    a.scale_log2 = scale_log2;
    a.B = d->num_seqs;
    a.s = p.s;
    a.H_q = d->num_q_heads;
    a.H_kv = d->num_kv_heads;
    a.rows = p.rows;
    a.num_pages = d->num_pages;
    a.max_context_len = d->max_context_len;
    a.n_slots = p.n_slots;
    a.min_rows = p.min_rows;
    a.max_q_len = d->max_q_len;
    a.n_split = p.n_split;
    a.split_units = p.split_units;
    a.wave_parts = p.wave_parts;
    pa::KernelEvents ev;
    ev.start = begin;
    ev.stop = p.stream ? nullptr : end;
    if ((p.shared ? pa::launch_q4_chunk(d->head_dim, a, stream, ev)
                  : pa::launch_q4_attn(d->dtype, d->head_dim, a, stream, ev)) != hipSuccess)
      return PA_EHIP;
    if (p.n_split > 1 && pa::launch_q4_merge(d->dtype, d->head_dim, a, stream) != hipSuccess) return PA_EHIP;
  }
  if (p.stream) {
    pa::Q4StreamArgs a{};
    const int workgroups = pa::q4_stream_workgroups(d->dtype, d->head_dim, p.s, &a.cus);
    if (workgroups <= 0) return PA_EHIP;
    a.k_pages = static_cast<const uint8_t*>(k_pages);
    a.v_pages = static_cast<const uint8_t*>(v_pages);
    a.ws_o = reinterpret_cast<float*>(ws);
    a.ws_ml = reinterpret_cast<float*>(ws + p.st_o);
    a.ws_flag = reinterpret_cast<unsigned long long*>(ws + p.st_o + p.st_ml);
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
      a.block_table = block_table + (int64_t)b * d->max_pages_per_seq;
      a.context_lens = context_lens + b;
      // (query_start_loc counts rows of the call; a decode call's rows are its sequences)
      a.query_start_loc = varlen ? query_start_loc + b : nullptr;
      a.rows = varlen ? p.rows : a.B;
      a.q = static_cast<const char*>(q) + (varlen ? 0 : b * row_bytes);
      a.out = static_cast<char*>(out) + (varlen ? 0 : b * row_bytes);
      a.key = pa::new_call_key();
      pa::KernelEvents ev;
      ev.start = b == 0 && !p.chunks ? begin : nullptr;
      ev.stop = b + a.B == d->num_seqs ? end : nullptr;
      if (pa::launch_q4_stream(d->dtype, d->head_dim, p.s, a, workgroups, stream, ev) != hipSuccess) return PA_EHIP;
    }
  }
  if (joined != nullptr) (void)hipEventRecord(joined, stream);
  return PA_OK;
}

}  // namespace

extern "C" {

int pa_q4_tile_bytes(int32_t head_dim, size_t* bytes) {
  if (bytes == nullptr) return PA_EINVAL;
  if (head_dim != 64 && head_dim != 128) return PA_ENOTSUP;
  *bytes = (size_t)pa::q4_tile_bytes(head_dim);
  return PA_OK;
}

int pa_kv_append_q4(const void* k_new, const void* v_new, const int32_t* block_table, const int32_t* context_lens,
                    const int32_t* query_start_loc, void* k_pages, void* v_pages, const pa_dims_t* dims, hipStream_t stream) {
  return rows_call(k_new, v_new, block_table, context_lens, query_start_loc, k_pages, v_pages, dims, stream,
                   pa::launch_q4_append);
}

int pa_kv_read_q4(const void* k_pages, const void* v_pages, const int32_t* block_table, const int32_t* context_lens,
                  const int32_t* query_start_loc, void* k_out, void* v_out, const pa_dims_t* dims, hipStream_t stream) {
  return rows_call(k_out, v_out, block_table, context_lens, query_start_loc, const_cast<void*>(k_pages),
                   const_cast<void*>(v_pages), dims, stream, pa::launch_q4_read);
}

int pa_workspace_size_q4(const pa_dims_t* dims, size_t* bytes) {
  if (bytes == nullptr) return PA_EINVAL;
  Plan p;
  const bool varlen = dims != nullptr && (dims->max_q_len > 1 || (dims->num_q_rows != 0 && dims->num_q_rows != dims->num_seqs));
  const int rc = plan(dims, varlen, &p);
  if (rc != PA_OK) return rc;
  *bytes = p.bytes();
  return PA_OK;
}

int paged_attn_q4(const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                  const int32_t* context_lens, float scale, void* out, const pa_dims_t* dims, void* workspace,
                  size_t workspace_bytes, hipStream_t stream, const pa_timing_t* timing) {
  return attend(q, k_pages, v_pages, block_table, context_lens, nullptr, scale, out, dims, workspace, workspace_bytes, stream,
                timing, false);
}

int paged_attn_varlen_q4(const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                         const int32_t* context_lens, const int32_t* query_start_loc, float scale, void* out,
                         const pa_dims_t* dims, void* workspace, size_t workspace_bytes, hipStream_t stream,
                         const pa_timing_t* timing) {
  return attend(q, k_pages, v_pages, block_table, context_lens, query_start_loc, scale, out, dims, workspace, workspace_bytes,
                stream, timing, true);
}

}  // extern "C"
