/*
 * pagedattn_q8.h -- the paged KV cache held in 8 bits with a scale for each page and
 * head: quantise new rows as they are written, read rows back, and attend (decode rows
 * and causal prompt chunks).  Beside pagedattn.h, whose conventions hold here too: device
 * pointers, buffers owned by the caller, work enqueued on `stream` and not waited for,
 * host validation before any HIP call, 0 or a negative error code.  The block table,
 * context lengths and query_start_loc are the same arrays.
 *
 * Format.  The 16 tokens of a page share, for each KV head and for K and V each, a
 * power-of-two scale 2^e, stored as the byte e + 127; elements are e4m3 (the OCP 8-bit
 * float: 4 exponent bits of bias 7, 3 mantissa bits, 448 the largest, 127 and 255 NaN).
 * With a = max |x| over the finite x that the page holds of the head, a = m 2^k and
 * 1 <= m < 2,
 *   e = k - 8 where m <= 1.75, else k - 7;  kept within -110 .. 119
 * (-110 for a page of zeros), so that a lies within (224, 448] 2^e.  An x is held as
 * x / 2^e to the nearest e4m3, ties to even, 448 where it is more; an infinity or a NaN
 * as NaN.  (A float for the elements: tokens of a page differ in size, and one of 2^-10
 * of the page's largest still has its four significant bits.  A power of two for the
 * scale: values of other pages' scales are exact in bf16, and so is their rescaling but
 * for the smallest.)
 *
 * A row written to slot 0 of a page begins it: its scale is that of the rows which the
 * call writes to it.  A call that writes later slots of a page keeps its scale where
 * that is large enough; where the new rows need a larger one the page takes that, and
 * the earlier slots' values (below the call's first slot of the page) are rounded to it
 * once more.  So a page's scale is that of the largest value written since it was begun.
 *
 * A token's K and V take head_dim bytes each per KV head and a byte per 16 tokens.
 *
 * Layout.  k_pages and v_pages: uint8 [num_pages][num_kv_heads][16 head_dim], 16-byte
 * aligned.  scales: uint8 [num_pages][num_kv_heads][2], K's byte then V's, 2-byte
 * aligned.  The code of dim d of token t is byte
 *   K:  ((d / 16) * 16 + t) * 16 + d % 16
 *   V:  (d / 64) * 1024 + ((t / 4) * 16 + d % 32 / 2) * 16 + (d / 32 % 2) * 8 + (d % 2) * 4 + t % 4
 * of a (page, KV head) tile.  (The orders in which a wave's lanes hold matrix-core
 * operands: lane l of a wave reads bytes 16 l .. 16 l + 15 of each KiB, with no exchange
 * between lanes.)  A page with a scale byte outside 17 .. 246, which no call writes, may
 * read as anything.
 *
 * dims (pa_dims_t): num_pages, num_kv_heads, head_dim (64 or 128), page_size (16),
 * max_pages_per_seq and max_context_len describe the cache as in pagedattn.h;
 * dtype (PA_BF16 or PA_FP32) is the type of the dense arrays: k_new, v_new,
 * k_out, v_out, q and out.  pages_per_split must be 0.  Arrays that a call writes
 * overlap none that it reads.  Calls of more work than a launch can have threads are
 * refused, PA_ENOTSUP: appends and reads from 2^26 - 4 groups of rows on, where a single
 * row of a decode call is a group, of a call with query_start_loc 16 appended rows or 4
 * read ones are, and each sequence counts two more (so somewhat below 2^30 appended or
 * 2^28 read rows).
 */
#ifndef PAGEDATTN_Q8_H
#define PAGEDATTN_Q8_H

#include "pagedattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Quantise new rows into the cache: pa_kv_append with 8-bit pools.  Sequence b
 * writes its rows (query_start_loc[b] .. query_start_loc[b+1]-1, or row b where
 * query_start_loc is NULL) at the LAST L_b positions of its context.
 *   k_new, v_new     [rows][num_kv_heads][head_dim]   device, read, 16-byte aligned
 *   k_pages, v_pages, scales                          device, updated in place
 * A sequence whose chunk is longer than its context or whose context exceeds
 * max_context_len is not written, nor rows whose page entry lies outside
 * [0, num_pages).  Slots after a call's last one of a page keep every byte, and so do
 * the slots before its first where the scale stays.  A page must not be written for two
 * sequences of one call (pages that sequences share are whole, and never written again).
 * Errors: PA_EINVAL, PA_ENOTSUP, PA_EHIP. */
int pa_kv_append_q8(const void *k_new, const void *v_new, const int32_t *block_table,
                    const int32_t *context_lens, const int32_t *query_start_loc, void *k_pages,
                    void *v_pages, uint8_t *scales, const pa_dims_t *dims, hipStream_t stream);

/* Read rows back: the values that the cache holds at the positions which
 * pa_kv_append_q8 with the same arguments writes, so the last L_b positions of
 * each context (all of it with L_b = context_lens[b]); exact in either type.
 *   k_out, v_out     [rows][num_kv_heads][head_dim]   device, written, 16-byte aligned
 * Rows of a sequence whose chunk is longer than its context or whose context
 * exceeds max_context_len, and rows whose page entry lies outside [0, num_pages),
 * are NaN.  Rows of no sequence (behind the last one, or of an empty decode
 * context) are left as they were.
 * Errors: PA_EINVAL, PA_ENOTSUP, PA_EHIP. */
int pa_kv_read_q8(const void *k_pages, const void *v_pages, const uint8_t *scales,
                  const int32_t *block_table, const int32_t *context_lens,
                  const int32_t *query_start_loc, void *k_out, void *v_out, const pa_dims_t *dims,
                  hipStream_t stream);

/* Bytes of device workspace that a paged_attn_q8 / paged_attn_varlen_q8 call with
 * these dims needs, 64 MiB and an alignment at most.  A call whose dims carry chunked
 * rows (max_q_len > 1 or num_q_rows != num_seqs) is sized as varlen.  Host only; no HIP
 * call. */
int pa_workspace_size_q8(const pa_dims_t *dims, size_t *bytes);

/* Decode attention over the 8-bit cache: paged_attn with 8-bit pools.  Products are
 * formed from the values that the cache stands for, without rounding those, on the
 * matrix cores with fp32 accumulation; softmax bases and sums are fp32, and so are the
 * scores: scale q.k log2 e may be up to 2^27 in magnitude (its steps there are 8; beyond,
 * an output may be NaN).  Queries:
 * bf16 ones as they are, fp32 ones as sums of three bf16 parts.  Softmax weights: for bf16 outputs in fp16 where every V
 * of the step is exact in fp16 (scales 2^-15 .. 2^7) and as two bf16 parts elsewhere,
 * for fp32 outputs as three bf16 parts.  Weighted sums do not overflow: an output is
 * finite wherever the weighted mean is.  (A row that sees a page whose V has a scale of
 * 2^56 or more loses what V below 2^-78 beside it would add.)  The same inputs give the
 * same bits.
 * GQA group size num_q_heads / num_kv_heads in {1, 2, 4, 6, 8}.  A row that sees
 * no key (context 0) is zeros; a row of a context above max_context_len, or that
 * sees a page entry outside [0, num_pages), is NaN.  q and out are 16-byte
 * aligned.
 * Errors: PA_EINVAL, PA_ENOTSUP, PA_ENOSPC, PA_EHIP. */
int paged_attn_q8(const void *q, const void *k_pages, const void *v_pages, const uint8_t *scales,
                  const int32_t *block_table, const int32_t *context_lens, float scale, void *out,
                  const pa_dims_t *dims, void *workspace, size_t workspace_bytes,
                  hipStream_t stream, const pa_timing_t *timing);

/* Causal chunks and decode rows in one call over the 8-bit cache:
 * paged_attn_varlen with 8-bit pools.  Row j of a chunk of length L in a context C
 * attends to positions 0 .. C - L + j; keys that a row does not see never reach
 * it, whatever they hold (NaN included), though they share their page's scale.  Rows of a
 * chunk longer than its
 * context or than max_q_len are NaN, rows of no sequence are left as they were.
 * max_context_len, beside bounding the contexts, decides how the chunks' work is divided,
 * so it should be no larger than they need.
 * Errors: PA_EINVAL, PA_ENOTSUP, PA_ENOSPC, PA_EHIP. */
int paged_attn_varlen_q8(const void *q, const void *k_pages, const void *v_pages,
                         const uint8_t *scales, const int32_t *block_table,
                         const int32_t *context_lens, const int32_t *query_start_loc, float scale,
                         void *out, const pa_dims_t *dims, void *workspace,
                         size_t workspace_bytes, hipStream_t stream, const pa_timing_t *timing);

#ifdef __cplusplus
}
#endif

#endif /* PAGEDATTN_Q8_H */
