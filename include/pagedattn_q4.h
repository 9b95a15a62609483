/*
 * pagedattn_q4.h -- the paged KV cache held in 4 bits: quantise new rows as they
 * are written, read rows back, and attend (decode rows and causal prompt
 * chunks).  Beside pagedattn.h, whose conventions hold here too: device pointers,
 * buffers owned by the caller, work enqueued on `stream` and not waited for,
 * host validation before any HIP call, 0 or a negative error code.  The block
 * table, context lengths and query_start_loc are the same arrays.
 *
 * Format (the OCP microscaling format with E2M1 elements).  Each (token, KV head)
 * vector of K and of V is cut into blocks of 32 consecutive dims that share a
 * power-of-two scale.  With a = max |x| over the block, a = m 2^k and
 * 1 <= m < 2, the scale is 2^e with
 *   e = k - 2 where m <= 1.75, else k - 1;  kept within -125 .. 125
 * (e = 0 for a block of zeros), stored as the byte e + 127.  An element is stored
 * as its sign (bit 3) and the code (bits 2..0) of the nearest of
 *   0, 0.5, 1, 1.5, 2, 3, 4, 6
 * to |x| / 2^e, ties to the even code.  (m <= 1.75 puts a at up to 7 2^e, which
 * rounds to 6 2^e and is off by no more than the half step of the elements
 * above 4; a smaller e would clip, a larger one would waste a code.)  The value it
 * stands for, sign * code's value * 2^e, is exact in bf16 and in fp32.  A block
 * that holds an infinity or a NaN gets the byte 255 and codes 0: every element
 * of it reads as NaN.  Bytes 253 and 254 are never written.
 *
 * A token's K and V take D / 2 + D / 32 bytes each per KV head, 68 at D = 128
 * (256 in bf16).
 *
 * Layout of k_pages and v_pages: uint8 [num_pages][num_kv_heads][tile], 16-byte
 * aligned, where a tile of 16 tokens holds 8 D bytes of codes and then D / 2
 * bytes of scales (1,088 bytes at D = 128, 544 at 64: pa_q4_tile_bytes).  Two dims
 * share a byte, the even one in the low half.  With w = D / 8, the codes of dims
 * 2 m and 2 m + 1 of token t are byte
 *   K:  ((m / w) * 16 + t) * w + m % w
 *   V:  ((t / 4) * 16 + m % 16) * w + 4 * (m / 16) + t % 4
 * and the scale of block j of token t is byte 8 D + t * (D / 32) + j of either.
 * (The orders in which a wave's lanes hold matrix-core operands: lane l of a
 * wave reads bytes l w .. l w + w - 1 of a tile, with no exchange between lanes.)
 *
 * dims (pa_dims_t): num_pages, num_kv_heads, head_dim (64 or 128), page_size (16),
 * max_pages_per_seq and max_context_len describe the cache as in pagedattn.h;
 * dtype (PA_BF16 or PA_FP32) is the type of the dense arrays: k_new, v_new,
 * k_out, v_out, q and out.  pages_per_split must be 0.  Arrays that a call writes
 * overlap none that it reads.  Calls of more work than a launch can have threads
 * (appends and reads from 2^26 single rows or 2^28 rows of chunks on) are refused:
 * PA_ENOTSUP.
 */
#ifndef PAGEDATTN_Q4_H
#define PAGEDATTN_Q4_H

#include "pagedattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of one (page, KV head) tile.  Host only.
 * Errors: PA_EINVAL (null pointer), PA_ENOTSUP (head_dim). */
int pa_q4_tile_bytes(int32_t head_dim, size_t *bytes);

/* Quantise new rows into the cache: pa_kv_append with 4-bit pools.  Sequence b
 * writes its rows (query_start_loc[b] .. query_start_loc[b+1]-1, or row b where
 * query_start_loc is NULL) at the LAST L_b positions of its context.
 *   k_new, v_new     [rows][num_kv_heads][head_dim]   device, read, 16-byte aligned
 *   k_pages, v_pages 4-bit pools, see above           device, updated in place
 * A sequence whose chunk is longer than its context or whose context exceeds
 * max_context_len is not written, nor a row whose page entry lies outside
 * [0, num_pages).  Slots that no row names keep every byte.  Two rows of one call
 * must not name the same slot.
 * Errors: PA_EINVAL, PA_ENOTSUP, PA_EHIP. */
int pa_kv_append_q4(const void *k_new, const void *v_new, const int32_t *block_table,
                    const int32_t *context_lens, const int32_t *query_start_loc, void *k_pages,
                    void *v_pages, const pa_dims_t *dims, hipStream_t stream);

/* Read rows back: the values that the cache holds at the positions which
 * pa_kv_append_q4 with the same arguments writes, so the last L_b positions of
 * each context (all of it with L_b = context_lens[b]).
 *   k_out, v_out     [rows][num_kv_heads][head_dim]   device, written, 16-byte aligned
 * Rows of a sequence whose chunk is longer than its context or whose context
 * exceeds max_context_len, and rows whose page entry lies outside [0, num_pages),
 * are NaN.  Rows of no sequence (behind the last one, or of an empty decode
 * context) are left as they were.
 * Errors: PA_EINVAL, PA_ENOTSUP, PA_EHIP. */
int pa_kv_read_q4(const void *k_pages, const void *v_pages, const int32_t *block_table,
                  const int32_t *context_lens, const int32_t *query_start_loc, void *k_out,
                  void *v_out, const pa_dims_t *dims, hipStream_t stream);

/* Bytes of device workspace that a paged_attn_q4 / paged_attn_varlen_q4 call with
 * these dims needs, 64 MiB and an alignment at most.  A call whose dims carry chunked
 * rows (max_q_len > 1 or num_q_rows != num_seqs) is sized as varlen.  Host only; no HIP
 * call. */
int pa_workspace_size_q4(const pa_dims_t *dims, size_t *bytes);

/* Decode attention over the 4-bit cache: paged_attn with 4-bit pools.  Products are
 * formed from the values that the cache stands for, without rounding those, on the
 * matrix cores with fp32 accumulation; softmax bases and sums are fp32, and so are the
 * scores: scale q.k log2 e may be up to 2^27 in magnitude (its steps there are 8; beyond,
 * an output may be NaN).  Queries:
 * bf16 ones as they are, except at head_dim 128, where a query is two e4m3 parts of
 * its row's scale (an error of at most 2^-22 of the row's largest, or 2^-135); fp32 ones as
 * sums of three bf16 parts.  Softmax weights: for bf16 outputs in fp16 where every V
 * of the step is exact in fp16 (scales 2^-23 .. 2^8) and as two bf16 parts elsewhere,
 * for fp32 outputs as three bf16 parts.  Weighted sums do not overflow: an output is
 * finite wherever the weighted mean is.  (A row that sees a V of 2^64 or more, or a NaN
 * block of V, loses what V below 2^-78 beside it would add.)  The same inputs give the
 * same bits.
 * GQA group size num_q_heads / num_kv_heads in {1, 2, 4, 6, 8}.  A row that sees
 * no key (context 0) is zeros; a row of a context above max_context_len, or that
 * sees a page entry outside [0, num_pages), is NaN.  q and out are 16-byte
 * aligned.
 * Errors: PA_EINVAL, PA_ENOTSUP, PA_ENOSPC, PA_EHIP. */
int paged_attn_q4(const void *q, const void *k_pages, const void *v_pages,
                  const int32_t *block_table, const int32_t *context_lens, float scale, void *out,
                  const pa_dims_t *dims, void *workspace, size_t workspace_bytes,
                  hipStream_t stream, const pa_timing_t *timing);

/* Causal chunks and decode rows in one call over the 4-bit cache:
 * paged_attn_varlen with 4-bit pools.  Row j of a chunk of length L in a context C
 * attends to positions 0 .. C - L + j; keys that a row does not see never reach
 * it, whatever they hold (NaN blocks included).  Rows of a chunk longer than its
 * context or than max_q_len are NaN, rows of no sequence are left as they were.
 * max_context_len, beside bounding the contexts, decides how the chunks' work is divided,
 * so it should be no larger than they need: chunks of few rows or keys take up to two
 * and a half times as long under a bound of 32,768 tokens or more (one prompt of 700 rows
 * 41 us instead of 19), also where decode rows beside them need it.
 * Errors: PA_EINVAL, PA_ENOTSUP, PA_ENOSPC, PA_EHIP. */
int paged_attn_varlen_q4(const void *q, const void *k_pages, const void *v_pages,
                         const int32_t *block_table, const int32_t *context_lens,
                         const int32_t *query_start_loc, float scale, void *out,
                         const pa_dims_t *dims, void *workspace, size_t workspace_bytes,
                         hipStream_t stream, const pa_timing_t *timing);

#ifdef __cplusplus
}
#endif

#endif /* PAGEDATTN_Q4_H */
