/*
 * pa_rope.h -- rotary positions of new query and key rows, the step before the cache
 * write (pa_kv_append and its siblings) and attention.  Beside pagedattn.h, whose
 * conventions hold here too.
 *
 * With n = rot_dim / 2 pairs, pair i of a head's vector, (x, y), at position p becomes
 *   factor * (x cos a - y sin a,  y cos a + x sin a),   a = p * inv_freq[i]
 * where the pair is dims i and i + n (interleaved = 0) or dims 2 i and 2 i + 1
 * (interleaved = 1).  Dims from rot_dim on stay as they are.
 *
 * inv_freq is in 64 bits, and so are the angles until whole turns are taken off them: a
 * frequency or a product rounded to 32 bits is off by 2^-24 of itself, at position 2^20
 * 1/16 of a radian.  The angles' error is at most 1.3 2^-52 of a (three roundings to 2^-53,
 * that of 1 / 2 pi among them); cosine and sine are in 32 bits, the
 * products and sums too, and a result is rounded once to the type.
 */
#ifndef PA_ROPE_H
#define PA_ROPE_H

#include "pagedattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How rows are rotated (host memory, read during the call only). */
typedef struct pa_rope {
  const double *inv_freq;  /* device, [rot_dim / 2], 8-byte aligned: radians per token */
  float factor;            /* of the rotated dims; finite */
  int32_t rot_dim;         /* even, 2 .. head_dim */
  int32_t interleaved;     /* 0: pair i is dims i, i + rot_dim / 2; 1: dims 2 i, 2 i + 1 */
  int64_t q_stride;        /* elements from a row to the next: at least num_q_heads * head_dim, */
  int64_t k_stride;        /* or 0 for just that (keys: num_kv_heads); whole 16 bytes */
  int64_t q_out_stride;
  int64_t k_out_stride;
} pa_rope_t;

/* Rotate rows of queries and keys.
 *   q      [rows][num_q_heads][head_dim]   device, read, rows q_stride apart
 *   k      [rows][num_kv_heads][head_dim]  device, read, rows k_stride apart
 *   q_out, k_out  the same shapes          device, written
 * All 16-byte aligned.  q and q_out may both be NULL (keys alone), so may k and k_out.
 * An output may be its input (q_out == q with the same stride), and q and k may be parts
 * of the same rows (as a joint projection leaves them); apart from that no written element
 * may be a read or written one elsewhere.
 *
 * Positions: where `positions` (device, int32 [rows]) is not NULL they are those, every
 * row of the call is rotated, and context_lens and query_start_loc are not read.  Else row
 * query_start_loc[b] + j is at position context_lens[b] - L_b + j (where pa_kv_append
 * writes it); with query_start_loc NULL (decode) row b is at context_lens[b] - 1.  Rows
 * of a sequence whose chunk is longer than its context, or whose context exceeds
 * max_context_len, are NaN; rows of no sequence (behind the last one, or of an empty
 * decode context) are left as they were.
 *
 * Uses num_seqs, num_q_heads, num_kv_heads, head_dim (64 or 128), max_context_len, dtype
 * and num_q_rows of dims: the rows are num_q_rows with query_start_loc or positions
 * (num_seqs where positions come with num_q_rows = 0), else num_seqs.
 * Errors: PA_EINVAL, PA_ENOTSUP, PA_EHIP. */
int pa_rope(const void *q, const void *k, const int32_t *positions, const int32_t *context_lens,
            const int32_t *query_start_loc, void *q_out, void *k_out, const pa_rope_t *rope,
            const pa_dims_t *dims, hipStream_t stream);

/* Frequencies for contexts of the trained length and beyond. */
typedef enum {
  PA_ROPE_PLAIN = 0,  /* base^(-2 i / rot_dim) */
  PA_ROPE_LINEAR = 1, /* those / stretch: positions squeezed into the trained range */
  PA_ROPE_BASE = 2,   /* a larger base, base * stretch^(rot_dim / (rot_dim - 2)): the slowest
                         pair is slowed by stretch, the fastest not */
  PA_ROPE_TURNS = 3,  /* pairs of at most low_turns turns in the trained length slowed by
                         stretch, of at least high_turns left, between them a ramp over the
                         turns */
  PA_ROPE_PAIRS = 4   /* the same ends, the ramp over the pairs' index between the last
                         whole index before the one of high_turns turns and the first after
                         that of low_turns; factor 0.1 ln(stretch) + 1 */
} pa_rope_kind_t;

typedef struct pa_rope_scaling {
  int32_t kind;            /* pa_rope_kind_t */
  int32_t rot_dim;         /* even, 2 .. 65536 */
  double base;             /* > 1 (10000 as a rule) */
  double stretch;          /* >= 1; how often the trained length fits the contexts */
  double trained_context;  /* tokens, > 0 (TURNS and PAIRS) */
  double low_turns;        /* 0 < low_turns < high_turns (TURNS and PAIRS) */
  double high_turns;
} pa_rope_scaling_t;

/* inv_freq_host [rot_dim / 2] and the factor (1 but for PA_ROPE_PAIRS), both written.
 * Host only; no HIP call.  Errors: PA_EINVAL (a null pointer, a field out of its range or
 * not finite; fields that the kind does not use are not looked at). */
int pa_rope_frequencies(const pa_rope_scaling_t *scaling, double *inv_freq_host, float *factor);

#ifdef __cplusplus
}
#endif

#endif /* PA_ROPE_H */
