// Chunk rows over the 8-bit paged cache for gfx950 (format in pagedattn_q8.h; the kernel is
// pa_q_attn.h's, design in pa_q4_attn.hip).
//
// A wave converts K and V of a unit for its columns, 64 instructions at head_dim 128: beside
// 16 products where it has 16 columns, and in large calls (bf16) beside 32 for 32, of which
// two waves fit a SIMD (216 registers; three at head_dim 64).  Issue bounds both, as it does
// the 4-bit cache's.  With 16, 223 vector and matrix instructions a unit, set-up included,
// where that has 332: one chunk of 700 rows, 32 query heads over 8, 15 us (265 TFLOP/s; 18
// there), of 64 rows on 1,500 tokens 12, 16 of 8 on 2,000 17; of 2,048 in fp32 95, at head_dim
// 64 65.  With 32: 8 chunks of 2,048 rows on 8-1,998 tokens 624-643 us on four machines (875-901
// TFLOP/s of the causal halves' work, 74 to 76 % of the rate of a large library product),
// where a unit takes 165 vector and 33 matrix instructions (150 and 32 in the loop): alone
// the first, four cycles each, would be 335 us of a SIMD's time and the second 270, and two waves hide
// little of each other.  On 0, 290, .. 2,030 tokens 580 us (944 TFLOP/s), at head_dim 64 354
// (772); one of 4,000 takes 143, 2 of 120 on 20,000 97.
//
// Scores of K's codes as e4m3 operands, with the query in two parts, took as long and drop bits
// (pa_q8_tile.h).
#include "pa_q8_tile.h"
#include "pa_q_attn.h"

namespace pa {

extern template const void* q_attn_pick<q8::Format, uint16_t, 64>(int);
extern template const void* q_attn_pick<q8::Format, float, 128>(int);
extern template const void* q_attn_pick<q8::Format, float, 64>(int);
template const void* q_attn_pick<q8::Format, uint16_t, 128>(int);

template hipError_t launch_q_attn<q8::Format>(int, int, const QAttnArgs&, hipStream_t, KernelEvents);

}  // namespace pa
