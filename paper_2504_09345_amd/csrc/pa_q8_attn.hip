// Chunk rows over the 8-bit paged cache for gfx950 (format in pagedattn_q8.h; the kernel is
// pa_q_attn.h's, design in pa_q4_attn.hip).
//
// Every wave converts K and V for its 16 columns, 64 instructions of a unit at head_dim 128
// beside 16 products, so issue bounds it as it does the 4-bit cache's, with 223 vector
// instructions a unit, set-up included, instead of 332: one chunk of 700 rows, 32 query
// heads over 8, 15 us (265 TFLOP/s; 18 there), of 64 rows on 1,500 tokens 12, 4 of 56 on
// 3,000 25; of 2,048 in fp32 95, at head_dim 64 65.  Large calls share the conversions
// (pa_q8_chunk.hip).
#include "pa_q8_tile.h"
#include "pa_q_attn.h"

namespace pa {

extern template const void* q_attn_pick<q8::Format, uint16_t, 64>();
extern template const void* q_attn_pick<q8::Format, float, 128>();
extern template const void* q_attn_pick<q8::Format, float, 64>();
template const void* q_attn_pick<q8::Format, uint16_t, 128>();

template hipError_t launch_q_attn<q8::Format>(int, int, const QAttnArgs&, hipStream_t, KernelEvents);

}  // namespace pa
