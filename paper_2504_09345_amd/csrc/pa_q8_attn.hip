// Chunk rows over the 8-bit paged cache for gfx950 (format in pagedattn_q8.h; the kernel is
// pa_q_attn.h's, design in pa_q4_attn.hip).
#include "pa_q8_tile.h"
#include "pa_q_attn.h"

namespace pa {

extern template const void* q_attn_pick<q8::Format, uint16_t, 64>();
extern template const void* q_attn_pick<q8::Format, float, 128>();
extern template const void* q_attn_pick<q8::Format, float, 64>();
template const void* q_attn_pick<q8::Format, uint16_t, 128>();

template hipError_t launch_q_attn<q8::Format>(int, int, const QAttnArgs&, hipStream_t, KernelEvents);

}  // namespace pa
