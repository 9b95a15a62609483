// The 4-bit cache's attention kernels, bf16 at head dim 64 (design in pa_q4_attn.hip).
#include "pa_q4_tile.h"
#include "pa_q_attn.h"

namespace pa {

template const void* q_attn_pick<q4::Format, uint16_t, 64>(int);

}  // namespace pa
