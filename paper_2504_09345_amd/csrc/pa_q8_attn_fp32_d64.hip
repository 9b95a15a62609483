// The 8-bit cache's attention kernels, fp32 at head dim 64 (design in pa_q8_attn.hip).
#include "pa_q8_tile.h"
#include "pa_q_attn.h"

namespace pa {

template const void* q_attn_pick<q8::Format, float, 64>(int);

}  // namespace pa
