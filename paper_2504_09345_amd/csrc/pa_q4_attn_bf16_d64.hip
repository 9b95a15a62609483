// The 4-bit cache's attention kernels, bf16 at head dim 64 (design in pa_q4_attn.hip).
#include "pa_q4_attn.h"

namespace pa {

template const void* q4_attn_pick<uint16_t, 64>();

}  // namespace pa
