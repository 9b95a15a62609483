// The 4-bit cache's attention kernels, fp32 at head dim 128 (design in pa_q4_attn.hip).
#include "pa_q4_attn.h"

namespace pa {

template const void* q4_attn_pick<float, 128>();

}  // namespace pa
