// The 4-bit cache's decode kernels, bf16 at head dim 64 (design in pa_q4_stream.hip).
#include "pa_q4_stream.h"

namespace pa {

template const void* q4_stream_pick<uint16_t, 64>(int);

}  // namespace pa
