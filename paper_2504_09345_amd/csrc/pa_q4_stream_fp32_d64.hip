// The 4-bit cache's decode kernels, fp32 at head dim 64 (design in pa_q4_stream.hip).
#include "pa_q4_stream.h"

namespace pa {

template const void* q4_stream_pick<float, 64>(int);

}  // namespace pa
