// The 4-bit cache's decode kernels, fp32 at head dim 128 (design in pa_q4_stream.hip).
#include "pa_q4_stream.h"

namespace pa {

template const void* q4_stream_pick<float, 128>(int);

}  // namespace pa
