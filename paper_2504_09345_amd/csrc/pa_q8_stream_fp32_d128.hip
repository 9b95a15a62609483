// The 8-bit cache's decode kernels, fp32 at head dim 128 (design in pa_q8_stream.hip).
#include "pa_q8_tile.h"
#include "pa_q_stream.h"

namespace pa {

template const void* q_stream_pick<q8::Format, float, 128>(int);

}  // namespace pa
