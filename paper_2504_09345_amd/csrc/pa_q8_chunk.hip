// The 8-bit cache's kernels of large calls' chunk rows (design in pa_q_chunk.h).
#include "pa_q8_tile.h"
#include "pa_q_chunk.h"

namespace pa {

template hipError_t launch_q_chunk<q8::Format>(int, const QAttnArgs&, hipStream_t, KernelEvents);

}  // namespace pa
