// Decode rows over the 8-bit paged cache for gfx950 (format in pagedattn_q8.h; the kernel
// is pa_q_stream.h's, design in pa_q4_stream.hip).
#include "pa_q8_tile.h"
#include "pa_q_stream.h"

namespace pa {

extern template const void* q_stream_pick<q8::Format, uint16_t, 64>(int);
extern template const void* q_stream_pick<q8::Format, float, 128>(int);
extern template const void* q_stream_pick<q8::Format, float, 64>(int);
template const void* q_stream_pick<q8::Format, uint16_t, 128>(int);

template int q_stream_workgroups<q8::Format>(int, int, int, int*);
template hipError_t launch_q_stream<q8::Format>(int, int, int, const QStreamArgs&, int, hipStream_t, KernelEvents);

}  // namespace pa
