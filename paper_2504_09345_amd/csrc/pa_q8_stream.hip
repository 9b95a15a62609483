// Decode rows over the 8-bit paged cache for gfx950 (format in pagedattn_q8.h; the kernel
// is pa_q_stream.h's, design in pa_q4_stream.hip).
//
// A unit is 8 KiB of K and V at head_dim 128, two 16-byte loads a lane and page of each,
// which become operands by conversions alone: K as bf16, V as fp16 where its scales allow.
// A page's two scale bytes are loaded beside K, a unit ahead too, and stay in the caches.
// With twice the 4-bit cache's bytes a unit and four fifths of its vector and matrix
// instructions (158 and 202, set-up included: no query in parts, one scale a page) HBM is the bound sooner:
// 256 sequences of 512-2,048 tokens, 32 query heads over 8, 683 MB in 110 us, 6.2 TB/s,
// where loads of this pattern alone reach 6.4 (the 4-bit cache's 361 MB take 69); 512 of
// 256-4,096 beside chunks 2.28 GB in 357, 6.4.
// Few long contexts stay far from it: at head_dim 64 in fp32, 64 query heads over 8, 4 of
// 8,192-32,768 tokens are 68 MB in 24 us.  The same call on 2,048 tokens takes 12.7 already:
// launch, lengths and entries, and the join of some nine records an item; from there on it
// grows with the bytes at 5.9 TB/s.  (In bf16 21 us, with 32 heads 19: three parts of the
// queries and weights are not what bounds it.)
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
