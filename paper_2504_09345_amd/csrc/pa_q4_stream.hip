// Decode rows over the 4-bit paged cache for gfx950 (format in pagedattn_q4.h): a
// persistent grid in which every team of waves streams an equal contiguous range of
// the batch's (sequence, head block, unit) triples, as the stream-K kernel of the
// 16-bit cache does (pa_stream.hip: equal bytes per workgroup whatever the context
// lengths, items cut by a range's ends joined by the part that arrives last, one
// launch), with another inner loop:
//
//  * A unit is two pages (32 tokens) of one KV head, 4.3 KiB of K and V at head_dim
//    128: softmax and the products' bookkeeping are paid once per 32 tokens, and the
//    PV product's k dimension is filled by them.
//  * The codes lie in memory as the lanes hold the matrix-core operands, so the
//    waves share nothing: no LDS tiles, no barrier per unit.  A wave's K registers
//    are loaded again as soon as the scores are formed and V's after the PV
//    products, one unit ahead, and four waves per SIMD keep 70 KB per CU in flight.
#include "pa_q4_stream.h"

#include <algorithm>
#include <atomic>

namespace pa {

extern template const void* q4_stream_pick<uint16_t, 64>(int);
extern template const void* q4_stream_pick<float, 128>(int);
extern template const void* q4_stream_pick<float, 64>(int);
template const void* q4_stream_pick<uint16_t, 128>(int);

static const void* q4_stream_fn(int dtype, int D, int s) {
  if (dtype == 0 && D == 128) return q4_stream_pick<uint16_t, 128>(s);
  if (dtype == 0 && D == 64) return q4_stream_pick<uint16_t, 64>(s);
  if (dtype == 1 && D == 128) return q4_stream_pick<float, 128>(s);
  if (dtype == 1 && D == 64) return q4_stream_pick<float, 64>(s);
  return nullptr;
}

// (a property of the kernel and the device, so it is asked for once: the two
// queries take as long as the rest of a small call on the host)
int q4_stream_workgroups(int dtype, int D, int s) {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices][2][2][9];
  int dev = 0, cus = 0, per_cu = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 0;
  std::atomic<int>* at = dev >= 0 && dev < kDevices && dtype >= 0 && dtype < 2 && s <= 8 ? &known[dev][dtype][D / 128][s] : nullptr;
  int n = at != nullptr ? at->load(std::memory_order_relaxed) : 0;
  if (n > 0) return n;
  const void* fn = q4_stream_fn(dtype, D, s);
  if (fn == nullptr || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, fn, kQ4StreamThreads, 0) != hipSuccess)
    return 0;
  n = std::min(cus * per_cu, kQ4StreamGroups);
  if (at != nullptr) at->store(n, std::memory_order_relaxed);
  return n;
}

hipError_t launch_q4_stream(int dtype, int D, int s, const Q4StreamArgs& a, int workgroups, hipStream_t st,
                            KernelEvents ev) {
  const void* fn = q4_stream_fn(dtype, D, s);
  if (fn == nullptr || workgroups <= 0) return hipErrorInvalidValue;
  void* args[] = {const_cast<Q4StreamArgs*>(&a)};
  hipError_t e = hipExtLaunchKernel(fn, dim3(workgroups), dim3(kQ4StreamThreads), args, 0, st, ev.start, ev.stop, 0);
  return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace pa
