// Decode rows over the 4-bit paged cache for gfx950 (format in pagedattn_q4.h): a
// persistent grid in which every wave streams an equal contiguous range of the batch's
// (sequence, KV head, unit) triples: equal bytes per wave whatever the context lengths.
//
//  * A unit is two pages (32 tokens) of one KV head, 4.3 KiB of K and V at head_dim
//    128: softmax and the products' bookkeeping are paid once per 32 tokens, and the
//    PV product's k dimension is filled by them.  The group's query heads are the
//    columns of the products (S of 16).
//  * The codes lie in memory as the lanes hold the matrix-core operands, and the units'
//    page entries in a register each of 64 lanes, so the waves share nothing: no LDS
//    tiles, no table, no barrier while streaming.  A wave's K registers are loaded again
//    as soon as the scores are formed and V's after the PV products.  Loading two units
//    at a time changed nothing (256 sequences: 78 us and 77), so bytes under way are not
//    the bound.
//  * A wave has a range, not a head of a range that eight waves share: the parts of an
//    item cut by the ranges' ends are then mostly waves of one workgroup, which meet in
//    LDS, and only items cut by a workgroup's ends go through memory, where a level of
//    the join costs 3-4 us.  Measured with eight waves of one range each and with a wave
//    each, 32 query heads over 8, bf16: 8 sequences of 512-2,048 tokens 22.1 us and
//    14.0, 256 of those 75.0 and 69.6, 4 of 8,192-32,768 29.5 and 23.6.  (Two waves on
//    two heads of one range each: 14.9, 68.0 and 24.9.)
//  * Where a batch has few short items, a workgroup takes each whole, its eight waves a
//    part of the units: nothing goes through memory then, and a call is 1.1-2.7 us
//    shorter (kQ4AloneUnits).
//  * Of a SIMD's waves the oldest issues first; left alone, the older half of a
//    workgroup ended its ranges 7 us before the younger one on 256 sequences, which then
//    streamed with half of the loads under way.  The waves take turns instead, a unit
//    each (64 sequences at 64 heads of 64 dims in fp32: 27 us instead of 35).
//
// 256 sequences of 512-2,048 tokens, 361 MB of codes and scales: 69 us.  With longer
// contexts the time grows with the bytes at 6.4-6.5 TB/s (512 sequences of 512-8,192
// tokens 2.4 GB in 401 us, of 1,024-16,384 4.9 GB in 780), the rate that loads of this
// pattern alone reach; the rest, some 13 us here, is launch, lengths and entries (3), the
// first units' loads and the joins of the last ranges (4-8).
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
int q4_stream_workgroups(int dtype, int D, int s, int* cus) {
  constexpr int kDevices = 64;
  static std::atomic<int64_t> known[kDevices][2][2][9];  // workgroups, and the CUs above them
  int dev = 0, n_cus = 0, per_cu = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 0;
  std::atomic<int64_t>* at = dev >= 0 && dev < kDevices && dtype >= 0 && dtype < 2 && s <= 8 ? &known[dev][dtype][D / 128][s] : nullptr;
  const int64_t have = at != nullptr ? at->load(std::memory_order_relaxed) : 0;
  if (have > 0) {
    *cus = (int)(have >> 32);
    return (int)have;
  }
  const void* fn = q4_stream_fn(dtype, D, s);
  if (fn == nullptr || hipDeviceGetAttribute(&n_cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, fn, kQ4StreamThreads, 0) != hipSuccess)
    return 0;
  const int n = std::min(n_cus * per_cu, kQ4StreamGroups);
  if (at != nullptr) at->store((int64_t)n_cus << 32 | n, std::memory_order_relaxed);
  *cus = n_cus;
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
