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
//    shorter (kQAloneUnits).
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
#include "pa_q4_tile.h"
#include "pa_q_stream.h"

namespace pa {

extern template const void* q_stream_pick<q4::Format, uint16_t, 64>(int);
extern template const void* q_stream_pick<q4::Format, float, 128>(int);
extern template const void* q_stream_pick<q4::Format, float, 64>(int);
template const void* q_stream_pick<q4::Format, uint16_t, 128>(int);

template int q_stream_workgroups<q4::Format>(int, int, int, int*);
template hipError_t launch_q_stream<q4::Format>(int, int, int, const QStreamArgs&, int, hipStream_t, KernelEvents);

}  // namespace pa
