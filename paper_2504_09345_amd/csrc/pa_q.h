// Arguments and launchers of the kernels of the caches held in few bits (internal to
// libpagedattn.so; the formats are described in pagedattn_q4.h and pagedattn_q8.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pa_kernels.h"

namespace pa {

// Bytes of a (page, KV head) tile.
constexpr int q4_tile_bytes(int D) { return 8 * D + D / 2; }
constexpr int q8_tile_bytes(int D) { return 16 * D; }

// HIP launches fewer than 2^32 threads in a dimension.
constexpr int64_t kQMaxThreads = ((int64_t)1 << 32) - 1;

// The cache write and its mirror, the read.
struct QRowsArgs {
  const void* k_rows;  // [rows][H_kv][D]; written by the read
  const void* v_rows;
  uint8_t* k_pages;
  uint8_t* v_pages;
  const int32_t* block_table;
  const int32_t* context_lens;
  const int32_t* query_start_loc;  // nullptr: row b is position context_lens[b] - 1
  int64_t bt_stride;
  int B, rows, H_kv, num_pages, max_context_len;
  uint8_t* scales;  // (of a format that has them beside the tiles)
};
constexpr int kQRowsWaves = 4;  // waves of a workgroup, each with the rows of a slot
constexpr int kQRowsGroup = 4;  // tokens of a slot at least, whose V bytes are a word
// Slots of a call, of `group` tokens each.
constexpr int64_t q_row_slots(bool varlen, int64_t rows, int64_t seqs, int group = kQRowsGroup) {
  return varlen ? rows / group + 2 * seqs : rows;
}
hipError_t launch_q4_append(int dtype, int D, const QRowsArgs& a, hipStream_t st);
hipError_t launch_q4_read(int dtype, int D, const QRowsArgs& a, hipStream_t st);
hipError_t launch_q8_append(int dtype, int D, const QRowsArgs& a, hipStream_t st);
hipError_t launch_q8_read(int dtype, int D, const QRowsArgs& a, hipStream_t st);

constexpr int kQUnit = 2 * 16;  // tokens of a step: two pages

// Chunk rows.  An item is a KV head's 16 or 32 columns (query row, head of the group) of
// one sequence, or 128 in a workgroup that shares V, over a part of its keys.
struct QAttnArgs {
  const void* q;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const int32_t* block_table;
  const int32_t* context_lens;
  const int32_t* query_start_loc;
  void* out;
  float* ws_o;   // [rows][H_q][n_split][D] unnormalised outputs of parts
  float* ws_ml;  // [rows][H_q][n_split][2] (base in log2 units, sum)
  int64_t bt_stride;
  float scale_log2;
  int B, s /* heads of a group */, H_q, H_kv, rows, num_pages, max_context_len;
  int n_slots;   // items of a KV head, at most
  int min_rows;  // sequences of fewer rows are the stream kernel's
  int max_q_len;
  int n_split, split_units;
  int blocks;      // column blocks of an item
  int wave_parts;  // waves (1, 2 or 4) that share an item's units, where they do not share V
  const uint8_t* scales;
};
constexpr int kQWaves = 4;  // waves of a workgroup: each has an item of its own, 2 or 4 share one, or all share V

// Query rows of an item of so many column blocks (of 16).
constexpr int q_positions(int blocks, int s) { return 16 * blocks / s; }
constexpr int kQChunkBlocks = 2 * kQWaves;  // of a workgroup that shares V's operands (launch_q_chunk)

// The formats (pa_q4_tile.h, pa_q8_tile.h), by which the kernels are instantiated.
namespace q4 { struct Format; }
namespace q8 { struct Format; }

template <class F> hipError_t launch_q_attn(int dtype, int D, const QAttnArgs& a, hipStream_t st, KernelEvents ev);
template <class F> hipError_t launch_q_chunk(int D, const QAttnArgs& a, hipStream_t st, KernelEvents ev);  // bf16
hipError_t launch_q_merge(int dtype, int D, const QAttnArgs& a, hipStream_t st);
template <class F, typename T, int D> const void* q_attn_pick(int blocks);

// The persistent kernel of decode rows (sequences of one row): (sequence, KV head,
// unit) triples of the whole batch in equal contiguous ranges, one per wave.
struct QStreamArgs {
  const void* q;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const int32_t* block_table;
  const int32_t* context_lens;
  const int32_t* query_start_loc;  // nullptr: decode
  void* out;
  // of each workgroup and slot (0: the item that its start cuts, 1: that its end cuts)
  float* ws_o;   // S * D floats (QRecord's order)
  float* ws_ml;  // (base in log2 units, sum) of the S heads
  unsigned long long* ws_flag;  // a counter per workgroup, kQCounterStride apart
  CounterKey key;
  int64_t bt_stride;
  float scale_log2;
  int B, H_q, H_kv, rows, num_pages, max_context_len;
  int max_q_len;  // longer chunks are NaN rows, where write_long
  int cus;        // of the device
  int write_long;
  const uint8_t* scales;
};
constexpr int kQStreamSeqs = 4096;    // sequences of a launch
constexpr int kQStreamGroups = 512;   // workgroups of a launch
constexpr int kQStreamThreads = 512;  // of a workgroup
// Units per wave below which a CU's second workgroup stays without a range (head_dim 64,
// where two fit).  One and two, 32 query heads over 8 in bf16: 64 sequences of 512-2,048
// tokens (5 units a wave of both) 18.8 us and 19.0, 4 of 8,192-32,768 (5) 17.3 and 19.8,
// 128 of 512-2,048 (10) 28.5 and 27.1, 256 (20) 48.8 and 47.6, 512 of 1,024-4,096 (80)
// 157 and 149; in fp32, 64 heads over 8: 64 of 256-2,048 (4) 23.4 and 24.6, 128 of
// 512-2,048 (10) 38.0 and 38.0, 256 (20) 61.4 and 62.6.  (8 bits, fp32: 4 of
// 8,192-32,768 23.4 and 25.2.)
constexpr int kQFewUnits = 8;
// A workgroup takes an item whole, where there are no more items than CUs, if the longest
// has at most so many units more than a workgroup's equal share: a wave's 3.5
// units more are what the join through memory costs.  Whole and shared, 32 query heads
// over 8 in bf16: 1 sequence of 200 tokens 8.4 us and 9.8, of 1,000 10.8 and 10.4, of
// 2,000 13.9 and 11.6; 8 of 200-500 9.5 and 10.6, of 512-2,048 14.5 and 13.5; 32 of
// 100-500 10.6 and 13.3, of 512-2,048 16.4 and 18.5.  (8 bits: 1 of 200 8.6 and 10.4; 32
// of 100-500 11.3 and 13.8, of 512-2,048 19.1 and 21.7; with 14 or 56 units instead of 28
// none is shorter.)
constexpr int kQAloneUnits = 28;
constexpr int kQCounterStride = 16;   // 128 bytes: atomics on one line follow each other 30 ns apart
static_assert(kQStreamGroups <= kStreamMaxGrid, "a cut item's groups of records");

// Workgroups that the current device holds at once, at most as many as a launch may
// have, and its CUs; 0 on error.
template <class F> int q_stream_workgroups(int dtype, int D, int s, int* cus);
template <class F> hipError_t launch_q_stream(int dtype, int D, int s, const QStreamArgs& a, int workgroups, hipStream_t st, KernelEvents ev);
template <class F, typename T, int D> const void* q_stream_pick(int s);

// A call's key (pa_counter.h), its own among the process's.
CounterKey new_call_key();

}  // namespace pa
