// Arguments and launchers of the 4-bit cache's kernels (internal to
// libpagedattn.so; the format is described in pagedattn_q4.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pa_kernels.h"

namespace pa {

constexpr int q4_tile_bytes(int D) { return 8 * D + D / 2; }

// The cache write and its mirror, the read.
struct Q4RowsArgs {
  const void* k_rows;  // [rows][H_kv][D]; written by the read
  const void* v_rows;
  uint8_t* k_pages;
  uint8_t* v_pages;
  const int32_t* block_table;
  const int32_t* context_lens;
  const int32_t* query_start_loc;  // nullptr: row b is position context_lens[b] - 1
  int64_t bt_stride;
  int B, rows, H_kv, num_pages, max_context_len;
};
hipError_t launch_q4_append(int dtype, int D, const Q4RowsArgs& a, hipStream_t st);
hipError_t launch_q4_read(int dtype, int D, const Q4RowsArgs& a, hipStream_t st);

// Attention.  A wave takes an item, a KV head's 16 NB columns (query row, head of
// the group) of one sequence, over a part of its keys.
struct Q4AttnArgs {
  const void* q;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const int32_t* block_table;
  const int32_t* context_lens;
  const int32_t* query_start_loc;  // nullptr: decode
  void* out;
  float* ws_o;   // [rows][H_q][n_split][D] unnormalised outputs of parts
  float* ws_ml;  // [rows][H_q][n_split][2] (base in log2 units, sum)
  int64_t bt_stride;
  float scale_log2;
  int B, s /* heads of a group */, H_q, H_kv, rows, num_pages, max_context_len;
  int n_slots;  // row blocks, at most (q4_slot)
  int n_split, split_units;
};
constexpr int kQ4Unit = 2 * 16;  // tokens of a step: two pages

// Column blocks (of 16) that a wave holds.
constexpr int kQ4BlocksMax = 4;
constexpr int q4_positions(int blocks, int s) { return 16 * blocks / s; }  // query rows of an item

hipError_t launch_q4_attn(int dtype, int D, int blocks, const Q4AttnArgs& a, hipStream_t st, KernelEvents ev);
hipError_t launch_q4_merge(int dtype, int D, const Q4AttnArgs& a, hipStream_t st);

}  // namespace pa
