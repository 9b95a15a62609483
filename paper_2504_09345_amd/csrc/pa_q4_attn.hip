// Attention over the 4-bit paged cache for gfx950 (format in pagedattn_q4.h):
// softmax(scale q.K^T) V per query row and head, K and V the values that the cache
// stands for, causal over a sequence's cached keys.
//
// A wave holds 16 NB columns, each a query row and a query head of one KV head's
// group, and streams the keys in units of two pages (32 tokens):
//   S^T[token][column] = K . Q^T    v_mfma_f32_16x16x32_bf16, K the A operand
//   O^T[dim][column]  += V^T . P^T  the same product, P in two bf16 parts
//                                   (three for fp32 outputs)
// The codes lie in memory in the order in which lanes hold these operands, so a
// page is one 16-byte load per lane for K and one for V and becomes operands by
// conversions alone: v_cvt_scalef32_pk_bf16_fp4 turns a byte into two bf16 with
// the block's scale applied, exactly.  No LDS, no barrier; every wave is alone.
#include "pa_q4_attn.h"

namespace pa {

extern template const void* q4_attn_pick<uint16_t, 64>();
extern template const void* q4_attn_pick<float, 128>();
extern template const void* q4_attn_pick<float, 64>();
template const void* q4_attn_pick<uint16_t, 128>();

static const void* q4_attn_fn(int dtype, int D) {
  if (dtype == 0 && D == 128) return q4_attn_pick<uint16_t, 128>();
  if (dtype == 0 && D == 64) return q4_attn_pick<uint16_t, 64>();
  if (dtype == 1 && D == 128) return q4_attn_pick<float, 128>();
  if (dtype == 1 && D == 64) return q4_attn_pick<float, 64>();
  return nullptr;
}

hipError_t launch_q4_attn(int dtype, int D, const Q4AttnArgs& a, hipStream_t st, KernelEvents ev) {
  const void* fn = q4_attn_fn(dtype, D);
  if (fn == nullptr) return hipErrorInvalidValue;
  const int64_t parts = (int64_t)a.H_kv * a.n_split;
  const int items = kQ4Waves / a.wave_parts;  // of a workgroup
  const int64_t grid = (a.n_slots + items - 1) / items * parts;
  void* args[] = {const_cast<Q4AttnArgs*>(&a)};
  hipError_t e = hipExtLaunchKernel(fn, dim3((uint32_t)grid), dim3(64 * kQ4Waves), args, 0, st, ev.start, ev.stop, 0);
  return e != hipSuccess ? e : hipGetLastError();
}

hipError_t launch_q4_merge(int dtype, int D, const Q4AttnArgs& a, hipStream_t st) {
  const uint32_t grid = (uint32_t)(((int64_t)a.rows * a.H_q + 3) / 4);
  if (dtype == 0 && D == 128) q4_merge_kernel<uint16_t, 128><<<grid, 256, 0, st>>>(a);
  else if (dtype == 0 && D == 64) q4_merge_kernel<uint16_t, 64><<<grid, 256, 0, st>>>(a);
  else if (dtype == 1 && D == 128) q4_merge_kernel<float, 128><<<grid, 256, 0, st>>>(a);
  else if (dtype == 1 && D == 64) q4_merge_kernel<float, 64><<<grid, 256, 0, st>>>(a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace pa
