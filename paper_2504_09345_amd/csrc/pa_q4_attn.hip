// Attention over the 4-bit paged cache for gfx950 (format in pagedattn_q4.h):
// softmax(scale q.K^T) V per query row and head, K and V the values that the cache
// stands for, causal over a sequence's cached keys.
//
// A wave holds 16 columns, each a query row and a query head of one KV head's group,
// and streams the keys in units of two pages (32 tokens):
//   S^T[token][column] = K . Q^T    K the A operand: at head_dim 128 and bf16 the codes
//                                   themselves with their scales, beside two e4m3 parts
//                                   of the query (v_mfma_scale_f32_16x16x128_f8f6f4, 2
//                                   of 33 cycles per page; as bf16 4 of 17, and 16
//                                   conversions); else K as bf16, exactly
//   O^T[dim][column]  += V^T . P^T  V and P in fp16 (v_mfma_f32_16x16x32_f16) where all
//                                   of the unit's V is exact in it, else in bf16, P in
//                                   two parts (three for fp32 outputs)
// The codes lie in memory in the order in which lanes hold these operands, so a page is
// one 16-byte load per lane for K and one for V and becomes operands by conversions
// alone: v_cvt_scalef32_pk_f16_fp4 turns a byte into two values with the block's scale
// applied, exactly.  No exchange between lanes but for a base that moves.
//
// What bounds it is issue: a unit takes some 190 vector instructions (96 of them V's
// conversion) and 12 products, about 1,300 cycles, which two or three waves of a SIMD
// overlap little.  So large calls share V's conversion (pa_q4_chunk.hip).  Where a call
// has fewer items than the GPU holds waves, 2 or 4 waves of a workgroup share an item's
// units and join their sums in LDS.
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
