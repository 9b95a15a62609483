// The 8-bit cache's format (pagedattn_q8.h): a wave's share of two pages, its values as
// matrix-core operands, and the products of 32 tokens.
#pragma once

#include "pa_q_tile.h"

namespace pa {
namespace q8 {

using namespace q;

// Codes 2 H and 2 H + 1 of w times scale, as two bf16 or two fp16.
template <int H, bool F16>
__device__ __forceinline__ uint32_t pair_of(uint32_t w, float scale) {
  if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, H != 0));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, H != 0));
}

}  // namespace q8
}  // namespace pa
