// Pages of 4 bits: the codes' way back, which the rows (pages.hip) and the attention
// (exact.hip) share.
#pragma once

#include <hip/hip_runtime.h>

namespace pkv {

// Eight values of 4 bits as bfloat16, exactly: the codes of w, the scale's exponent.
__device__ __forceinline__ uint4 values4(uint32_t w, float scale) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)));
}

}  // namespace pkv
