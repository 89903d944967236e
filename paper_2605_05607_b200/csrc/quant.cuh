// bf16 / fp32 -> E4M3 with one scale for many values: the arithmetic that the quantising kernels share.
#pragma once
#include "common.cuh"

#include <cuda_bf16.h>
#include <cuda_fp8.h>

namespace tcmoe {

__device__ __forceinline__ uint8_t to_e4m3(float v, float scale) {
  return (uint8_t)__nv_cvt_float_to_fp8(__fdiv_rn(v, scale), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float scale_of(float amax) { return amax == 0.f ? 1.f : __fdiv_rn(amax, 448.f); }

// Two codes at once, the low byte that of `a`.  fl32(v / scale) comes from the reciprocal, which the whole row shares, by
// Markstein's correction (P. Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", IBM J. Res.
// Dev. 34, 1990): with inv = RN(1 / s) and q within an ulp of v / s, RN(q + (v - q s) * inv), the residual exact, is RN(v / s) as long
// as nothing leaves the normal range.  Values so small that the residual does round to code 0 either way.  (Taking the code
// where both ends of an error interval around v * inv agree was no faster than dividing: quotients of 8-bit significands
// tie exactly too often, and one lane's division stops its warp.)
__device__ __forceinline__ uint32_t to_e4m3_pair(float a, float b, float inv, float scale) {
  float qa = a * inv, qb = b * inv;
#pragma unroll
  for (int i = 0; i < 2; ++i) {   // the first step makes q faithful, the second is the one that rounds correctly
    qa = fmaf(fmaf(-qa, scale, a), inv, qa);
    qb = fmaf(fmaf(-qb, scale, b), inv, qb);
  }
  return __nv_cvt_float2_to_fp8x2(make_float2(copysignf(qa, a), copysignf(qb, b)),   // -0 stays -0
                                  __NV_SATFINITE, __NV_E4M3);
}
// Scales for which to_e4m3_pair is exact: neither the reciprocal nor a residual leaves the normal range.  (False for a NaN.)
__device__ __forceinline__ bool e4m3_pair_exact(float scale) { return scale >= 0x1p-80f && scale < 0x1p100f; }

}  // namespace tcmoe
