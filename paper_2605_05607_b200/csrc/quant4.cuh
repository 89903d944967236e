// E2M1 elements with a power-of-two scale per 32 of them (MXFP4): conversions shared by the quantising kernels and the FP4 products.
#pragma once
#include "common.cuh"

#include <cuda_bf16.h>
#include <cuda_fp4.h>

namespace tcmoe {
namespace fp4 {

__host__ __device__ constexpr int chunks(int K) { return 2 * ((K + 255) / 256); }   // scale chunks (128 of K) along K, whole stages

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
  return m;
}
// larger magnitudes of two pairs of bf16, NaN if either is
__device__ __forceinline__ uint32_t max_nan2(uint32_t magnitudes, uint32_t pair) {
  uint32_t m;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(magnitudes), "r"(pair & 0x7FFF7FFFu));
  return m;
}
// E8M0 byte of a block whose largest magnitude is `top`: floor(log2(top)) is the exponent field, and subnormals (field 0) lie below the lowest scale
__device__ __forceinline__ uint32_t scale_byte(float top) {
  const uint32_t field = __float_as_uint(top) >> 23;
  if (field == 255u) return 255u;   // infinite or NaN
  if (top == 0.f) return 127u;
  return field > 2u ? field - 2u : 0u;
}
// 2^-ex, always a normal number (ex <= 125); 0 for the NaN scale, so that its codes are zeros or, of infinities and NaN, any
__device__ __forceinline__ float inverse(uint32_t byte) { return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23); }
// 2^ex: 2^-127 is subnormal
__device__ __forceinline__ float scale_of_byte(uint32_t byte) {
  return byte == 0u ? __uint_as_float(0x00400000u) : byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte << 23);
}

__device__ __forceinline__ float half_of(uint32_t pair, int h) { return __uint_as_float(h ? pair & 0xFFFF0000u : pair << 16); }   // of two bf16
__device__ __forceinline__ void unpack8(const uint4& raw, float (&f)[8]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f[2 * q] = half_of(w[q], 0);
    f[2 * q + 1] = half_of(w[q], 1);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  uint4 raw;
  __nv_bfloat162* p = reinterpret_cast<__nv_bfloat162*>(&raw);
#pragma unroll
  for (int q = 0; q < 4; ++q) p[q] = __floats2bfloat162_rn(f[2 * q], f[2 * q + 1]);
  return raw;
}

// eight codes, the first in the lowest four bits
__device__ __forceinline__ uint32_t codes8(const float (&f)[8], float inv) {
  uint32_t c = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    c |= (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(f[2 * q] * inv, f[2 * q + 1] * inv), __NV_E2M1, cudaRoundNearest) << (8 * q);
  return c;
}
// the codes of two (scaled) values, the first in the low half
__device__ __forceinline__ uint32_t code2(float a, float b) {
  return (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(a, b), __NV_E2M1, cudaRoundNearest);
}
// An 8 x 8 transpose of 4-bit pieces over eight neighbouring lanes: piece i of lane l becomes piece l of lane i.
__device__ __forceinline__ uint32_t transpose8(uint32_t v, int lane) {
  // exchange halves with the lane 4 away, then bytes with the one 2 away, then pieces with the neighbour
  uint32_t o = __shfl_xor_sync(0xFFFFFFFFu, v, 4);
  v = (lane & 4) ? (v & 0xFFFF0000u) | (o >> 16) : (v & 0x0000FFFFu) | (o << 16);
  o = __shfl_xor_sync(0xFFFFFFFFu, v, 2);
  v = (lane & 2) ? (v & 0xFF00FF00u) | ((o >> 8) & 0x00FF00FFu) : (v & 0x00FF00FFu) | ((o << 8) & 0xFF00FF00u);
  o = __shfl_xor_sync(0xFFFFFFFFu, v, 1);
  return (lane & 1) ? (v & 0xF0F0F0F0u) | ((o >> 4) & 0x0F0F0F0Fu) : (v & 0x0F0F0F0Fu) | ((o << 4) & 0xF0F0F0F0u);
}
__device__ __forceinline__ void values8(uint32_t codes, float scale, float (&f)[8]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(codes >> (8 * q)), __NV_E2M1);
    f[2 * q] = __half2float(__half(__half_raw{h.x})) * scale;
    f[2 * q + 1] = __half2float(__half(__half_raw{h.y})) * scale;
  }
}

}  // namespace fp4
}  // namespace tcmoe
