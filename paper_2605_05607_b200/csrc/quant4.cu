// Microscaled 4-bit floating point (OCP Microscaling Formats, version 1.0: MXFP4), the format of the FP4 form of the expert FFN:
//   32 neighbouring values of K share a power of two: exponent ex = clamp(floor(log2(max|v|)) - 2, -127, 125), held as the byte
//   ex + 127 (E8M0); 127 for a block of zeros; 255 (NaN, which is then what all of the block reads as) if a value is not finite
//   element = E2M1 of v * 2^-ex, round to nearest even, saturating at 6; two per byte, the lower K in the low half
// Scaling by a power of two is exact, so a code is rounded once and a restatement takes the same decisions bit for bit.
//
// Activation rows keep their scales row-major, [rows, K / 32].  The expert products read scales as the tensor cores take them: a
// chunk of 512 bytes holds 128 rows (or weight columns) x 4 scales (128 of K), byte (row % 32) * 16 + (row / 32) * 4 + scale % 4, and
// chunks follow each other along K, an even number of them (a pipeline stage is 256 of K; the chunks past K hold 127).
#include "quant4.cuh"

namespace tcmoe {
namespace {

// 16 bytes (8 values) per lane, four lanes per block of 32.  The blocks of all rows follow each other in all three arrays, so rows play no part.
// Bound by memory: 2.53 bytes per value.
constexpr int QROWS_UNROLL = 4;
__global__ void __launch_bounds__(256) quantize_rows_fp4_kernel(const uint4* __restrict__ src, uint32_t* __restrict__ dst,
                                                                uint8_t* __restrict__ scale, long long vecs) {
  grid_dependency_sync();
  const long long step = (long long)gridDim.x * 256;
  for (long long v0 = (long long)blockIdx.x * 256 + threadIdx.x; v0 - threadIdx.x < vecs; v0 += QROWS_UNROLL * step) {
    uint4 raw[QROWS_UNROLL];
#pragma unroll
    for (int i = 0; i < QROWS_UNROLL; ++i) raw[i] = v0 + i * step < vecs ? __ldg(src + v0 + i * step) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < QROWS_UNROLL; ++i) {
      float f[8], top = 0.f;
      fp4::unpack8(raw[i], f);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fp4::max_nan(top, fabsf(f[j]));
      top = fp4::max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = fp4::max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      const uint32_t b = fp4::scale_byte(top);
      const long long v = v0 + i * step;
      if (v < vecs) {
        dst[v] = fp4::codes8(f, fp4::inverse(b));
        if ((v & 3) == 0) scale[v >> 2] = (uint8_t)b;
      }
    }
  }
}

__global__ void __launch_bounds__(256) dequantize_rows_fp4_kernel(const uint32_t* __restrict__ src, const uint8_t* __restrict__ scale,
                                                                  uint4* __restrict__ dst, long long vecs) {
  grid_dependency_sync();
  const long long step = (long long)gridDim.x * 256;
  for (long long v0 = (long long)blockIdx.x * 256 + threadIdx.x; v0 < vecs; v0 += QROWS_UNROLL * step) {
    uint32_t c[QROWS_UNROLL];
    uint8_t b[QROWS_UNROLL];
#pragma unroll
    for (int i = 0; i < QROWS_UNROLL; ++i)
      if (v0 + i * step < vecs) {
        c[i] = __ldg(src + v0 + i * step);
        b[i] = __ldg(scale + ((v0 + i * step) >> 2));
      }
#pragma unroll
    for (int i = 0; i < QROWS_UNROLL; ++i)
      if (v0 + i * step < vecs) {
        float f[8];
        fp4::values8(c[i], fp4::scale_of_byte(b[i]), f);
        dst[v0 + i * step] = fp4::pack8(f);
      }
  }
}

// Weights [E, K, N] (N contiguous) -> codes [E, N, K / 2] and scale chunks [E, ceil(N / 128), 2 ceil(K / 256), 512].  A block takes 256 of K x 64
// columns; a warp 32 of K, a lane two columns, whose 32 values it holds in registers.  Codes go through shared memory so that a column
// leaves in 128-byte runs.  Bound by memory and by issue slots (61 % busy with conversions): 32 x 4096 x 1536 to codes and back 187 us, 177 with the
// maxima of both columns taken at once (5.8 TB/s).
constexpr int WT_PITCH = 128 + 16;   // bytes per column in shared memory: neighbouring columns four banks apart
__global__ void __launch_bounds__(256) quantize_weights_fp4_kernel(const uint32_t* __restrict__ w, uint4* __restrict__ wq,
                                                                   uint8_t* __restrict__ scale, int K, int N) {
  __shared__ __align__(16) uint8_t codes_s[64 * WT_PITCH];
  __shared__ __align__(8) uint8_t scale_s[2][32][2][4];   // [chunk][column % 32][column / 32 of the block's two][scale of the chunk]
  grid_dependency_sync();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int e = blockIdx.z, n0 = blockIdx.x * 64, k0 = blockIdx.y * 256 + warp * 32, n = n0 + 2 * lane;
  uint32_t raw[32];
  const bool in = n < N && k0 < K;
  const uint32_t* src = w + (((size_t)e * K + k0) * N + n) / 2;
#pragma unroll
  for (int i = 0; i < 32; ++i) raw[i] = in ? __ldg(src + (size_t)i * (N / 2)) : 0u;
  uint32_t top = 0;   // of either column
#pragma unroll
  for (int i = 0; i < 32; ++i) top = fp4::max_nan2(top, raw[i]);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t b = fp4::scale_byte(fp4::half_of(top, h));
    const float inv = fp4::inverse(b);
    uint32_t c[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = fp4::half_of(raw[q * 8 + j], h);
      c[q] = fp4::codes8(f, inv);
    }
    const int col = 2 * lane + h;
    *reinterpret_cast<uint4*>(codes_s + col * WT_PITCH + warp * 16) = make_uint4(c[0], c[1], c[2], c[3]);
    scale_s[warp >> 2][col & 31][col >> 5][warp & 3] = (uint8_t)b;
  }
  __syncthreads();
  const int kb0 = blockIdx.y * 8;   // first block of 32 of the tile
  if (n0 < N) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = threadIdx.x + 256 * i, col = at >> 3, piece = at & 7;
      if (n0 + col < N && (kb0 + piece) * 32 < K)
        wq[((size_t)e * N + n0 + col) * (K / 32) + kb0 + piece] = *reinterpret_cast<const uint4*>(codes_s + col * WT_PITCH + piece * 16);
    }
  }
  if (threadIdx.x < 64) {
    const int chunk = threadIdx.x >> 5;
    const size_t c = ((size_t)e * ((N + 127) / 128) + n0 / 128) * fp4::chunks(K) + blockIdx.y * 2 + chunk;
    *reinterpret_cast<uint2*>(scale + c * 512 + lane * 16 + (n0 & 64) / 8) = *reinterpret_cast<const uint2*>(scale_s[chunk][lane]);
  }
}

__global__ void __launch_bounds__(256) dequantize_weights_fp4_kernel(const uint4* __restrict__ wq, const uint8_t* __restrict__ scale,
                                                                     uint32_t* __restrict__ w, int K, int N) {
  __shared__ __align__(16) uint8_t codes_s[64 * WT_PITCH];
  __shared__ __align__(8) uint8_t scale_s[2][32][2][4];
  grid_dependency_sync();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int e = blockIdx.z, n0 = blockIdx.x * 64, k0 = blockIdx.y * 256 + warp * 32, n = n0 + 2 * lane, kb0 = blockIdx.y * 8;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int at = threadIdx.x + 256 * i, col = at >> 3, piece = at & 7;
    if (n0 + col < N && (kb0 + piece) * 32 < K)
      *reinterpret_cast<uint4*>(codes_s + col * WT_PITCH + piece * 16) = __ldg(wq + ((size_t)e * N + n0 + col) * (K / 32) + kb0 + piece);
  }
  if (threadIdx.x < 64) {
    const int chunk = threadIdx.x >> 5;
    const size_t c = ((size_t)e * ((N + 127) / 128) + n0 / 128) * fp4::chunks(K) + blockIdx.y * 2 + chunk;
    *reinterpret_cast<uint2*>(scale_s[chunk][lane]) = *reinterpret_cast<const uint2*>(scale + c * 512 + lane * 16 + (n0 & 64) / 8);
  }
  __syncthreads();
  if (n >= N || k0 >= K) return;
  const int col = 2 * lane;
  const float s0 = fp4::scale_of_byte(scale_s[warp >> 2][col & 31][col >> 5][warp & 3]);
  const float s1 = fp4::scale_of_byte(scale_s[warp >> 2][(col + 1) & 31][col >> 5][warp & 3]);
  const uint4 c0 = *reinterpret_cast<const uint4*>(codes_s + col * WT_PITCH + warp * 16);
  const uint4 c1 = *reinterpret_cast<const uint4*>(codes_s + (col + 1) * WT_PITCH + warp * 16);
  const uint32_t a[4] = {c0.x, c0.y, c0.z, c0.w}, b[4] = {c1.x, c1.y, c1.z, c1.w};
  uint32_t* dst = w + (((size_t)e * K + k0) * N + n) / 2;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float f[8], g[8];
    fp4::values8(a[q], s0, f);
    fp4::values8(b[q], s1, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(f[j], g[j]);
      dst[(size_t)(q * 8 + j) * (N / 2)] = *reinterpret_cast<const uint32_t*>(&v);
    }
  }
}

unsigned flat_grid(long long vecs) {
  const long long blocks = (vecs + 256 * QROWS_UNROLL - 1) / (256 * QROWS_UNROLL), cap = (long long)sm_count() * 16;
  return (unsigned)(blocks < cap ? blocks : cap);
}

}  // namespace

cudaError_t launch_quantize_rows_fp4(const void* src, long long rows, int cols, void* dst, void* scale, cudaStream_t st) {
  const long long vecs = rows * (cols / 8);
  if (vecs <= 0) return cudaSuccess;
  return launch_pdl(quantize_rows_fp4_kernel, dim3(flat_grid(vecs)), dim3(256), 0, st, static_cast<const uint4*>(src),
                    static_cast<uint32_t*>(dst), static_cast<uint8_t*>(scale), vecs);
}

cudaError_t launch_dequantize_rows_fp4(const void* src, const void* scale, long long rows, int cols, void* dst, cudaStream_t st) {
  const long long vecs = rows * (cols / 8);
  if (vecs <= 0) return cudaSuccess;
  return launch_pdl(dequantize_rows_fp4_kernel, dim3(flat_grid(vecs)), dim3(256), 0, st, static_cast<const uint32_t*>(src),
                    static_cast<const uint8_t*>(scale), static_cast<uint4*>(dst), vecs);
}

// the grid covers whole scale chunks: 128 columns, 256 of K
static dim3 weight_grid(int E, int K, int N) { return dim3((unsigned)((N + 127) / 128 * 2), (unsigned)((K + 255) / 256), (unsigned)E); }

cudaError_t launch_quantize_weights_fp4(const void* w, int E, int K, int N, void* wq, void* scale, cudaStream_t st) {
  return launch_pdl(quantize_weights_fp4_kernel, weight_grid(E, K, N), dim3(256), 0, st, static_cast<const uint32_t*>(w),
                    static_cast<uint4*>(wq), static_cast<uint8_t*>(scale), K, N);
}

cudaError_t launch_dequantize_weights_fp4(const void* wq, const void* scale, int E, int K, int N, void* w, cudaStream_t st) {
  return launch_pdl(dequantize_weights_fp4_kernel, weight_grid(E, K, N), dim3(256), 0, st, static_cast<const uint4*>(wq),
                    static_cast<const uint8_t*>(scale), static_cast<uint32_t*>(w), K, N);
}

}  // namespace tcmoe
