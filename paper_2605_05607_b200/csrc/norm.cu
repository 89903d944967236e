// Root-mean-square norm of the residual stream, the step in front of the layer, with the residual's addition, an E4M3 output with one
// scale per row (the operand of the FP8 experts), and its backward pass.
//     s = x + residual                    fp32; leaves as bf16 (the residual stream of the next block)
//     rstd = 1 / sqrt(mean(s^2) + eps)
//     y = (s * w) * rstd                  leaves as bf16 and / or as codes of y / scale, scale = max|y| / 448
// Everything is computed from the fp32 sum: y and the codes are rounded once each, from fp32 (codes of the rounded y would round twice).
// The product with w comes first so that one pass has both sums of the row: rounding is monotone, so max|y| is (max|s * w|) * rstd to the bit.
//
// Bound by memory: every input is read once into registers and every output written once.
#include "quant.cuh"
#include "quant4.cuh"

namespace tcmoe {
namespace {

constexpr int VEC = 8;   // elements per thread and load: 16 bytes of bf16
static_assert(NORM_COLS == 4 * 16 * 32 * VEC, "the widest kernels hold a row in registers");

struct NormArgs {
  const uint4 *x, *res;
  const void* w;
  int w32;                // weights in fp32 (else bf16)
  float eps;
  long long rows;
  int vec_per_row;
  uint4 *res_out, *y;     // may be the inputs themselves: a row is in registers before any of it is written
  uint2* yq;
  float *scale, *rstd;
};

using fp4::max_nan;
using fp4::pack8;
using fp4::unpack8;
__device__ __forceinline__ void load_w(const void* w, int w32, int v, float (&f)[VEC]) {
  if (w32) {
    const float4 a = __ldg(static_cast<const float4*>(w) + 2 * v), b = __ldg(static_cast<const float4*>(w) + 2 * v + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
    unpack8(__ldg(static_cast<const uint4*>(w) + v), f);
  }
}

// WARPS warps per row, KEEP vectors of 8 per lane: at most KEEP * WARPS * 256 columns, all in registers.  WARPS == 1: eight rows per block.
template <int KEEP, int WARPS, bool RES, bool QUANT>
__global__ void __launch_bounds__(WARPS == 1 ? 256 : WARPS * 32) rmsnorm_kernel(const NormArgs a) {
  grid_dependency_sync();
  constexpr int LANES = WARPS * 32;
  __shared__ float2 part[2][WARPS];
  const int lane = WARPS == 1 ? threadIdx.x & 31 : threadIdx.x;   // of the row's threads
  const int rpb = blockDim.x / LANES;
  int flip = 0;
  for (long long r = (long long)blockIdx.x * rpb + (WARPS == 1 ? threadIdx.x >> 5 : 0); r < a.rows; r += (long long)gridDim.x * rpb) {
    const long long base = r * a.vec_per_row;
    uint4 xv[KEEP], rv[RES ? KEEP : 1];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int v = lane + LANES * i;
      if (v < a.vec_per_row) {
        xv[i] = a.x[base + v];
        if (RES) rv[i] = a.res[base + v];
      }
    }
    float s[KEEP][VEC];
    float sum = 0.f, top = 0.f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int v = lane + LANES * i;
      if (v < a.vec_per_row) {
        unpack8(xv[i], s[i]);
        if (RES) {
          float t[VEC];
          unpack8(rv[i], t);
#pragma unroll
          for (int j = 0; j < VEC; ++j) s[i][j] += t[j];
          if (a.res_out != nullptr) a.res_out[base + v] = pack8(s[i]);
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum = fmaf(s[i][j], s[i][j], sum);
        float w[VEC];
        load_w(a.w, a.w32, v, w);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          s[i][j] *= w[j];
          if (QUANT) top = max_nan(top, fabsf(s[i][j]));
        }
      }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
      if (QUANT) top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, off));
    }
    if (WARPS > 1) {   // two buffers: the next row's sums do not overwrite what a slow warp still reads
      if ((lane & 31) == 0) part[flip][lane >> 5] = make_float2(sum, top);
      __syncthreads();
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        const float2 q = part[flip][i];
        sum += q.x;
        if (QUANT) top = max_nan(top, q.y);
      }
      flip ^= 1;
    }
    const float rstd = __frsqrt_rn(__fadd_rn(__fdiv_rn(sum, (float)(a.vec_per_row * VEC)), a.eps));
    if (lane == 0 && a.rstd != nullptr) a.rstd[r] = rstd;
    float sc = 1.f, inv = 1.f;
    bool exact = true;
    if (QUANT) {
      sc = __fdiv_rn(__fmul_rn(top, rstd), 448.f);
      if (sc == 0.f) sc = 1.f;   // a row of zeros, or one so small that the scale is: all codes are 0
      if (lane == 0) a.scale[r] = sc;
      exact = e4m3_pair_exact(sc);
      inv = __frcp_rn(sc);
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int v = lane + LANES * i;
      if (v < a.vec_per_row) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[i][j] = __fmul_rn(s[i][j], rstd);
        if (!QUANT || a.y != nullptr) a.y[base + v] = pack8(s[i]);
        if (QUANT) {
          uint32_t c[4];
#pragma unroll
          for (int q = 0; q < 4; ++q)
            c[q] = exact ? to_e4m3_pair(s[i][2 * q], s[i][2 * q + 1], inv, sc)
                         : (uint32_t)to_e4m3(s[i][2 * q], sc) | ((uint32_t)to_e4m3(s[i][2 * q + 1], sc) << 8);
          a.yq[base + v] = make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
        }
      }
    }
  }
}

// Backward: with g = dy * w and xhat = s * rstd,
//     dx = rstd * (g - xhat * mean(g * xhat)) + dres,      dw = sum over rows of dy * xhat.
// A block walks rows with its columns fixed, so a thread adds up its columns' dw in registers; the blocks' sums are joined by a second
// kernel in a fixed order (no atomics: the same bits every time).
struct NormBwdArgs {
  const uint4 *dy, *dres, *s;
  const void* w;
  int w32;
  const float* rstd;
  int rows, vec_per_row;
  uint4* dx;
  float* part;            // [grid, columns]
};

template <int KEEP, int WARPS, bool SKIP>
__global__ void __launch_bounds__(WARPS * 32) rmsnorm_backward_kernel(const NormBwdArgs a) {
  grid_dependency_sync();
  constexpr int LANES = WARPS * 32;
  __shared__ float part[2][WARPS];
  const int lane = threadIdx.x;
  float dw[KEEP][VEC];
#pragma unroll
  for (int i = 0; i < KEEP; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) dw[i][j] = 0.f;
  int flip = 0;
  const float n = (float)(a.vec_per_row * VEC);
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const long long base = (long long)r * a.vec_per_row;
    uint4 dyv[KEEP], sv[KEEP], kv[SKIP ? KEEP : 1];
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int v = lane + LANES * i;
      if (v < a.vec_per_row) {
        dyv[i] = a.dy[base + v];
        sv[i] = a.s[base + v];
        if (SKIP) kv[i] = a.dres[base + v];
      }
    }
    const float rstd = __ldg(a.rstd + r);
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int v = lane + LANES * i;
      if (v < a.vec_per_row) {
        float dy[VEC], s[VEC], w[VEC];
        unpack8(dyv[i], dy);
        unpack8(sv[i], s);
        load_w(a.w, a.w32, v, w);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float t = dy[j] * (s[j] * rstd);
          dw[i][j] += t;
          dot = fmaf(t, w[j], dot);
        }
      }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, off);
    if (WARPS > 1) {
      if ((lane & 31) == 0) part[flip][lane >> 5] = dot;
      __syncthreads();
      dot = 0.f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) dot += part[flip][i];
      flip ^= 1;
    }
    const float mean = dot / n;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int v = lane + LANES * i;
      if (v < a.vec_per_row) {
        float dy[VEC], s[VEC], w[VEC], k[VEC];
        unpack8(dyv[i], dy);
        unpack8(sv[i], s);
        load_w(a.w, a.w32, v, w);
        if (SKIP) unpack8(kv[i], k);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float g = (dy[j] * w[j] - (s[j] * rstd) * mean) * rstd;
          s[j] = SKIP ? g + k[j] : g;
        }
        a.dx[base + v] = pack8(s);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < KEEP; ++i) {
    const int v = lane + LANES * i;
    if (v < a.vec_per_row) {
      float4* out = reinterpret_cast<float4*>(a.part + (long long)blockIdx.x * a.vec_per_row * VEC) + 2 * v;
      out[0] = make_float4(dw[i][0], dw[i][1], dw[i][2], dw[i][3]);
      out[1] = make_float4(dw[i][4], dw[i][5], dw[i][6], dw[i][7]);
    }
  }
}

// dw[c] = sum over the blocks' partial rows: 32 columns per block, eight warps share the rows.
__global__ void __launch_bounds__(256) rmsnorm_dw_kernel(const float* __restrict__ part, int parts, int cols, float* __restrict__ dw) {
  grid_dependency_sync();
  __shared__ float sum_s[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (c < cols) {
#pragma unroll 4
    for (int r = warp; r < parts; r += 8) sum += part[(long long)r * cols + c];
  }
  sum_s[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && c < cols) {
#pragma unroll
    for (int i = 1; i < 8; ++i) sum += sum_s[i][lane];
    dw[c] = sum;
  }
}

template <bool RES, bool QUANT>
cudaError_t launch_norm(const NormArgs& a, cudaStream_t st) {
  const long long cap = (long long)sm_count() * 16;
  auto go = [&](auto kernel, int threads, int rpb) {
    const long long blocks = (a.rows + rpb - 1) / rpb;
    return launch_pdl(kernel, dim3((unsigned)(blocks < cap ? blocks : cap)), dim3(threads), 0, st, a);
  };
  const int cols = a.vec_per_row * VEC;
  if (cols <= 512) return go(rmsnorm_kernel<2, 1, RES, QUANT>, 256, 8);
  if (cols <= 1024) return go(rmsnorm_kernel<4, 1, RES, QUANT>, 256, 8);
  if (cols <= 2048) return go(rmsnorm_kernel<2, 4, RES, QUANT>, 128, 1);
  if (cols <= 4096) return go(rmsnorm_kernel<4, 4, RES, QUANT>, 128, 1);
  if (cols <= 8192) return go(rmsnorm_kernel<4, 8, RES, QUANT>, 256, 1);
  return go(rmsnorm_kernel<4, 16, RES, QUANT>, 512, 1);   // NORM_COLS
}

template <bool SKIP>
cudaError_t launch_norm_bwd(const NormBwdArgs& a, int grid, cudaStream_t st) {
  const int cols = a.vec_per_row * VEC;
  auto go = [&](auto kernel, int threads) { return launch_pdl(kernel, dim3(grid), dim3(threads), 0, st, a); };
  if (cols <= 512) return go(rmsnorm_backward_kernel<1, 2, SKIP>, 64);
  if (cols <= 1024) return go(rmsnorm_backward_kernel<1, 4, SKIP>, 128);
  if (cols <= 2048) return go(rmsnorm_backward_kernel<1, 8, SKIP>, 256);
  if (cols <= 4096) return go(rmsnorm_backward_kernel<2, 8, SKIP>, 256);
  if (cols <= 8192) return go(rmsnorm_backward_kernel<2, 16, SKIP>, 512);
  return go(rmsnorm_backward_kernel<4, 16, SKIP>, 512);   // NORM_COLS
}

}  // namespace

cudaError_t launch_rmsnorm(const void* x, const void* res, const void* w, bool w32, float eps, long long rows, int cols, void* res_out,
                           void* y, void* yq, float* scale, float* rstd, cudaStream_t st) {
  if (rows <= 0) return cudaSuccess;
  const NormArgs a{static_cast<const uint4*>(x), static_cast<const uint4*>(res), w, w32 ? 1 : 0, eps, rows, cols / VEC,
                   static_cast<uint4*>(res_out), static_cast<uint4*>(y), static_cast<uint2*>(yq), scale, rstd};
  if (res != nullptr) return yq != nullptr ? launch_norm<true, true>(a, st) : launch_norm<true, false>(a, st);
  return yq != nullptr ? launch_norm<false, true>(a, st) : launch_norm<false, false>(a, st);
}

int rmsnorm_parts(long long rows) { return (int)(rows < NORM_PARTS ? rows : NORM_PARTS); }

cudaError_t launch_rmsnorm_backward(const void* dy, const void* dres, const void* s, const void* w, bool w32, const float* rstd,
                                    long long rows, int cols, void* dx, float* dw, float* part, cudaStream_t st) {
  const int parts = rmsnorm_parts(rows);
  if (parts > 0) {
    const NormBwdArgs a{static_cast<const uint4*>(dy), static_cast<const uint4*>(dres), static_cast<const uint4*>(s), w, w32 ? 1 : 0, rstd,
                        (int)rows, cols / VEC, static_cast<uint4*>(dx), part};
    const cudaError_t e = dres != nullptr ? launch_norm_bwd<true>(a, parts, st) : launch_norm_bwd<false>(a, parts, st);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(rmsnorm_dw_kernel, dim3((cols + 31) / 32), dim3(256), 0, st, static_cast<const float*>(part), parts, cols, dw);
}

}  // namespace tcmoe
