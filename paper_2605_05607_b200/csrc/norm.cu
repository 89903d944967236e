// Root-mean-square norm of the residual stream, the step in front of the layer, with the residual's addition, an E4M3 output with one
// scale per row (the operand of the FP8 experts), and its backward pass.
//     s = x + residual                    fp32; leaves as bf16 (the residual stream of the next block)
//     rstd = 1 / sqrt(mean(s^2) + eps)     NaN, and with it the row, where the sum is not finite
//     y = (s * w) * rstd                  leaves as bf16 and / or as codes of y / scale, scale = max|y| / 448
// Everything is computed from the fp32 sum: y and the codes are rounded once each, from fp32 (codes of the rounded y would round twice).
// The product with w comes first so that one pass has both sums of the row: rounding is monotone, so max|y| is (max|s * w|) * rstd to the bit.
//
// Bound by memory: every input is read once into registers and every output written once.  16384 rows of 4096 with residual, bf16 and E4M3 outputs
// 106 us (5.7 TB/s); rows on their way through shared memory instead (as in the backward pass below) took 117.
#include "ptx.cuh"
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
    // A sum that is not finite would give 0, and a row of zeros that look like a result; with eps = 0, squares that vanish an infinity.  NaN both.
    const float var = __fadd_rn(__fdiv_rn(sum, (float)(a.vec_per_row * VEC)), a.eps);
    const float rstd = var > 0.f && var <= 3.402823466e38f ? __frsqrt_rn(var) : __uint_as_float(0x7FC00000u);
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
  long long rows;
  int vec_per_row;
  uint4* dx;
  float* part;            // [grid, columns]
};

// Rows come through shared memory, STAGES of them on their way per block: every thread copies (cp.async) the vectors that it will use itself, so it waits
// for its own copies and for nobody.  Loaded into registers instead, a row at a time, 8192 rows of 4096 with dres took 67 us, 49 so.
// WARPS warps per row, or (FIT) as many as the block has; WARPS == 1: eight rows per block, whose dw are joined at the end (16000 rows of 512 with two warps per row: 35.9 us, 18.6 so).
// Without dres two blocks of 512 fit an SM by their shared memory, so they are held to the registers for it (64, 82 left alone: 8370 rows of 7168 103 us, 70
// so); with dres shared memory leaves room for one, and fewer registers cost (8370 of 7168 79 us, 116 so).
template <int KEEP, int WARPS, int STAGES, bool SKIP, bool FIT>
__global__ void __launch_bounds__(WARPS == 1 ? 256 : WARPS * 32, WARPS == 16 && KEEP <= 2 && !SKIP ? 2 : 0) rmsnorm_backward_kernel(const NormBwdArgs a) {
  extern __shared__ __align__(16) uint4 ring_s[];   // per row of the block: [STAGES][dy, s, dres][vec_per_row]
  constexpr int STREAMS = SKIP ? 3 : 2, TEAMS = WARPS == 1 ? 8 : 1;
  const int LANES = FIT ? blockDim.x : WARPS * 32;
  __shared__ float part[2][WARPS];
  grid_dependency_sync();
  const int lane = WARPS == 1 ? threadIdx.x & 31 : threadIdx.x, team = WARPS == 1 ? threadIdx.x >> 5 : 0, n_vec = a.vec_per_row;
  const long long r0 = (long long)blockIdx.x * TEAMS + team, step = (long long)gridDim.x * TEAMS;   // sums with them pass 32 bits at the largest row counts
  uint4* ring = ring_s + team * STAGES * STREAMS * n_vec;
  const uint4* const from[3] = {a.dy, a.s, a.dres};
  auto fetch = [&](long long r, int stage) {
    if (r < a.rows) {
#pragma unroll
      for (int q = 0; q < STREAMS; ++q)
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
          const int v = lane + LANES * i;
          if (v < n_vec) ptx::cp_async_16(ptx::smem_u32(ring + (stage * STREAMS + q) * n_vec + v), from[q] + r * n_vec + v, 16);
        }
    }
    ptx::cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < STAGES; ++i) fetch(r0 + i * step, i);
  float2 dw[KEEP][VEC / 2], w[KEEP][VEC / 2];
#pragma unroll
  for (int i = 0; i < KEEP; ++i) {
    float f[VEC] = {};
    if (lane + LANES * i < n_vec) load_w(a.w, a.w32, lane + LANES * i, f);
#pragma unroll
    for (int j = 0; j < VEC; j += 2) {
      dw[i][j / 2] = make_float2(0.f, 0.f);
      w[i][j / 2] = make_float2(f[j], f[j + 1]);
    }
  }
  int flip = 0, stage = 0;
  const float n = (float)(n_vec * VEC);
  float rstd = r0 < a.rows ? __ldg(a.rstd + r0) : 0.f;
  for (long long r = r0; r < a.rows; r += step) {
    const float next = r + step < a.rows ? __ldg(a.rstd + r + step) : 0.f;
    ptx::cp_async_wait<STAGES - 1>();   // this row's copies of this thread
    uint4 dyv[KEEP], sv[KEEP], kv[SKIP ? KEEP : 1];
    float2 dots = make_float2(0.f, 0.f);   // sum of dy * s * w, over even and odd columns
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int v = lane + LANES * i;
      if (v < n_vec) {
        dyv[i] = ring[(stage * STREAMS) * n_vec + v];
        sv[i] = ring[(stage * STREAMS + 1) * n_vec + v];
        if (SKIP) kv[i] = ring[(stage * STREAMS + 2) * n_vec + v];
        float dy[VEC], s[VEC];
        unpack8(dyv[i], dy);
        unpack8(sv[i], s);
#pragma unroll
        for (int j = 0; j < VEC; j += 2) {
          const float2 t = __fmul2_rn(make_float2(dy[j], dy[j + 1]), make_float2(s[j], s[j + 1]));
          dw[i][j / 2] = __ffma2_rn(t, make_float2(rstd, rstd), dw[i][j / 2]);
          dots = __ffma2_rn(t, w[i][j / 2], dots);
        }
      }
    }
    float dot = dots.x + dots.y;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, off);
    if (WARPS > 1) {   // two buffers: the next row's sums do not overwrite what a slow warp still reads
      if ((lane & 31) == 0) part[flip][lane >> 5] = dot;
      __syncthreads();
      dot = 0.f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i)
        if (!FIT || i * 32 < LANES) dot += part[flip][i];
      flip ^= 1;
    }
    fetch(r + STAGES * step, stage);   // the stage's values are in registers (their sum has been used)
    if (++stage == STAGES) stage = 0;
    const float c = -(dot / n) * rstd * rstd;   // dx = rstd * (dy * w + c * s) + dres
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int v = lane + LANES * i;
      if (v < n_vec) {
        float dy[VEC], s[VEC], k[VEC];
        unpack8(dyv[i], dy);
        unpack8(sv[i], s);
        if (SKIP) unpack8(kv[i], k);
#pragma unroll
        for (int j = 0; j < VEC; j += 2) {
          const float2 g = __fmul2_rn(make_float2(dy[j], dy[j + 1]), w[i][j / 2]), s2 = make_float2(s[j], s[j + 1]), c2 = make_float2(c, c);
          const float2 t = __ffma2_rn(s2, c2, g), r2 = make_float2(rstd, rstd);
          const float2 o = SKIP ? __ffma2_rn(t, r2, make_float2(k[j], k[j + 1])) : __fmul2_rn(t, r2);
          s[j] = o.x;
          s[j + 1] = o.y;
        }
        a.dx[r * n_vec + v] = pack8(s);
      }
    }
    rstd = next;
  }
  if (WARPS == 1) {   // the block's eight sums, a column at a time, in the order of the warps
    ptx::cp_async_wait<0>();
    __syncthreads();
    float* sums = reinterpret_cast<float*>(ring_s);   // [8][columns]: fits, as a warp's ring has STAGES * STREAMS * 2 >= 4 bytes per column
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int v = lane + LANES * i;
      if (v < n_vec)
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) reinterpret_cast<float2*>(sums)[(team * n_vec + v) * VEC / 2 + j] = dw[i][j];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < n_vec * VEC; c += 256) {
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < TEAMS; ++t) sum += sums[t * n_vec * VEC + c];
      a.part[(long long)blockIdx.x * n_vec * VEC + c] = sum;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < KEEP; ++i) {
    const int v = lane + LANES * i;
    if (v < n_vec) {
      float4* out = reinterpret_cast<float4*>(a.part + (long long)blockIdx.x * n_vec * VEC) + 2 * v;
      out[0] = make_float4(dw[i][0].x, dw[i][0].y, dw[i][1].x, dw[i][1].y);
      out[1] = make_float4(dw[i][2].x, dw[i][2].y, dw[i][3].x, dw[i][3].y);
    }
  }
}

// dw[c] = sum over the blocks' partial rows: 32 columns per block, whose warps share the rows (a load of each is on its way at once: eight
// warps instead of 32 took 10 us for 592 partial rows of 4096).
__global__ void __launch_bounds__(1024) rmsnorm_dw_kernel(const float* __restrict__ part, int parts, int cols, float* __restrict__ dw) {
  grid_dependency_sync();
  __shared__ float sum_s[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (c < cols) {
#pragma unroll 10
    for (int r = warp; r < parts; r += 32) sum += part[(long long)r * cols + c];
  }
  sum_s[warp][lane] = sum;
  __syncthreads();
  sum = sum_s[lane][warp];
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
  if (lane == 0 && blockIdx.x * 32 + warp < cols) dw[blockIdx.x * 32 + warp] = sum;
}

template <bool RES, bool QUANT>
cudaError_t launch_norm(const NormArgs& a, cudaStream_t st) {
  const int cols = a.vec_per_row * VEC;
  // Blocks per SM before they take a second row, us with 16 / 64: 32768 rows of 2000, bf16 alone, 52.2 / 49.6, 16357 of 4096 51.3 / 47.7; with residual and
  // both outputs 102.5 / 101.7; 9347 of 7168 110.9 / 113.1, 32768 of 512 28.6 / 29.4.
  const long long cap = (long long)sm_count() * (cols > 1024 && cols <= 4096 ? 64 : 16);
  auto go = [&](auto kernel, int threads, int rpb) {
    const long long blocks = (a.rows + rpb - 1) / rpb;
    return launch_pdl(kernel, dim3((unsigned)(blocks < cap ? blocks : cap)), dim3(threads), 0, st, a);
  };
  if (cols <= 512) return go(rmsnorm_kernel<2, 1, RES, QUANT>, 256, 8);
  if (cols <= 1024) return go(rmsnorm_kernel<4, 1, RES, QUANT>, 256, 8);
  if (cols <= 2048) return go(rmsnorm_kernel<2, 4, RES, QUANT>, 128, 1);
  if (cols <= 4096) return go(rmsnorm_kernel<4, 4, RES, QUANT>, 128, 1);
  if (cols <= 8192) return go(rmsnorm_kernel<4, 8, RES, QUANT>, 256, 1);
  // to NORM_COLS; us with 256 / 512 threads per row: 4187 rows of 16000, bf16 alone, 53.5 / 79.4, with residual and both outputs (spilled) 160 / 115
  if constexpr (RES) return go(rmsnorm_kernel<4, 16, RES, QUANT>, 512, 1);
  else return go(rmsnorm_kernel<8, 8, RES, QUANT>, 256, 1);
}

// Blocks of the backward pass: `teams` rows at a time each, no more than there is room for.
constexpr int rmsnorm_blocks(long long rows, int teams, int resident) {
  const long long blocks = (rows + teams - 1) / teams, most = resident < NORM_PARTS ? resident : NORM_PARTS;
  return (int)(blocks < most ? blocks : most);
}
static_assert(rmsnorm_blocks((1ll << 31) - 1, 8, 592) == 592 && rmsnorm_blocks(9, 8, 592) == 2, "up to the largest row count");

constexpr int NORM_SMEM = 226 * 1024;   // an SM's, less what the system and the kernel itself take of a block's 227 KiB
// Blocks per SM as shared memory, registers and NORM_PARTS (four per SM) allow.
template <bool SKIP>
cudaError_t launch_norm_bwd(const NormBwdArgs& a, int* parts, cudaStream_t st) {
  const int cols = a.vec_per_row * VEC;
  auto go = [&](auto kernel, int threads, int stages, int teams = 1) {
    const int smem = teams * stages * (SKIP ? 3 : 2) * cols * 2;
    if (smem > 40 * 1024) {   // beyond 48 KiB with what the kernel declares itself; always the most, as another thread may be about to launch with more than this
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, NORM_SMEM);
      if (e != cudaSuccess) return e;
    }
    const int per_sm = max(1, min(min(4, 1152 / threads), NORM_SMEM / (smem + 1280)));
    *parts = rmsnorm_blocks(a.rows, teams, per_sm * sm_count());
    return launch_pdl(kernel, dim3(*parts), dim3(threads), smem, st, a);
  };
  // Threads as a row needs them instead of the whole 256 or 512, where that leaves room for another block or a tenth fewer; us, whole / fit: with dres 39893
  // rows of 1504 97 / 94, 23076 of 2600 106 / 100, 12000 of 5000 110 / 100, 8370 of 7168 88 / 79; without 23076 of 2600 88 / 84, 12000 of 5000 82 / 77.
  // Where it does not, the count known in advance is better: with dres 16483 of 3640 97 / 100, 14648 of 4096 84 / 88, 5000 of 12000 93 / 96, without
  // 9146 of 6560 73 / 76.
  auto fit = [&](int keep) { return ((a.vec_per_row + keep - 1) / keep + 31) & ~31; };
  if (cols <= 512) return go(rmsnorm_backward_kernel<2, 1, 4, SKIP, false>, 256, 4, 8);
  if (cols <= 1024) return go(rmsnorm_backward_kernel<4, 1, 3, SKIP, false>, 256, 3, 8);
  if (cols <= 2048)
    return fit(1) < 256 ? go(rmsnorm_backward_kernel<1, 8, 4, SKIP, true>, fit(1), 4) : go(rmsnorm_backward_kernel<1, 8, 4, SKIP, false>, 256, 4);
  if (cols <= 4096)
    return fit(1) <= 384 ? go(rmsnorm_backward_kernel<1, 16, 4, SKIP, true>, fit(1), 4) : go(rmsnorm_backward_kernel<1, 16, 4, SKIP, false>, 512, 4);
  if (cols <= 8192)   // without dres four stages leave one block per SM: 7500 of 8000 99 us, 72 so
    return fit(2) <= (SKIP ? 448 : 384) ? go(rmsnorm_backward_kernel<2, 16, 3, SKIP, true>, fit(2), 3) : go(rmsnorm_backward_kernel<2, 16, 3, SKIP, false>, 512, 3);
  return go(rmsnorm_backward_kernel<4, 16, 2, SKIP, false>, 512, 2);   // NORM_COLS
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
  int parts = 0;
  if (rows > 0) {
    const NormBwdArgs a{static_cast<const uint4*>(dy), static_cast<const uint4*>(dres), static_cast<const uint4*>(s), w, w32 ? 1 : 0, rstd,
                        rows, cols / VEC, static_cast<uint4*>(dx), part};
    const cudaError_t e = dres != nullptr ? launch_norm_bwd<true>(a, &parts, st) : launch_norm_bwd<false>(a, &parts, st);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(rmsnorm_dw_kernel, dim3((cols + 31) / 32), dim3(1024), 0, st, static_cast<const float*>(part), parts, cols, dw);
}

}  // namespace tcmoe
