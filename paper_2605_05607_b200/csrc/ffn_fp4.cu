// FP4 form of the expert FFN: E2M1 elements, a power of two per 32 of K, on the block-scaled tensor-core instructions (tcgen05
// kind::mxf4), which take the scales along and accumulate the scaled products in fp32:
//     GEMM-1  h[r, n] = silu(a_r . W1[e][:, n]) * (a_r . W3[e][:, n]), quantised in the epilogue: h exists in 4 bits only
//     GEMM-2  o[r, n] = w_r * (h_r . W2[e][:, n])
//
// The weights are the M side of the UMMAs (two of 128 columns: the same columns of W1 and of W3, or neighbouring ones of W2), the tile's rows
// the N side, rounded up to 16: experts of a few rows, which stream weights, pay for no padded rows, and 32 neighbouring columns of h
// lie in the 32 lanes of a warp, which quantises them without shared memory.
//
// A pipeline stage holds 256 of K: 128 bytes per row of either operand (packed, 128-byte swizzle, by TMA) and their scales in chunks of 128
// rows x 4 (512 bytes, by untiled bulk copies, in the layout that tcgen05.cp spreads over TMEM).  The scales' TMEM columns belong to the
// stage: when a stage is filled again, the UMMAs that read its scales have completed.
//
// One persistent CTA per SM takes every 148th tile.  SHARE, for layers with fewer tiles than SMs: the stages of all tiles, one tile after the other, are
// divided evenly among the CTAs.  A tile that several of them share leaves as fp32 parts; per epilogue warp, the one that writes the last part adds
// them up, in the order of K whoever is last, puts the sums back into its accumulator and goes on as if they were its own.  GEMM-2 of one token,
// top-2 of 4096 x 14336 (32 tiles): 31 us, 22 so.  (With all layers divided this way, 64 tokens, top-8 of 128 experts of 4096 x 1536, took
// 218 us instead of 211: neighbouring CTAs no longer stream neighbouring columns.  A form of its own, because the larger code alone costs the others
// up to 4 us: instructions that are missed in the cache wait behind the weights that are on their way.)
//
// TMEM: two accumulator buffers of 2 x 96 columns, then 24 columns of scales per stage.  Warp roles: 0-7 epilogue, 8 TMA, 9 UMMA and TMEM
// owner.  One persistent CTA per SM; every wait is bounded.
#include "ffn_fp4.cuh"

#include <atomic>

namespace tcmoe {
namespace ffn {
namespace {

constexpr int W_BYTES = 128 * 128;                  // one half of the weight tile: 128 columns x 256 of K
constexpr int X_BYTES = 128 * F4_ROWS;              // the tile's rows
constexpr int SF_BYTES = F4_SF_BYTES;
constexpr int STAGE_BYTES = 2 * W_BYTES + X_BYTES + 3 * SF_BYTES;   // W W X sfX sfW sfW
constexpr int NSTAGE = 4;
constexpr int SF_COLS = 24;                         // TMEM columns of a stage's scales
constexpr int BUF_COLS = 2 * F4_ROWS;               // of an accumulator buffer
constexpr int SF_TMEM = 2 * BUF_COLS;
static_assert(SF_TMEM + NSTAGE * SF_COLS <= 512, "TMEM");
static_assert(X_BYTES % 1024 == 0, "swizzle atoms");
constexpr int NUM_BARS = 2 * NSTAGE + 4;
constexpr int EPI_WARPS = 8, TMA_WARP = EPI_WARPS, MMA_WARP = EPI_WARPS + 1;
constexpr int THREADS = (EPI_WARPS + 2) * 32;
constexpr int TABLE_BYTES = (2 * (MAX_E + 1) * 4 + 15) & ~15;
constexpr int SMEM_BYTES = 1024 + NSTAGE * STAGE_BYTES + NUM_BARS * 8 + 64 + TABLE_BYTES + EPI_WARPS * F4Out<F4_ROWS, 2>::BYTES;
static_assert(SMEM_BYTES <= 232448, "shared memory of an SM");
constexpr uint32_t HINT = 1000;

struct F4Tile {
  int e, mt, row0, rows, c0, halves;   // expert, row tile over all experts, first row, rows; first 128-column chunk, halves in use
};

template <bool GLU, bool SHARE>
__global__ void __launch_bounds__(THREADS, 1)
ffn_fp4_kernel(const __grid_constant__ CUtensorMap map_wa, const __grid_constant__ CUtensorMap map_wb,
               const __grid_constant__ F4RowMaps xmaps, const F4Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + NSTAGE * STAGE_BYTES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + NUM_BARS);
  int* abort_s = reinterpret_cast<int*>(tmem_slot + 1);
  int* tp_s = reinterpret_cast<int*>(tmem_slot + 16);
  int* eoff_s = tp_s + (MAX_E + 1);
  const uint32_t smem_base = ptx::smem_u32(smem), bar_base = ptx::smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (NSTAGE + s); };
  auto tfull_bar = [&](int b) { return bar_base + 8u * (2 * NSTAGE + b); };
  auto tempty_bar = [&](int b) { return bar_base + 8u * (2 * NSTAGE + 2 + b); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < NSTAGE; ++s) {
      ptx::mbar_init(full_bar(s), 1);    // TMA thread (expect_tx)
      ptx::mbar_init(empty_bar(s), 1);   // tcgen05.commit
    }
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(tfull_bar(b), 1);             // tcgen05.commit
      ptx::mbar_init(tempty_bar(b), EPI_WARPS);    // one lane per epilogue warp
    }
    ptx::fence_mbar_init();
  }
  if (warp == TMA_WARP && lane == 0) {
    ptx::prefetch_tensormap(&map_wa);
    ptx::prefetch_tensormap(&map_wb);
  }
  if (warp == MMA_WARP) {
    ptx::tmem_alloc(ptx::smem_u32(tmem_slot), 512);
    ptx::tmem_relinquish();
  }
  grid_dependency_sync();   // nothing above touches global data
  f4_load_offsets(p.expert_offsets, p.E, eoff_s);
  __syncthreads();
  if (warp == 0) f4_tile_table(eoff_s, p.E, F4_ROWS, tp_s, lane);
  if (threadIdx.x == 32) *abort_s = p.status[ST_ABORT];
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int n_tiles = GLU ? p.NC : (p.NC + 1) / 2;   // column tiles: one chunk of W1 and of W3, or two of W2
  const int KB = (p.K + F4_BK - 1) / F4_BK;
  // Items of this CTA: every gridDim.x-th tile, or (SHARE) the tiles that its share of the stages of all tiles lies in.
  const int grid = (int)gridDim.x, total = tp_s[p.E] * n_tiles;
  const int per = SHARE ? (total * KB + grid - 1) / grid : 0;
  const int u0 = min(total * KB, (int)blockIdx.x * per), u1 = min(total * KB, u0 + per), w0 = SHARE ? u0 / KB : (int)blockIdx.x;
  const int items = SHARE ? (u1 + KB - 1) / KB - w0 : (total - w0 + grid - 1) / grid;
  auto tile_at = [&](int j) { return SHARE ? w0 + j : w0 + j * grid; };
  auto kb_begin = [&](int j) { return SHARE ? max(0, u0 - (w0 + j) * KB) : 0; };
  auto kb_end = [&](int j) { return SHARE ? min(KB, u1 - (w0 + j) * KB) : KB; };
  volatile int* abort_flag = abort_s;
  const volatile int* global_abort = p.status + ST_ABORT;
  auto timeout = [&](int detail) {
    report_error(p.status, DEV_TIMEOUT, GLU ? KID_GEMM1 : KID_GEMM2, detail, blockIdx.x);
    p.status[ST_ABORT] = 1;
    *abort_flag = 1;
  };
  // expert by expert, and inside one column tile by column tile, rows fastest: CTAs that run together share weights in L2
  auto tile_of = [&](int w, int from) {   // from: an expert at or before the tile's
    const int lo = f4_expert_from(tp_s, from, n_tiles, w);
    const uint32_t local = (uint32_t)(w - tp_s[lo] * n_tiles), mts = (uint32_t)(tp_s[lo + 1] - tp_s[lo]), c = local / mts;
    F4Tile t;
    t.e = lo;
    const int m = (int)(local - c * mts);
    t.mt = tp_s[lo] + m;
    t.row0 = eoff_s[lo] + m * F4_ROWS;
    t.rows = min(F4_ROWS, eoff_s[lo + 1] - t.row0);
    t.c0 = GLU ? (int)c : 2 * (int)c;
    t.halves = GLU ? 2 : min(2, p.NC - t.c0);
    return t;
  };

  if (warp < EPI_WARPS) {
    // ================================ epilogue: lane = column, TMEM column = row ================================
    const int quarter = warp & 3, turn = warp >> 2;
    const uint32_t out_mem = ptx::smem_u32(tp_s) + TABLE_BYTES + (uint32_t)(warp * F4Out<F4_ROWS, 2>::BYTES);   // GEMM-2
    int tl = 0;
    F4Tile t{}, next{};
    float rw[(F4Out<F4_ROWS, 2>::TURNS + 1) / 2];
    // slot 2 i: the part of CTA i's first tile, which began before it; slot 2 i + 1: that of its last, which goes on behind it
    auto slot = [&](int i, int r0) {
      return p.part + ((size_t)i * p.part_rows + r0) * 256 + quarter * 32 + lane;   // per row: 128 columns of either half
    };
    if (items > 0) {
      next = tile_of(tile_at(0), 0);
      if (!GLU) f4_fetch_weights<F4_ROWS, 2>(p, next.row0, next.rows, turn, lane, rw);
    }
    // Looked at once, alike for all lanes: the wait's shuffle, which ends the loop after an abort, wants the whole warp.
    const bool go = __all_sync(0xFFFFFFFFu, !*abort_flag);
    for (; go && tl < items; ++tl) {
      t = next;
      if (!GLU) f4_keep_weights<F4_ROWS, 2>(rw, out_mem, lane);
      if (tl + 1 < items) {
        next = tile_of(tile_at(tl + 1), t.e);
        if (!GLU) f4_fetch_weights<F4_ROWS, 2>(p, next.row0, next.rows, turn, lane, rw);
      }
      const int buf = tl & 1;
      if (!ptx::mbar_wait_warp<false, HINT>(tfull_bar(buf), (tl >> 1) & 1, abort_flag, global_abort)) { timeout(1); break; }
      ptx::tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * BUF_COLS);
      const bool whole = !SHARE || (kb_begin(tl) == 0 && kb_end(tl) == KB);
      bool mine = true;   // the sums are complete and this warp's to finish
      if constexpr (SHARE) {
        if (!whole && turn * 16 < t.rows) {
          const int w = tile_at(tl), first = w * KB / per, last = ((w + 1) * KB - 1) / per;   // CTAs that share the tile
#pragma unroll 1
          for (int r0 = turn * 16; r0 < t.rows; r0 += 32) {
            uint32_t a[16], b[16];
            ptx::tmem_ld16(taddr + r0, a);
            ptx::tmem_ld16(taddr + F4_ROWS + r0, b);
            ptx::tmem_ld_wait_on(a, b);
            float* to = slot(2 * blockIdx.x + (kb_begin(tl) == 0 ? 1 : 0), r0);
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (r0 + r < t.rows) {
                __stcg(to + r * 256, __uint_as_float(a[r]));
                __stcg(to + r * 256 + 128, __uint_as_float(b[r]));
              }
          }
          __threadfence();
          __syncwarp();
          int before = 0;
          if (lane == 0) before = atomicAdd(p.arrived + first * EPI_WARPS + warp, 1);
          mine = __shfl_sync(0xFFFFFFFFu, before, 0) == last - first;
          __threadfence();
          for (int r0 = turn * 16; mine && r0 < t.rows; r0 += 32)
#pragma unroll 1
            for (int r = r0; r < min(r0 + 16, t.rows); ++r) {   // back into the accumulator, four parts on their way at once
              float a = 0.f, b = 0.f;
#pragma unroll 1
              for (int i0 = first; i0 <= last; i0 += 4) {
                float va[4], vb[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const float* from = slot(2 * min(i0 + i, last) + (i0 + i == first ? 1 : 0), r);
                  va[i] = i0 + i <= last ? __ldcg(from) : 0.f;
                  vb[i] = i0 + i <= last ? __ldcg(from + 128) : 0.f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) { a += va[i]; b += vb[i]; }
              }
              ptx::tmem_st1(taddr + r, __float_as_uint(a));
              ptx::tmem_st1(taddr + F4_ROWS + r, __float_as_uint(b));
            }
          ptx::tmem_st_wait();
        }
      }
#pragma unroll 1
      for (int r0 = turn * 16; mine && r0 < t.rows; r0 += 32) {   // the two warps of a quarter take turns
        uint32_t a[16], b[16];
        ptx::tmem_ld16(taddr + r0, a);
        ptx::tmem_ld16(taddr + F4_ROWS + r0, b);
        ptx::tmem_ld_wait_on(a, b);
        if (GLU) {
          // Block of 32 columns = the warp, a row at a time, each step for all 16 rows before the next: one row after the other, the chain of a row's
          // reduction left two warps per scheduler idle two thirds of the time (9819 tokens on 64 experts of 576 x 2656, GEMM-1 alone on this form:
          // 139 us, 66 so).  Lane r has the scale of row r.
          const bool in = t.c0 * 128 + quarter * 32 < p.N;   // N is a multiple of 32
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            const float2 h = silu_mul2(__uint_as_float(a[r]), __uint_as_float(a[r + 1]), __uint_as_float(b[r]), __uint_as_float(b[r + 1]));
            a[r] = __float_as_uint(h.x);
            a[r + 1] = __float_as_uint(h.y);
          }
          uint32_t top = 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, a[r] & 0x7FFFFFFFu);   // as numbers: of magnitudes the same order, NaN above all
            if ((lane & 15) == r) top = m;
          }
          const uint32_t sb = fp4::scale_byte(__uint_as_float(top));
          const float inv = fp4::inverse(sb);
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            uint32_t mine = 0;   // this column's codes of eight rows
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              const int r = g * 8 + i;
              mine |= fp4::code2(__uint_as_float(a[r]) * __shfl_sync(0xFFFFFFFFu, inv, r),
                                 __uint_as_float(a[r + 1]) * __shfl_sync(0xFFFFFFFFu, inv, r + 1)) << (4 * i);
            }
            mine = fp4::transpose8(mine, lane);     // lane l of eight: row l, the columns of its group of eight
            const int row = r0 + g * 8 + (lane & 7);
            if (row < t.rows && in)
              p.hq[(size_t)(t.row0 + row) * (size_t)(p.N / 8) + t.c0 * 16 + quarter * 4 + (lane >> 3)] = mine;
          }
          const int row = r0 + lane;
          if (lane < 16 && row < t.rows) {
            uint8_t* sf = p.sfh + f4_scale_at(t.mt, row, F4_ROWS, fp4::chunks(p.N), t.c0) + quarter;
            sf[0] = in ? (uint8_t)sb : 127;
            if (t.c0 + 1 == p.NC && (p.NC & 1)) sf[512] = 127;   // the chunk past the last column is part of a stage
          }
        } else {
          const int col0 = t.c0 * 128 + quarter * 32;
          f4_store_rows<F4_ROWS, 2>(p, a, out_mem, r0 >> 5, lane, t.row0 + r0, t.rows - r0, col0);
          if (t.halves > 1) f4_store_rows<F4_ROWS, 2>(p, b, out_mem, r0 >> 5, lane, t.row0 + r0, t.rows - r0, col0 + 128);
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(tempty_bar(buf));
    }
  } else if (warp == TMA_WARP) {
    // ================================ TMA producer ================================
    if (lane == 0) {
      uint32_t it = 0;
      int e = 0;
      for (int j = 0; j < items && !*abort_flag; ++j) {
        const F4Tile t = tile_of(tile_at(j), e);
        e = t.e;
        const int box = (t.rows + 31) / 32;   // rows by 32; what the stage held behind them reaches no stored row
        const uint32_t bytes = (uint32_t)(t.halves * (W_BYTES + SF_BYTES) + box * 32 * 128 + SF_BYTES);
        const size_t wc0 = (size_t)t.e * p.NC + t.c0, wc1 = GLU ? wc0 : wc0 + 1;
        bool ok = true;
        const int end = kb_end(j);
        for (int kb = kb_begin(j); kb < end; ++kb, ++it) {
          const int s = it % NSTAGE;
          if (!ptx::mbar_wait<false, HINT>(empty_bar(s), ((it / NSTAGE) & 1) ^ 1, abort_flag, global_abort)) {
            timeout(2); ok = false; break;
          }
          const uint32_t sw = smem_base + s * STAGE_BYTES, sx = sw + 2 * W_BYTES, sf = sx + X_BYTES, bar = full_bar(s);
          ptx::mbar_arrive_expect_tx(bar, bytes);
          ptx::tma_load_3d(sw, &map_wa, bar, kb * 128, t.c0 * 128, t.e);
          ptx::bulk_load(sf + SF_BYTES, p.sfa + (wc0 * KB + kb) * SF_BYTES, SF_BYTES, bar);
          if (t.halves > 1) {
            ptx::tma_load_3d(sw + W_BYTES, &map_wb, bar, kb * 128, GLU ? t.c0 * 128 : t.c0 * 128 + 128, t.e);
            ptx::bulk_load(sf + 2 * SF_BYTES, p.sfb + (wc1 * KB + kb) * SF_BYTES, SF_BYTES, bar);
          }
          ptx::tma_load_2d(sx, &xmaps.m[box - 1], bar, kb * 128, t.row0);
          ptx::bulk_load(sf, p.sfx + ((size_t)t.mt * KB + kb) * SF_BYTES, SF_BYTES, bar);
        }
        if (!ok) break;
      }
    }
  } else if (warp == MMA_WARP) {
    // ================================ UMMA issuer: the warp walks the loop, one elected lane issues ================================
    const bool elected = ptx::elect_one();
    const uint32_t base = __shfl_sync(0xFFFFFFFFu, smem_base, 0), tmem = __shfl_sync(0xFFFFFFFFu, tmem_base, 0);
    const uint64_t w_desc = desc_at(desc_base(16, 1024), base), x_desc = desc_at(desc_base(16, 1024), base + 2 * W_BYTES);
    const uint64_t sf_desc = scale_desc(base + 2 * W_BYTES + X_BYTES);
    int s = 0, tl = 0, e = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (; ok && tl < items && !*abort_flag; ++tl) {
      const int buf = tl & 1;
      const F4Tile t = tile_of(tile_at(tl), e);
      e = t.e;
      if (!ptx::mbar_wait(tempty_bar(buf), ((tl >> 1) & 1) ^ 1, abort_flag, global_abort)) { timeout(3); break; }
      ptx::tc_fence_after();
      const uint32_t d = tmem + (uint32_t)(buf * BUF_COLS);
      const int n = (t.rows + 15) & ~15;
      const uint32_t id0 = idesc_f4(128, n, 0), id1 = idesc_f4(128, n, 2);
      const int begin = kb_begin(tl), end = kb_end(tl);
      for (int kb = begin; kb < end; ++kb) {
        if (!ptx::mbar_wait(full_bar(s), ph, abort_flag, global_abort)) { timeout(4); ok = false; break; }
        ptx::tc_fence_after();
        if (elected) {
          const uint64_t so = (uint64_t)(s * (STAGE_BYTES >> 4));
          const uint32_t sf = tmem + (uint32_t)(SF_TMEM + s * SF_COLS);   // X chunks, W half 0 chunks, W half 1 chunks: four columns each
#pragma unroll
          for (int i = 0; i < 6; ++i)
            if (i < 4 || t.halves > 1) ptx::tmem_copy_scales(sf + 4 * i, sf_desc + so + (uint64_t)(i * (512 >> 4)));
#pragma unroll
          for (int k = 0; k < 4; ++k) {   // 64 of K: 32 bytes inside the swizzle row
            const uint32_t id = (k & 1) ? id1 : id0, ch = (uint32_t)(4 * (k >> 1));
            ptx::umma_f4(d, w_desc + so + 2 * k, x_desc + so + 2 * k, id, sf + 8 + ch, sf + ch, kb > begin || k > 0);
            if (t.halves > 1)
              ptx::umma_f4(d + F4_ROWS, w_desc + so + (W_BYTES >> 4) + 2 * k, x_desc + so + 2 * k, id, sf + 16 + ch, sf + ch, kb > begin || k > 0);
          }
          ptx::umma_commit(empty_bar(s));   // free the stage when these UMMAs have read it
        }
        if (++s == NSTAGE) { s = 0; ph ^= 1u; }
      }
      if (ok && elected) ptx::umma_commit(tfull_bar(buf));
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (*abort_flag || *global_abort) {
    // abort path only: give bulk copies and UMMAs still in flight time to land before the CTA retires
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
  }
  __syncthreads();
  if (warp == MMA_WARP) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem_base, 512);
  }
}

// Quantised rows, gathered into expert-sorted order, their scales into the chunks of the row tiles, and the rows' gate weights.  A warp takes `chunk`
// neighbouring rows.  Only the scales need the tables of the experts, so those are built while the first rows are on their way.
__global__ void __launch_bounds__(256) fp4_sort_kernel(const uint4* __restrict__ xq, const uint8_t* __restrict__ sx, int a_rows,
                                                       const int32_t* __restrict__ gather_idx, int gather_div,
                                                       const int32_t* __restrict__ expert_offsets, int E, int K, int capacity, int tile_rows,
                                                       int chunk, uint4* xs, uint8_t* sfx, const float* __restrict__ topk_w,
                                                       const int32_t* __restrict__ row_pair, float* row_w, int32_t* arrived, int n_arrived,
                                                       int32_t* status) {
  __shared__ int eoff[MAX_E + 1], tp[MAX_E + 1];
  grid_dependency_sync();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int KB = K / 32, words = fp4::chunks(K);              // scale bytes of a row, and its 4-byte words in the chunks
  const long long r0 = ((long long)blockIdx.x * 8 + warp) * chunk;
  const int n = (int)max(0ll, min((long long)chunk, min((long long)__ldg(expert_offsets + E), (long long)capacity) - r0));   // rows of this warp
  f4_load_offsets(expert_offsets, E, eoff);
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < n_arrived; i += 256) arrived[i] = 0;   // for the products behind this kernel
  int src = -1;
  if (lane < n) {
    const int r = (int)r0 + lane;
    src = __ldg(gather_idx + r);
    if (gather_div > 1) src /= gather_div;
    if (src < 0 || src >= a_rows) {
      report_error(status, DEV_INDEX_OUT_OF_RANGE, KID_GEMM1, src, r);
      src = -1;
    }
    if (row_w != nullptr) {   // nothing is read with a number that lies outside the batch
      const int pair = __ldg(row_pair + r);
      const bool valid = pair >= 0 && pair < capacity;
      if (!valid) report_error(status, DEV_INDEX_OUT_OF_RANGE, KID_GEMM1, pair, r);
      row_w[r] = valid ? __ldg(topk_w + pair) : 0.f;
    }
  }
  for (int j = 0; j < n; ++j) {
    const int s = __shfl_sync(0xFFFFFFFFu, src, j);
    if (s < 0) continue;
    const uint4* from = xq + (size_t)s * KB;
    uint4* to = xs + (size_t)(r0 + j) * KB;
#pragma unroll 4
    for (int v = lane; v < KB; v += 32) to[v] = __ldg(from + v);
  }
  __syncthreads();
  if (warp == 0) f4_tile_table(eoff, E, tile_rows, tp, lane);
  __syncthreads();
  if (n == 0) return;
  const bool whole = KB % 4 == 0 && (reinterpret_cast<uintptr_t>(sx) & 3) == 0;
  int e = 0;
  for (int hi = E; hi - e > 1;) {   // the first row's expert: the last that starts at or before it, and is not empty
    const int mid = (e + hi) >> 1;
    if (eoff[mid] <= (int)r0) e = mid; else hi = mid;
  }
  for (int j = 0; j < n; ++j) {
    const int s = __shfl_sync(0xFFFFFFFFu, src, j), r = (int)r0 + j;
    while (eoff[e + 1] <= r) ++e;
    if (s < 0) continue;
    uint8_t* sf = sfx + f4_scale_at(tp[e], r - eoff[e], tile_rows, words, 0);
    const uint8_t* from = sx + (size_t)s * KB;
    for (int c = lane; c < words; c += 32) {
      uint32_t v = 0x7F7F7F7Fu;
      if (4 * c < KB) {
        if (whole) v = __ldg(reinterpret_cast<const uint32_t*>(from + 4 * c));
        else
          for (int i = 0; i < 4 && 4 * c + i < KB; ++i) v = (v & ~(0xFFu << (8 * i))) | ((uint32_t)__ldg(from + 4 * c + i) << (8 * i));
      }
      *reinterpret_cast<uint32_t*>(sf + (size_t)c * 512) = v;
    }
  }
}

template <bool GLU, bool SHARE>
cudaError_t launch_form(const F4Params& p, const void* wa, const void* wb, const void* rows, long long n_rows, cudaStream_t st) {
  static std::atomic<bool> attr_set[MAX_DEVICES];   // per device; setting it twice is harmless
  const int dev = current_device();
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(ffn_fp4_kernel<GLU, SHARE>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
    if (e != cudaSuccess) return e;
    attr_set[dev].store(true, std::memory_order_release);
  }
  CUtensorMap m_a, m_b;
  F4RowMaps x{};
  if (!make_weight_map_fp8(&m_a, wa, p.E, p.N, p.K / 2, 128)) return cudaErrorInvalidValue;
  m_b = m_a;
  if (GLU && !make_weight_map_fp8(&m_b, wb, p.E, p.N, p.K / 2, 128)) return cudaErrorInvalidValue;
  for (int i = 0; i < F4_ROWS / 32; ++i)
    if (!make_act_map(&x.m[i], rows, n_rows, p.K / 2, true, 32 * (i + 1))) return cudaErrorInvalidValue;
  ProfileScope prof(GLU ? KID_GEMM1 : KID_GEMM2, st);
  return launch_pdl(ffn_fp4_kernel<GLU, SHARE>, dim3(min(sm_count(), F4_CTAS)), dim3(THREADS), SMEM_BYTES, st, m_a, m_b, x, p);
}

template <bool GLU>
cudaError_t launch_gemm(const F4Params& p, const void* wa, const void* wb, const void* rows, long long n_rows, bool share, cudaStream_t st) {
  return share ? launch_form<GLU, true>(p, wa, wb, rows, n_rows, st) : launch_form<GLU, false>(p, wa, wb, rows, n_rows, st);
}

}  // namespace
}  // namespace ffn

long long fp4_row_sets(const Shape& s) {
  const long long P = (long long)s.T * s.k, e = s.E < P ? s.E : P;
  const long long one = P / ffn::F4_ROWS + e, two = 2 * (P / ffn::F4_PAIR_ROWS2 + e);   // every expert's last tile may be a part
  return one > two ? one : two;
}

// CTA pairs from 128 rows per expert on.  FFN on single CTAs / pairs, us, rows per expert in brackets: 1500 skewed tokens, top-2 of 64 x 2048 x 2048 (47)
// 97 / 117, 3000, top-2 of 64 x 2048 x 2048 (94) 108 / 120, 3200, top-4 of 128 x 2048 x 1024 (100) 133 / 133, 3318 on 32 x 1888 x 7168 (104) 217 / 198, 1777
// skewed, top-4 of 64 x 2880 x 2880 (111) 225 / 252, 450, top-2 of 8 x 4096 x 4096 (112) 66 / 66, 1000 skewed, top-4 of 32 x 1024 x 1024 (125) 37 / 41,
// 4096, top-2 of 64 x 2048 x 2048 (128) 135 / 128, 2900, top-2 of 32 x 2880 x 2880 (181) 156 / 135, 800, top-2 of 8 x 2048 x 7168 (200) 77 / 67, 3600
// skewed on 16 x 4096 x 1536 (225) 81 / 79.  Near the rule the routing decides: 1900, top-8 of 128 x 4096 x 1536 (119) even 349 / 318, skewed 328 / 364.
// (Both forms side by side, each for the experts of its kind, gained nothing where routing is skewed and lost where tiles are few.)
static bool fp4_pairs(const Shape& s) { return (long long)s.T * s.k >= 128ll * s.E; }

// Whether a product's tiles (at most row_tiles * ceil(N / width)) are shared.  A CTA streams at most 63 KB/us, all together 6.5 TB/s: tiles that leave SMs
// idle take KB * 0.55 us whole, tiles * KB * 0.0052 us shared and then about 4 us for their parts.
static bool fp4_share(const Shape& s, int K, int N, int width) {
  const long long P = (long long)s.T * s.k, row_tiles = P / ffn::F4_ROWS + (s.E < P ? s.E : P);
  const long long tiles = row_tiles * ((N + width - 1) / width), KB = (K + ffn::F4_BK - 1) / ffn::F4_BK;
  return !fp4_pairs(s) && KB * (105 - tiles) > 770;
}
static bool fp4_share1(const Shape& s) { return fp4_share(s, s.d, s.f, 128); }
static bool fp4_share2(const Shape& s) { return fp4_share(s, s.f, s.d, 256); }
static int fp4_part_rows(const Shape& s) {
  const long long P = (long long)s.T * s.k;
  return P < ffn::F4_ROWS ? (int)(P + 15) & ~15 : ffn::F4_ROWS;
}
static bool fp4_shares(const Shape& s) { return fp4_share1(s) || fp4_share2(s); }
// Rows that parts are reserved for: those of the largest batch of at most s.T tokens that shares tiles (0 if none does), so that a workspace for many
// tokens serves fewer.  Tiles only grow with the tokens, so batches share up to some number of tokens, and F4_ROWS rows are the most.
static int fp4_reserved_rows(const Shape& s) {
  Shape b = s;
  b.T = min(s.T, (ffn::F4_ROWS + s.k - 1) / s.k);
  if (b.T > 0 && !fp4_shares(b)) {
    int hi = b.T;   // does not share
    b.T = 1;
    if (!fp4_shares(b)) b.T = 0;
    while (hi - b.T > 1 && b.T > 0) {
      const int low = b.T;
      b.T = (low + hi) / 2;
      if (!fp4_shares(b)) {
        hi = b.T;
        b.T = low;
      }
    }
  }
  return b.T > 0 ? fp4_part_rows(b) : 0;
}
size_t fp4_part_bytes(const Shape& s) { return (size_t)2 * ffn::F4_CTAS * fp4_reserved_rows(s) * 256 * 4; }
size_t fp4_arrived_bytes(const Shape& s) { return fp4_reserved_rows(s) > 0 ? (size_t)2 * ffn::F4_CTAS * 8 * 4 : 0; }

cudaError_t launch_expert_ffn_fp4(const Shape& s, const FfnArgs& a, const Fp4Args& q, cudaStream_t st) {
  if (s.T == 0) return cudaSuccess;
  const int P = s.T * s.k;
  const bool pairs = fp4_pairs(s);
  const int rows1 = pairs ? ffn::F4_PAIR_ROWS1 : ffn::F4_ROWS, rows2 = pairs ? ffn::F4_PAIR_ROWS2 : ffn::F4_ROWS;
  float* row_w = a.topk_w != nullptr ? q.row_w : nullptr;
  // rows per warp: one as long as all of them are resident at once; 131072 rows of 4096, us with 1 / 2 / 4 / 8 / 16: 122 / 94 / 89 / 95 / 116
  const int chunk = P >= 8 * 64 * sm_count() ? 4 : 1;
  cudaError_t e = launch_pdl(ffn::fp4_sort_kernel, dim3((unsigned)((P + 8 * chunk - 1) / (8 * chunk))), dim3(256), 0, st, static_cast<const uint4*>(a.a_src),
                             q.sx, a.a_rows, a.gather_idx, a.gather_div, a.expert_offsets, s.E, s.d, P, rows1, chunk, static_cast<uint4*>(a.xs), q.sfx,
                             a.topk_w, a.row_pair, row_w, q.arrived, fp4_shares(s) ? 2 * ffn::F4_CTAS * 8 : 0, a.status);
  if (e != cudaSuccess) return e;
  ffn::F4Params g1{};
  g1.expert_offsets = a.expert_offsets;
  g1.E = s.E;
  g1.K = s.d;
  g1.N = s.f;
  g1.NC = (s.f + 127) / 128;
  g1.sfx = q.sfx;
  g1.sfa = q.s1;
  g1.sfb = q.s3;
  g1.hq = static_cast<uint32_t*>(a.h);
  g1.sfh = q.sfh;
  g1.h_rows = rows2;
  g1.part = q.part;
  g1.part_rows = fp4_part_rows(s);
  g1.arrived = q.arrived;
  g1.status = a.status;
  e = pairs ? ffn::launch_fp4_pair(true, g1, a.w1, a.w3, a.xs, P, fp4_row_sets(s), st) : ffn::launch_gemm<true>(g1, a.w1, a.w3, a.xs, P, fp4_share1(s), st);
  if (e != cudaSuccess) return e;
  ffn::F4Params g2{};
  g2.expert_offsets = a.expert_offsets;
  g2.E = s.E;
  g2.K = s.f;
  g2.N = s.d;
  g2.NC = (s.d + 127) / 128;
  g2.sfx = q.sfh;
  g2.sfa = g2.sfb = q.s2;
  g2.out = static_cast<__nv_bfloat16*>(a.o);
  g2.row_w = row_w;
  g2.part = q.part;
  g2.part_rows = g1.part_rows;
  g2.arrived = q.arrived + ffn::F4_CTAS * 8;
  g2.status = a.status;
  return pairs ? ffn::launch_fp4_pair(false, g2, a.w2, a.w2, a.h, P, fp4_row_sets(s), st) : ffn::launch_gemm<false>(g2, a.w2, a.w2, a.h, P, fp4_share2(s), st);
}

}  // namespace tcmoe
