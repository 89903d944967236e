// The FP4 expert products on CTA pairs (cluster of 2, tcgen05 cta_group::2), for experts of many rows; formats as in ffn_fp4.cu.
//
// At 4 bits the tensor cores outrun L2: what bounds the products is the bytes that a tile fetches per operation, so tiles are as large
// as TMEM allows next to the scales.
//   GEMM-1  256 rows (M, 128 in each CTA) x 128 columns of W1 and the same of W3 (N = 256, CTA 0 holds those of W1, CTA 1 those of W3): every CTA has
//           both products of its rows, a thread one row, and 32 neighbouring columns, a block of the quantisation, in its registers.
//           One accumulator of 256 columns (a second does not fit beside the scales): the epilogue takes it into registers, 128 per thread,
//           lets the next tile start, and works from there.
//   GEMM-2  256 columns of W2 (M) x up to 208 rows (N, rounded up to 16: no padded rows), two accumulators.  TMEM has room for the scales of four of its six
//           stages: the UMMAs that read a slot's are waited for before it is filled again.  (With 192 rows and five stages, 4096 tokens, top-2 of 8 experts
//           of 14336 x 4096: 240 us, 207 so; 1024 rows are five tiles instead of six.)
// Two warps feed a stage, one its operands and one their scales: with five copies per stage one thread was busy for 400 of a stage's 512 cycles.
// Pair protocol, barriers and the abort path are those of ffn_gemm2.cu; rank 0 issues every UMMA and copy of scales to TMEM.
#include "ffn_fp4.cuh"

#include <atomic>

namespace tcmoe {
namespace ffn {
namespace {

constexpr int W_BYTES = 128 * 128;                 // this CTA's 128 weight columns x 256 of K
constexpr int SF_COLS = 24;                        // TMEM columns of a stage's scales
constexpr int TABLE_BYTES = (3 * (MAX_E + 1) * 4 + 15) & ~15;
constexpr uint32_t HINT = 4000;

template <bool GLU> struct Geo {
  // Eight: GEMM-1's hold 128 accumulator columns each in registers; GEMM-2's took 567 us with sixteen for 131072 rows of 1536 and 128 experts of 1536 x
  // 4096, 540 with eight (the board is at its power limit).
  static constexpr int EPI_WARPS = 8, SHARES = EPI_WARPS / 4;
  static constexpr int TMA_WARP = EPI_WARPS, MMA_WARP = EPI_WARPS + 1, SF_WARP = EPI_WARPS + 2, THREADS = (EPI_WARPS + 3) * 32;
  using Out = F4Out<F4_PAIR_ROWS2, SHARES>;   // GEMM-2
  static constexpr int TILE_ROWS = GLU ? F4_PAIR_ROWS1 : F4_PAIR_ROWS2;
  static constexpr int X_BYTES = 128 * TILE_ROWS / 2;
  static constexpr int STAGE_BYTES = W_BYTES + X_BYTES + 3 * F4_SF_BYTES;   // W, X, scales
  static constexpr int NSTAGE = 6, SLOTS = GLU ? 6 : 4;   // stages, and those whose scales fit TMEM
  static constexpr int MOST_ROWS = TILE_ROWS / 2;          // of a CTA
  static constexpr int BUFS = GLU ? 1 : 2;
  static constexpr int BUF_COLS = GLU ? 256 : F4_PAIR_ROWS2;
  static constexpr int SF_TMEM = BUFS * BUF_COLS;
  static constexpr int NUM_BARS = 2 * NSTAGE + 2 * BUFS;
  static constexpr int SMEM_BYTES = 1024 + NSTAGE * STAGE_BYTES + NUM_BARS * 8 + 64 + TABLE_BYTES + (GLU ? 0 : EPI_WARPS * Out::BYTES);
  static_assert(SF_TMEM + SLOTS * SF_COLS <= 512, "TMEM");
  static_assert(SMEM_BYTES <= 232448, "shared memory of an SM");
  static_assert(STAGE_BYTES % 1024 == 0 && X_BYTES % 1024 == 0, "swizzle atoms");
};

struct PairTile {
  int e, tile, row0, rows, lr0, c0;   // expert, row tile over all experts, first row, rows left from it on, first row inside the expert, first chunk
};

template <bool GLU>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Geo<GLU>::THREADS, 1)
ffn_fp4_pair_kernel(const __grid_constant__ CUtensorMap map_wa, const __grid_constant__ CUtensorMap map_wb,
                    const __grid_constant__ CUtensorMap map_sfa, const __grid_constant__ CUtensorMap map_sfb,
                    const __grid_constant__ CUtensorMap map_sfx, const __grid_constant__ F4RowMaps xmaps, const F4Params p) {
  using G = Geo<GLU>;
  constexpr int NSTAGE = G::NSTAGE, EPI_WARPS = G::EPI_WARPS, TMA_WARP = G::TMA_WARP, MMA_WARP = G::MMA_WARP, SF_WARP = G::SF_WARP;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + NSTAGE * G::STAGE_BYTES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + G::NUM_BARS);
  int* abort_s = reinterpret_cast<int*>(tmem_slot + 1);
  int* tp_s = reinterpret_cast<int*>(tmem_slot + 16);
  int* eoff_s = tp_s + (MAX_E + 1);
  int* hp_s = eoff_s + (MAX_E + 1);   // GEMM-1: tiles of the product that reads h
  const uint32_t smem_base = ptx::smem_u32(smem), bar_base = ptx::smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (NSTAGE + s); };
  auto tfull_bar = [&](int b) { return bar_base + 8u * (2 * NSTAGE + b); };
  auto tempty_bar = [&](int b) { return bar_base + 8u * (2 * NSTAGE + G::BUFS + b); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)ptx::cluster_ctarank();
  const int cluster_id = blockIdx.x >> 1, num_clusters = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < NSTAGE; ++s) {
      ptx::mbar_init(full_bar(s), 2);    // the leader's two TMA threads (expect_tx for both CTAs)
      ptx::mbar_init(empty_bar(s), 1);   // tcgen05.commit
    }
    for (int b = 0; b < G::BUFS; ++b) {
      ptx::mbar_init(tfull_bar(b), 1);                 // tcgen05.commit
      ptx::mbar_init(tempty_bar(b), 2 * EPI_WARPS);    // one lane per epilogue warp, both CTAs
    }
    ptx::fence_mbar_init();
  }
  if (warp == TMA_WARP && lane == 0) {
    ptx::prefetch_tensormap(&map_wa);
    ptx::prefetch_tensormap(&map_wb);
    ptx::prefetch_tensormap(&map_sfa);
    ptx::prefetch_tensormap(&map_sfb);
    ptx::prefetch_tensormap(&map_sfx);
  }
  if (warp == MMA_WARP) {
    ptx::tmem_alloc_pair(ptx::smem_u32(tmem_slot), 512);
    ptx::tmem_relinquish_pair();
  }
  grid_dependency_sync();   // nothing above touches global data
  f4_load_offsets(p.expert_offsets, p.E, eoff_s);
  __syncthreads();
  if (warp == 0) f4_tile_table(eoff_s, p.E, G::TILE_ROWS, tp_s, lane);
  if (GLU && warp == 1) f4_tile_table(eoff_s, p.E, p.h_rows, hp_s, lane);
  if (threadIdx.x == 64) *abort_s = p.status[ST_ABORT];
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();   // the peer's barriers are initialised before anything signals them
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int n_tiles = GLU ? p.NC : (p.NC + 1) / 2;
  const int total = tp_s[p.E] * n_tiles;
  const int KB = (p.K + F4_BK - 1) / F4_BK;
  volatile int* abort_flag = abort_s;
  const volatile int* global_abort = p.status + ST_ABORT;
  auto timeout = [&](int detail) {
    report_error(p.status, DEV_TIMEOUT, GLU ? KID_GEMM1 : KID_GEMM2, detail, blockIdx.x);
    p.status[ST_ABORT] = 1;
    *abort_flag = 1;
  };
  // Expert by expert; inside one, row tiles in groups of about 2048 rows, and in a group column tile by column tile, rows fastest: pairs that
  // run together share the weights of a column tile, and a group's rows stay in L2.
  auto tile_of = [&](int w, int from) {   // from: an expert at or before the tile's
    constexpr int MG = 2048 / G::TILE_ROWS;
    PairTile t;
    t.e = f4_expert_from(tp_s, from, n_tiles, w);
    uint32_t local = (uint32_t)(w - tp_s[t.e] * n_tiles);
    const int mts = tp_s[t.e + 1] - tp_s[t.e], g = mts > MG ? (int)(local / (uint32_t)(MG * n_tiles)) : 0;
    local -= (uint32_t)(g * MG * n_tiles);
    const uint32_t gsize = (uint32_t)min(MG, mts - g * MG), c = local / gsize;
    const int m = g * MG + (int)(local - c * gsize);
    t.tile = tp_s[t.e] + m;
    t.lr0 = m * G::TILE_ROWS;
    t.row0 = eoff_s[t.e] + t.lr0;
    t.rows = min(G::TILE_ROWS, eoff_s[t.e + 1] - t.row0);
    t.c0 = GLU ? (int)c : 2 * (int)c;
    return t;
  };

  if (warp < EPI_WARPS) {
    // ================================ epilogue (both CTAs) ================================
    const int quarter = warp & 3, half = warp >> 2;
    const uint32_t out_mem = ptx::smem_u32(tp_s) + TABLE_BYTES + (uint32_t)(warp * G::Out::BYTES);   // GEMM-2
    int tl = 0;
    PairTile t{}, next{};
    float rw[(G::Out::TURNS + 1) / 2];
    if (cluster_id < total) {
      next = tile_of(cluster_id, 0);
      if constexpr (!GLU) f4_fetch_weights<F4_PAIR_ROWS2, G::SHARES>(p, next.row0, next.rows, half, lane, rw);
    }
    // Looked at once, alike for all lanes: the wait's shuffle, which ends the loop after an abort, wants the whole warp.
    const bool go = __all_sync(0xFFFFFFFFu, !*abort_flag);
    for (int w = cluster_id; go && w < total; w += num_clusters, ++tl) {
      t = next;
      if constexpr (!GLU) f4_keep_weights<F4_PAIR_ROWS2, G::SHARES>(rw, out_mem, lane);
      if (w + num_clusters < total) {
        next = tile_of(w + num_clusters, t.e);
        if constexpr (!GLU) f4_fetch_weights<F4_PAIR_ROWS2, G::SHARES>(p, next.row0, next.rows, half, lane, rw);
      }
      const int buf = GLU ? 0 : tl & 1;
      const uint32_t phase = GLU ? tl & 1 : (tl >> 1) & 1;
      if (!ptx::mbar_wait_warp<false, HINT>(tfull_bar(buf), phase, abort_flag, global_abort)) { timeout(1); break; }
      ptx::tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * G::BUF_COLS);
      if constexpr (GLU) {
        // lane = row, columns 64 half .. + 63 of both products
        uint32_t a[2][32], b[2][32];
        auto load = [&](uint32_t (&a0)[32], uint32_t (&a1)[32], uint32_t (&b0)[32], uint32_t (&b1)[32]) {
          ptx::tmem_ld32(taddr + half * 64, a0);
          ptx::tmem_ld32(taddr + half * 64 + 32, a1);
          ptx::tmem_ld32(taddr + 128 + half * 64, b0);
          ptx::tmem_ld32(taddr + 128 + half * 64 + 32, b1);
          ptx::tmem_ld_wait_on(a0, a1);
          ptx::tmem_ld_wait_on(b0, b1);
        };
        load(a[0], a[1], b[0], b[1]);
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_cluster_relaxed(ptx::mapa(tempty_bar(0), 0));
        const int row = rank * BM + quarter * 32 + lane;
        uint32_t codes[2][4], scales = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float top = 0.f;
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float2 h = silu_mul2(__uint_as_float(a[i][j]), __uint_as_float(a[i][j + 1]), __uint_as_float(b[i][j]), __uint_as_float(b[i][j + 1]));
            top = fp4::max_nan(top, fp4::max_nan(fabsf(h.x), fabsf(h.y)));
            a[i][j] = __float_as_uint(h.x);
            a[i][j + 1] = __float_as_uint(h.y);
          }
          const bool in = t.c0 * 128 + half * 64 + i * 32 < p.N;
          const uint32_t sb = in ? fp4::scale_byte(top) : 127u;
          const float inv = fp4::inverse(sb);
          scales |= sb << (8 * i);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(a[i][q * 8 + j]);
            codes[i][q] = fp4::codes8(f, inv);
          }
        }
        if (row < t.rows) {
          uint32_t* dst = p.hq + (size_t)(t.row0 + row) * (size_t)(p.N / 8) + t.c0 * 16 + half * 8;
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (t.c0 * 128 + half * 64 + i * 32 < p.N) *reinterpret_cast<uint4*>(dst + 4 * i) = make_uint4(codes[i][0], codes[i][1], codes[i][2], codes[i][3]);
          uint8_t* sf = p.sfh + f4_scale_at(hp_s[t.e], t.lr0 + row, p.h_rows, fp4::chunks(p.N), t.c0) + half * 2;
          *reinterpret_cast<uint16_t*>(sf) = (uint16_t)scales;
          if (t.c0 + 1 == p.NC && (p.NC & 1)) *reinterpret_cast<uint16_t*>(sf + 512) = 0x7F7F;   // the chunk past the last column is part of a stage
        }
      } else {
        // lane = column of this CTA's 128, TMEM column = row; the warps of a quarter take turns
        const int col0 = (t.c0 + rank) * 128 + quarter * 32;
#pragma unroll 1
        for (int r0 = half * 16, i = 0; r0 < t.rows; r0 += 16 * G::SHARES, ++i) {
          uint32_t a[16];
          ptx::tmem_ld16(taddr + r0, a);
          ptx::tmem_ld_wait_on(a);
          f4_store_rows<G::TILE_ROWS, G::SHARES>(p, a, out_mem, i, lane, t.row0 + r0, t.rows - r0, col0);
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_cluster_relaxed(ptx::mapa(tempty_bar(buf), 0));
      }
    }
  } else if (warp == TMA_WARP || warp == SF_WARP) {
    // ================================ TMA producers (both CTAs): operands, and their scales ================================
    if (lane == 0) {
      const bool scales = warp == SF_WARP;
      int s = 0, e = 0;
      uint32_t ph = 1;
      bool ok = true;
      for (int w = cluster_id; ok && w < total && !*abort_flag; w += num_clusters) {
        const PairTile t = tile_of(w, e);
        e = t.e;
        // rows of this CTA and its first one; boxes of 32 (what the stage held behind them reaches no stored row)
        const int n = (t.rows + 15) & ~15, first = GLU ? rank * BM : rank * (n / 2);
        auto blocks32 = [&](int r) { return GLU ? (min(max(t.rows - r * BM, 0), BM) + 31) >> 5 : (n / 2 + 31) >> 5; };
        const int mine = blocks32(rank);
        auto box_rows = [&](int blocks) { return min(32 * blocks, G::MOST_ROWS); };
        const int sets = t.rows > 128 ? 2 : 1;                                         // of the tile's scales
        const bool cols = GLU || t.c0 + rank < p.NC, both = GLU || t.c0 + 1 < p.NC;    // this CTA has weight columns; both have
        // of both CTAs: the leader announces them, the peer's copies only complete them
        const uint32_t bytes = scales ? ((GLU ? 4u : both ? 2u : 1u) + (GLU ? 1 : 2) * (uint32_t)sets) * F4_SF_BYTES
                                      : (both ? 2u : 1u) * W_BYTES + (uint32_t)(box_rows(blocks32(0)) + box_rows(blocks32(1))) * 128;
        const int wc = t.e * p.NC + t.c0, set0 = 2 * t.tile;
        for (int kb = 0; kb < KB; ++kb) {
          if (!ptx::mbar_wait<false, HINT>(empty_bar(s), ph, abort_flag, global_abort)) {
            timeout(2); ok = false; break;
          }
          const uint32_t sw = smem_base + s * G::STAGE_BYTES, sx = sw + W_BYTES, sf = sx + G::X_BYTES;
          const uint32_t bar = ptx::mapa(full_bar(s), 0);
          if (rank == 0) ptx::mbar_arrive_expect_tx(full_bar(s), bytes);
          if (!scales) {
            if (cols) ptx::tma_load_3d_pair(sw, GLU && rank != 0 ? &map_wb : &map_wa, bar, kb * 128, (GLU ? t.c0 : t.c0 + rank) * 128, t.e);
            if (mine > 0) ptx::tma_load_2d_pair(sx, &xmaps.m[mine - 1], bar, kb * 128, t.row0 + first);
          } else if constexpr (GLU) {
            if (mine > 0) ptx::tma_load_2d_pair(sf, &map_sfx, bar, 0, ((set0 + rank) * KB + kb) * 2);
            ptx::tma_load_2d_pair(sf + F4_SF_BYTES, &map_sfa, bar, 0, (wc * KB + kb) * 2);
            ptx::tma_load_2d_pair(sf + 2 * F4_SF_BYTES, &map_sfb, bar, 0, (wc * KB + kb) * 2);
          } else {
            if (cols) ptx::tma_load_2d_pair(sf + 2 * F4_SF_BYTES, &map_sfa, bar, 0, ((wc + rank) * KB + kb) * 2);
            ptx::tma_load_2d_pair(sf, &map_sfx, bar, 0, (set0 * KB + kb) * 2);
            if (sets > 1) ptx::tma_load_2d_pair(sf + F4_SF_BYTES, &map_sfx, bar, 0, ((set0 + 1) * KB + kb) * 2);
          }
          if (++s == NSTAGE) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == MMA_WARP) {
    // ================================ UMMA issuer (leader CTA only): the warp walks the loop, one elected lane issues ================================
    if (rank == 0) {
      const bool elected = ptx::elect_one();
      const uint32_t base = __shfl_sync(0xFFFFFFFFu, smem_base, 0), tmem = __shfl_sync(0xFFFFFFFFu, tmem_base, 0);
      const uint64_t w_desc = desc_at(desc_base(16, 1024), base), x_desc = desc_at(desc_base(16, 1024), base + W_BYTES);
      const uint64_t sf_desc = scale_desc(base + W_BYTES + G::X_BYTES);
      int s = 0, tl = 0, e = 0, slot = 0, old = 0, it = 0;   // old: the stage whose scales had the slot before
      uint32_t ph = 0, old_ph = 0;
      bool ok = true;
      for (int w = cluster_id; ok && w < total && !*abort_flag; w += num_clusters, ++tl) {
        const int buf = GLU ? 0 : tl & 1;
        const uint32_t phase = GLU ? tl & 1 : (tl >> 1) & 1;
        const PairTile t = tile_of(w, e);
        e = t.e;
        if (!ptx::mbar_wait_cluster(tempty_bar(buf), phase ^ 1, abort_flag, global_abort)) { timeout(3); break; }
        ptx::tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(buf * G::BUF_COLS);
        const int n = GLU ? 256 : (t.rows + 15) & ~15;
        const uint32_t id0 = idesc_f4(256, n, 0), id1 = idesc_f4(256, n, 2);
        for (int kb = 0; kb < KB; ++kb) {
          if (!ptx::mbar_wait_cluster<HINT>(full_bar(s), ph, abort_flag, global_abort)) { timeout(4); ok = false; break; }
          if (G::SLOTS < NSTAGE && it++ >= G::SLOTS) {
            if (!ptx::mbar_wait_cluster<HINT>(empty_bar(old), old_ph, abort_flag, global_abort)) { timeout(5); ok = false; break; }
            if (++old == NSTAGE) { old = 0; old_ph ^= 1u; }
          }
          ptx::tc_fence_after();
          if (elected) {
            const uint64_t so = (uint64_t)(s * (G::STAGE_BYTES >> 4));
            const uint32_t sf = tmem + (uint32_t)(G::SF_TMEM + slot * SF_COLS);
            // Shared memory: three sets of two chunks.  TMEM, columns: GEMM-1 rows 0 4, W1 | W3 of one 128 of K side by side 8 12, 16 20;
            // GEMM-2 the two sets of rows side by side 0 4, 8 12, W2 16 20.
            constexpr int at[6] = {0, GLU ? 4 : 8, GLU ? 8 : 4, GLU ? 16 : 12, GLU ? 12 : 16, 20};
#pragma unroll
            for (int i = 0; i < 6; ++i) ptx::tmem_copy_scales_pair(sf + at[i], sf_desc + so + (uint64_t)(i * (512 >> 4)));
#pragma unroll
            for (int k = 0; k < 4; ++k) {   // 64 of K: 32 bytes inside the swizzle row
              const uint32_t id = (k & 1) ? id1 : id0, j = (uint32_t)(k >> 1);
              if constexpr (GLU) ptx::umma_f4_pair(d, x_desc + so + 2 * k, w_desc + so + 2 * k, id, sf + 4 * j, sf + 8 + 8 * j, (kb | k) != 0);
              else ptx::umma_f4_pair(d, w_desc + so + 2 * k, x_desc + so + 2 * k, id, sf + 16 + 4 * j, sf + 8 * j, (kb | k) != 0);
            }
            ptx::umma_commit_both(empty_bar(s));   // free the stage in both CTAs once these UMMAs have read it
          }
          if (++s == NSTAGE) { s = 0; ph ^= 1u; }
          if (++slot == G::SLOTS) slot = 0;
        }
        if (ok && elected) ptx::umma_commit_both(tfull_bar(buf));   // accumulator complete, both CTAs
      }
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (*abort_flag || *global_abort) {
    // abort path only: give bulk copies still in flight time to land before the CTAs retire
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
  }
  ptx::cluster_sync();   // neither CTA leaves while its peer may still touch its shared memory / TMEM
  if (warp == MMA_WARP) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem_base, 512);
  }
}

template <bool GLU>
cudaError_t launch(const F4Params& p, const void* wa, const void* wb, const void* rows, long long n_rows, long long row_sets, cudaStream_t st) {
  using G = Geo<GLU>;
  static std::atomic<int> grid_of[MAX_DEVICES];   // per device, 0 = not set up yet; doing it twice is harmless
  std::atomic<int>& cached = grid_of[current_device()];
  int grid = cached.load(std::memory_order_acquire);
  if (grid == 0) {
    const cudaError_t e = cudaFuncSetAttribute(ffn_fp4_pair_kernel<GLU>, cudaFuncAttributeMaxDynamicSharedMemorySize, G::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    int clusters = 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(sm_count() & ~1);
    cfg.blockDim = dim3(G::THREADS);
    cfg.dynamicSmemBytes = G::SMEM_BYTES;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&clusters, ffn_fp4_pair_kernel<GLU>, &cfg) != cudaSuccess || clusters <= 0) {
      (void)cudaGetLastError();
      clusters = sm_count() / 2;
    }
    grid = 2 * min(clusters, sm_count() / 2);
    cached.store(grid, std::memory_order_release);
  }
  CUtensorMap m_a, m_b, m_sa, m_sb, m_sx;
  F4RowMaps x;
  const long long w_chunks = (long long)p.E * p.NC * fp4::chunks(p.K);
  if (!make_weight_map_fp8(&m_a, wa, p.E, p.N, p.K / 2, 128) || !make_scale_map(&m_sa, p.sfa, w_chunks) ||
      !make_scale_map(&m_sx, p.sfx, row_sets * fp4::chunks(p.K)))
    return cudaErrorInvalidValue;
  m_b = m_a;
  m_sb = m_sa;
  if (GLU && (!make_weight_map_fp8(&m_b, wb, p.E, p.N, p.K / 2, 128) || !make_scale_map(&m_sb, p.sfb, w_chunks))) return cudaErrorInvalidValue;
  for (int i = 0; i < 4; ++i)
    if (!make_act_map(&x.m[i], rows, n_rows, p.K / 2, true, min(32 * (i + 1), G::MOST_ROWS))) return cudaErrorInvalidValue;
  ProfileScope prof(GLU ? KID_GEMM1 : KID_GEMM2, st);
  return launch_pdl(ffn_fp4_pair_kernel<GLU>, dim3(grid), dim3(G::THREADS), G::SMEM_BYTES, st, m_a, m_b, m_sa, m_sb, m_sx, x, p);
}

}  // namespace

cudaError_t launch_fp4_pair(bool glu, const F4Params& p, const void* wa, const void* wb, const void* rows, long long n_rows,
                            long long row_sets, cudaStream_t st) {
  return glu ? launch<true>(p, wa, wb, rows, n_rows, row_sets, st) : launch<false>(p, wa, wb, rows, n_rows, row_sets, st);
}

}  // namespace ffn
}  // namespace tcmoe
