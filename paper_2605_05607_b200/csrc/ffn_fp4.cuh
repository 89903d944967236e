// Pieces shared by the FP4 expert products (ffn_fp4.cu: one CTA per tile; ffn_fp4_pair.cu: CTA pairs).
#pragma once
#include "ffn_common.cuh"
#include "quant4.cuh"

namespace tcmoe {
namespace ffn {

constexpr int F4_BK = 256;                          // K per pipeline stage: 128 bytes per row of either operand
constexpr int F4_SF_BYTES = 1024;                   // scales of 128 rows over a stage, two chunks
// Rows of a tile.  The scales of a row tile lie together, in one or two sets of chunks of 128 rows: whoever writes them needs the tile of the product that reads them.
constexpr int F4_ROWS = 96;          // single CTA: two accumulators of 2 x 96 columns and the scales of four stages fit TMEM
constexpr int F4_PAIR_ROWS1 = 256;   // GEMM-1 on pairs: rows are the M side
constexpr int F4_PAIR_ROWS2 = 208;   // GEMM-2 on pairs: two accumulators of 208 columns and the scales of four stages

constexpr int F4_CTAS = 160;         // CTAs of the single-CTA products, at most (they have two slots for parts of tiles each)

struct F4RowMaps { CUtensorMap m[4]; };   // boxes of 32, 64, 96 rows, and of as many as a CTA's half of a pair tile

struct F4Params {
  const int32_t* expert_offsets;
  int E, K, N;              // K: elements
  int NC;                   // 128-column chunks of the weights
  const uint8_t* sfx;       // scale chunks of the row tiles
  const uint8_t *sfa, *sfb; // of the weights (GEMM-1: W1, W3)
  uint32_t* hq;             // GEMM-1: codes of h [P, N / 8 words], and their scale chunks per row tile of h_rows rows (GEMM-2's)
  uint8_t* sfh;
  int h_rows;
  __nv_bfloat16* out;       // GEMM-2: o [P, N]
  const float* row_w;       // gate weight of every sorted row; NULL: 1
  float* part;              // single CTAs: parts of tiles, two slots of part_rows rows x 256 columns per CTA
  int part_rows;
  int32_t* arrived;         // [F4_CTAS, 8 warps] parts of a tile that have been written, zero before the launch
  int32_t* status;
};

// Where the scales of row `lr` of an expert are whose tiles (of `rows` rows) start at `tile0`: the first byte of its word in chunk c.
__host__ __device__ __forceinline__ size_t f4_scale_at(int tile0, int lr, int rows, int chunks, int c) {
  const int in = lr % rows;
  const size_t set = (size_t)(tile0 + lr / rows) * (rows > 128 ? 2 : 1) + (in >> 7);
  return (set * (size_t)chunks + c) * 512 + (in & 31) * 16 + ((in & 127) >> 5) * 4;
}

// Instruction descriptor of kind::mxf4: A, B E2M1, both K-major, scales E8M0; the scale pair of an instruction's 64 of K is bytes id, id + 1 of the columns.
__host__ __device__ constexpr uint32_t idesc_f4(int m, int n, int id) {
  return ((uint32_t)id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 7) << 27) |
         ((uint32_t)id << 29);
}
// 32 rows of 16 bytes in shared memory, no swizzle: eight-row groups 128 bytes apart
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem_addr) {
  return (uint64_t)((smem_addr & 0x3FFFF) >> 4) | ((uint64_t)(128 >> 4) << 16) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
}

// Expert offsets into shared memory, by all threads of the block: one memory latency for any number of experts.  A barrier has to follow.
__device__ __forceinline__ void f4_load_offsets(const int32_t* expert_offsets, int E, int* eoff) {
  for (int i = threadIdx.x; i <= E; i += blockDim.x) eoff[i] = __ldcg(expert_offsets + i);
}
// silu(a) * b = (a / (1 + 2^(-a log2 e))) * b of two values: products and sums two at a time (f32x2)
__device__ __forceinline__ float2 silu_mul2(float a0, float a1, float b0, float b1) {
  float2 h;
  asm("{\n\t.reg .b64 a, b, t, c;\n\t.reg .f32 x, y;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "mov.b64 c, {%6, %6};\n\tmul.rn.f32x2 t, a, c;\n\t"
      "mov.b64 {x, y}, t;\n\tex2.approx.ftz.f32 x, x;\n\tex2.approx.ftz.f32 y, y;\n\tmov.b64 t, {x, y};\n\t"
      "mov.b64 c, {%7, %7};\n\tadd.rn.f32x2 t, t, c;\n\t"
      "mov.b64 {x, y}, t;\n\trcp.approx.ftz.f32 x, x;\n\trcp.approx.ftz.f32 y, y;\n\tmov.b64 t, {x, y};\n\t"
      "mul.rn.f32x2 t, a, t;\n\tmul.rn.f32x2 t, t, b;\n\tmov.b64 {%0, %1}, t;\n\t}"
      : "=f"(h.x), "=f"(h.y)
      : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(-1.4426950408889634f), "f"(1.f));
  return h;
}

// Tiles of `rows` rows per expert, exclusive prefix (tp[E] = all of them), by one warp.
__device__ __forceinline__ void f4_tile_table(const int* eoff, int E, int rows, int* tp, int lane) {
  int base = 0;
  for (int e0 = 0; e0 < E; e0 += 32) {
    const int e = e0 + lane;
    const int tiles = e < E ? (eoff[e + 1] - eoff[e] + rows - 1) / rows : 0;
    int sum = tiles;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int u = __shfl_up_sync(0xFFFFFFFFu, sum, off);
      if (lane >= off) sum += u;
    }
    if (e < E) tp[e] = base + sum - tiles;
    base += __shfl_sync(0xFFFFFFFFu, sum, 31);
  }
  if (lane == 0) tp[E] = base;
}

// The expert whose tiles hold task w (tp[e] * n_tiles <= w < tp[e + 1] * n_tiles), looked for from expert `e` on: a warp's tasks ascend, and a search
// over all experts for each took longer than the main loop of K = 256.
__device__ __forceinline__ int f4_expert_from(const int* tp, int e, int n_tiles, int w) {
  while (tp[e + 1] * n_tiles <= w) ++e;
  return e;
}

// GEMM-2's epilogue: lane = column, TMEM column = row.  Two or four warps share a quarter of the columns and take turns of 16 rows; each has its own piece of
// shared memory: the gate weights of its rows, then a buffer of 16 rows x 32 columns, two rows to a word.
//
// The weights are in the order of the rows (written by the kernel that sorts them) and are fetched a tile ahead: two dependent loads per 16 rows in the
// epilogue itself took 1.1 us each, five times the main loop of K = 1536 in all.  What bounds the epilogue then is the load / store unit, so
// rows leave it in few instructions: 4 loads of weights, 8 stores of two rows' bf16 pair and 2 loads of eight columns per 16 x 32 values, and
// 16-byte stores to o.  131072 rows of 4096 columns on CTA pairs take 430 us at K = 512, 464 at 768, 550 at 1536, 1590 at 6144: up to about K = 1536 the chain of a
// turn, and not the walk over K, sets the time (o alone takes 164 at the copy rate).
constexpr int F4_OUT_PITCH = 36;   // words per two rows: lanes that load neighbouring rows use different banks
template <int ROWS, int SHARES> struct F4Out {   // SHARES warps share a quarter
  static constexpr int TURNS = (ROWS + 16 * SHARES - 1) / (16 * SHARES);
  static constexpr int BYTES = TURNS * 64 + 8 * F4_OUT_PITCH * 4;
};
// Lane l of w[i] has row 16 (share + SHARES (j / 16)) + j % 16, j = 32 i + l.
template <int ROWS, int SHARES, int N>
__device__ __forceinline__ void f4_fetch_weights(const F4Params& p, int row0, int rows, int share, int lane, float (&w)[N]) {
  static_assert(N == (F4Out<ROWS, SHARES>::TURNS + 1) / 2, "32 lanes: 16 rows of two turns");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = 32 * i + lane, r = 16 * (share + SHARES * (at >> 4)) + (at & 15);
    w[i] = p.row_w != nullptr && r < rows ? __ldcg(p.row_w + row0 + r) : 1.f;
  }
}
template <int ROWS, int SHARES, int N>
__device__ __forceinline__ void f4_keep_weights(const float (&w)[N], uint32_t mem, int lane) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (32 * i + lane < 16 * F4Out<ROWS, SHARES>::TURNS) ptx::st_shared_b32(mem + 4 * (32 * i + lane), __float_as_uint(w[i]));
  __syncwarp();
}
// turn `i` of the warp: 16 rows from row0 on, of which `rows` exist
template <int ROWS, int SHARES>
__device__ __forceinline__ void f4_store_rows(const F4Params& p, const uint32_t (&acc)[16], uint32_t mem, int i, int lane, int row0, int rows, int col0) {
  const uint32_t buf = mem + F4Out<ROWS, SHARES>::TURNS * 64;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint4 w = ptx::ld_shared_v4(mem + i * 64 + q * 16);
    const uint32_t two[2] = {pack2(__uint_as_float(w.x) * __uint_as_float(acc[4 * q]), __uint_as_float(w.y) * __uint_as_float(acc[4 * q + 1])),
                             pack2(__uint_as_float(w.z) * __uint_as_float(acc[4 * q + 2]), __uint_as_float(w.w) * __uint_as_float(acc[4 * q + 3]))};
    ptx::st_shared_b32(buf + ((2 * q) * F4_OUT_PITCH + lane) * 4, two[0]);
    ptx::st_shared_b32(buf + ((2 * q + 1) * F4_OUT_PITCH + lane) * 4, two[1]);
  }
  __syncwarp();
  const int col = col0 + (lane & 3) * 8, r = 2 * (lane >> 2);
  const uint4 a = ptx::ld_shared_v4(buf + ((lane >> 2) * F4_OUT_PITCH + (lane & 3) * 8) * 4);
  const uint4 b = ptx::ld_shared_v4(buf + ((lane >> 2) * F4_OUT_PITCH + (lane & 3) * 8 + 4) * 4);
  __syncwarp();
  if (col < p.N) {
    __nv_bfloat16* o = p.out + (size_t)(row0 + r) * (size_t)p.N + col;
    if (r < rows)
      *reinterpret_cast<uint4*>(o) = make_uint4(__byte_perm(a.x, a.y, 0x5410), __byte_perm(a.z, a.w, 0x5410), __byte_perm(b.x, b.y, 0x5410),
                                                __byte_perm(b.z, b.w, 0x5410));
    if (r + 1 < rows)
      *reinterpret_cast<uint4*>(o + p.N) = make_uint4(__byte_perm(a.x, a.y, 0x7632), __byte_perm(a.z, a.w, 0x7632), __byte_perm(b.x, b.y, 0x7632),
                                                      __byte_perm(b.z, b.w, 0x7632));
  }
}

cudaError_t launch_fp4_pair(bool glu, const F4Params& p, const void* wa, const void* wb, const void* rows, long long n_rows,
                            long long row_sets, cudaStream_t st);

}  // namespace ffn
}  // namespace tcmoe
