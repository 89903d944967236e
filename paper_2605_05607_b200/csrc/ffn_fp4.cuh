// Parameters of the FP4 expert products.
#pragma once
#include "common.cuh"
#include "quant4.cuh"

#include <cuda.h>

namespace tcmoe {
namespace ffn {

constexpr int F4_ROWS = 96;   // rows of a tile: two accumulators of 2 x 96 columns and the scales of four stages fit TMEM

struct F4RowMaps { CUtensorMap m[F4_ROWS / 32]; };   // boxes of 32, 64, 96 rows

struct F4Params {
  const int32_t* expert_offsets;
  int E, K, N;              // K: elements
  int NC;                   // 128-column chunks of the weights
  const uint8_t* sfx;       // scale chunks of the row tiles
  const uint8_t *sfa, *sfb; // of the weights (GEMM-1: W1, W3)
  uint32_t* hq;             // GEMM-1: codes of h [P, N / 8 words], and their scale chunks per row tile
  uint8_t* sfh;
  __nv_bfloat16* out;       // GEMM-2: o [P, N]
  const float* topk_w;      // NULL: 1
  const int32_t* row_pair;
  int32_t* status;
};

}  // namespace ffn
}  // namespace tcmoe
