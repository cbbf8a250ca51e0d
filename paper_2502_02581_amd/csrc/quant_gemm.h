// Argument blocks of the products of block-scaled tensors (see quant_format.h).
#pragma once

#include "gemm_plan.h"
#include "quant_format.h"

namespace moe {

// C[rows, N] = A[rows, K] B_g[N, K]^T over the row tiles of a plan, or (no plan) over the rows of groups that offsets delimit, or (neither) over n_rows
// rows of one group.  K is whole blocks: rows of codes are padded with zeros.
struct QuantGemm {
  const RowTile* tiles;
  const int32_t *n_tiles, *offsets;
  int32_t n_rows, n_groups;
  int32_t height, tail;                  // one group: rows of a tile (256, 128 or 64); pieces (1, 2 or 4) that tiles of the last round are cut into
  int32_t n_parts, k_part, part_blocks;  // K is summed in n_parts parts of k_part blocks; launch blocks of a part
  float* part;                           // n_parts > 1: fp32 sums [n_parts][n_rows][N]
  int32_t N, nk;           // columns, blocks of K
  const uint8_t *A, *As;   // rows of lda codes and las exponents
  int64_t lda, las;
  const int32_t* a_index;  // row r reads row a_index[r] / a_index_div (NULL: row r)
  int32_t a_index_div, a_src_rows;  // of so many rows
  const uint8_t *B[2], *Bs[2];  // [1]: second matrix of a dual product
  int64_t ldb, b_group;         // bytes of a row, of a group
  int64_t lbs, bs_group;        // the same of the exponents
  void* out[3];
  const void* in[2];
  int64_t ldc;
  uint8_t *q[2], *qs[2];   // where the quantised outputs go (QuantOut): rows of ldq codes and lds exponents, the bytes of whole blocks of N
  int64_t ldq, lds;
  const float* c_scale;    // activation-backward epilogues: row r is scaled by c_scale[a_index[r]]
};

}  // namespace moe
