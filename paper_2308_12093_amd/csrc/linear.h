// The product with bias, activation and residual: what its files share.
#pragma once

#include "gemm_half_kernel.h"
#include "rows8.h"

namespace gnn {

using half_parts::Linear;

// Z = X W + bias, X [M][K] with the row_tops of tops_launch (not read where K < kShortReduction), W [K][N]; `out` says what becomes of
// it.  Backward (not of GNN_ACT_NONE) fills `tops` of D: linear_row_parts(M, N) parts a row.  K >= 4 and gemm_half_fits.
size_t linear_half_workspace_bytes(int64_t N, int64_t K);
int linear_row_parts(int64_t n, int64_t k);
gnn_status_t linear_half_launch(int act, int64_t M, int64_t N, int64_t K, const float *X, const unsigned *row_tops, const float *W,
                                const float *bias, const Linear &out, const Tops &tops, void *workspace, hipStream_t st);

}  // namespace gnn
