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

// The same products on parts in one scale (half_pair.h), where pair_product_fits: of many aligned rows.
bool pair_product_fits(int64_t M, int64_t N, int64_t K, const float *A);
size_t pair_workspace_bytes(int64_t N, int64_t K);
// A and X have rows of K floats, a multiple of 4, of which the KB first are those of B and W and the others zeros.
// C [M][N] = A [M][K] B^T, B [N][KB]; row_tops: of A, `parts` of them
gnn_status_t pair_plain_launch(int64_t M, int64_t N, int64_t K, int64_t KB, const float *A, const unsigned *row_tops, int parts, const float *B, float *C,
                               void *workspace, hipStream_t st);
int pair_row_parts(int64_t N);
gnn_status_t pair_linear_launch(int act, int64_t M, int64_t N, int64_t K, int64_t KB, const float *X, const unsigned *row_tops, int parts, const float *W,
                                const float *bias, const Linear &out, const Tops &tops, void *workspace, hipStream_t st);

// C [M][N] = A^T B, A [K][M], or NULL: `held` with its columns; B [K][N]; sums [N] = the column sums of B unless it is NULL; a_tops (not of
// `held`), b_tops: largest magnitudes of their columns, of B with each row times held's scale.
bool pair_tn_fits(int64_t M, int64_t N, int64_t K, bool held);
int64_t pair_tn_least_rows(int64_t M, int64_t N);      // no K below this fits
size_t pair_tn_workspace_bytes(int64_t M, int64_t N, int64_t K);
gnn_status_t pair_tn_launch(int64_t M, int64_t N, int64_t K, const float *A, const Rows8 &held, const unsigned *a_tops, const float *B,
                            const unsigned *b_tops, float *C, float *sums, void *workspace, hipStream_t st);

}  // namespace gnn
