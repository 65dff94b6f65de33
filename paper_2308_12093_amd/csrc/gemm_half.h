// Products on the fp16 matrix instruction with fp32 operands, sums and results (gemm_half.hip): what the gated block needs.
#pragma once

#include "gated.h"

namespace gnn {

// Largest magnitudes, as the bits of floats (which order like them, infinities and NaN last).
//   rows: [part][n], of a part of each row (the whole row: of its parts' largest)
//   cols: [block of top_rows(n) rows][columns]
struct Tops {
    unsigned *rows, *cols;             // either may be NULL: not wanted
};
// Few rows in smaller blocks, so that there are enough of them for the chip.
constexpr int64_t kTopRowsLine = 32768;
__host__ __device__ constexpr int top_rows(int64_t n) { return n < kTopRowsLine ? 32 : 128; }
static inline int64_t top_blocks(int64_t n) { return ceil_div(n, top_rows(n)); }
// of n rows or fewer: just below the line there are more blocks than from it on
static inline int64_t most_top_blocks(int64_t n) {
    const int64_t below = top_blocks(n < kTopRowsLine ? n : kTopRowsLine - 1), all = top_blocks(n);
    return all > below ? all : below;
}

// Rows a block takes where only rows' largest magnitudes are wanted, or none: four for each group of lanes, and more where a grid
// of these would have 2^24 blocks of 256 threads, which it cannot.
static inline int64_t free_rows(int64_t n, int lanes, int64_t parts) {
    int64_t rows = 4 * (256 / lanes);
    while (ceil_div(n, rows) * parts >= (int64_t)1 << 24) rows *= 2;
    return rows;
}

// columns of B as a product reads it: element (k, n) at k * sk + n * sn
struct HalfOperand {
    const float *p;
    long sk, sn;
};

// A product of two parts each is off by up to 8 u (u = 2^-24) where one of floats is by u at most, but is rounded less often on its way
// into the sum.  Root mean square of the errors of sums of K products of normal numbers, in u sqrt(K): parts 1.4 for K = 4 to 32, 1.5
// for 64, 1.7 for 128; a chain of float multiplications and additions 0.7 for 4, 1.2 for 16, 1.5 for 24, 1.7 for 32, 3.4 for
// 128.  So shorter reductions than this, one step of the kernels, are formed in float: [A | U] of the gated block on the
// fp32 instruction, A^T B in plain code, D W^T in gemm_launch.
constexpr int64_t kShortReduction = 32;
bool gemm_half_fits(int64_t M, int64_t N);
// scratch of a product: the parts of B and their exponents; parts of the reduction
size_t gemm_half_workspace_bytes(int64_t N, int64_t K);
size_t gemm_half_gated_workspace_bytes(int64_t half, int64_t K);
// largest magnitudes of X [n][m], top_parts(m, X) parts a row
int top_parts(int64_t m, const float *X);
gnn_status_t tops_launch(int64_t n, int m, const float *X, const Tops &tops, hipStream_t st);

// C [M][N] = A [M][K] B^T, B [N][K]; row_tops: of A, `parts` of them.  K >= 4 and gemm_half_fits.
gnn_status_t gemm_half_launch(int64_t M, int64_t N, int64_t K, const float *A, const unsigned *row_tops, int parts, const float *B,
                              float *C, void *workspace, hipStream_t st);
// [A | U] = X W + bias, X [M][K] with the row_tops of tops_launch (not read where K < kShortReduction), W [K][2 half]; `out` says
// what becomes of it.  Backward fills
// `tops` of D: gated_row_parts(n, half) parts a row.
int gated_row_parts(int64_t n, int64_t half);
gnn_status_t gemm_half_gated_launch(int64_t M, int64_t K, const float *X, const unsigned *row_tops, const float *W,
                                    const float *bias, const Gated &out, const Tops &tops, void *workspace, hipStream_t st);
// C [M][N] = A^T B, A [K][M], B [K][N]; sums [N] = the column sums of B unless it is NULL; a_tops, b_tops: their columns', not read
// where K < kShortReduction.
bool gemm_half_tn_fits(int64_t M, int64_t N, int64_t K);
size_t gemm_half_tn_workspace_bytes(int64_t M, int64_t N, int64_t K);
gnn_status_t gemm_half_tn_launch(int64_t M, int64_t N, int64_t K, const float *A, const unsigned *a_tops, const float *B,
                                 const unsigned *b_tops, float *C, float *sums, void *workspace, hipStream_t st);

}  // namespace gnn
