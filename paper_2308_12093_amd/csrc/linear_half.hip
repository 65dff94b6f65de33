// act(X W + b) + R, and dY .* act'(X W + b), in the epilogue of the product on the fp16 matrix instruction (gemm_half_kernel.h).  Outputs are
// stored through the caches, large ones too: past them 2^18 x 16 -> 256 takes 69 us as well, 2^20 x 128 -> 64 249, 65536 x 512 -> 2048 at any
// alignment with residual and Z 752.
#include "linear.h"

namespace gnn {

using namespace half_parts;

size_t linear_half_workspace_bytes(int64_t N, int64_t K) { return half_parts_bytes(N, K) + half_exps_bytes(N); }

int linear_row_parts(int64_t n, int64_t k) { return (int)ceil_div(k, 32 * half_tiles(n, k)); }

gnn_status_t linear_half_launch(int act, int64_t M, int64_t N, int64_t K, const float *X, const unsigned *row_tops, const float *W,
                                const float *bias, const Linear &out, const Tops &tops, void *workspace, hipStream_t st) {
    HalfProduct g{};
    set_product(g, M, N, K, workspace);
    g.A = X; g.row_tops = row_tops; g.top_parts = top_parts(K, X);
    g.B = HalfOperand{W, (long)N, 1};
    g.bias = bias;
    g.linear = out;
    g.tops = tops;
    const bool back = out.D != nullptr;
    const int rows = K < kShortReduction ? kShort : K % 4 == 0 && K < 1 << 24 && aligned16(X) ? kCopied : kLoaded;
    const int w = half_tiles(M, N);
    if (rows != kShort) GNN_TRY(split_weights(g, w, 0, st));
    const dim3 grid = product_grid(g);
#define LINEAR_CASE(NT_, ROWS_, ACT_)                                                                                       \
    if (w == NT_ && rows == ROWS_ && act == ACT_) {                                                                         \
        if constexpr (ACT_ != GNN_ACT_NONE)                                                                                 \
            if (back) hipLaunchKernelGGL((gemm_half_kernel<NT_, kLinearBackward, ROWS_, ACT_>), grid, dim3(256), 0, st, g); \
        if (!back) hipLaunchKernelGGL((gemm_half_kernel<NT_, kLinearForward, ROWS_, ACT_>), grid, dim3(256), 0, st, g);     \
    }
#define LINEAR_CASES(NT_, ROWS_)                                                                                   \
    LINEAR_CASE(NT_, ROWS_, GNN_ACT_NONE) LINEAR_CASE(NT_, ROWS_, GNN_ACT_RELU) LINEAR_CASE(NT_, ROWS_, GNN_ACT_ELU)  \
    LINEAR_CASE(NT_, ROWS_, GNN_ACT_SIGMOID) LINEAR_CASE(NT_, ROWS_, GNN_ACT_SILU) LINEAR_CASE(NT_, ROWS_, GNN_ACT_GELU)
    LINEAR_CASES(2, kLoaded) LINEAR_CASES(2, kCopied) LINEAR_CASES(2, kShort)
    LINEAR_CASES(4, kLoaded) LINEAR_CASES(4, kCopied) LINEAR_CASES(4, kShort)
#undef LINEAR_CASES
#undef LINEAR_CASE
    return launch_status();
}

}  // namespace gnn
