// Y = act(X W^T + b) + R of rows in 8 bits and weights in 8 bits: sums of integers, which are exact, on v_mfma_i32_32x32x32_i8, and
// fp32 from the scales on.
#include "activation.h"
#include "rows8.h"

namespace gnn {
namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));

struct Product8 {
    int M, N, K;
    long ld;                           // bytes between rows of X and of W
    Rows8 X, W;                        // W: a row for each column of Y
    const float *bias, *R;
    float *Y;
    int tiles_n;
};

// Four wavefronts per 32 rows and 32 columns of Y share the reduction: a lane takes 16 consecutive bytes of its row of X and of its row
// of W straight into registers (the lane halves the first and the second 16 of 32), what lies behind K in them is made zero in X.
template <int ACT>
__global__ void __launch_bounds__(256)
linear8_few_kernel(Product8 g) {
    __shared__ intx4 sums[4][4][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l = lane % 32, half = lane / 32;
    const int m0 = (int)(blockIdx.x / g.tiles_n) * 32, j = (int)(blockIdx.x % g.tiles_n) * 32 + l;
    const int all = (g.K + 31) / 32, first = all * wave / 4, total = all * (wave + 1) / 4;
    const int8_t *x = g.X.q + (size_t)min(m0 + l, g.M - 1) * g.ld, *w = g.W.q + (size_t)min(j, g.N - 1) * g.ld;
    intx16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0;
    for (int step = first; step < total; ++step) {
        const int k = step * 32 + 16 * half, at = min(k, (int)g.ld - 16);
        intx4 a = *reinterpret_cast<const intx4 *>(x + at);
        const intx4 b = *reinterpret_cast<const intx4 *>(w + at);
        if (k + 16 > g.K) {                                // bytes of word i that are before K
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int left = g.K - k - 4 * i;
                a[i] = left >= 4 ? a[i] : left <= 0 ? 0 : a[i] & ((1 << 8 * left) - 1);
            }
        }
        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[wave][i][lane] = intx4{acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]};
    __syncthreads();
    if (j >= g.N) return;
    const intx4 z = (sums[0][wave][lane] + sums[1][wave][lane]) + (sums[2][wave][lane] + sums[3][wave][lane]);
    const float scale = g.W.scale[j], bias = g.bias ? g.bias[j] : 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int m = m0 + 8 * wave + 4 * half + v;
        if (m >= g.M) continue;
        float y, slope;
        activate<ACT, false>(fmaf((float)z[v] * g.X.scale[m], scale, bias), y, slope);
        const size_t at = (size_t)m * g.N + j;
        g.Y[at] = g.R ? y + g.R[at] : y;
    }
}

}  // namespace

// sums of f_in products of 127 x 127 in 32 bits; blocks of 32 x 32
bool linear8_fits(int64_t n, int64_t m, int64_t k) {
    return m <= 1 << 17 && k <= 1 << 21 && ceil_div(n, 32) * ceil_div(k, 32) < (int64_t)1 << 24;
}

gnn_status_t linear8_forward_launch(int act, int n, int m, int k, const Rows8 &X, const Rows8 &W, const float *b, const float *R, float *Y,
                                    hipStream_t st) {
    if (n <= 0) return GNN_OK;
    const Product8 g{n, k, m, (long)rows8_stride(m), X, W, b, R, Y, (int)ceil_div(k, 32)};
    const dim3 grid((unsigned)(ceil_div(n, 32) * g.tiles_n));
#define LINEAR8_CASE(ACT_) \
    if (act == ACT_) hipLaunchKernelGGL(linear8_few_kernel<ACT_>, grid, dim3(256), 0, st, g);
    LINEAR8_CASE(GNN_ACT_NONE) LINEAR8_CASE(GNN_ACT_RELU) LINEAR8_CASE(GNN_ACT_ELU)
    LINEAR8_CASE(GNN_ACT_SIGMOID) LINEAR8_CASE(GNN_ACT_SILU) LINEAR8_CASE(GNN_ACT_GELU)
#undef LINEAR8_CASE
    return launch_status();
}

}  // namespace gnn
