// The gated feed-forward block H = act(X W_gate + b_gate) * (X W_up + b_up), forward and backward.
#include "common.h"

namespace gnn {
namespace {

// the gate's activation g and its derivative dg at a
__device__ __forceinline__ void gate_of(int gate, float a, float &g, float &dg) {
    if (gate == GNN_GATE_GELU) {
        const float below = 0.5f * (1.f + erff(a * 0.70710678118654752f));
        g = a * below;
        dg = fmaf(a * 0.39894228040143268f, expf(-0.5f * a * a), below);
        return;
    }
    const float s = 1.f / (1.f + expf(-a));
    g = gate == GNN_GATE_SILU ? a * s : s;
    dg = gate == GNN_GATE_SILU ? s * fmaf(a, 1.f - s, 1.f) : s * (1.f - s);
}

__global__ void __launch_bounds__(256)
gated_combine_kernel(long n, int k, int gate, const float *__restrict__ Z, float *__restrict__ H) {
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n * k; i += (long)gridDim.x * 256) {
        const long row = i / k;
        const float *z = Z + row * 2 * k + (i - row * k);
        float g, dg;
        gate_of(gate, z[0], g, dg);
        H[i] = g * z[k];
    }
}

// D = [dH U act'(A) | dH act(A)]; D may be Z
__global__ void __launch_bounds__(256)
gated_split_kernel(long n, int k, int gate, const float *Z, const float *__restrict__ dH, float *D) {
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n * k; i += (long)gridDim.x * 256) {
        const long row = i / k, at = row * 2 * k + (i - row * k);
        const float u = Z[at + k], d = dH[i];
        float g, dg;
        gate_of(gate, Z[at], g, dg);
        D[at] = d * u * dg;
        D[at + k] = d * g;
    }
}

unsigned blocks_of(int64_t count) { return (unsigned)(ceil_div(count, 256) < 1 << 20 ? ceil_div(count, 256) : 1 << 20); }

}  // namespace

size_t gated_workspace_bytes(bool backward, int64_t n, int64_t m, int64_t k) {
    const size_t z = align_up((size_t)n * 2 * k * sizeof(float));
    if (!backward) return z + gemm_workspace_bytes(0, 0, n, 2 * k, m);
    size_t most = gemm_workspace_bytes(0, 0, n, 2 * k, m);
    for (size_t b : {gemm_workspace_bytes(0, 1, n, m, 2 * k), gemm_workspace_bytes(1, 0, m, 2 * k, n),
                     colsum_workspace_bytes(n, (int)(2 * k))})
        if (b > most) most = b;
    return z + most;
}

gnn_status_t gated_forward_launch(int gate, int n, int m, int k, const float *X, const float *W, const float *b, float *H,
                                  float *Z, void *workspace, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    Carver carve(workspace);
    float *z = carve.take<float>((size_t)n * 2 * k);
    if (Z) z = Z;
    GNN_TRY(gemm_launch(0, 0, n, 2 * (int64_t)k, m, X, W, z, b, 0, carve.take<char>(0), st));
    hipLaunchKernelGGL(gated_combine_kernel, dim3(blocks_of((int64_t)n * k)), dim3(256), 0, st, (long)n, k, gate, z, H);
    return launch_status();
}

gnn_status_t gated_backward_launch(int gate, int n, int m, int k, const float *X, const float *W, const float *b,
                                   const float *Z, const float *dH, float *dW, float *db, float *dX, void *workspace,
                                   hipStream_t st) {
    if (n <= 0) {
        GNN_TRY(fill_zero_launch((int64_t)m * 2 * k, dW, st));
        return db ? fill_zero_launch(2 * (int64_t)k, db, st) : GNN_OK;
    }
    Carver carve(workspace);
    float *d = carve.take<float>((size_t)n * 2 * k);
    void *rest = carve.take<char>(0);
    if (!Z) {
        GNN_TRY(gemm_launch(0, 0, n, 2 * (int64_t)k, m, X, W, d, b, 0, rest, st));
        Z = d;
    }
    hipLaunchKernelGGL(gated_split_kernel, dim3(blocks_of((int64_t)n * k)), dim3(256), 0, st, (long)n, k, gate, Z, dH, d);
    GNN_TRY(launch_status());
    if (dX) GNN_TRY(gemm_launch(0, 1, n, m, 2 * (int64_t)k, d, W, dX, nullptr, 0, rest, st));
    GNN_TRY(gemm_launch(1, 0, m, 2 * (int64_t)k, n, X, d, dW, nullptr, 0, rest, st));
    return db ? colsum_launch(n, 2 * k, d, db, rest, st) : GNN_OK;
}

}  // namespace gnn
