// The gated feed-forward block H = act(X W_gate + b_gate) .* (X W_up + b_up), forward and backward.  Its large products are
// those of gemm_split.hip (forward, and backward where [A | U] was not kept, with the block's own epilogue) and gemm.hip.
#include "gated.h"

namespace gnn {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx4u __attribute__((ext_vector_type(4), aligned(4)));

constexpr int KB = 32;                 // reduction indices of a step: lane half h takes 16 h .. 16 h + 15

// Few rows: four wavefronts per 32 rows and 32 columns of H share the reduction, operands straight from memory into
// registers two steps ahead (the two lane halves of v_mfma_f32_32x32x2_f32 take 16 consecutive indices each), one launch, no
// scratch.  A wavefront has the sums of the gate and of the other projection for the same elements.
template <bool BACK>
__global__ void __launch_bounds__(256)
gated_few_kernel(int M, int K, const float *__restrict__ X, const float *__restrict__ W, const float *__restrict__ bias, Gated g,
                 int tiles_n) {
    constexpr int AHEAD = 2;
    __shared__ floatx4 sums[4][2][4][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l = lane % 32, half = lane / 32;
    const int m0 = (int)(blockIdx.x / tiles_n) * 32, j = (int)(blockIdx.x % tiles_n) * 32 + l, jj = min(j, g.half - 1);
    const int all = (K + KB - 1) / KB, first = all * wave / 4, total = all * (wave + 1) / 4;
    const float *x = X + (size_t)min(m0 + l, M - 1) * K, *w = W + jj;       // what is past the end re-reads the last
    const size_t ld = 2 * (size_t)g.half;
    float xs[AHEAD][16], ga[AHEAD][16], up[AHEAD][16];
    auto load = [&](int step, int s) __attribute__((always_inline)) {
        const int k0 = step * KB + 16 * half;
        if (k0 + 16 <= K) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const floatx4u v = *reinterpret_cast<const floatx4u *>(x + k0 + 4 * i);
                xs[s][4 * i] = v.x; xs[s][4 * i + 1] = v.y; xs[s][4 * i + 2] = v.z; xs[s][4 * i + 3] = v.w;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                ga[s][i] = w[(k0 + i) * ld];
                up[s][i] = w[(k0 + i) * ld + g.half];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                xs[s][i] = k0 + i < K ? x[k0 + i] : 0.f;
                ga[s][i] = k0 + i < K ? w[(k0 + i) * ld] : 0.f;
                up[s][i] = k0 + i < K ? w[(k0 + i) * ld + g.half] : 0.f;
            }
        }
    };
    floatx16 a, u;
#pragma unroll
    for (int v = 0; v < 16; ++v) a[v] = u[v] = 0.f;
#pragma unroll
    for (int s = 0; s < AHEAD; ++s)
        if (first + s < total) load(first + s, s);
    for (int step = first; step < total; step += AHEAD) {
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            if (step + s < total) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    a = __builtin_amdgcn_mfma_f32_32x32x2f32(xs[s][i], ga[s][i], a, 0, 0, 0);
                    u = __builtin_amdgcn_mfma_f32_32x32x2f32(xs[s][i], up[s][i], u, 0, 0, 0);
                }
                if (step + s + AHEAD < total) load(step + s + AHEAD, s);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        sums[wave][0][i][lane] = floatx4{a[4 * i], a[4 * i + 1], a[4 * i + 2], a[4 * i + 3]};
        sums[wave][1][i][lane] = floatx4{u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]};
    }
    __syncthreads();
    if (j >= g.half) return;
    // a wavefront finishes a quarter of the tile: accumulator register v of lane (half, l) is row 8 (v / 4) + 4 half + v % 4
    floatx4 s[2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
        s[p] = (sums[0][p][wave][lane] + sums[1][p][wave][lane]) + (sums[2][p][wave][lane] + sums[3][p][wave][lane]) +
               (bias ? bias[p * g.half + j] : 0.f);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int m = m0 + 8 * wave + 4 * half + v;
        if (m >= M) continue;
        float act, slope = 0.f;
        gate_of<BACK>(g.gate, s[0][v], act, slope);
        const size_t at = (size_t)m * g.half + j, two = (size_t)m * 2 * g.half + j;
        if constexpr (BACK) {
            const float dh = g.dH[at];
            g.D[two] = dh * s[1][v] * slope;
            g.D[two + g.half] = dh * act;
        } else {
            g.H[at] = act * s[1][v];
            if (g.Z) {
                g.Z[two] = s[0][v];
                g.Z[two + g.half] = s[1][v];
            }
        }
    }
}

// D from the [A | U] that forward has kept, VEC columns a thread
template <int VEC>
__global__ void __launch_bounds__(256)
gated_gradient_kernel(long n, int k, int gate, const float *__restrict__ Z, const float *__restrict__ dH, float *__restrict__ D) {
    const int groups = k / VEC;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n * groups; i += (long)gridDim.x * 256) {
        const long row = i / groups, at = row * 2 * k + (i - row * groups) * VEC;
        float a[VEC], u[VEC], d[VEC];
        if constexpr (VEC == 4) {
            const float4 x = *reinterpret_cast<const float4 *>(Z + at), y = *reinterpret_cast<const float4 *>(Z + at + k);
            const float4 z = *reinterpret_cast<const float4 *>(dH + i * VEC);
            a[0] = x.x; a[1] = x.y; a[2] = x.z; a[3] = x.w;
            u[0] = y.x; u[1] = y.y; u[2] = y.z; u[3] = y.w;
            d[0] = z.x; d[1] = z.y; d[2] = z.z; d[3] = z.w;
        } else {
            a[0] = Z[at]; u[0] = Z[at + k]; d[0] = dH[i];
        }
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            float g, dg;
            gate_of<true>(gate, a[v], g, dg);
            a[v] = d[v] * u[v] * dg;
            u[v] = d[v] * g;
        }
        if constexpr (VEC == 4) {
            *reinterpret_cast<float4 *>(D + at) = make_float4(a[0], a[1], a[2], a[3]);
            *reinterpret_cast<float4 *>(D + at + k) = make_float4(u[0], u[1], u[2], u[3]);
        } else {
            D[at] = a[0]; D[at + k] = u[0];
        }
    }
}

bool gated_few(int64_t n, int64_t m, int64_t k) {
    return m < 4 || ceil_div(n, 32) * ceil_div(k, 32) <= 512 || !gemm_gated_fits(n, k);
}

// [A | U] and what becomes of it
gnn_status_t project(int64_t n, int64_t m, const float *X, const float *W, const float *b, const Gated &g, void *workspace,
                     hipStream_t st) {
    if (!gated_few(n, m, g.half)) return gemm_gated_launch(n, m, X, W, b, g, workspace, st);
    const int64_t tiles_n = ceil_div(g.half, 32), blocks = ceil_div(n, 32) * tiles_n;
    auto kernel = g.D ? gated_few_kernel<true> : gated_few_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, (int)n, (int)m, X, W, b, g, (int)tiles_n);
    return launch_status();
}

}  // namespace

bool gated_fits(bool backward, int64_t n, int64_t m, int64_t k) {
    if (gated_few(n, m, k) ? ceil_div(n, 32) * ceil_div(k, 32) >= (int64_t)1 << 24 : !gemm_fits(n, 2 * k, m)) return false;
    return !backward || (gemm_fits(n, m, 2 * k) && gemm_tn_split_fits(m, 2 * k, n));
}

// What n rows take, or fewer: a product of few rows needs no scratch, one of more the parts of W.
size_t gated_workspace_bytes(bool backward, int64_t n, int64_t m, int64_t k) {
    size_t most = gated_few(n, m, k) ? kAlign : gemm_gated_workspace_bytes(k, m);
    if (!backward) return most;
    for (size_t b : {gemm_workspace_bytes(0, 1, n, m, 2 * k), gemm_tn_split_workspace_bytes(m, 2 * k, n)})
        if (b > most) most = b;
    return align_up((size_t)n * 2 * k * sizeof(float)) + most;
}

gnn_status_t gated_forward_launch(int gate, int n, int m, int k, const float *X, const float *W, const float *b, float *H,
                                  float *Z, void *workspace, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    return project(n, m, X, W, b, Gated{k, gate, H, Z, nullptr, nullptr}, workspace, st);
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
    if (Z) {
        const bool vec = k % 4 == 0 && aligned16(Z) && aligned16(dH);
        int64_t blocks = ceil_div((int64_t)n * k / (vec ? 4 : 1), 256);
        if (blocks > 1 << 20) blocks = 1 << 20;
        auto kernel = vec ? gated_gradient_kernel<4> : gated_gradient_kernel<1>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, (long)n, k, gate, Z, dH, d);
        GNN_TRY(launch_status());
    } else {
        GNN_TRY(project(n, m, X, W, b, Gated{k, gate, nullptr, nullptr, dH, d}, rest, st));
    }
    if (dX) GNN_TRY(gemm_launch(0, 1, n, m, 2 * (int64_t)k, d, W, dX, nullptr, 0, rest, st));
    return gemm_tn_split_launch(m, 2 * (int64_t)k, n, X, d, dW, db, rest, st);
}

}  // namespace gnn
