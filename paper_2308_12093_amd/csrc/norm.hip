// Dropout, layer norm and the two around a residual connection, forward and backward.
#include "dropout.h"

namespace gnn {
namespace {

// Four consecutive floats of a row of f, at any 4-byte aligned address; zeros past the row's end.
typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float4 load4(const float *row, int c, int f) {
    if (c + 4 <= f) {
        const float4u v = *reinterpret_cast<const float4u *>(row + c);
        return make_float4(v.x, v.y, v.z, v.w);
    }
    return make_float4(row[c], c + 1 < f ? row[c + 1] : 0.f, c + 2 < f ? row[c + 2] : 0.f, 0.f);
}

__device__ __forceinline__ void store4(float *row, int c, int f, float4 v) {
    if (c + 4 <= f) {
        *reinterpret_cast<float4u *>(row + c) = float4u{v.x, v.y, v.z, v.w};
        return;
    }
    row[c] = v.x;
    if (c + 1 < f) row[c + 1] = v.y;
    if (c + 2 < f) row[c + 2] = v.z;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

__device__ __forceinline__ float activation(float z, int act) {
    if (act == kActRelu) return fmaxf(z, 0.f);
    if (act == kActElu) return z > 0.f ? z : expm1f(z);
    return z;
}
__device__ __forceinline__ float slope(float z, int act) {
    if (act == kActRelu) return z > 0.f ? 1.f : 0.f;
    if (act == kActElu) return z > 0.f ? 1.f : expf(z);
    return 1.f;
}

__global__ void __launch_bounds__(256)
dropout_kernel(int n, int f, const float *X, const float *R, Dropout drop, float *Y) {
    const DropoutWords words(drop);
    const long groups = (f + 3) / 4, total = (long)n * groups;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long)gridDim.x * 256) {
        const long row = i / groups;
        const int g = (int)(i - row * groups), c = 4 * g;
        float4 x = words.apply(load4(X + row * f, c, f), (uint32_t)row, g);
        if (R) {
            const float4 r = load4(R + row * f, c, f);
            x = make_float4(x.x + r.x, x.y + r.y, x.z + r.z, x.w + r.w);
        }
        store4(Y + row * f, c, f, x);
    }
}

// One wavefront per row, which it reads three times.  With R: H = R + dropout(X) first, and no dropout after.
__global__ void __launch_bounds__(256)
norm_forward_kernel(int n, int f, const float *X, const float *R, const float *__restrict__ gamma,
                    const float *__restrict__ beta, float eps, int act, Dropout drop, float *H, float *Y, float *stat) {
    const DropoutWords words(drop);
    const int lane = threadIdx.x % 64;
    const long row = (long)blockIdx.x * 4 + threadIdx.x / 64;
    if (row >= n) return;
    const float *x = X + row * f;
    float sum = 0.f;
    for (int c = 4 * lane; c < f; c += 256) {
        float4 v = load4(x, c, f);
        if (R) {
            const float4 r = load4(R + row * f, c, f);
            v = words.apply(v, (uint32_t)row, c / 4);
            v = make_float4(v.x + r.x, v.y + r.y, v.z + r.z, v.w + r.w);
            store4(H + row * f, c, f, v);
            if (c + 4 > f) v = load4(H + row * f, c, f);
        }
        sum += (v.x + v.y) + (v.z + v.w);
    }
    if (R) x = H + row * f;
    const float mean = wave_sum(sum) / (float)f;
    float square = 0.f;
    for (int c = 4 * lane; c < f; c += 256)
        for (int j = 0; j < 4 && c + j < f; ++j) square = fmaf(x[c + j] - mean, x[c + j] - mean, square);
    const float rstd = 1.f / sqrtf(wave_sum(square) / (float)f + eps);
    if (lane == 0) { stat[2 * row] = mean; stat[2 * row + 1] = rstd; }
    for (int c = 4 * lane; c < f; c += 256) {
        float z[4] = {0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < 4 && c + j < f; ++j)
            z[j] = activation(fmaf((x[c + j] - mean) * rstd, gamma ? gamma[c + j] : 1.f, beta ? beta[c + j] : 0.f), act);
        float4 y = make_float4(z[0], z[1], z[2], z[3]);
        if (!R) y = words.apply(y, (uint32_t)row, c / 4);
        store4(Y + row * f, c, f, y);
    }
}

// dY through the dropout and the activation behind the norm
__device__ __forceinline__ void norm_gradient(const DropoutWords &words, bool after, const float *x, const float *dy, long row,
                                              int c, int f, float mean, float rstd, const float *gamma, const float *beta,
                                              int act, float (&xhat)[4], float (&dz)[4]) {
    float4 d = load4(dy, c, f);
    if (after) d = words.apply(d, (uint32_t)row, c / 4);
    const float g[4] = {d.x, d.y, d.z, d.w};
    for (int j = 0; j < 4; ++j) {
        xhat[j] = c + j < f ? (x[c + j] - mean) * rstd : 0.f;
        const float z = c + j < f ? fmaf(xhat[j], gamma ? gamma[c + j] : 1.f, beta ? beta[c + j] : 0.f) : 0.f;
        dz[j] = c + j < f ? g[j] * slope(z, act) : 0.f;
    }
}

// One wavefront per row: dR = dH + rstd (g - mean(g) - xhat mean(g xhat)), g = dZ gamma; dX = dR, dropped with `before`.
__global__ void __launch_bounds__(256)
norm_backward_kernel(int n, int f, const float *X, const float *__restrict__ stat, const float *__restrict__ gamma,
                     const float *__restrict__ beta, int act, Dropout drop, bool before, const float *dY, const float *dH,
                     float *dR, float *dX) {
    const DropoutWords words(drop);
    const int lane = threadIdx.x % 64;
    const long row = (long)blockIdx.x * 4 + threadIdx.x / 64;
    if (row >= n) return;
    const float mean = stat[2 * row], rstd = stat[2 * row + 1];
    float s1 = 0.f, s2 = 0.f;
    float xhat[4], dz[4];
    for (int c = 4 * lane; c < f; c += 256) {
        norm_gradient(words, !before, X + row * f, dY + row * f, row, c, f, mean, rstd, gamma, beta, act, xhat, dz);
        for (int j = 0; j < 4 && c + j < f; ++j) {
            const float g = dz[j] * (gamma ? gamma[c + j] : 1.f);
            s1 += g;
            s2 = fmaf(g, xhat[j], s2);
        }
    }
    s1 = wave_sum(s1) / (float)f;
    s2 = wave_sum(s2) / (float)f;
    for (int c = 4 * lane; c < f; c += 256) {
        norm_gradient(words, !before, X + row * f, dY + row * f, row, c, f, mean, rstd, gamma, beta, act, xhat, dz);
        float o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < 4 && c + j < f; ++j) {
            o[j] = rstd * ((dz[j] * (gamma ? gamma[c + j] : 1.f) - s1) - xhat[j] * s2);
            if (dH) o[j] += dH[row * f + c + j];
        }
        float4 v = make_float4(o[0], o[1], o[2], o[3]);
        if (dR) store4(dR + row * f, c, f, v);
        if (before) v = words.apply(v, (uint32_t)row, c / 4);
        if (dX) store4(dX + row * f, c, f, v);
    }
}

constexpr int kNormBlocks = 256;       // partial rows of the weights' gradients

// part[block] = [sum dZ xhat | sum dZ] over every kNormBlocks-th row
__global__ void __launch_bounds__(256)
norm_sums_kernel(int n, int f, const float *X, const float *__restrict__ stat, const float *__restrict__ gamma,
                 const float *__restrict__ beta, int act, Dropout drop, bool after, const float *dY, double *part) {
    const DropoutWords words(drop);
    for (int c = 4 * threadIdx.x; c < f; c += 1024) {
        double a[4] = {0, 0, 0, 0}, b[4] = {0, 0, 0, 0};
        for (long row = blockIdx.x; row < n; row += gridDim.x) {
            float xhat[4], dz[4];
            norm_gradient(words, after, X + row * f, dY + row * f, row, c, f, stat[2 * row], stat[2 * row + 1], gamma, beta,
                          act, xhat, dz);
            for (int j = 0; j < 4; ++j) { a[j] += (double)dz[j] * xhat[j]; b[j] += dz[j]; }
        }
        for (int j = 0; j < 4 && c + j < f; ++j) {
            part[(size_t)blockIdx.x * 2 * f + c + j] = a[j];
            part[(size_t)blockIdx.x * 2 * f + f + c + j] = b[j];
        }
    }
}

__global__ void __launch_bounds__(256)
norm_sums_final_kernel(int f, int blocks, const double *__restrict__ part, float *dgamma, float *dbeta) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= 2 * f) return;
    double s = 0.0;
    for (int b = 0; b < blocks; ++b) s += part[(size_t)b * 2 * f + c];
    float *out = c < f ? dgamma : dbeta;
    if (out) out[c < f ? c : c - f] = (float)s;
}

__global__ void rng_advance_kernel(uint64_t *state, uint64_t by) { state[1] += by; }

}  // namespace

gnn_status_t rng_advance_launch(uint64_t *state, uint64_t by, hipStream_t st) {
    hipLaunchKernelGGL(rng_advance_kernel, dim3(1), dim3(1), 0, st, state, by);
    return launch_status();
}

gnn_status_t dropout_launch(int n, int f, const float *X, const float *R, const Dropout &drop, float *Y, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    int64_t blocks = ceil_div((int64_t)n * ((f + 3) / 4), 256);
    if (blocks > 1 << 20) blocks = 1 << 20;
    hipLaunchKernelGGL(dropout_kernel, dim3((unsigned)blocks), dim3(256), 0, st, n, f, X, R, drop, Y);
    return launch_status();
}

gnn_status_t norm_forward_launch(int n, int f, const float *X, const float *R, const float *gamma, const float *beta,
                                 float eps, int act, const Dropout &drop, float *H, float *Y, float *stat, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    hipLaunchKernelGGL(norm_forward_kernel, dim3((unsigned)ceil_div(n, 4)), dim3(256), 0, st, n, f, X, R, gamma, beta, eps, act,
                       drop, H, Y, stat);
    return launch_status();
}

size_t norm_workspace_bytes(int64_t n, int64_t f) { return align_up((size_t)kNormBlocks * 2 * f * sizeof(double)); }

gnn_status_t norm_backward_launch(int n, int f, const float *X, const float *stat, const float *gamma, const float *beta,
                                  int act, const Dropout &drop, bool before, const float *dY, const float *dH, float *dR,
                                  float *dX, float *dgamma, float *dbeta, void *workspace, hipStream_t st) {
    double *part = static_cast<double *>(workspace);
    if (dgamma || dbeta) {                                 // before dX, which may lie over dY
        hipLaunchKernelGGL(norm_sums_kernel, dim3(kNormBlocks), dim3(256), 0, st, n, f, X, stat, gamma, beta, act, drop,
                           !before, dY, part);
        GNN_TRY(launch_status());
        hipLaunchKernelGGL(norm_sums_final_kernel, dim3((unsigned)ceil_div(2 * (int64_t)f, 256)), dim3(256), 0, st, f, kNormBlocks,
                           part, dgamma, dbeta);
        GNN_TRY(launch_status());
    }
    if (n <= 0 || (!dR && !dX)) return GNN_OK;
    hipLaunchKernelGGL(norm_backward_kernel, dim3((unsigned)ceil_div(n, 4)), dim3(256), 0, st, n, f, X, stat, gamma, beta, act,
                       drop, before, dY, dH, dR, dX);
    return launch_status();
}

}  // namespace gnn
