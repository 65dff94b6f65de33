// The product with its epilogue, Y = act(X W + b) + R, forward and backward: which kernels a call takes, and its workspace.  Products of many
// aligned rows are those of pair_product.hip and pair_tn.hip; of rows at any alignment, narrow outputs and reductions of one step those of
// gemm_half_kernel.h (linear_half.hip) and gemm_half_tn.hip; of few rows they are here and in gemm.hip.
#include "linear.h"
#include "rows.h"

namespace gnn {
namespace {

using namespace half_parts;

// Few rows: four wavefronts per 32 rows and 32 columns of Y share the reduction, operands straight from memory into
// registers two steps ahead (the two lane halves of v_mfma_f32_32x32x2_f32 take P consecutive indices each), one launch, no scratch.
// While tiles are few, bound by the launch and two waits for memory (1 x 256 -> 512 4.0 us, 3.4 a launch in a graph of fifty); then by the
// loads, 32 rows at a time by lanes, and the instruction on the fullest CU (3001 x 203 -> 259 with GELU and residual 12.4 us, 13.7 with R
// loaded behind the sums).
template <bool BACK, int ACT>
__global__ void __launch_bounds__(256)
linear_few_kernel(int M, int N, int K, const float *__restrict__ X, const float *__restrict__ W, const float *__restrict__ bias, Linear g,
                  int tiles_n) {
    constexpr int AHEAD = 2, P = 8;            // steps ahead; indices of a step for each lane half
    __shared__ floatx4 sums[4][4][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l = lane % 32, half = lane / 32;
    const int m0 = (int)(blockIdx.x / tiles_n) * 32, j = (int)(blockIdx.x % tiles_n) * 32 + l;
    const int all = (K + 2 * P - 1) / (2 * P), first = all * wave / 4, total = all * (wave + 1) / 4;
    const float *x = X + (size_t)min(m0 + l, M - 1) * K, *w = W + min(j, N - 1);       // what is past the end re-reads the last
    const size_t ld = N;
    float xs[AHEAD][P], ws[AHEAD][P];
    auto load = [&](int step, int s) __attribute__((always_inline)) {
        const int k0 = (2 * step + half) * P;
        if (k0 + P <= K) {
#pragma unroll
            for (int i = 0; i < P / 4; ++i) {
                const float4u v = *reinterpret_cast<const float4u *>(x + k0 + 4 * i);
                xs[s][4 * i] = v.x; xs[s][4 * i + 1] = v.y; xs[s][4 * i + 2] = v.z; xs[s][4 * i + 3] = v.w;
            }
#pragma unroll
            for (int i = 0; i < P; ++i) ws[s][i] = w[(k0 + i) * ld];
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                xs[s][i] = k0 + i < K ? x[k0 + i] : 0.f;
                ws[s][i] = k0 + i < K ? w[(k0 + i) * ld] : 0.f;
            }
        }
    };
    floatx16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
    for (int s = 0; s < AHEAD; ++s)
        if (first + s < total) load(first + s, s);
    // a wavefront finishes a quarter of the tile: accumulator register v of lane (half, l) is row 8 (v / 4) + 4 half + v % 4; what it adds
    // or multiplies by is under way beside the sums
    const int row = m0 + 8 * wave + 4 * half, col = min(j, N - 1);
    const float *beside = BACK ? g.dY : g.R;
    float with[4] = {0.f, 0.f, 0.f, 0.f};
    const float b = bias ? bias[col] : 0.f;
    if (beside) {
#pragma unroll
        for (int v = 0; v < 4; ++v) with[v] = beside[(size_t)min(row + v, M - 1) * N + col];
    }
    for (int step = first; step < total; step += AHEAD) {
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            if (step + s < total) {
#pragma unroll
                for (int i = 0; i < P; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(xs[s][i], ws[s][i], acc, 0, 0, 0);
                if (step + s + AHEAD < total) load(step + s + AHEAD, s);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[wave][i][lane] = floatx4{acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]};
    __syncthreads();
    if (j >= N) return;
    const floatx4 z = (sums[0][wave][lane] + sums[1][wave][lane]) + (sums[2][wave][lane] + sums[3][wave][lane]) + b;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (row + v >= M) continue;
        float y, slope;
        activate<ACT, BACK>(z[v], y, slope);
        const size_t at = (size_t)(row + v) * N + j;
        if constexpr (BACK) {
            g.D[at] = with[v] * slope;
        } else {
            if (g.Z) g.Z[at] = z[v];
            g.Y[at] = g.R ? y + with[v] : y;
        }
    }
}

// D = dY .* act'(Z) from the Z that forward has kept, as it is or in 8 bits, and the largest magnitudes of its rows and of its columns,
// those with each row times row_scale.  A block takes `rows` rows (top_rows where columns' are wanted) and 256 columns, `lanes` lanes a
// row, four columns each; the `parts` blocks of the same rows stand side by side.  D NULL: not wanted (it is dY).  Bound by memory: 65536 x
// 2048 with SiLU 1.6 GB in 304 us, 5.3 TB/s; Z and dY are read past the caches, to leave the place to D, which the products read next (335 us; where D is dY they read it
// from memory).
template <bool ALIGNED, int ACT, bool HELD>
__global__ void __launch_bounds__(256)
linear_gradient_kernel(long n, int k, int lanes, int rows, int parts, const float *__restrict__ Z, Rows8 held, const float *__restrict__ dY,
                       const float *__restrict__ row_scale, float *__restrict__ D, Tops tops) {
    __shared__ unsigned across[256][4];
    const int gl = threadIdx.x & (lanes - 1), grp = threadIdx.x / lanes, groups = 256 / lanes;
    const int part = blockIdx.x % parts, block = blockIdx.x / parts, c = (part * 64 + gl) * 4;
    const long r0 = (long)block * rows, r1 = min(n, r0 + rows), ld = rows8_stride(k);
    auto read = [&](const float *row) __attribute__((always_inline)) {
        if constexpr (!ALIGNED) return rows::load4(row, c, k);
        const floatx4 v = __builtin_nontemporal_load(reinterpret_cast<const floatx4 *>(row + c));
        return make_float4(v.x, v.y, v.z, v.w);
    };
    unsigned top[4] = {0, 0, 0, 0};
    constexpr int U = 4;                                   // rows under way
    for (long first = r0; first < r1; first += U * groups) {
        float4 z[U], d[U];
        float factor[U];
        unsigned most[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long row = first + i * groups + grp;
            factor[i] = 1.f;
            z[i] = d[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (row >= r1 || c >= k) continue;
            if (row_scale) factor[i] = row_scale[row];
            d[i] = read(dY + row * k);
            if constexpr (ACT != GNN_ACT_NONE && !HELD) z[i] = read(Z + row * k);
            if constexpr (ACT != GNN_ACT_NONE && HELD) {   // what lies behind a row's end is any integer, but dY is zero there
                const float s = held.scale[row];
                const float4 x = integers(*reinterpret_cast<const unsigned *>(held.q + row * ld + c));
                const float4 e = held.columns ? rows::load4(held.columns, c, k) : make_float4(1.f, 1.f, 1.f, 1.f);
                z[i] = make_float4(x.x * s * e.x, x.y * s * e.y, x.z * s * e.z, x.w * s * e.w);
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long row = first + i * groups + grp;
            float4 &v = d[i];
            if constexpr (ACT != GNN_ACT_NONE) {
                float y, s[4];
                activate<ACT, true>(z[i].x, y, s[0]);
                activate<ACT, true>(z[i].y, y, s[1]);
                activate<ACT, true>(z[i].z, y, s[2]);
                activate<ACT, true>(z[i].w, y, s[3]);
                v = make_float4(v.x * s[0], v.y * s[1], v.z * s[2], v.w * s[3]);
            }
            most[i] = largest(v);
            top[0] = max(top[0], magnitude(v.x * factor[i]));
            top[1] = max(top[1], magnitude(v.y * factor[i]));
            top[2] = max(top[2], magnitude(v.z * factor[i]));
            top[3] = max(top[3], magnitude(v.w * factor[i]));
            if (!D || row >= r1 || c >= k) continue;
            if constexpr (ALIGNED) *reinterpret_cast<float4 *>(D + row * k + c) = v;
            else rows::store4(D + row * k, c, k, v);
        }
        if (!tops.rows) continue;
        for (int q = lanes >> 1; q > 0; q >>= 1)
#pragma unroll
            for (int i = 0; i < U; ++i) most[i] = max(most[i], (unsigned)__shfl_xor((int)most[i], q, 64));
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long row = first + i * groups + grp;
            if (gl == 0 && row < r1) tops.rows[(size_t)part * n + row] = most[i];
        }
    }
    if (!tops.cols) return;
#pragma unroll
    for (int v = 0; v < 4; ++v) across[threadIdx.x][v] = top[v];
    __syncthreads();
    if (grp == 0)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            for (int q = 1; q < groups; ++q) top[v] = max(top[v], across[q * lanes + gl][v]);
            if (c + v < k) tops.cols[(size_t)block * k + c + v] = top[v];
        }
}

// The whole backward pass of a small product in one launch: blocks of 32 x 32 elements of dX, then of dW, whose eight wavefronts share the
// reduction as above; D = dY .* act'(Z) is formed where it is read, and so is X from its integers.  What such a pass takes is
// launches: 61 x 11 -> 768 in 8 bits 16.7 us by way of X and D in floats, gnn_gemm's products and a sum of their parts.
struct SmallBack {
    int n, m, k, tiles_x, tiles_k, tiles_dx;               // tiles_dx: blocks of dX, in front
    const float *X;                                        // NULL: from `x8`
    Rows8 x8;
    const float *W, *Z;                                    // Z NULL: from `z8`
    Rows8 z8;
    const float *dY;
    float *dW, *db, *dX;                                   // db: or NULL
};

template <int ACT, bool HELD>
__global__ void __launch_bounds__(512)
linear_small_back_kernel(SmallBack g) {
    constexpr int WAVES = 8, AHEAD = 2, P = 8;
    __shared__ floatx4 sums[WAVES][4][64];
    __shared__ float s_db[WAVES][32];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l = lane % 32, half = lane / 32;
    const bool weights = (int)blockIdx.x >= g.tiles_dx;    // uniform
    const int block = weights ? (int)blockIdx.x - g.tiles_dx : (int)blockIdx.x, across = weights ? g.tiles_k : g.tiles_x;
    const int r0 = block / across * 32, c0 = block % across * 32, K = weights ? g.n : g.k;
    const int all = (K + 2 * P - 1) / (2 * P), first = all * wave / WAVES, total = all * (wave + 1) / WAVES;
    const long z_ld = rows8_stride(g.k), x_ld = rows8_stride(g.m);
    floatx16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
    float db = 0.f;
    auto d_of = [&](float dy, float z) __attribute__((always_inline)) {
        if constexpr (ACT == GNN_ACT_NONE) return dy;
        float y, slope;
        activate<ACT, true>(z, y, slope);
        return dy * slope;
    };
    // P operands of each of two matrices, and what the second (dW) or first (dX) has to be formed from
    float a[AHEAD][P], b[AHEAD][P], z[AHEAD][P];
    if (weights) {
        const int m = min(r0 + l, g.m - 1), j = min(c0 + l, g.k - 1);
        const float column = ACT != GNN_ACT_NONE && HELD && g.z8.columns ? g.z8.columns[j] : 1.f;
        auto load = [&](int step, int s) __attribute__((always_inline)) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int row = (2 * step + half) * P + p;
                const bool in = row < g.n;
                const size_t i = in ? row : 0;             // what is past the end is read from the first row and not used
                a[s][p] = g.X ? g.X[i * g.m + m] : (float)g.x8.q[i * x_ld + m] * g.x8.scale[i];
                b[s][p] = g.dY[i * g.k + j];
                if constexpr (ACT != GNN_ACT_NONE)
                    z[s][p] = HELD ? (float)g.z8.q[i * z_ld + j] * g.z8.scale[i] * column : g.Z[i * g.k + j];
                if (!in) a[s][p] = b[s][p] = z[s][p] = 0.f;
            }
        };
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
            if (first + s < total) load(first + s, s);
        for (int step = first; step < total; step += AHEAD) {
#pragma unroll
            for (int s = 0; s < AHEAD; ++s)
                if (step + s < total) {
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const float d = d_of(b[s][p], z[s][p]);
                        db += d;
                        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[s][p], d, acc, 0, 0, 0);
                    }
                    if (step + s + AHEAD < total) load(step + s + AHEAD, s);
                }
        }
    } else {
        const size_t i = min(r0 + l, g.n - 1), c = min(c0 + l, g.m - 1);
        const float scale = ACT != GNN_ACT_NONE && HELD ? g.z8.scale[i] : 1.f;
        const float *dy = g.dY + i * g.k, *zs = HELD || ACT == GNN_ACT_NONE ? nullptr : g.Z + i * g.k, *w = g.W + c * g.k;
        const int8_t *q = HELD ? g.z8.q + i * z_ld : nullptr;
        auto load = [&](int step, int s) __attribute__((always_inline)) {
            const int k0 = (2 * step + half) * P;
            if (k0 + P <= g.k) {
#pragma unroll
                for (int h = 0; h < P; h += 4) {
                    const float4u u = *reinterpret_cast<const float4u *>(dy + k0 + h), v = *reinterpret_cast<const float4u *>(w + k0 + h);
                    float4u e = {0.f, 0.f, 0.f, 0.f};
                    if constexpr (ACT != GNN_ACT_NONE && !HELD) e = *reinterpret_cast<const float4u *>(zs + k0 + h);
                    if constexpr (ACT != GNN_ACT_NONE && HELD) {
                        const float4 f = integers(*reinterpret_cast<const unsigned *>(q + k0 + h));
                        e = float4u{f.x * scale, f.y * scale, f.z * scale, f.w * scale};
                        if (g.z8.columns) e *= *reinterpret_cast<const float4u *>(g.z8.columns + k0 + h);
                    }
#pragma unroll
                    for (int p = 0; p < 4; ++p) { a[s][h + p] = u[p]; b[s][h + p] = v[p]; z[s][h + p] = e[p]; }
                }
            } else {
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const bool in = k0 + p < g.k;
                    a[s][p] = in ? dy[k0 + p] : 0.f;
                    b[s][p] = in ? w[k0 + p] : 0.f;
                    z[s][p] = 0.f;
                    if constexpr (ACT != GNN_ACT_NONE) {
                        if (in) z[s][p] = HELD ? (float)q[k0 + p] * scale * (g.z8.columns ? g.z8.columns[k0 + p] : 1.f) : zs[k0 + p];
                    }
                }
            }
        };
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
            if (first + s < total) load(first + s, s);
        for (int step = first; step < total; step += AHEAD) {
#pragma unroll
            for (int s = 0; s < AHEAD; ++s)
                if (step + s < total) {
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(d_of(a[s][p], z[s][p]), b[s][p], acc, 0, 0, 0);
                    if (step + s + AHEAD < total) load(step + s + AHEAD, s);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[wave][i][lane] = floatx4{acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]};
    db += __shfl_xor(db, 32, 64);
    if (half == 0) s_db[wave][l] = db;
    __syncthreads();
    if (weights && g.db && r0 == 0 && wave == 0 && half == 0 && c0 + l < g.k) {
        float s = 0.f;
        for (int w = 0; w < WAVES; ++w) s += s_db[w][l];
        g.db[c0 + l] = s;
    }
    // four wavefronts finish a quarter of the tile each: accumulator register v of lane (half, l) is row 8 (v / 4) + 4 half + v % 4
    const int col = c0 + l, rows = weights ? g.m : g.n, cols = weights ? g.k : g.m;
    if (wave >= 4 || col >= cols) return;
    floatx4 s = sums[0][wave][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += sums[w][wave][lane];
    float *out = weights ? g.dW : g.dX;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int row = r0 + 8 * wave + 4 * half + v;
        if (row < rows) out[(size_t)row * cols + col] = weights && !g.X && g.x8.columns ? s[v] * g.x8.columns[row] : s[v];
    }
}

// the other kernels read four indices at a time
bool too_narrow(int64_t m, int64_t k) { return m < 4 || k < 4; }
// Tiles of 32 x 32 of Y up to which the kernels for few rows are the faster; their time goes with tiles times f_in, where the others begin at
// three launches forward (one below 32 features) and six backward.  Few rows / others in us, forward with SiLU and Z: 128000 x 32 -> 64,
// 8000 tiles, 21 / 23; 256000, 16000, 39 / 37; 32000 x 64 -> 256, 8000, 24.6 / 24.2; 16000 x 128 -> 128, 2000, 14.4 / 17.0; 32000, 4000,
// 23 / 21; 1984 x 256 -> 1024, 2000, 20.8 / 20.8; 1984 x 512 -> 512, 1000, 19.8 / 24.8; 4000, 2000, 35 / 27; 992 x 1024 -> 1024, 1000,
// 33.5 / 37.7; 1984, 2000, 63 / 40; 7104 x 203 -> 259, 2000, 22.2 / 23.7.  Backward from Z: 32000 x 64 -> 256, 8000, 71 / 76; 64000, 16000,
// 112 / 97; 32000 x 128 -> 128, 4000, 60 / 61; 4000 x 256 -> 256, 1000, 45 / 54; 8000, 2000, 67 / 64; 992 x 512 -> 512, 500, 42 / 54;
// 1984, 1000, 68 / 65; 480 x 1024 -> 1024, 500, 53 / 66; 992, 1000, 87 / 73; 3552 x 203 -> 259, 1000, 47 / 51.
int64_t few_tiles(bool backward, int64_t m) { return m < 32 ? 8000 : backward ? 500000 / m + 150 : 380000 / m + 650; }
// weights whose gradient is better off in float than through partial products of doubles and the pass over those, however few the rows
bool wide_weights(int64_t m, int64_t k) { return !too_narrow(m, k) && m * k >= 1 << 19; }
// D W^T is a product of the layers
bool short_columns(int64_t k) { return k < kShortReduction; }
bool linear_few(bool backward, int64_t n, int64_t m, int64_t k) {
    return too_narrow(m, k) || ceil_div(n, 32) * ceil_div(k, 32) <= few_tiles(backward, m);
}
// the rows up to which a backward pass takes them
int64_t few_rows(int64_t n, int64_t m, int64_t k) {
    if (too_narrow(m, k)) return n;
    const int64_t rows = 32 * (few_tiles(true, m) / ceil_div(k, 32));
    return n < rows ? n : rows;
}

#define BY_ACT(ACT_, KERNEL_, ...)                                             \
    ((ACT_) == GNN_ACT_RELU      ? KERNEL_(GNN_ACT_RELU, __VA_ARGS__)          \
     : (ACT_) == GNN_ACT_ELU     ? KERNEL_(GNN_ACT_ELU, __VA_ARGS__)           \
     : (ACT_) == GNN_ACT_SIGMOID ? KERNEL_(GNN_ACT_SIGMOID, __VA_ARGS__)       \
     : (ACT_) == GNN_ACT_SILU    ? KERNEL_(GNN_ACT_SILU, __VA_ARGS__) : KERNEL_(GNN_ACT_GELU, __VA_ARGS__))
#define FEW_KERNEL(ACT_, BACK_) linear_few_kernel<BACK_, ACT_>
#define GRADIENT_KERNEL(ACT_, ALIGNED_, HELD_) linear_gradient_kernel<ALIGNED_, ACT_, HELD_>

gnn_status_t few(int act, int64_t n, int64_t m, int64_t k, const float *X, const float *W, const float *b, const Linear &g, hipStream_t st) {
    const int64_t tiles_n = ceil_div(k, 32), blocks = ceil_div(n, 32) * tiles_n;
    auto kernel = g.D ? BY_ACT(act, FEW_KERNEL, true) : act == GNN_ACT_NONE ? linear_few_kernel<false, GNN_ACT_NONE> : BY_ACT(act, FEW_KERNEL, false);
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, (int)n, (int)k, (int)m, X, W, b, g, (int)tiles_n);
    return launch_status();
}

gnn_status_t gradient(int act, int64_t n, int k, const float *Z, const Rows8 &held, const float *dY, const float *row_scale, float *D,
                      const Tops &tops, int *parts, hipStream_t st) {
    const bool aligned = k % 4 == 0 && aligned16(Z) && aligned16(dY);
    int lanes = 1;
    while (lanes < 64 && lanes * 4 < k) lanes <<= 1;
    *parts = (int)ceil_div(k, 256);
    const int rows = tops.cols ? top_rows(n) : (int)free_rows(n, lanes, *parts);
    auto kernel = act == GNN_ACT_NONE ? (aligned ? linear_gradient_kernel<true, GNN_ACT_NONE, false> : linear_gradient_kernel<false, GNN_ACT_NONE, false>)
                  : Z ? (aligned ? BY_ACT(act, GRADIENT_KERNEL, true, false) : BY_ACT(act, GRADIENT_KERNEL, false, false))
                      : (aligned ? BY_ACT(act, GRADIENT_KERNEL, true, true) : BY_ACT(act, GRADIENT_KERNEL, false, true));
    hipLaunchKernelGGL(kernel, dim3((unsigned)(ceil_div(n, rows) * *parts)), dim3(256), 0, st, (long)n, k, lanes, rows, *parts, Z, held,
                       dY, row_scale, D, tops);
    return launch_status();
}

// of X W, whichever kernel forms it
size_t product_bytes(int64_t k, int64_t m) {
    const size_t pair = pair_workspace_bytes(k, m), half = linear_half_workspace_bytes(k, m);
    return pair > half ? pair : half;
}

int64_t four(int64_t width) { return (width + 3) / 4 * 4; }

// Rows of `m` floats with zeros behind them up to a multiple of four, and their largest magnitudes unless `tops` is NULL: [part of 256
// columns][row].  `lanes` lanes a row, four columns each.  30000 x 301, 72 MB: 17 us with the magnitudes, from and to the caches.
__global__ void __launch_bounds__(256)
pad_rows_kernel(long n, int m, int lanes, int rows, int parts, const float *__restrict__ X, float *__restrict__ out, unsigned *__restrict__ tops) {
    const int gl = threadIdx.x & (lanes - 1), grp = threadIdx.x / lanes, groups = 256 / lanes;
    const int part = blockIdx.x % parts, c = (part * 64 + gl) * 4;
    const long r0 = (long)(blockIdx.x / parts) * rows, r1 = min(n, r0 + rows), ld = (m + 3) / 4 * 4;
    constexpr int U = 4;                                   // rows under way
    for (long first = r0; first < r1; first += U * groups) {
        float4 x[U];
        unsigned most[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long row = first + i * groups + grp;
            x[i] = row < r1 && c < m ? rows::load4(X + row * m, c, m) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long row = first + i * groups + grp;
            if (row < r1 && c < m) *reinterpret_cast<float4 *>(out + row * ld + c) = x[i];
            most[i] = largest(x[i]);
        }
        if (!tops) continue;
        for (int q = lanes >> 1; q > 0; q >>= 1)
#pragma unroll
            for (int i = 0; i < U; ++i) most[i] = max(most[i], (unsigned)__shfl_xor((int)most[i], q, 64));
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long row = first + i * groups + grp;
            if (gl == 0 && row < r1) tops[(size_t)part * n + row] = most[i];
        }
    }
}

gnn_status_t pad_rows(int64_t n, int m, const float *X, float *out, unsigned *tops, hipStream_t st) {
    int lanes = 1;
    while (lanes < 64 && lanes * 4 < m) lanes <<= 1;
    const int parts = (int)ceil_div(m, 256), rows = (int)free_rows(n, lanes, parts);
    hipLaunchKernelGGL(pad_rows_kernel, dim3((unsigned)(ceil_div(n, rows) * parts)), dim3(256), 0, st, (long)n, m, lanes, rows, parts, X, out, tops);
    return launch_status();
}

// Whether a product of rows that are no multiple of four floats is one of rows that are, in `space`: 30000 x 301 -> 1000 forward 199 us
// from the rows as they are (gemm_half_kernel.h, which lanes read themselves).
bool padded(int64_t M, int64_t N, int64_t K, const float *space) {
    return K % 4 != 0 && K >= kShortReduction && pair_product_fits(M, N, four(K), space);
}

// forward's room for rows of X with zeros behind them, in floats
int64_t forward_space(int64_t n, int64_t m, int64_t k) { return padded(n, k, m, nullptr) ? n * four(m) : 0; }

// Backward's room beside D, in floats, for one of these after the other: X in 8 bits brought to floats, of as many rows as do not go to
// dW as the integers they are (all up to some number); rows of X, and of D, with zeros behind them.  No less for a larger n.
int64_t backward_space(int64_t n, int64_t m, int64_t k) {
    int64_t rows = n;
    if (!linear_few(true, n, m, k) && pair_tn_fits(m, k, n, true)) {
        rows = pair_tn_least_rows(m, k) - 1;
        if (few_rows(n, m, k) > rows) rows = few_rows(n, m, k);
    }
    int64_t most = rows * m;
    if (padded(n, k, m, nullptr) && n * four(m) > most) most = n * four(m);
    if (padded(n, m, k, nullptr) && n * four(k) > most) most = n * four(k);
    return most;
}

// act(X W + b) + R, or D and its largest magnitudes, `parts` a row.  x_rows: room for the largest magnitudes of X's rows, filled where
// `known`; space: n four(m) floats where X is padded.
gnn_status_t product(int act, int64_t n, int64_t m, int64_t k, const float *X, unsigned *x_rows, bool known, const float *W, const float *b,
                     const Linear &g, const Tops &tops, int *parts, float *space, void *workspace, hipStream_t st) {
    const bool pad = padded(n, k, m, space), pair = pad || pair_product_fits(n, k, m, X);
    *parts = pair ? pair_row_parts(k) : linear_row_parts(n, k);
    if (pad) GNN_TRY(pad_rows(n, (int)m, X, space, known ? nullptr : x_rows, st));
    else if (!known && m >= kShortReduction) GNN_TRY(tops_launch(n, (int)m, X, Tops{x_rows, nullptr}, st));
    const int x_parts = pad && !known ? (int)ceil_div(m, 256) : top_parts(m, X);
    if (pair) return pair_linear_launch(act, n, k, four(m), m, pad ? space : X, x_rows, x_parts, W, b, g, tops, workspace, st);
    return linear_half_launch(act, n, k, m, X, x_rows, W, b, g, tops, workspace, st);
}

// Rows and widths up to which one launch is the faster; its time goes with n times the blocks.  One launch / the others in us, SiLU from
// floats and from 8 bits: 128 x 64 -> 64 5.8 / 15.0, 5.5 / 17.7; 512 x 64 -> 64 8.3 / 15.3, 12.3 / 19.9; 1024 13.7 / 15.5, 21.9 / 18.0;
// 2048 25 / 16; 512 x 256 -> 1024 21 / 36, 23 / 40; 1024 29 / 41, 43 / 45; 128 x 1024 -> 1024 17 / 40, 21 / 44; 512 51 / 53, 66 / 58;
// 1 x 1024 -> 2048 18.7 / 19.2, 21.5 / 21.6.
bool small_back(bool held, int64_t n, int64_t m, int64_t k) {
    return n <= (held ? 512 : 1024) && k <= 2048 && n * ceil_div(m, 32) * (ceil_div(n, 32) + ceil_div(k, 32)) <= 800000;
}

gnn_status_t small_backward(int act, int64_t n, int64_t m, int64_t k, const float *X, const Rows8 &X8, const float *W, const float *Z,
                            const Rows8 &Z8, const float *dY, float *dW, float *db, float *dX, hipStream_t st) {
    const int tiles_x = (int)ceil_div(m, 32), tiles_k = (int)ceil_div(k, 32), tiles_dx = dX ? (int)ceil_div(n, 32) * tiles_x : 0;
    const SmallBack g{(int)n, (int)m, (int)k, tiles_x, tiles_k, tiles_dx, X, X8, W, Z, Z8, dY, dW, db, dX};
#define SMALL_KERNEL(ACT_, HELD_) linear_small_back_kernel<ACT_, HELD_>
    auto kernel = act == GNN_ACT_NONE ? linear_small_back_kernel<GNN_ACT_NONE, false>
                  : Z ? BY_ACT(act, SMALL_KERNEL, false) : BY_ACT(act, SMALL_KERNEL, true);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles_dx + tiles_x * tiles_k)), dim3(512), 0, st, g);
    return launch_status();
}

// scratch of a backward pass behind D and X
struct Backward {
    unsigned *x_rows, *x_cols, *d_rows, *d_cols;
    void *rest;
    size_t bytes;
    Backward(char *at, int64_t n, int64_t m, int64_t k) {
        Carver carve(at);
        x_rows = carve.take<unsigned>(n * ceil_div(m, 64));
        x_cols = carve.take<unsigned>(most_top_blocks(n) * m);
        d_rows = carve.take<unsigned>(n * (ceil_div(k, 64) + 1));  // those of `product`, of `gradient` or top_parts
        d_cols = carve.take<unsigned>(most_top_blocks(n) * k);
        rest = carve.take<char>(0);
        size_t most = product_bytes(k, four(m));
        for (size_t b : {pair_workspace_bytes(m, four(k)), pair_tn_workspace_bytes(m, k, n), gemm_half_workspace_bytes(m, k), gemm_half_tn_workspace_bytes(m, k, n), gemm_workspace_bytes(0, 1, n, m, k)})
            if (b > most) most = b;
        bytes = carve.off + most;
    }
};

}  // namespace

// A grid has less than 2^32 threads, 2^24 blocks of 256: the kernels for few rows take 32 x 32 elements of Y a block, columns' largest
// magnitudes are formed in blocks of 32 rows and 64 columns at least.
bool linear_fits(bool backward, int64_t n, int64_t m, int64_t k) {
    if (m > 1 << 21 || k > 1 << 21) return false;
    const int64_t rows = ceil_div(n, 32), most = (int64_t)1 << 24;
    if (linear_few(backward, n, m, k))
        return rows * ceil_div(k, 32) < most && (!backward || (gemm_fits(n, m, k) && gemm_half_tn_fits(m, k, n)));
    return rows * ceil_div(m > k ? m : k, 64) < most && gemm_half_fits(n, k) &&
           (!backward || ((short_columns(k) ? gemm_fits(n, m, k) : gemm_half_fits(n, m)) && gemm_half_tn_fits(m, k, n)));
}

// What n rows take, or fewer: a product of few rows needs less.
size_t linear_workspace_bytes(bool backward, int64_t n, int64_t m, int64_t k) {
    if (!backward)
        return linear_few(false, n, m, k) ? kAlign
                                          : align_up((size_t)n * ceil_div(m, 64) * sizeof(unsigned)) +
                                                align_up((size_t)forward_space(n, m, k) * sizeof(float)) + product_bytes(k, four(m));
    const size_t d = align_up((size_t)n * k * sizeof(float)) + align_up((size_t)backward_space(n, m, k) * sizeof(float));
    size_t most = 0;
    const int64_t small = few_rows(n, m, k);
    if (small > 0 && !wide_weights(m, k)) {
        const size_t tn = gemm_workspace_bytes(1, 0, m, k, small);         // a row of sums per chunk is an m-th of it
        most = tn + align_up(tn / m);
        const size_t x = gemm_workspace_bytes(0, 1, small, m, k);
        if (x > most) most = x;
    }
    if (!linear_few(true, n, m, k) || wide_weights(m, k)) {
        const Backward w(nullptr, n, m, k);
        if (w.bytes > most) most = w.bytes;
    }
    return d + most;
}

gnn_status_t linear_forward_launch(int act, int n, int m, int k, const float *X, const float *W, const float *b, const float *R, float *Y,
                                   float *Z, void *workspace, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    const Linear g{R, Y, Z, nullptr, nullptr};
    if (linear_few(false, n, m, k)) return few(act, n, m, k, X, W, b, g, st);
    Carver carve(workspace);
    unsigned *x_rows = carve.take<unsigned>((size_t)n * ceil_div(m, 64));
    float *space = carve.take<float>(forward_space(n, m, k));
    int parts;
    return product(act, n, m, k, X, x_rows, false, W, b, g, Tops{nullptr, nullptr}, &parts, space, carve.take<char>(0), st);
}

gnn_status_t linear_backward_launch(int act, int n, int m, int k, const float *X, const Rows8 &X8, const float *W, const float *b,
                                    const float *Z, const Rows8 &Z8, const float *dY, float *dW, float *db, float *dX, void *workspace,
                                    hipStream_t st) {
    if (n <= 0) {
        GNN_TRY(fill_zero_launch((int64_t)m * k, dW, st));
        return db ? fill_zero_launch(k, db, st) : GNN_OK;
    }
    Carver carve(workspace);
    float *d_space = carve.take<float>((size_t)n * k), *x_space = carve.take<float>(backward_space(n, m, k));
    const bool plain = act == GNN_ACT_NONE, kept = Z || Z8.q;
    const float *d = plain ? dY : d_space;
    const Linear g{nullptr, nullptr, nullptr, dY, d_space};
    if (small_back(!X, n, m, k)) {
        if (plain || kept) return small_backward(act, n, m, k, X, X8, W, Z, Z8, dY, dW, db, dX, st);
        GNN_TRY(few(act, n, m, k, X, W, b, g, st));
        return small_backward(GNN_ACT_NONE, n, m, k, X, X8, W, nullptr, no_rows8(), d, dW, db, dX, st);
    }
    const bool is_few = linear_few(true, n, m, k), pair_tn = !is_few && pair_tn_fits(m, k, n, !X);
    const float *row_scale = nullptr;                      // what X8's rows are to be taken times, where its integers are read as they are
    if (!X && pair_tn) {
        row_scale = X8.scale;
    } else if (!X) {
        GNN_TRY(dequantize_rows_launch(n, m, X8, x_space, st));
        X = x_space;
    }
    const bool one_step = n < kShortReduction;             // X^T D does without largest magnitudes
    int parts = 0;
    if (is_few) {
        void *rest = carve.take<char>(0);
        const bool wide = wide_weights(m, k);
        const Backward w(static_cast<char *>(rest), n, m, k);
        const Tops of_d{nullptr, wide && !one_step ? w.d_cols : nullptr};
        if (!plain && kept) {
            GNN_TRY(gradient(act, n, k, Z, Z8, dY, nullptr, d_space, of_d, &parts, st));
        } else {
            if (!plain) GNN_TRY(few(act, n, m, k, X, W, b, g, st));
            if (of_d.cols) GNN_TRY(tops_launch(n, k, d, of_d, st));
        }
        if (dX) GNN_TRY(gemm_launch(0, 1, n, m, k, d, W, dX, nullptr, 0, wide ? w.rest : rest, st));
        if (wide) {
            if (!one_step) GNN_TRY(tops_launch(n, m, X, Tops{nullptr, w.x_cols}, st));
            return gemm_half_tn_launch(m, k, n, X, w.x_cols, d, w.d_cols, dW, db, w.rest, st);
        }
        GemmExtras extras{};
        extras.sums = db;
        extras.workspace = static_cast<char *>(rest) + gemm_workspace_bytes(1, 0, m, k, n);
        return gemm_launch(1, 0, m, k, n, X, d, dW, nullptr, 0, rest, st, nullptr, 0, 0, nullptr, nullptr, &extras);
    }
    const Backward w(static_cast<char *>(workspace) + carve.off, n, m, k);
    const Tops of_x{plain || kept || m < kShortReduction ? nullptr : w.x_rows, one_step || !X ? nullptr : w.x_cols}, of_d{w.d_rows, w.d_cols};
    if (of_x.rows || of_x.cols) GNN_TRY(tops_launch(n, m, X, of_x, st));
    if (plain && !row_scale) {
        GNN_TRY(tops_launch(n, k, dY, of_d, st));
        parts = top_parts(k, dY);
    } else if (plain || kept) {
        GNN_TRY(gradient(act, n, k, Z, Z8, dY, row_scale, plain ? nullptr : d_space, of_d, &parts, st));
    } else {
        GNN_TRY(product(act, n, m, k, X, w.x_rows, of_x.rows != nullptr, W, b, g, of_d, &parts, x_space, w.rest, st));
    }
    if (dX && short_columns(k)) {
        GNN_TRY(gemm_launch(0, 1, n, m, k, d, W, dX, nullptr, 0, w.rest, st));
    } else if (dX && X != x_space && padded(n, m, k, x_space)) {
        GNN_TRY(pad_rows(n, k, d, x_space, nullptr, st));
        GNN_TRY(pair_plain_launch(n, m, four(k), k, x_space, w.d_rows, parts, W, dX, w.rest, st));
    } else if (dX && pair_product_fits(n, m, k, d)) {
        GNN_TRY(pair_plain_launch(n, m, k, k, d, w.d_rows, parts, W, dX, w.rest, st));
    } else if (dX) GNN_TRY(gemm_half_launch(n, m, k, d, w.d_rows, parts, W, dX, w.rest, st));
    if (pair_tn) return pair_tn_launch(m, k, n, X, X8, w.x_cols, d, w.d_cols, dW, db, w.rest, st);
    return gemm_half_tn_launch(m, k, n, X, w.x_cols, d, w.d_cols, dW, db, w.rest, st);
}

}  // namespace gnn
