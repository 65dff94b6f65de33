// The gated feed-forward block H = act(X W_gate + b_gate) .* (X W_up + b_up), forward and backward.  Its large products are
// those of gemm_half.hip (forward, and backward where [A | U] was not kept, with the block's own epilogue) and of
// gemm_half_tn.hip; those of few rows are here and in gemm.hip.
#include "gemm_half.h"

namespace gnn {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx4u __attribute__((ext_vector_type(4), aligned(4)));


// Few rows: four wavefronts per 32 rows and 32 columns of H share the reduction, operands straight from memory into
// registers two steps ahead (the two lane halves of v_mfma_f32_32x32x2_f32 take P consecutive indices each), one launch, no
// scratch.  A wavefront has the sums of the gate and of the other projection for the same elements.  While tiles are few, bound by
// the launch and two waits for memory (1 x 256 -> 512 4.9 us); then by no one thing: 3001 x 203 -> 259, 18.2 us, four blocks on the
// fullest CU, takes 15.9 with no loads of X, 13.4 with none of W, and its matrix instructions alone 5.5; X in whole lines, which
// would have to pass through LDS, 17.5.  Steps of 16 indices leave room for a fourth wavefront per SIMD where 32 take 158
// registers (20.8 us); steps of 8, four ahead, 17.4, but 1 x 256 -> 512 5.3.
template <bool BACK, int GATE>
__global__ void __launch_bounds__(256)
gated_few_kernel(int M, int K, const float *__restrict__ X, const float *__restrict__ W, const float *__restrict__ bias, Gated g,
                 int tiles_n) {
    constexpr int AHEAD = 2, P = 8;            // steps ahead; indices of a step for each lane half
    __shared__ floatx4 sums[4][2][4][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l = lane % 32, half = lane / 32;
    const int m0 = (int)(blockIdx.x / tiles_n) * 32, j = (int)(blockIdx.x % tiles_n) * 32 + l, jj = min(j, g.half - 1);
    const int all = (K + 2 * P - 1) / (2 * P), first = all * wave / 4, total = all * (wave + 1) / 4;
    const float *x = X + (size_t)min(m0 + l, M - 1) * K, *w = W + jj;       // what is past the end re-reads the last
    const size_t ld = 2 * (size_t)g.half;
    float xs[AHEAD][P], ga[AHEAD][P], up[AHEAD][P];
    auto load = [&](int step, int s) __attribute__((always_inline)) {
        const int k0 = (2 * step + half) * P;
        if (k0 + P <= K) {
#pragma unroll
            for (int i = 0; i < P / 4; ++i) {
                const floatx4u v = *reinterpret_cast<const floatx4u *>(x + k0 + 4 * i);
                xs[s][4 * i] = v.x; xs[s][4 * i + 1] = v.y; xs[s][4 * i + 2] = v.z; xs[s][4 * i + 3] = v.w;
            }
#pragma unroll
            for (int i = 0; i < P; ++i) {
                ga[s][i] = w[(k0 + i) * ld];
                up[s][i] = w[(k0 + i) * ld + g.half];
            }
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) {
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
                for (int i = 0; i < P; ++i) {
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
        gate_of<GATE, BACK>(s[0][v], act, slope);
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

// D from the [A | U] that forward has kept, and the largest magnitudes of its rows and columns.  A block takes `rows` rows
// (top_rows where these are wanted) and 64 VEC columns of each half, `lanes` lanes a row; the `parts`
// blocks of the same rows stand side by side.  Bound by memory: 65536 x 1024 1.34 GB in 248 us, 5.4 TB/s.
template <int VEC, int GATE>
__global__ void __launch_bounds__(256)
gated_gradient_kernel(long n, int k, int lanes, int rows, int parts, const float *__restrict__ Z, const float *__restrict__ dH,
                      float *__restrict__ D, Tops tops) {
    __shared__ unsigned across[256][2 * VEC];
    const int gl = threadIdx.x & (lanes - 1), grp = threadIdx.x / lanes, groups = 256 / lanes;
    const int part = blockIdx.x % parts, block = blockIdx.x / parts, c = (part * 64 + gl) * VEC;
    const long r0 = (long)block * rows, r1 = min(n, r0 + rows);
    unsigned top[2 * VEC];
#pragma unroll
    for (int v = 0; v < 2 * VEC; ++v) top[v] = 0;
    constexpr int U = 4;                                   // rows under way
    for (long first = r0; first < r1; first += U * groups) {
        float a[U][VEC], u[U][VEC], d[U][VEC];
        unsigned most[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long row = first + i * groups + grp, at = row * 2 * k + c;
#pragma unroll
            for (int v = 0; v < VEC; ++v) a[i][v] = u[i][v] = d[i][v] = 0.f;
            if (row >= r1 || c >= k) continue;
            if constexpr (VEC == 4) {
                const float4 x = *reinterpret_cast<const float4 *>(Z + at), y = *reinterpret_cast<const float4 *>(Z + at + k);
                const float4 z = *reinterpret_cast<const float4 *>(dH + row * k + c);
                a[i][0] = x.x; a[i][1] = x.y; a[i][2] = x.z; a[i][3] = x.w;
                u[i][0] = y.x; u[i][1] = y.y; u[i][2] = y.z; u[i][3] = y.w;
                d[i][0] = z.x; d[i][1] = z.y; d[i][2] = z.z; d[i][3] = z.w;
            } else {
                a[i][0] = Z[at]; u[i][0] = Z[at + k]; d[i][0] = dH[row * k + c];
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long row = first + i * groups + grp, at = row * 2 * k + c;
            most[i] = 0;
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                float g, dg;
                gate_of<GATE, true>(a[i][v], g, dg);
                a[i][v] = d[i][v] * u[i][v] * dg;
                u[i][v] = d[i][v] * g;
                const unsigned ta = __float_as_uint(a[i][v]) & 0x7fffffffu, tu = __float_as_uint(u[i][v]) & 0x7fffffffu;
                top[v] = max(top[v], ta);
                top[VEC + v] = max(top[VEC + v], tu);
                most[i] = max(most[i], max(ta, tu));
            }
            if (row >= r1 || c >= k) continue;
            if constexpr (VEC == 4) {
                *reinterpret_cast<float4 *>(D + at) = make_float4(a[i][0], a[i][1], a[i][2], a[i][3]);
                *reinterpret_cast<float4 *>(D + at + k) = make_float4(u[i][0], u[i][1], u[i][2], u[i][3]);
            } else {
                D[at] = a[i][0]; D[at + k] = u[i][0];
            }
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
    for (int v = 0; v < 2 * VEC; ++v) across[threadIdx.x][v] = top[v];
    __syncthreads();
    if (grp == 0 && c < k)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            for (int q = 1; q < groups; ++q) {
                top[v] = max(top[v], across[q * lanes + gl][v]);
                top[VEC + v] = max(top[VEC + v], across[q * lanes + gl][VEC + v]);
            }
            tops.cols[(size_t)block * 2 * k + c + v] = top[v];
            tops.cols[(size_t)block * 2 * k + k + c + v] = top[VEC + v];
        }
}

// the other kernels read four indices at a time, of f_in and of 2 f_out
bool too_narrow(int64_t m, int64_t k) { return m < 4 || k < 2; }
// Tiles of 32 x 32 of H up to which the kernels for few rows are the faster, forward and back together; their time goes with tiles times
// f_in, where the others begin at three launches forward (one below 32 features) and six or seven backward.  Few rows / others in us,
// forward, with backward from Z: 40000 x 8 -> 64, 2500 tiles, 9.8 / 12.6, 54 / 76; 128000, 8000, 25.3 / 17.5, 119 / 120; 176000, 11000,
// 34 / 26, 161 / 159; 16000 x 31 -> 256, 4000, 17.0 / 17.5, 82 / 84; 60000 x 40 -> 64, 3750, 17.8 / 22.0, 79 / 100; 120000, 7500, 32 /
// 36, 138 / 140; 16000 x 64 -> 256, 4000, 20.7 / 21.9, 96 / 100; 24000, 6000, 29.3 / 25.7, 132 / 114; 32000 x 96 -> 96, 3000, 22.8 / 23.9,
// 101 / 100; 16000 x 128 -> 128, 2000, 19.5 / 18.0, 89 / 91; 4000 x 256 -> 256, 1000, 18.2 / 18.8, 86 / 87; 6000, 1504, 26.5 / 21.3,
// 125 / 93; 1500 x 512 -> 512, 752, 23.9 / 26.5, 98 / 99; 1984, 992, 32 / 27, 125 / 103.
int64_t few_tiles(int64_t m) { return m < 32 ? 8000 : 260000 / m; }
// Weights whose gradient is better off in float than through partial products of doubles and the pass over those, however few
// the rows, forward and back, doubles / float: 1 x 512 -> 1024 57 / 27 us, 256 rows 75 / 63; half as many weights, 1 x 256 -> 512, 28
// through doubles and 33 through parts of floats.
bool wide_weights(int64_t m, int64_t k) { return !too_narrow(m, k) && m * 2 * k >= 1 << 19; }
// D W^T is a product of the layers
bool short_columns(int64_t k) { return 2 * k < kShortReduction; }
bool gated_few(int64_t n, int64_t m, int64_t k) { return too_narrow(m, k) || ceil_div(n, 32) * ceil_div(k, 32) <= few_tiles(m); }

#define BY_GATE(GATE_, KERNEL_, ARG_)                                        \
    ((GATE_) == GNN_GATE_SIGMOID ? KERNEL_<ARG_, GNN_GATE_SIGMOID>           \
     : (GATE_) == GNN_GATE_SILU  ? KERNEL_<ARG_, GNN_GATE_SILU> : KERNEL_<ARG_, GNN_GATE_GELU>)

gnn_status_t few(int64_t n, int64_t m, const float *X, const float *W, const float *b, const Gated &g, hipStream_t st) {
    const int64_t tiles_n = ceil_div(g.half, 32), blocks = ceil_div(n, 32) * tiles_n;
    auto kernel = g.D ? BY_GATE(g.gate, gated_few_kernel, true) : BY_GATE(g.gate, gated_few_kernel, false);
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, (int)n, (int)m, X, W, b, g, (int)tiles_n);
    return launch_status();
}

gnn_status_t gradient(int64_t n, int k, int gate, const float *Z, const float *dH, float *D, const Tops &tops, int *parts,
                      hipStream_t st) {
    const bool vec = k % 4 == 0 && aligned16(Z) && aligned16(dH);
    int lanes = 1;
    while (lanes < 64 && lanes * (vec ? 4 : 1) < k) lanes <<= 1;
    *parts = (int)ceil_div(k, vec ? 256 : 64);
    const int rows = tops.cols ? top_rows(n) : (int)free_rows(n, lanes, *parts);
    auto kernel = vec ? BY_GATE(gate, gated_gradient_kernel, 4) : BY_GATE(gate, gated_gradient_kernel, 1);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(ceil_div(n, rows) * *parts)), dim3(256), 0, st, (long)n, k, lanes, rows, *parts,
                       Z, dH, D, tops);
    return launch_status();
}

// scratch of a backward pass behind D
struct Backward {
    unsigned *x_rows, *x_cols, *d_rows, *d_cols;
    void *rest;
    size_t bytes;
    Backward(char *at, int64_t n, int64_t m, int64_t k) {
        Carver carve(at);
        x_rows = carve.take<unsigned>(n * ceil_div(m, 64));
        x_cols = carve.take<unsigned>(most_top_blocks(n) * m);
        d_rows = carve.take<unsigned>(n * ceil_div(k, 32));      // gated_row_parts(n, k), or those of `gradient`
        d_cols = carve.take<unsigned>(most_top_blocks(n) * 2 * k);
        rest = carve.take<char>(0);
        size_t most = gemm_half_gated_workspace_bytes(k, m);
        for (size_t b : {gemm_half_workspace_bytes(m, 2 * k), gemm_half_tn_workspace_bytes(m, 2 * k, n), gemm_workspace_bytes(0, 1, n, m, 2 * k)})
            if (b > most) most = b;
        bytes = carve.off + most;
    }
};

}  // namespace

// A grid has less than 2^32 threads, 2^24 blocks of 256: the kernels for few rows take 32 x 32 elements of H a block, columns' largest
// magnitudes are formed in blocks of 32 rows and 64 columns at least.
bool gated_fits(bool backward, int64_t n, int64_t m, int64_t k) {
    if (m > 1 << 21 || k > 1 << 21) return false;
    const int64_t rows = ceil_div(n, 32), most = (int64_t)1 << 24;
    if (gated_few(n, m, k))
        return rows * ceil_div(k, 32) < most && (!backward || (gemm_fits(n, m, 2 * k) && gemm_half_tn_fits(m, 2 * k, n)));
    return rows * ceil_div(m > k ? m : k, 64) < most && gemm_half_fits(n, 2 * k) &&
           (!backward || ((short_columns(k) ? gemm_fits(n, m, 2 * k) : gemm_half_fits(n, m)) && gemm_half_tn_fits(m, 2 * k, n)));
}

// What n rows take, or fewer: a product of few rows needs less.
size_t gated_workspace_bytes(bool backward, int64_t n, int64_t m, int64_t k) {
    if (!backward) return gated_few(n, m, k) ? kAlign : align_up((size_t)n * ceil_div(m, 64) * sizeof(unsigned)) + gemm_half_gated_workspace_bytes(k, m);
    const size_t d = align_up((size_t)n * 2 * k * sizeof(float));
    size_t most = 0;
    // the rows up to which the kernels for few rows run
    const int64_t rows = too_narrow(m, k) ? n : 32 * (few_tiles(m) / ceil_div(k, 32)), small = n < rows ? n : rows;
    if (small > 0 && !wide_weights(m, k)) {
        const size_t tn = gemm_workspace_bytes(1, 0, m, 2 * k, small);     // a row of sums per chunk is an m-th of it
        most = tn + align_up(tn / m);
        const size_t x = gemm_workspace_bytes(0, 1, small, m, 2 * k);
        if (x > most) most = x;
    }
    if (!gated_few(n, m, k) || wide_weights(m, k)) {
        const Backward w(nullptr, n, m, k);
        if (w.bytes > most) most = w.bytes;
    }
    return d + most;
}

gnn_status_t gated_forward_launch(int gate, int n, int m, int k, const float *X, const float *W, const float *b, float *H,
                                  float *Z, void *workspace, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    const Gated g{k, gate, H, Z, nullptr, nullptr};
    if (gated_few(n, m, k)) return few(n, m, X, W, b, g, st);
    Carver carve(workspace);
    const Tops tops{carve.take<unsigned>((size_t)n * ceil_div(m, 64)), nullptr};
    if (m >= kShortReduction) GNN_TRY(tops_launch(n, m, X, tops, st));
    return gemm_half_gated_launch(n, m, X, tops.rows, W, b, g, Tops{nullptr, nullptr}, carve.take<char>(0), st);
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
    const Gated g{k, gate, nullptr, nullptr, dH, d};
    const bool one_step = n < kShortReduction;             // X^T D does without largest magnitudes
    int parts = 0;
    if (gated_few(n, m, k)) {
        void *rest = carve.take<char>(0);
        const bool wide = wide_weights(m, k);
        const Backward w(static_cast<char *>(rest), n, m, k);
        const Tops of_d{nullptr, wide && !one_step ? w.d_cols : nullptr};
        if (Z) {
            GNN_TRY(gradient(n, k, gate, Z, dH, d, of_d, &parts, st));
        } else {
            GNN_TRY(few(n, m, X, W, b, g, st));
            if (of_d.cols) GNN_TRY(tops_launch(n, 2 * k, d, of_d, st));
        }
        if (dX) GNN_TRY(gemm_launch(0, 1, n, m, 2 * (int64_t)k, d, W, dX, nullptr, 0, wide ? w.rest : rest, st));
        if (wide) {
            if (!one_step) GNN_TRY(tops_launch(n, m, X, Tops{nullptr, w.x_cols}, st));
            return gemm_half_tn_launch(m, 2 * (int64_t)k, n, X, w.x_cols, d, w.d_cols, dW, db, w.rest, st);
        }
        GemmExtras extras{};
        extras.sums = db;
        extras.workspace = static_cast<char *>(rest) + gemm_workspace_bytes(1, 0, m, 2 * (int64_t)k, n);
        return gemm_launch(1, 0, m, 2 * (int64_t)k, n, X, d, dW, nullptr, 0, rest, st, nullptr, 0, 0, nullptr, nullptr, &extras);
    }
    const Backward w(static_cast<char *>(workspace) + carve.off, n, m, k);
    const Tops of_x{Z || m < kShortReduction ? nullptr : w.x_rows, one_step ? nullptr : w.x_cols}, of_d{w.d_rows, w.d_cols};
    if (of_x.rows || of_x.cols) GNN_TRY(tops_launch(n, m, X, of_x, st));
    if (Z) {
        GNN_TRY(gradient(n, k, gate, Z, dH, d, of_d, &parts, st));
    } else {
        GNN_TRY(gemm_half_gated_launch(n, m, X, w.x_rows, W, b, g, of_d, w.rest, st));
        parts = gated_row_parts(n, k);
    }
    if (dX && short_columns(k)) GNN_TRY(gemm_launch(0, 1, n, m, 2 * (int64_t)k, d, W, dX, nullptr, 0, w.rest, st));
    else if (dX) GNN_TRY(gemm_half_launch(n, m, 2 * (int64_t)k, d, w.d_rows, parts, W, dX, w.rest, st));
    return gemm_half_tn_launch(m, 2 * (int64_t)k, n, X, w.x_cols, d, w.d_cols, dW, db, w.rest, st);
}

}  // namespace gnn
