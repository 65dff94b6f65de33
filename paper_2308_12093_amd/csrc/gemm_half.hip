// Products of fp32 matrices on the fp16 matrix instruction (half_parts.h), for the gated block: X W with the gate behind it, and
// D W^T.
#include "gemm_half_kernel.h"

namespace gnn {
namespace {

using namespace half_parts;

// ---- parts of B -------------------------------------------------------------------------------------------
// out: [32-column tile][step][instruction][part][lane][8]; lane (half, l): column 32 tile + l, indices 32 step + 16 half +
// 8 instruction + 0..7; zeros past N and K.  exps[32 tile + l]: the column's power of two.
// halves: B is [B_gate | B_up], and `halves` consecutive tiles hold columns of the one and the same columns of the other.
// A block of 1024 threads finds the largest magnitudes of its tile's columns and writes kPartSteps steps of it.
constexpr int kPartSteps = 16;

template <bool TB>
__global__ void __launch_bounds__(1024)
half_weights_kernel(int N, int K, int steps, HalfOperand b, int halves, char *__restrict__ out, int *__restrict__ exps) {
    __shared__ unsigned top[32];
    const int t = threadIdx.x, lane = t % 64, l = lane % 32, half = lane / 32, ins = t / 64 % 2, sub = t / 128;
    int n = blockIdx.x * 32 + l;
    if (halves) {
        const int c = blockIdx.x % halves, pair = halves / 2, j = ((int)blockIdx.x / halves * pair + c % pair) * 32 + l;
        n = j < N / 2 ? j + (c < pair ? 0 : N / 2) : N;
    }
    auto fetch = [&](int step, float (&x)[8]) __attribute__((always_inline)) {
        const int k0 = step * KB + 16 * half + 8 * ins;
        const float *at = b.p + k0 * b.sk + n * b.sn;
        if (TB && n < N && k0 + 8 <= K) {
            const float4u u = *reinterpret_cast<const float4u *>(at), v = *reinterpret_cast<const float4u *>(at + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[j] = u[j]; x[4 + j] = v[j]; }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = n < N && k0 + j < K ? at[j * (TB ? 1 : b.sk)] : 0.f;
        }
    };
    if (t < 32) top[t] = 0;
    __syncthreads();
    float x[8];
    if constexpr (TB) {                                    // a column is a row in memory: a wavefront reads two of the 32
        const int c = t / 64 * 2;
        unsigned both[2] = {0, 0};
#pragma unroll 4
        for (int k = 4 * lane; k < K; k += 256)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                // the last four where fewer are left; a column past the end is the last one again
                const float4u v = *reinterpret_cast<const float4u *>(b.p + min(k, K - 4) + (long)min((int)blockIdx.x * 32 + c + i, N - 1) * b.sn);
#pragma unroll
                for (int j = 0; j < 4; ++j) both[i] = max(both[i], __float_as_uint(v[j]) & 0x7fffffffu);
            }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) both[i] = max(both[i], (unsigned)__shfl_xor((int)both[i], d, 64));
            if (lane == 0) top[c + i] = both[i];
        }
    } else {
        unsigned most = 0;
        for (int s = sub; s < steps; s += 8) {
            fetch(s, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(x[j]) & 0x7fffffffu);
        }
        most = max(most, (unsigned)__shfl_xor((int)most, 32, 64));
        if (half == 0) atomicMax(&top[l], most);
    }
    __syncthreads();
    const int e = exponent_of(top[l]);
    if (blockIdx.y == 0 && t < 32) exps[blockIdx.x * 32 + t] = e;
    const float scale = power_of_two(e), scale2 = power_of_two(e + 11);
    char *to = out + (size_t)blockIdx.x * steps * kTileBytes + lane * 16;
    const int end = min(steps, ((int)blockIdx.y + 1) * kPartSteps);
    for (int s = blockIdx.y * kPartSteps + sub; s < end; s += 8) {
        half8 part[2];
        fetch(s, x);
        halves8(x, scale, scale2, part);
#pragma unroll
        for (int p = 0; p < 2; ++p)
            *reinterpret_cast<half8 *>(to + (size_t)s * kTileBytes + (ins * 2 + p) * kFragBytes) = part[p];
    }
}

// ---- largest magnitudes -----------------------------------------------------------------------------------
// A block reads `rows` rows (top_rows where the columns' are wanted) and 64 VEC columns, `lanes` lanes a row; the `parts` blocks of
// the same rows stand side by side.  65536 x 512, 134 MB: of the rows 25 us, 5.3 TB/s, of the
// columns 35.
template <int VEC>
__global__ void __launch_bounds__(256)
tops_kernel(long n, int m, int lanes, int rows, int parts, const float *__restrict__ X, Tops tops) {
    __shared__ unsigned across[256][VEC];
    const int gl = threadIdx.x & (lanes - 1), grp = threadIdx.x / lanes, groups = 256 / lanes;
    const int part = blockIdx.x % parts, block = blockIdx.x / parts, c = (part * 64 + gl) * VEC;
    const long r0 = (long)block * rows, r1 = min(n, r0 + rows);
    unsigned top[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) top[v] = 0;
    constexpr int U = 4;                                   // rows under way (8: 32 and 35 us)
    for (long first = r0; first < r1; first += U * groups) {
        unsigned x[U][VEC], most[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long row = first + i * groups + grp;
#pragma unroll
            for (int v = 0; v < VEC; ++v) x[i][v] = 0;
            if (row >= r1 || c >= m) continue;
            if constexpr (VEC == 4) {
                const uintx4 u = *reinterpret_cast<const uintx4 *>(X + row * m + c);
                x[i][0] = u.x; x[i][1] = u.y; x[i][2] = u.z; x[i][3] = u.w;
            } else {
                x[i][0] = __float_as_uint(X[row * m + c]);
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            most[i] = 0;
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                x[i][v] &= 0x7fffffffu;
                top[v] = max(top[v], x[i][v]);
                most[i] = max(most[i], x[i][v]);
            }
        }
        if (!tops.rows) continue;
        for (int d = lanes >> 1; d > 0; d >>= 1)
#pragma unroll
            for (int i = 0; i < U; ++i) most[i] = max(most[i], (unsigned)__shfl_xor((int)most[i], d, 64));
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long row = first + i * groups + grp;
            if (gl == 0 && row < r1) tops.rows[(size_t)part * n + row] = most[i];
        }
    }
    if (!tops.cols) return;
#pragma unroll
    for (int v = 0; v < VEC; ++v) across[threadIdx.x][v] = top[v];
    __syncthreads();
    if (grp == 0 && c < m)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            for (int k = 1; k < groups; ++k) top[v] = max(top[v], across[k * lanes + gl][v]);
            tops.cols[(size_t)block * m + c + v] = top[v];
        }
}

// sum of the parts of a split reduction
__global__ void __launch_bounds__(256)
sum_splits_kernel(long count, int splits, const float *__restrict__ part, float *__restrict__ C) {
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    float a = 0.f, b = 0.f;
    int s = 0;
    for (; s + 1 < splits; s += 2) {
        a += part[s * count + i];
        b += part[(s + 1) * count + i];
    }
    if (s < splits) a += part[s * count + i];
    C[i] = a + b;
}

// Parts of a long reduction where its tiles leave most of the chip idle, four steps of it at least: 1024 x 512 x 2048 65 -> 22 us, the sum
// of the parts among them.
constexpr int64_t kSplitBlocks = 512;
int plain_splits(int64_t tiles, int64_t steps) {
    if (tiles >= kSplitBlocks / 2) return 1;
    int64_t splits = kSplitBlocks / tiles;
    if (splits > steps / 4) splits = steps / 4;
    return splits < 1 ? 1 : (int)splits;
}
constexpr size_t kSplitBytes = kSplitBlocks * 128 * 64 * sizeof(float);    // their tiles have two column tiles

}  // namespace

gnn_status_t half_parts::split_weights(const HalfProduct &g, int tiles, int halves, hipStream_t st) {
    const dim3 grid((unsigned)(g.tiles_n * tiles), (unsigned)ceil_div(g.steps, kPartSteps));
    auto kernel = g.B.sk == 1 ? half_weights_kernel<true> : half_weights_kernel<false>;
    hipLaunchKernelGGL(kernel, grid, dim3(1024), 0, st, g.N, g.K, g.steps, g.B, halves, const_cast<char *>(g.parts),
                       const_cast<int *>(g.exps));
    return launch_status();
}

// a grid has less than 2^32 threads
bool gemm_half_fits(int64_t M, int64_t N) {
    return N <= INT32_MAX / 4 && M <= INT32_MAX - 256 && ceil_div(M, 128) * ceil_div(N, 64) < ((int64_t)1 << 24) - 8;
}

size_t gemm_half_workspace_bytes(int64_t N, int64_t K) { return half_parts_bytes(N, K) + half_exps_bytes(N) + kSplitBytes; }
size_t gemm_half_gated_workspace_bytes(int64_t half, int64_t K) { return half_parts_bytes(2 * half, K) + half_exps_bytes(2 * half); }

int top_parts(int64_t m, const float *X) { return (int)ceil_div(m, m % 4 == 0 && aligned16(X) ? 256 : 64); }

gnn_status_t tops_launch(int64_t n, int m, const float *X, const Tops &tops, hipStream_t st) {
    const bool vec = m % 4 == 0 && aligned16(X);
    int lanes = 1;
    while (lanes < 64 && lanes * (vec ? 4 : 1) < m) lanes <<= 1;
    const int parts = top_parts(m, X), rows = tops.cols ? top_rows(n) : (int)free_rows(n, lanes, parts);
    hipLaunchKernelGGL(vec ? tops_kernel<4> : tops_kernel<1>, dim3((unsigned)(ceil_div(n, rows) * parts)), dim3(256), 0, st, (long)n,
                       m, lanes, rows, parts, X, tops);
    return launch_status();
}

gnn_status_t gemm_half_launch(int64_t M, int64_t N, int64_t K, const float *A, const unsigned *row_tops, int parts, const float *B,
                              float *C, void *workspace, hipStream_t st) {
    HalfProduct g{};
    set_product(g, M, N, K, workspace);
    g.A = A; g.row_tops = row_tops; g.top_parts = parts;
    g.B = HalfOperand{B, 1, (long)K};
    g.C = C;
    g.stream = (size_t)M * N * sizeof(float) > kStreamBytes;
    const int w = half_tiles(M, N), splits = plain_splits((int64_t)g.tiles_m * g.tiles_n, g.steps);
    if (splits > 1) {
        g.split_steps = (int)ceil_div(g.steps, splits);
        g.splits = (int)ceil_div(g.steps, g.split_steps);
        g.C = reinterpret_cast<float *>(static_cast<char *>(workspace) + half_parts_bytes(N, K) + half_exps_bytes(N));
    }
    GNN_TRY(split_weights(g, w, 0, st));
    const bool aligned = K % 4 == 0 && K < 1 << 24 && aligned16(A);
    auto kernel = w == 2 ? (aligned ? gemm_half_kernel<2, kPlain, kCopied, 0> : gemm_half_kernel<2, kPlain, kLoaded, 0>)
                                     : (aligned ? gemm_half_kernel<4, kPlain, kCopied, 0> : gemm_half_kernel<4, kPlain, kLoaded, 0>);
    hipLaunchKernelGGL(kernel, product_grid(g), dim3(256), 0, st, g);
    GNN_TRY(launch_status());
    if (g.splits == 1) return GNN_OK;
    hipLaunchKernelGGL(sum_splits_kernel, dim3((unsigned)ceil_div(M * N, 256)), dim3(256), 0, st, (long)(M * N), g.splits, g.C, C);
    return launch_status();
}

int gated_row_parts(int64_t n, int64_t half) { return (int)ceil_div(half, 16 * half_tiles(n, 2 * half)); }

gnn_status_t gemm_half_gated_launch(int64_t M, int64_t K, const float *X, const unsigned *row_tops, const float *W,
                                    const float *bias, const Gated &out, const Tops &tops, void *workspace, hipStream_t st) {
    HalfProduct g{};
    const int64_t N = 2 * (int64_t)out.half;
    const int w = half_tiles(M, N);
    set_product(g, M, N, K, workspace);
    g.tiles_n = (int)ceil_div(out.half, 16 * w);
    g.A = X; g.row_tops = row_tops; g.top_parts = top_parts(K, X);
    g.B = HalfOperand{W, (long)N, 1};
    g.bias = bias;
    g.gated = out;
    g.tops = tops;
    g.stream = !out.D && (size_t)M * N * sizeof(float) > kStreamBytes;      // D is read next
    const bool back = out.D != nullptr;
    const int rows = K < kShortReduction ? kShort : K % 4 == 0 && K < 1 << 24 && aligned16(X) ? kCopied : kLoaded;
    if (rows != kShort) GNN_TRY(split_weights(g, w, w, st));
    const dim3 grid = product_grid(g);
#define GATED_CASE(NT_, ROWS_, GATE_)                                                                                       \
    if (w == NT_ && rows == ROWS_ && out.gate == GATE_) {                                                                   \
        if (back) hipLaunchKernelGGL((gemm_half_kernel<NT_, kGateBackward, ROWS_, GATE_>), grid, dim3(256), 0, st, g);      \
        else hipLaunchKernelGGL((gemm_half_kernel<NT_, kGateForward, ROWS_, GATE_>), grid, dim3(256), 0, st, g);            \
    }
#define GATED_CASES(NT_, ROWS_) \
    GATED_CASE(NT_, ROWS_, GNN_GATE_SIGMOID) GATED_CASE(NT_, ROWS_, GNN_GATE_SILU) GATED_CASE(NT_, ROWS_, GNN_GATE_GELU)
    GATED_CASES(2, kLoaded) GATED_CASES(2, kCopied) GATED_CASES(2, kShort)
    GATED_CASES(4, kLoaded) GATED_CASES(4, kCopied) GATED_CASES(4, kShort)
#undef GATED_CASES
#undef GATED_CASE
    return launch_status();
}

}  // namespace gnn
