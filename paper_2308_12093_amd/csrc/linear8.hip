// Y = act(X W^T + b) + R of rows in 8 bits and weights in 8 bits: sums of integers, which are exact, on v_mfma_i32_32x32x32_i8, and
// fp32 from the scales on.
#include <type_traits>

#include "activation.h"
#include "half_parts.h"
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
    int tiles_m, tiles_n;
};

// bytes of word i of four that stand before K, the others zero; k: the index of the first
__device__ __forceinline__ intx4 before(intx4 a, int k, int K) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int left = K - k - 4 * i;
        a[i] = left >= 4 ? a[i] : left <= 0 ? 0 : a[i] & ((1 << 8 * left) - 1);
    }
    return a;
}

// A block of four wavefronts owns 128 rows and 128 columns of Y, a wavefront 64 x 64.  Per step of 64 indices the block copies its rows of
// X and of W to LDS, 16 rows of 64 bytes an instruction, without touching registers, a step ahead; one barrier a step.  A row's four
// 16-byte pieces lie in the order piece ^ (row / 4 mod 4), so that the reads of sixteen rows fall on different banks.
// Four blocks a CU, which fall out of step: while some read and multiply others write.  65536 x 512 -> 2048 with SiLU and residual 1.1 GB
// in 231 us, 4.8 TB/s, the matrix cores busy for 13 %; of 4096 indices 1.5 POP/s, for LDS is longer at work than they.  What it spent
// its time on before: R's loads behind branches (801 -> 351 us, with LDS in place of lanes' own loads), then 64-bit addresses, comparisons
// of rows and columns for each element and an exact sigmoid (2400 vector instructions a wavefront, now 750).
template <int ACT>
__global__ void __launch_bounds__(256, ACT == GNN_ACT_GELU ? 3 : 4)
linear8_kernel(Product8 g) {
    __shared__ __align__(16) char x0[8192];
    __shared__ __align__(16) char x1[8192];
    __shared__ __align__(16) char w0[8192];
    __shared__ __align__(16) char w1[8192];
    __shared__ float x_scale[128];
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t / 64), lane = t % 64, l = lane % 32, half = lane / 32;
    const long tiles = (long)g.tiles_m * g.tiles_n, id = half_parts::xcd_tile(tiles);
    if (id >= tiles) return;
    const int m0 = (int)(id / g.tiles_n) * 128, n0 = (int)(id % g.tiles_n) * 128, steps = (int)((g.ld + 63) / 64), ld = (int)g.ld;
    // this wavefront's rows of X and of W, 16 an instruction; past the end the last again, and past a row's end its last piece again
    const char *x = reinterpret_cast<const char *>(g.X.q) + (size_t)m0 * ld, *w = reinterpret_cast<const char *>(g.W.q) + (size_t)n0 * ld;
    const int piece = 16 * (lane % 4 ^ lane / 16);
    unsigned x_row[2], w_row[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = 32 * wave + 16 * i + lane / 4;
        x_row[i] = (unsigned)min(r, g.M - 1 - m0) * ld;
        w_row[i] = (unsigned)min(r, g.N - 1 - n0) * ld;
    }
    auto copy = [](const char *base, unsigned offset, char *to) __attribute__((always_inline)) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + offset),
                                         (__attribute__((address_space(3))) void *)to, 16, 0, 0);
    };
    auto stage = [&](int step, char *xs, char *ws) __attribute__((always_inline)) {
        const unsigned at = min(step * 64 + piece, ld - 16);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            copy(x, x_row[i] + at, xs + (2 * wave + i) * 1024);
            copy(w, w_row[i] + at, ws + (2 * wave + i) * 1024);
        }
    };
    if (t < 128) x_scale[t] = g.X.scale[min(m0 + t, g.M - 1)];
    stage(0, x0, w0);
    intx16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
    const int wm = wave / 2, wn = wave % 2;
    // piece p of row r of a 32-row tile
    auto fragment = [&](const char *from, int tile, int p) __attribute__((always_inline)) {
        return *reinterpret_cast<const intx4 *>(from + (tile * 32 + l) * 64 + ((p ^ (l / 4)) & 3) * 16);
    };
    auto turn = [&](int step, const char *xs, const char *ws, char *next_x, char *next_w) __attribute__((always_inline)) {
        // this wavefront's copies of the step have arrived; after the barrier everyone's have, and the other buffers, read in the step
        // before, are free
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (step + 1 < steps) stage(step + 1, next_x, next_w);
#pragma unroll
        for (int ins = 0; ins < 2; ++ins) {
            intx4 a[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                a[i] = fragment(xs, 2 * wm + i, 2 * ins + half);
                b[i] = fragment(ws, 2 * wn + i, 2 * ins + half);
            }
            if ((step + 1) * 64 > g.K)
#pragma unroll
                for (int i = 0; i < 2; ++i) a[i] = before(a[i], step * 64 + 32 * ins + 16 * half, g.K);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[i], b[j], acc[i][j], 0, 0, 0);
        }
    };
    for (int step = 0; step < steps; step += 2) {
        turn(step, x0, w0, x1, w1);
        if (step + 1 < steps) turn(step + 1, x1, w1, x0, w0);
    }
    // accumulator register v of lane (half, l): row 8 (v / 4) + 4 half + v % 4, column l of its 32 x 32 tile.  Addresses are a scalar
    // base and the lane's own 32-bit offset; only blocks at an edge compare rows and columns.
    const int row0 = m0 + 64 * wm, col0 = n0 + 64 * wn;
    const size_t corner = (size_t)row0 * g.N + col0;
    const unsigned mine = 4u * half * (unsigned)g.N + l;
    auto at = [&](int i, int v, int j) __attribute__((always_inline)) { return corner + (size_t)(32 * i + 8 * (v / 4) + v % 4) * g.N + 32 * j; };
    float scale[2], bias[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int n = min(col0 + 32 * j + l, g.N - 1);
        scale[j] = g.W.scale[n];
        bias[j] = g.bias ? g.bias[n] : 0.f;
    }
    auto put = [&](int i, int v, int j, float r) __attribute__((always_inline)) {
        const float x = x_scale[64 * wm + 32 * i + 8 * (v / 4) + 4 * half + v % 4];
        float y, slope;
        activate<ACT, false>(fmaf((float)acc[i][j][v] * x, scale[j], bias[j]), y, slope);
        (g.Y + at(i, v, j))[mine] = y + r;
    };
    // The part of R that two tiles need is under way at once.  Where columns end inside, lanes are off for a tile; where rows do, element by
    // element.
    auto finish = [&](auto rows, auto columns) __attribute__((always_inline)) {
        constexpr bool ROWS = decltype(rows)::value, COLUMNS = decltype(columns)::value;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float r[2][16];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) r[j][v] = 0.f;
            if constexpr (ROWS && COLUMNS) {
                if (g.R)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
#pragma unroll
                        for (int j = 0; j < 2; ++j) r[j][v] = (g.R + at(i, v, j))[mine];
#pragma unroll
                for (int v = 0; v < 16; ++v)
#pragma unroll
                    for (int j = 0; j < 2; ++j) put(i, v, j, r[j][v]);
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (col0 + 32 * j + l >= g.N) continue;
                    if constexpr (ROWS) {
                        if (g.R)
#pragma unroll
                            for (int v = 0; v < 16; ++v) r[j][v] = (g.R + at(i, v, j))[mine];
#pragma unroll
                        for (int v = 0; v < 16; ++v) put(i, v, j, r[j][v]);
                    } else {
#pragma unroll
                        for (int v = 0; v < 16; ++v)
                            if (row0 + 32 * i + 8 * (v / 4) + 4 * half + v % 4 < g.M) put(i, v, j, g.R ? (g.R + at(i, v, j))[mine] : 0.f);
                    }
                }
            }
        }
    };
    if (row0 + 64 > g.M) finish(std::false_type(), std::false_type());
    else if (col0 + 64 > g.N) finish(std::true_type(), std::false_type());
    else finish(std::true_type(), std::true_type());
}

// Four wavefronts per 32 rows and 32 columns of Y share the reduction: a lane takes 16 consecutive bytes of its row of X and of its row
// of W straight into registers (the lane halves the first and the second 16 of 32), what lies behind K in them is made zero in X.
// 1 x 512 -> 1024 3.0 us, 2.5 a launch in a graph of fifty.  1024 x 512 -> 512 with residual 5.2, 5.9 with R and the scales
// loaded behind the sums; four steps under way gain nothing and cost 0.3 to 2 us where there are one or two.
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
    // a wavefront finishes a quarter of the tile; what it needs besides the sums is under way beside them
    const int row = m0 + 8 * wave + 4 * half, col = min(j, g.N - 1);
    float x_scale[4], with[4] = {0.f, 0.f, 0.f, 0.f};
    const float scale = g.W.scale[col], bias = g.bias ? g.bias[col] : 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) x_scale[v] = g.X.scale[min(row + v, g.M - 1)];
    if (g.R) {
#pragma unroll
        for (int v = 0; v < 4; ++v) with[v] = g.R[(size_t)min(row + v, g.M - 1) * g.N + col];
    }
    for (int step = first; step < total; ++step) {
        const int k = step * 32 + 16 * half, at = min(k, (int)g.ld - 16);
        intx4 a = *reinterpret_cast<const intx4 *>(x + at);
        const intx4 b = *reinterpret_cast<const intx4 *>(w + at);
        if (k + 16 > g.K) a = before(a, k, g.K);
        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[wave][i][lane] = intx4{acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]};
    __syncthreads();
    if (j >= g.N) return;
    const intx4 z = (sums[0][wave][lane] + sums[1][wave][lane]) + (sums[2][wave][lane] + sums[3][wave][lane]);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (row + v >= g.M) continue;
        float y, slope;
        activate<ACT, false>(fmaf((float)z[v] * x_scale[v], scale, bias), y, slope);
        g.Y[(size_t)(row + v) * g.N + j] = g.R ? y + with[v] : y;
    }
}

// Tiles of 32 x 32 of Y up to which the kernel for few rows is the faster: its time goes with tiles times f_in.  It / the other in us, with
// SiLU: 4096 x 128 -> 512, 2048 tiles, 6.0 / 5.7; 1024 x 512 -> 512, 512, 5.0 / 6.5; 2048, 1024, 7.3 / 6.7; 2048 x 1024 -> 256, 512,
// 6.6 / 8.3; 4096, 1024, 11.6 / 8.6; 512 x 2048 -> 1024, 512, 10.2 / 12.2; 1024, 1024, 18.1 / 12.5; 8192 x 203 -> 259, 2304, 8.4 / 8.8;
// 32768 x 64 -> 64, 2048, 4.9 / 11.9.
bool linear8_few(int64_t n, int64_t m, int64_t k) { return ceil_div(n, 32) * ceil_div(k, 32) <= 300 + 350000 / m; }

}  // namespace

// sums of f_in products of 127 x 127 in 32 bits; blocks of 32 x 32
bool linear8_fits(int64_t n, int64_t m, int64_t k) {
    return m <= 1 << 17 && k <= 1 << 21 && ceil_div(n, 32) * ceil_div(k, 32) < (int64_t)1 << 24;
}

gnn_status_t linear8_forward_launch(int act, int n, int m, int k, const Rows8 &X, const Rows8 &W, const float *b, const float *R, float *Y,
                                    hipStream_t st) {
    if (n <= 0) return GNN_OK;
    const bool few = linear8_few(n, m, k);
    const int tile = few ? 32 : 128;
    const Product8 g{n, k, m, (long)rows8_stride(m), X, W, b, R, Y, (int)ceil_div(n, tile), (int)ceil_div(k, tile)};
    const int64_t tiles = (int64_t)g.tiles_m * g.tiles_n;
    const dim3 grid((unsigned)(few ? tiles : 8 * ceil_div(tiles, 8)));
#define LINEAR8_CASE(ACT_)                                                                        \
    if (act == ACT_) {                                                                            \
        if (few) hipLaunchKernelGGL(linear8_few_kernel<ACT_>, grid, dim3(256), 0, st, g);         \
        else hipLaunchKernelGGL(linear8_kernel<ACT_>, grid, dim3(256), 0, st, g);                 \
    }
    LINEAR8_CASE(GNN_ACT_NONE) LINEAR8_CASE(GNN_ACT_RELU) LINEAR8_CASE(GNN_ACT_ELU)
    LINEAR8_CASE(GNN_ACT_SIGMOID) LINEAR8_CASE(GNN_ACT_SILU) LINEAR8_CASE(GNN_ACT_GELU)
#undef LINEAR8_CASE
    return launch_status();
}

}  // namespace gnn
