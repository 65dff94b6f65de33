// Products of many fp32 rows with weights on the fp16 matrix instruction (half_pair.h), and what becomes of them: C itself,
// act(X W + b) + R, dY .* act'(X W + b).
#include <type_traits>

#include "activation.h"
#include "half_pair.h"
#include "linear.h"

namespace gnn {
namespace {

using namespace half_pair;

// ---- parts of B -------------------------------------------------------------------------------------------
// out: [32-column tile][step][part][lane][8]; lane (half, l): column 32 tile + l, indices 16 step + 8 half + 0..7; zeros past N and K.
// exps[32 tile + l]: the column's power of two.  A block of 1024 threads finds the largest magnitudes of its tile's columns and writes
// kPartSteps steps of it.
constexpr int kPartSteps = 32;

template <bool TB>
__global__ void __launch_bounds__(1024)
pair_weights_kernel(int N, int K, int steps, HalfOperand b, char *__restrict__ out, int *__restrict__ exps) {
    __shared__ unsigned top[32];
    const int t = threadIdx.x, lane = t % 64, l = lane % 32, half = lane / 32, sub = t / 64;
    const int n = blockIdx.x * 32 + l;
    auto fetch = [&](int step, float (&x)[8]) __attribute__((always_inline)) {
        const int k0 = step * KP + 8 * half;
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
        for (int s = sub; s < steps; s += 16) {
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
    const float scale = power_of_two(e);
    char *to = out + (size_t)blockIdx.x * steps * kPairBytes + lane * 16;
    const int end = min(steps, ((int)blockIdx.y + 1) * kPartSteps);
    for (int s = blockIdx.y * kPartSteps + sub; s < end; s += 16) {
        half8 part[2];
        fetch(s, x);
        pairs8(x, scale, part);
#pragma unroll
        for (int p = 0; p < 2; ++p) *reinterpret_cast<half8 *>(to + (size_t)s * kPairBytes + p * 1024) = part[p];
    }
}

// ---- rows times weights -----------------------------------------------------------------------------------
struct PairProduct {
    int M, N, K, steps;                // K: floats between rows of A, zeros behind the first KB of them
    int KB;                            // indices that B has
    const float *A;
    const unsigned *row_tops;          // [top_parts][M]
    int top_parts;
    HalfOperand B;
    const char *parts;                 // of B
    const int *exps;
    const float *bias;
    int tiles_m, tiles_n;
    Linear linear;                     // Y: C
    Tops tops;                         // of D: 2 tiles_n parts a row
};

enum { kPlain, kForward, kBackward };

// A block of four wavefronts owns 128 rows and 64 NJ columns, a wavefront 64 rows and 32 NJ columns.  Per step of 16 indices the
// block copies its rows (64 bytes each, 16 rows an instruction) and the parts of its columns to LDS, without touching registers, a step ahead;
// one barrier a step.  A row's four 16-byte pieces lie in the order piece ^ (row / 4 mod 4), so that the reads of sixteen rows fall on
// different banks.  A lane reads eight consecutive floats of its two rows back and splits them.
// With NJ = 4 a step is 24 matrix instructions of 32 cycles to 4 + 8 reads of 1 KB, 6 copies and about 70 vector instructions of 4
// cycles; with NJ = 2 LDS is as long at work as the matrix cores.  65536 x 2048 -> 512 plain: 400 us when the card is cool, 344 TFLOP/s of the
// product and 1.03 PFLOP/s on the instruction, 465 us after some more of them: the clock falls to 1.8 GHz and below, the instruction is
// busy for 54 % of the cycles.  (In half_parts.h's two scales: 458 and 496.)  65536 x 512 -> 2048 with SiLU, residual and Z, 1.7 GB besides:
// 570 to 640 us.  Pairs of the next step between the matrix instructions, with three buffers in LDS: 399 and 461, D of 2^17 x 128 -> 256
// 105 instead of 98.
// K is a multiple of 4, below 2^22, and A 16-byte aligned.
template <int NJ, int OUT, int ACT>
__global__ void __launch_bounds__(256, NJ == 2 && OUT != kBackward ? 3 : 2)
pair_product_kernel(PairProduct g) {
    __shared__ __align__(16) char a_even[8192];
    __shared__ __align__(16) char a_odd[8192];
    __shared__ __align__(16) char b_even[2 * NJ * kPairBytes];
    __shared__ __align__(16) char b_odd[2 * NJ * kPairBytes];
    __shared__ int s_exp[128];
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t / 64), lane = t % 64, l = lane % 32, half = lane / 32;
    const long tiles = (long)g.tiles_m * g.tiles_n, id = xcd_tile(tiles);
    if (id >= tiles) return;
    const int wm = wave / 2, wn = wave % 2;
    const int m0 = (int)(id / g.tiles_n) * 128, ct0 = (int)(id % g.tiles_n) * 2 * NJ;        // first row, first column tile
    const int row0 = m0 + 64 * wm, col0 = (ct0 + NJ * wn) * 32;                               // the wavefront's
    // global -> LDS, 1 KB per wavefront and instruction, from a uniform base and a 32-bit offset
    auto copy = [](const char *base, unsigned offset, char *to) __attribute__((always_inline)) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + offset),
                                         (__attribute__((address_space(3))) void *)to, 16, 0, 0);
    };
    // rows past the end re-read the last, pieces past a row's end its last
    const char *base = reinterpret_cast<const char *>(g.A + (size_t)m0 * g.K);
    const int piece = 16 * (lane % 4 ^ lane / 16);
    unsigned mine[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) mine[i] = 4u * (unsigned)min(32 * wave + 16 * i + lane / 4, g.M - 1 - m0) * (unsigned)g.K;
    auto stage = [&](int step, char *as, char *bs) __attribute__((always_inline)) {
        const unsigned at = min(step * 64 + piece, 4 * g.K - 16);
#pragma unroll
        for (int i = 0; i < 2; ++i) copy(base, mine[i] + at, as + (2 * wave + i) * 1024);
        // the 4 NJ fragments of a step are dealt to the four wavefronts
#pragma unroll
        for (int i = 0; i < NJ; ++i) {
            const int f = NJ * wave + i;
            copy(g.parts + ((size_t)(ct0 + f / 2) * g.steps + step) * kPairBytes + f % 2 * 1024, lane * 16, bs + f * 1024);
        }
    };
    stage(0, a_even, b_even);
    if (t < 128) {
        unsigned top = 0;
        for (int p = 0; p < g.top_parts; ++p) top = max(top, g.row_tops[(size_t)p * g.M + min(m0 + t, g.M - 1)]);
        s_exp[t] = exponent_of(top);
    }
    floatx16 acc[2][NJ];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    __syncthreads();
    float scale[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) scale[i] = power_of_two(s_exp[64 * wm + 32 * i + l]);
    auto turn = [&](int step, const char *as, const char *bs, char *next_a, char *next_b) __attribute__((always_inline)) {
        // this wavefront's copies of the step have arrived; after the barrier everyone's have, and the other buffers,
        // read in the step before, are free
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (step + 1 < g.steps) stage(step + 1, next_a, next_b);
        half8 a[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            floatx4 raw[2];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                raw[p] = *reinterpret_cast<const floatx4 *>(as + (64 * wm + 32 * i + l) * 64 + ((2 * half + p) ^ (l / 4 & 3)) * 16);
                if ((step + 1) * KP > g.K && step * KP + 8 * half + 4 * p >= g.K) raw[p] = floatx4{0.f, 0.f, 0.f, 0.f};
            }
            pairs8({raw[0][0], raw[0][1], raw[0][2], raw[0][3], raw[1][0], raw[1][1], raw[1][2], raw[1][3]}, scale[i], a[i]);
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            half8 b[2];
#pragma unroll
            for (int p = 0; p < 2; ++p) b[p] = *reinterpret_cast<const half8 *>(bs + ((NJ * wn + j) * 2 + p) * 1024 + lane * 16);
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][1], b[0], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][0], b[1], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][0], b[0], acc[i][j], 0, 0, 0);
        }
    };
    for (int step = 0; step < g.steps; step += 2) {
        turn(step, a_even, b_even, a_odd, b_odd);
        if (step + 1 < g.steps) turn(step + 1, a_odd, b_odd, a_even, b_even);
    }
    float finite = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) finite = fmaf(acc[i][j][v], 0.f, finite);
    // accumulator register v of lane (half, l): row 8 (v / 4) + 4 half + v % 4, column l of its 32 x 32 tile.  Addresses are a scalar base and
    // the lane's own 32-bit offset; only blocks at an edge compare rows and columns.
    const size_t corner = (size_t)row0 * g.N + col0;
    const unsigned own = 4u * half * (unsigned)g.N + l;
    auto at = [&](int i, int j, int v) __attribute__((always_inline)) { return corner + (size_t)(32 * i + 8 * (v / 4) + v % 4) * g.N + 32 * j; };
    auto there = [&](int i, int j, int v) __attribute__((always_inline)) {
        return row0 + 32 * i + 8 * (v / 4) + 4 * half + v % 4 < g.M && col0 + 32 * j + l < g.N;
    };
    auto bias_of = [&](int j) __attribute__((always_inline)) { return OUT != kPlain && g.bias ? g.bias[min(col0 + 32 * j + l, g.N - 1)] : 0.f; };
    unsigned *s_top = reinterpret_cast<unsigned *>(b_even);        // of the block's columns
    if constexpr (OUT == kBackward) {
        __syncthreads();
        if (t < 64 * NJ) s_top[t] = 0;
        __syncthreads();
    }
    // the largest magnitudes of rows 32 i ..: over the 32 lanes of a row each step a lane hands on half of its rows and keeps the other
    // half; in the end lanes 2 v and 2 v + 1 have row v
    auto put_rows = [&](unsigned (&top)[16], int i) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 16, rows = 8; rows >= 1; d >>= 1, rows >>= 1) {
            const bool upper = l & d;
#pragma unroll
            for (int v = 0; v < rows; ++v) {
                const unsigned give = upper ? top[v] : top[v + rows], keep = upper ? top[v + rows] : top[v];
                top[v] = max(keep, (unsigned)__shfl_xor((int)give, d, 64));
            }
        }
        top[0] = max(top[0], (unsigned)__shfl_xor((int)top[0], 1, 64));
        const int v = l / 2, row = row0 + 32 * i + 4 * half + 8 * (v / 4) + v % 4;
        if (l % 2 == 0 && row < g.M) g.tops.rows[(size_t)(ct0 / NJ + wn) * g.M + row] = top[0];
    };
    // and of column tile j in rows 32 i ..: theirs, or through LDS those of the block
    auto put_cols = [&](unsigned top, int i, int j) __attribute__((always_inline)) {
        top = max(top, (unsigned)__shfl_xor((int)top, 32, 64));
        if (half != 0) return;
        if (top_rows(g.M) != 32) atomicMax(&s_top[(wn * NJ + j) * 32 + l], top);
        else if (row0 + 32 * i < g.M && col0 + 32 * j + l < g.N) g.tops.cols[(size_t)(row0 / 32 + i) * g.N + col0 + 32 * j + l] = top;
    };
    if (__any(finite != 0.f)) {                            // 0 x (inf or NaN) is NaN: one tile after the other on the fp32 instruction
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
            unsigned row_top[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) row_top[v] = 0;
#pragma unroll 1
            for (int j = 0; j < NJ; ++j) {
                const float *x = g.A + (size_t)min(row0 + 32 * i + l, g.M - 1) * g.K;
                const int n = col0 + 32 * j + l;
                const float *w = g.B.p + (long)min(n, g.N - 1) * g.B.sn, bias = bias_of(j);
                floatx16 f;
#pragma unroll
                for (int v = 0; v < 16; ++v) f[v] = 0.f;
#pragma unroll 1
                for (int k = 0; k < g.K; k += 2)           // K is even
                    f = __builtin_amdgcn_mfma_f32_32x32x2f32(x[k + half], n < g.N && k + half < g.KB ? w[(k + half) * g.B.sk] : 0.f, f, 0, 0, 0);
                unsigned col_top = 0;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    float y, slope = 0.f;
                    const float z = f[v] + bias;
                    activate<ACT, OUT == kBackward>(z, y, slope);
                    if (!there(i, j, v)) continue;
                    const size_t to = at(i, j, v) + own;
                    if constexpr (OUT == kBackward) {
                        const float d = g.linear.dY[to] * slope;
                        g.linear.D[to] = d;
                        row_top[v] = max(row_top[v], __float_as_uint(d) & 0x7fffffffu);
                        col_top = max(col_top, __float_as_uint(d) & 0x7fffffffu);
                    } else {
                        if (OUT == kForward && g.linear.Z) g.linear.Z[to] = z;
                        g.linear.Y[to] = OUT == kForward && g.linear.R ? y + g.linear.R[to] : y;
                    }
                }
                if constexpr (OUT == kBackward) put_cols(col_top, i, j);
            }
            if constexpr (OUT == kBackward) put_rows(row_top, i);
        }
    } else {
        int eb[NJ];
        float bias[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            eb[j] = g.exps[col0 + 32 * j + l];
            bias[j] = bias_of(j);
        }
        auto value = [&](int i, int j, int v) __attribute__((always_inline)) {
            return ldexpf(acc[i][j][v], -(s_exp[64 * wm + 32 * i + 8 * (v / 4) + 4 * half + v % 4] + eb[j]));
        };
        // one output, `other` its element of R or dY
        auto put = [&](int i, int j, int v, float other, unsigned &row_top, unsigned &col_top) __attribute__((always_inline)) {
            const float z = value(i, j, v) + bias[j];
            float y, slope = 0.f;
            activate<ACT, OUT == kBackward>(z, y, slope);
            if constexpr (OUT == kBackward) {
                const float d = other * slope;
                (g.linear.D + at(i, j, v))[own] = d;
                row_top = max(row_top, __float_as_uint(d) & 0x7fffffffu);
                col_top = max(col_top, __float_as_uint(d) & 0x7fffffffu);
            } else {
                if (OUT == kForward && g.linear.Z) (g.linear.Z + at(i, j, v))[own] = z;
                (g.linear.Y + at(i, j, v))[own] = OUT == kForward ? y + other : y;
            }
        };
        const float *from = OUT == kForward ? g.linear.R : g.linear.dY;
        // Two tiles at a time, what they need of R or dY under way at once.  Where columns end inside, lanes are off for a tile; where rows
        // do, element by element.
        auto finish = [&](auto rows, auto columns) __attribute__((always_inline)) {
            constexpr bool ROWS = decltype(rows)::value, COLUMNS = decltype(columns)::value;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                unsigned row_top[16];
#pragma unroll
                for (int v = 0; v < 16; ++v) row_top[v] = 0;
#pragma unroll
                for (int j0 = 0; j0 < NJ; j0 += 2) {
                    unsigned col_top[2] = {0, 0};
                    float r[2][16];
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int v = 0; v < 16; ++v) r[q][v] = 0.f;
                    if constexpr (ROWS && COLUMNS) {
                        if (OUT != kPlain && from)
#pragma unroll
                            for (int v = 0; v < 16; ++v)
#pragma unroll
                                for (int q = 0; q < 2; ++q) r[q][v] = (from + at(i, j0 + q, v))[own];
#pragma unroll
                        for (int v = 0; v < 16; ++v)
#pragma unroll
                            for (int q = 0; q < 2; ++q) put(i, j0 + q, v, r[q][v], row_top[v], col_top[q]);
                    } else {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            if (col0 + 32 * (j0 + q) + l >= g.N) continue;
                            if constexpr (ROWS) {
                                if (OUT != kPlain && from)
#pragma unroll
                                    for (int v = 0; v < 16; ++v) r[q][v] = (from + at(i, j0 + q, v))[own];
#pragma unroll
                                for (int v = 0; v < 16; ++v) put(i, j0 + q, v, r[q][v], row_top[v], col_top[q]);
                            } else {
#pragma unroll
                                for (int v = 0; v < 16; ++v)
                                    if (there(i, j0 + q, v))
                                        put(i, j0 + q, v, OUT != kPlain && from ? (from + at(i, j0 + q, v))[own] : 0.f, row_top[v], col_top[q]);
                            }
                        }
                    }
                    if constexpr (OUT == kBackward)
#pragma unroll
                        for (int q = 0; q < 2; ++q) put_cols(col_top[q], i, j0 + q);
                }
                if constexpr (OUT == kBackward) put_rows(row_top, i);
            }
        };
        if (row0 + 64 > g.M) finish(std::false_type(), std::false_type());
        else if (col0 + 32 * NJ > g.N) finish(std::true_type(), std::false_type());
        else finish(std::true_type(), std::true_type());
    }
    if constexpr (OUT == kBackward) {
        if (top_rows(g.M) == 32) return;
        __syncthreads();
        const int n = ct0 * 32 + t;
        if (t < 64 * NJ && n < g.N) g.tops.cols[(size_t)(m0 / 128) * g.N + n] = s_top[t];
    }
}

// 32-column tiles of a wavefront; the epilogue of a backward pass has registers for two.  Blocks that begin together also end together, and
// a short reduction leaves much of the time to memory at the end: more and smaller blocks fall out of step (2^17 x 128 -> 256 with ELU 71 ->
// 61 us, 30000 x 301 -> 1000 with SiLU, residual and Z 164 -> 146).
int pair_tiles(int64_t M, int64_t N, int64_t K) {
    const bool many = K > 512 || ceil_div(M, 128) * ceil_div(N, 256) >= 2048;
    return many && (N % 256 == 0 || N % 256 > 128) ? 4 : 2;
}
size_t parts_bytes(int64_t N, int64_t K) { return align_up((size_t)ceil_div(N, 256) * 8 * ceil_div(K, KP) * kPairBytes); }

gnn_status_t set_pair(PairProduct &g, int nj, int64_t M, int64_t N, int64_t K, int64_t KB, const float *A, const unsigned *row_tops, int parts, const HalfOperand &B,
                      void *workspace, hipStream_t st) {
    g.M = (int)M; g.N = (int)N; g.K = (int)K; g.KB = (int)KB; g.steps = (int)ceil_div(K, KP);
    g.A = A; g.row_tops = row_tops; g.top_parts = parts;
    g.B = B;
    char *at = static_cast<char *>(workspace);
    int *exps = reinterpret_cast<int *>(at + parts_bytes(N, K));
    g.parts = at; g.exps = exps;
    g.tiles_m = (int)ceil_div(M, 128); g.tiles_n = (int)ceil_div(N, 64 * nj);
    const dim3 grid((unsigned)(g.tiles_n * 2 * nj), (unsigned)ceil_div(g.steps, kPartSteps));
    hipLaunchKernelGGL(B.sk == 1 ? pair_weights_kernel<true> : pair_weights_kernel<false>, grid, dim3(1024), 0, st, g.N, g.KB, g.steps, B, at, exps);
    return launch_status();
}

dim3 pair_grid(const PairProduct &g) { return dim3((unsigned)(8 * ceil_div((int64_t)g.tiles_m * g.tiles_n, 8))); }

}  // namespace

// Blocks enough for the chip, whole lines of aligned rows, and reductions that parts are exact enough for.
bool pair_product_fits(int64_t M, int64_t N, int64_t K, const float *A) {
    if (K < kShortReduction || K % 4 != 0 || K >= 1 << 22 || !aligned16(A) || N <= 64 || N > 1 << 22 || M > INT32_MAX - 256) return false;
    const int64_t blocks = ceil_div(M, 128) * ceil_div(N, 64 * pair_tiles(M, N, K));
    return blocks >= 256 && blocks < ((int64_t)1 << 24) - 8;
}

size_t pair_workspace_bytes(int64_t N, int64_t K) { return parts_bytes(N, K) + align_up((size_t)ceil_div(N, 256) * 256 * sizeof(int)); }

int pair_row_parts(int64_t N) { return 2 * (int)ceil_div(N, 128); }

gnn_status_t pair_plain_launch(int64_t M, int64_t N, int64_t K, int64_t KB, const float *A, const unsigned *row_tops, int parts, const float *B, float *C,
                               void *workspace, hipStream_t st) {
    PairProduct g{};
    GNN_TRY(set_pair(g, pair_tiles(M, N, K), M, N, K, KB, A, row_tops, parts, HalfOperand{B, 1, (long)KB}, workspace, st));
    g.linear.Y = C;
    auto kernel = pair_tiles(M, N, K) == 4 ? pair_product_kernel<4, kPlain, GNN_ACT_NONE> : pair_product_kernel<2, kPlain, GNN_ACT_NONE>;
    hipLaunchKernelGGL(kernel, pair_grid(g), dim3(256), 0, st, g);
    return launch_status();
}

gnn_status_t pair_linear_launch(int act, int64_t M, int64_t N, int64_t K, int64_t KB, const float *X, const unsigned *row_tops, int parts, const float *W,
                                const float *bias, const Linear &out, const Tops &tops, void *workspace, hipStream_t st) {
    PairProduct g{};
    const bool back = out.D != nullptr, four = !back && pair_tiles(M, N, K) == 4;
    GNN_TRY(set_pair(g, four ? 4 : 2, M, N, K, KB, X, row_tops, parts, HalfOperand{W, (long)N, 1}, workspace, st));
    g.bias = bias;
    g.linear = out;
    g.tops = tops;
#define PAIR_CASE(ACT_)                                                                                                                  \
    if (act == ACT_) {                                                                                                                   \
        void (*kernel)(PairProduct) = pair_product_kernel<2, kBackward, ACT_>;                                                           \
        if (!back) kernel = four ? pair_product_kernel<4, kForward, ACT_> : pair_product_kernel<2, kForward, ACT_>;                      \
        hipLaunchKernelGGL(kernel, pair_grid(g), dim3(256), 0, st, g);                                                                   \
    }
    PAIR_CASE(GNN_ACT_NONE) PAIR_CASE(GNN_ACT_RELU) PAIR_CASE(GNN_ACT_ELU)
    PAIR_CASE(GNN_ACT_SIGMOID) PAIR_CASE(GNN_ACT_SILU) PAIR_CASE(GNN_ACT_GELU)
#undef PAIR_CASE
    return launch_status();
}

}  // namespace gnn
