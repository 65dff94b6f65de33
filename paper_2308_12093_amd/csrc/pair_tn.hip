// C = A^T B over all nodes on the fp16 matrix instruction (half_pair.h), A [K][M] in floats or in 8 bits, B [K][N] in floats.
#include "half_pair.h"
#include "linear.h"

namespace gnn {
namespace {

using namespace half_pair;

constexpr int64_t kChunkStep = 128;
// Rows of a chunk.  Its sums are in float, rounded up to six times per 32 rows; the chunks are added in double.
constexpr int64_t kMostRows = 4096;

struct PairTn {
    int M, N;
    long K, chunk;                     // chunk: a multiple of kChunkStep
    const float *A, *B;
    Rows8 held;                        // A where that is NULL: column m of row k is q[k][m] scale[k]
    const unsigned *a_tops, *b_tops;   // a_tops: not with `held`; b_tops: of B's rows times their scale then
    int tiles_m, tiles_n, splits;
    float *part;                       // [split][M][N]
    float *sums;                       // [split][N]: column sums of B, or NULL
};

// A block of four wavefronts owns 128 columns of A and 64 NJ of B over one chunk, a wavefront 64 x 32 NJ outputs.  Per step of 16 indices
// the block reads 16 rows of its columns (a lane eight rows of one column: rows of 128 bytes side by side), splits them in registers and
// shares the pairs through LDS in the order of the instruction's lanes, double-buffered, one barrier a step; the floats of a step are
// loaded two steps ahead.  With NJ = 4 there are 24 matrix instructions a step to 12 reads and 6 writes of 1 KB and about a hundred vector instructions.
// 512 x 2048 over 65536 rows 463 us cool and 532 warm, 0.89 and 0.78 PFLOP/s on the instruction, which is busy for 45 % of the cycles at
// 1.87 GHz (gemm_half_tn.hip: 550 and 685).
//
// HELD: an integer of 8 bits is one fp16 number, exactly, so A has one part, and there are 16 matrix instructions a step.  The scale
// of its row, from LDS, goes to the row of B before that is split.  A thread takes 4 columns of 2 rows, 4 bytes each.  A byte b + 128 behind 0x64 is
// the fp16 number 1024 + 128 + b.  512 x 1024 over 65536 rows 215 to 256 us; by way of floats 376, 41 for these and 22 for their largest
// magnitudes.
template <bool HELD, int NJ>
__global__ void __launch_bounds__(256, 2)
pair_tn_kernel(PairTn g) {
    constexpr int PA = HELD ? 1 : 2, BF = NJ / 2, FRAGS = HELD ? BF : 1 + BF;      // parts of A; 32-column tiles that a wavefront splits
    constexpr int A_BYTES = 4 * PA * 1024, STAGE = A_BYTES + 2 * NJ * kPairBytes, COLS = 64 * NJ;
    __shared__ __align__(16) char even[STAGE];
    __shared__ __align__(16) char odd[STAGE];
    __shared__ int s_exp[128 + COLS];
    __shared__ __align__(16) float s_rows[HELD ? kMostRows : 4];   // the scales of the chunk's rows, zeros to the end of the last step
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t / 64), lane = t % 64, l = lane % 32, half = lane / 32;
    // tiles of a chunk side by side: they read the same rows
    const long total = (long)g.tiles_m * g.tiles_n * g.splits, id = xcd_tile(total);
    if (id >= total) return;
    const int split = (int)(id / (g.tiles_m * g.tiles_n)), tile = (int)(id % (g.tiles_m * g.tiles_n));
    const int bm = tile / g.tiles_n * 128, bn = tile % g.tiles_n * COLS;
    const long k0 = split * g.chunk, k1 = min(g.K, k0 + g.chunk);
    for (int i = t; i < 128 + COLS; i += 256) {                   // the chunk's largest magnitudes
        const bool a = i < 128;
        if (HELD && a) { s_exp[i] = 0; continue; }
        const long width = a ? g.M : g.N;
        const unsigned *tops = a ? g.a_tops + min(bm + i, g.M - 1) : g.b_tops + min(bn + i - 128, g.N - 1);
        unsigned top = 0;
        const int each = top_rows(g.K);
        for (long b = k0 / each; b * each < k1; ++b) top = max(top, tops[b * width]);
        s_exp[i] = exponent_of(top);
    }
    if constexpr (HELD)
        for (int i = t; i < (int)(k1 - k0 + KP - 1) / KP * KP; i += 256) s_rows[i] = k0 + i < k1 ? g.held.scale[k0 + i] : 0.f;
    // 32-column tiles that this wavefront splits: FRAGS - BF of A, then BF of B.  Columns past the end re-read the last: their
    // results are not stored.
    unsigned at[FRAGS];                                    // bytes to this lane's first float, from the step's first row
    float scale[FRAGS];
    __syncthreads();
#pragma unroll
    for (int f = 0; f < FRAGS; ++f) {
        const bool a = f < FRAGS - BF;
        const int c = (a ? wave : 4 + BF * wave + f - (FRAGS - BF)) * 32 + l;
        at[f] = a ? 4 * ((unsigned)(8 * half) * g.M + min(bm + c, g.M - 1)) : 4 * ((unsigned)(8 * half) * g.N + min(bn + c - 128, g.N - 1));
        scale[f] = power_of_two(s_exp[c]);
    }
    const int ld = (int)rows8_stride(g.M);
    unsigned byte = 0;                                     // to this thread's four integers, from the step's first row
    if constexpr (HELD) byte = 2u * (t / 32) * ld + min(bm + 4 * (t % 32), ld - 4);
    float sum[BF] = {};
    const bool sums = g.sums && bm == 0;                   // uniform
    const long whole = k0 + (k1 - k0) / KP * KP;           // end of the steps that are complete

    struct Raw {
        float x[FRAGS][8];
        unsigned q[HELD ? 2 : 1];
    };
    auto load = [&](long k, Raw &r) __attribute__((always_inline)) {
        k = min(k, whole - KP);                            // the last complete step again after it: no branch, no use
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) {
            const bool a = f < FRAGS - BF;
            const float *p = a ? g.A + k * g.M : g.B + k * g.N;
            const long width = a ? g.M : g.N;
            unsigned mine = at[f];
            asm("" : "+v"(mine));                          // known to be 32 bits here: a scalar base and this offset, no 64-bit sum
#pragma unroll
            for (int j = 0; j < 8; ++j) r.x[f][j] = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p + j * width) + mine);
        }
        if constexpr (HELD) {
            const char *q = reinterpret_cast<const char *>(g.held.q) + k * ld;
            unsigned mine = byte;
            asm("" : "+v"(mine));
#pragma unroll
            for (int j = 0; j < 2; ++j) r.q[j] = *reinterpret_cast<const unsigned *>(q + j * (long)ld + mine);
        }
    };
    // the step's last rows, where they are fewer than 16; zeros behind them
    auto load_some = [&](long k, Raw &r) __attribute__((always_inline)) {
        const int left = (int)(k1 - k);
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) {
            const bool a = f < FRAGS - BF;
            const float *p = a ? g.A + k * g.M : g.B + k * g.N;
            const long width = a ? g.M : g.N;
#pragma unroll
            for (int j = 0; j < 8; ++j) r.x[f][j] = 8 * half + j < left ? p[j * width + at[f] / 4] : 0.f;
        }
        if constexpr (HELD) {
            const char *q = reinterpret_cast<const char *>(g.held.q) + k * ld + byte;
#pragma unroll
            for (int j = 0; j < 2; ++j) r.q[j] = 2 * (t / 32) + j < left ? *reinterpret_cast<const unsigned *>(q + j * (long)ld) : 0u;
        }
    };
    // the pairs of the step that begins with row k
    auto put = [&](long k, const Raw &r, char *to, bool count) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) {
            const bool a = f < FRAGS - BF;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = r.x[f][j];
            if (!a) {
                const float s = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                sum[f - (FRAGS - BF)] += count ? s : 0.f;
                if constexpr (HELD) {
                    const float *s = s_rows + (count ? (int)(k - k0) : 0) + 8 * half;
                    const floatx4 u = *reinterpret_cast<const floatx4 *>(s), v = *reinterpret_cast<const floatx4 *>(s + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) { x[j] *= u[j]; x[4 + j] *= v[j]; }
                }
            }
            half8 part[2];
            pairs8(x, scale[f], part);
            char *own = to + (a ? wave * PA * 1024 : A_BYTES + (BF * wave + f - (FRAGS - BF)) * kPairBytes) + lane * 16;
#pragma unroll
            for (int p = 0; p < 2; ++p) *reinterpret_cast<half8 *>(own + p * 1024) = part[p];
        }
        if constexpr (HELD) {
            const unsigned u = r.q[0] ^ 0x80808080u, v = r.q[1] ^ 0x80808080u;
            const int cg = t % 32, rg = t / 32;
            const half2v less = {(_Float16)-1152.f, (_Float16)-1152.f};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                // bytes: integer c of the first row, 0, integer c of the second, 0
                const unsigned w = __builtin_amdgcn_perm(v, u, 0x0c000c00u | c | (4 + c) << 16) | 0x64006400u;
                const half2v pair = __builtin_bit_cast(half2v, w) + less;
                *reinterpret_cast<half2v *>(to + cg / 8 * 1024 + (rg / 4 * 32 + (4 * cg + c) % 32) * 16 + 4 * (rg % 4)) = pair;
            }
        }
    };
    floatx16 acc[2][NJ];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    const int wm = wave / 2, wn = wave % 2;                // the wavefront's outputs: rows 64 wm .., columns 32 NJ wn ..
    auto multiply = [&](const char *buf) __attribute__((always_inline)) {
        half8 a[2][PA];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int p = 0; p < PA; ++p) a[i][p] = *reinterpret_cast<const half8 *>(buf + ((2 * wm + i) * PA + p) * 1024 + lane * 16);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            half8 b[2];
#pragma unroll
            for (int p = 0; p < 2; ++p) b[p] = *reinterpret_cast<const half8 *>(buf + A_BYTES + (NJ * wn + j) * kPairBytes + p * 1024 + lane * 16);
            if constexpr (!HELD)
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][PA - 1], b[0], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][0], b[1], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][0], b[0], acc[i][j], 0, 0, 0);
        }
    };
    // the products of the step in `buf`, and the pairs of the next into `next`, whose floats are then loaded for the one after it
    auto turn = [&](long k, const char *buf, char *next, Raw &r, bool more) __attribute__((always_inline)) {
        __syncthreads();
        multiply(buf);
        put(k + KP, r, next, more);
        __builtin_amdgcn_sched_barrier(0);                 // not one step's loads beside another's
        load(k + 3 * KP, r);
    };
    if (whole > k0) {
        Raw first, second;                                 // of even and of odd steps
        load(k0, first);
        load(k0 + KP, second);
        put(k0, first, even, true);
        load(k0 + 2 * KP, first);
        for (long k = k0; k < whole; k += 2 * KP) {
            turn(k, even, odd, second, k + KP < whole);
            if (k + KP < whole) turn(k + KP, odd, even, first, k + 2 * KP < whole);
        }
    }
    if (whole < k1) {
        Raw r;
        load_some(whole, r);
        __syncthreads();
        put(whole, r, even, true);
        __syncthreads();
        multiply(even);
    }
    float finite = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) finite = fmaf(acc[i][j][v], 0.f, finite);
    const int m0 = bm + 64 * wm, n0 = bn + 32 * NJ * wn;
    float *part = g.part + (size_t)split * g.M * g.N;
    if (__any(finite != 0.f)) {                            // 0 x (inf or NaN) is NaN: one tile after the other on the fp32 instruction
#pragma unroll 1
        for (int i = 0; i < 2; ++i)
#pragma unroll 1
            for (int j = 0; j < NJ; ++j) {
                const int m = min(m0 + 32 * i + l, g.M - 1), n = min(n0 + 32 * j + l, g.N - 1);
                floatx16 f;
#pragma unroll
                for (int v = 0; v < 16; ++v) f[v] = 0.f;
#pragma unroll 1
                for (long k = k0; k < k1; k += 2) {
                    const bool in = k + half < k1;
                    const long row = in ? k + half : k1 - 1;
                    float x, y = g.B[row * g.N + n];
                    if constexpr (HELD) {
                        x = (float)g.held.q[row * ld + m];
                        y *= g.held.scale[row];
                    } else {
                        x = g.A[row * g.M + m];
                    }
                    f = __builtin_amdgcn_mfma_f32_32x32x2f32(in ? x : 0.f, in ? y : 0.f, f, 0, 0, 0);
                }
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int mm = m0 + 32 * i + 8 * (v / 4) + 4 * half + v % 4;
                    if (mm < g.M && n0 + 32 * j + l < g.N) part[(size_t)mm * g.N + n] = f[v];
                }
            }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int dm = 32 * i + 8 * (v / 4) + 4 * half + v % 4, ea = HELD ? 0 : s_exp[64 * wm + dm];
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const int dn = 32 * j + l, eb = s_exp[128 + 32 * NJ * wn + dn];
                    if (m0 + dm < g.M && n0 + dn < g.N) part[(size_t)(m0 + dm) * g.N + n0 + dn] = ldexpf(acc[i][j][v], -(ea + eb));
                }
            }
    }
    if (sums) {                                            // the two lane halves of a column
#pragma unroll
        for (int f = 0; f < BF; ++f) {
            const float s = sum[f] + __shfl_xor(sum[f], 32, 64);
            const int n = bn + (BF * wave + f) * 32 + l;
            if (half == 0 && n < g.N) g.sums[(size_t)split * g.N + n] = s;
        }
    }
}

// out[i] = sum over the chunks, in double and in a fixed order; the outputs of C, each row times its factor (or not), then the column sums.
// 32 VEC outputs a block, eight lanes each.
template <int VEC>
__global__ void __launch_bounds__(256)
pair_reduce_kernel(long count, int N, int splits, const float *__restrict__ part, const float *__restrict__ factor, float *__restrict__ C,
                   long count2, const float *__restrict__ part2, float *__restrict__ sums) {
    __shared__ double red[8][32][VEC];
    const int o = threadIdx.x % 32, sl = threadIdx.x / 32;
    const long blocks = (count + 32 * VEC - 1) / (32 * VEC);
    const bool second = blockIdx.x >= blocks;
    const long i = ((second ? blockIdx.x - blocks : blockIdx.x) * 32L + o) * VEC, n = second ? count2 : count;
    const float *p = second ? part2 : part;
    double a[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) a[v] = 0.0;
    if (i < n)
        for (int s = sl; s < splits; s += 8) {
            if constexpr (VEC == 4) {
                const floatx4 x = *reinterpret_cast<const floatx4 *>(p + s * n + i);
#pragma unroll
                for (int v = 0; v < 4; ++v) a[v] += x[v];
            } else {
                a[0] += p[s * n + i];
            }
        }
#pragma unroll
    for (int v = 0; v < VEC; ++v) red[sl][o][v] = a[v];
    __syncthreads();
    if (sl == 0 && i < n) {
        const double times = factor && !second ? (double)factor[i / N] : 1.0;      // VEC columns of one row
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            double t = 0.0;
            for (int k = 0; k < 8; ++k) t += red[k][o][v];
            (second ? sums : C)[i + v] = (float)(t * times);
        }
    }
}

int tile_n(int64_t N) { return N <= 128 ? 128 : 256; }

// Chunks: enough blocks for the chip, at least eight steps each, at most kMostRows indices.
int64_t pair_chunks(int64_t M, int64_t N, int64_t K) {
    const int64_t tiles = ceil_div(M, 128) * ceil_div(N, tile_n(N));
    int64_t chunks = ceil_div(512, tiles);
    const int64_t most = ceil_div(K, kChunkStep), least = ceil_div(K, kMostRows);
    if (chunks > most) chunks = most;
    if (chunks < least) chunks = least;
    return chunks < 1 ? 1 : chunks;
}

}  // namespace

// so many rows that the chip's 256 CUs have a tile and a kChunkStep each
int64_t pair_tn_least_rows(int64_t M, int64_t N) {
    const int64_t rows = (ceil_div(256, ceil_div(M, 128) * ceil_div(N, tile_n(N))) - 1) * kChunkStep + 1;
    return rows > kShortReduction ? rows : kShortReduction;
}

// Reductions that parts are exact enough for, tiles of which not too much is empty, and enough of them times chunks of some length for
// the chip.  Fewer than four are so many chunks that their sums count: 128 x 256 over 2^17 rows 52 + 22 us, 51 + 12 in tiles of 128 x 128
// (gemm_half_tn.hip); but with A in 8 bits that would need it in floats first, and their largest magnitudes.
bool pair_tn_fits(int64_t M, int64_t N, int64_t K, bool held) {
    if (M > INT32_MAX / 4 || N > INT32_MAX / 4 || M <= 64 || N <= (held ? 64 : 128)) return false;
    const int64_t tiles = ceil_div(M, 128) * ceil_div(N, tile_n(N)), most = (int64_t)1 << 24;
    if (!held && tiles < 4) return false;
    return K >= pair_tn_least_rows(M, N) && tiles * pair_chunks(M, N, K) < most - 8 && ceil_div(M * N, 32) + ceil_div(N, 32) < most;
}

// no less for a larger K
size_t pair_tn_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    const int64_t chunks = pair_chunks(M, N, K);
    return align_up((size_t)chunks * M * N * sizeof(float)) + align_up((size_t)chunks * N * sizeof(float));
}

gnn_status_t pair_tn_launch(int64_t M, int64_t N, int64_t K, const float *A, const Rows8 &held, const unsigned *a_tops, const float *B,
                            const unsigned *b_tops, float *C, float *sums, void *workspace, hipStream_t st) {
    PairTn g{};
    const int64_t chunks = pair_chunks(M, N, K);
    g.M = (int)M; g.N = (int)N; g.K = K;
    g.chunk = ceil_div(ceil_div(K, chunks), kChunkStep) * kChunkStep;
    g.splits = (int)ceil_div(K, g.chunk);
    g.A = A; g.held = held; g.B = B; g.a_tops = a_tops; g.b_tops = b_tops;
    g.tiles_m = (int)ceil_div(M, 128); g.tiles_n = (int)ceil_div(N, tile_n(N));
    Carver carve(workspace);
    g.part = carve.take<float>((size_t)chunks * M * N);
    float *part2 = carve.take<float>((size_t)chunks * N);
    g.sums = sums ? part2 : nullptr;
    const dim3 grid((unsigned)(8 * ceil_div((int64_t)g.tiles_m * g.tiles_n * g.splits, 8)));
    auto kernel = A ? pair_tn_kernel<false, 4> : tile_n(N) == 256 ? pair_tn_kernel<true, 4> : pair_tn_kernel<true, 2>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, g);
    GNN_TRY(launch_status());
    const long count = (long)M * N, count2 = sums ? N : 0;
    const int vec = N % 4 == 0 ? 4 : 1;                    // the chunks lie N and M N floats apart in an aligned workspace
    hipLaunchKernelGGL(vec == 4 ? pair_reduce_kernel<4> : pair_reduce_kernel<1>,
                       dim3((unsigned)(ceil_div(count, 32 * vec) + ceil_div(count2, 32 * vec))), dim3(256), 0, st, count, (int)N, g.splits, g.part,
                       A ? nullptr : held.columns, C, count2, part2, sums);
    return launch_status();
}

}  // namespace gnn
