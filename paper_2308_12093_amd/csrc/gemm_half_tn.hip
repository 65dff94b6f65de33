// C = A^T B over all nodes, A [K][M], B [K][N], with fp32 operands and results, on the fp16 matrix instruction (half_parts.h).
#include "half_parts.h"

namespace gnn {
namespace {

using namespace half_parts;

constexpr int64_t kChunkStep = 128;
// Rows of a chunk.  Its sums are in float, rounded about twice per 32 rows, 256 times for 4096 of them, where a float chain
// is 4096 times; the chunks are added in double.  In doubles throughout, as the layers' products of this form: 512 x 2048 over 65536
// rows 2226 us where this takes 578.
constexpr int64_t kMostRows = 4096;

struct TnProduct {
    int M, N;
    long K, chunk;                     // chunk: a multiple of kChunkStep
    const float *A, *B;
    const unsigned *a_tops, *b_tops;
    int tiles_m, tiles_n, splits;
    float *part;                       // [split][M][N]
    float *sums;                       // [split][N]: column sums of B, or NULL
};

// A block of four wavefronts owns 64 TM x 64 TN outputs, a wavefront 32 TM x 32 TN, over one chunk.  Per step of 32 indices the block
// reads 32 rows of its columns (a lane eight rows of one column: rows of 128 bytes side by side), splits them in registers and
// shares the parts through LDS in the order of the instruction's lanes, 4 KB per 32 columns, double-buffered, one barrier a
// step: the products of a step stand between the parts of the next, whose floats were loaded two steps ahead.
template <int TM, int TN>
__global__ void __launch_bounds__(256, 2)
gemm_half_tn_kernel(TnProduct g) {
    constexpr int TILES = 2 * (TM + TN), FRAGS = TM + TN;  // 32-column tiles of the block; fragments of a wavefront
    __shared__ __align__(16) char even[TILES * kTileBytes];
    __shared__ __align__(16) char odd[TILES * kTileBytes];
    __shared__ int s_exp[TILES * 32];
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t / 64), lane = t % 64, l = lane % 32, half = lane / 32;
    // tiles of a chunk side by side: they read the same rows
    const long total = (long)g.tiles_m * g.tiles_n * g.splits, id = xcd_tile(total);
    if (id >= total) return;
    const int split = (int)(id / (g.tiles_m * g.tiles_n)), tile = (int)(id % (g.tiles_m * g.tiles_n));
    const int bm = tile / g.tiles_n, bn = tile % g.tiles_n;
    const long k0 = split * g.chunk, k1 = min(g.K, k0 + g.chunk);
    // columns past the end re-read the last: their results are not stored
    auto of_a = [&](int c) __attribute__((always_inline)) { return min(bm * 64 * TM + c, g.M - 1); };
    auto of_b = [&](int c) __attribute__((always_inline)) { return min(bn * 64 * TN + c, g.N - 1); };

    for (int i = t; i < TILES * 32; i += 256) {            // the chunk's largest magnitudes
        const bool a = i < 64 * TM;
        const unsigned *tops = a ? g.a_tops + of_a(i) : g.b_tops + of_b(i - 64 * TM);
        unsigned top = 0;
        const int each = top_rows(g.K);
        for (long b = k0 / each; b * each < k1; ++b) top = max(top, tops[b * (a ? g.M : g.N)]);
        s_exp[i] = exponent_of(top);
    }
    // fragment i of the wavefront: instruction (wave & 1) of 32-column tile wave / 2 + 2 i; tiles of A first
    unsigned at[FRAGS];                                    // bytes to this lane's first float, from the step's first row
    float scale[FRAGS], scale2[FRAGS];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FRAGS; ++i) {
        const int c = (wave / 2 + 2 * i) * 32 + l, down = 16 * (wave & 1) + 8 * half;
        at[i] = 4 * (i < TM ? (unsigned)down * g.M + of_a(c) : (unsigned)down * g.N + of_b(c - 64 * TM));
        scale[i] = power_of_two(s_exp[c]);
        scale2[i] = power_of_two(s_exp[c] + 11);
    }
    float sum[TN];
#pragma unroll
    for (int i = 0; i < TN; ++i) sum[i] = 0.f;
    const bool sums = g.sums && bm == 0;                   // uniform
    const long whole = k0 + (k1 - k0) / KB * KB;           // end of the steps that are complete
    auto load_one = [&](long k, int i, float (&x)[8]) __attribute__((always_inline)) {
        k = min(k, whole - KB);                            // the last complete step again after it: no branch, no use
        const float *p = i < TM ? g.A + k * g.M : g.B + k * g.N;
        const long ld = i < TM ? g.M : g.N;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p + j * ld) + at[i]);
    };
    auto load = [&](long k, float (&raw)[FRAGS][8]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < FRAGS; ++i) load_one(k, i, raw[i]);
    };
    floatx16 acc[TM][TN];
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    };
    clear();
    const int wm = wave / 2, wn = wave % 2;                // the wavefront's tiles: rows wm TM .., columns wn TN ..
    auto put = [&](const half8 (&part)[2], int i, char *to) __attribute__((always_inline)) {
        const int f = 2 * (wave / 2 + 2 * i) + (wave & 1);
#pragma unroll
        for (int p = 0; p < 2; ++p) *reinterpret_cast<half8 *>(to + (f * 2 + p) * kFragBytes + lane * 16) = part[p];
    };
    auto add_up = [&](const float (&x)[8], int i, bool count) __attribute__((always_inline)) {
        const float s = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        if (i >= TM) sum[i - TM] += count ? s : 0.f;
    };
    auto put_parts = [&](const float (&raw)[FRAGS][8], char *to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < FRAGS; ++i) {
            half8 part[2];
            halves8(raw[i], scale[i], scale2[i], part);
            put(part, i, to);
            add_up(raw[i], i, true);
        }
    };
    // The products of the step in `buf`, and between them the parts of the next (`raw`, into `next`), whose floats are then loaded
    // for the one after it.  A matrix instruction takes 32 cycles, in which its wavefront can issue eight others: they are
    // written, and kept (sched_barrier), in that order: left to itself the compiler issues all matrix instructions, then
    // all others (512 x 2048 over 65536 rows: 616 us; in this order 600, 229 TFLOP/s, 0.69 PFLOP/s on the instruction).
    auto turn = [&](long k, const char *buf, char *next, float (&raw)[FRAGS][8], bool more) __attribute__((always_inline)) {
        __syncthreads();
        half8 a[TM][2][2], b[TN][2][2];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                a[i][q / 2][q % 2] = *reinterpret_cast<const half8 *>(buf + ((wm * TM + i) * 4 + q) * kFragBytes + lane * 16);
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                b[j][q / 2][q % 2] = *reinterpret_cast<const half8 *>(buf + ((2 * TM + wn * TN + j) * 4 + q) * kFragBytes + lane * 16);
        floatx16 small[2];
#pragma unroll
        for (int n = 0; n < TM * TN; ++n) {                // tile n % TM, n / TM; part of the fragments n, n + TM TN, ..
            floatx16 &cross = small[n % 2], &last = small[1 - n % 2];
            const half8 (&x)[2][2] = a[n % TM], (&y)[2][2] = b[n / TM];
#pragma unroll
            for (int v = 0; v < 16; ++v) cross[v] = 0.f;
            half8 part[(FRAGS + TM * TN - 1) / (TM * TN)][2];
#pragma unroll
            for (int q = 0; q < 6; ++q) {
                if (q < 4) cross = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[q / 2][1 - q % 2], y[q / 2][q % 2], cross, 0, 0, 0);
                else acc[n % TM][n / TM] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[q - 4][0], y[q - 4][0], acc[n % TM][n / TM], 0, 0, 0);
#pragma unroll
                for (int i = n; i < FRAGS; i += TM * TN) {
                    if (q < 4) halves2(raw[i], 2 * q, scale[i], scale2[i], part[i / (TM * TN)]);
                    if (q == 3) put(part[i / (TM * TN)], i, next);
                    if (q == 4) add_up(raw[i], i, more);
                    if (q == 5) load_one(k + 3 * KB, i, raw[i]);
                }
                if (n > 0 && q >= 4)
#pragma unroll
                    for (int v = 8 * (q - 4); v < 8 * (q - 3); ++v)
                        acc[(n - 1) % TM][(n - 1) / TM][v] = fmaf(last[v], 0x1p-11f, acc[(n - 1) % TM][(n - 1) / TM][v]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int v = 0; v < 16; ++v)
            acc[TM - 1][TN - 1][v] = fmaf(small[(TM * TN - 1) % 2][v], 0x1p-11f, acc[TM - 1][TN - 1][v]);
    };
    if (whole > k0) {
        float ahead[2][FRAGS][8];                          // of even and of odd steps
        load(k0, ahead[0]);
        load(k0 + KB, ahead[1]);
        put_parts(ahead[0], even);
        load(k0 + 2 * KB, ahead[0]);
        for (long k = k0; k < whole; k += 2 * KB) {
            turn(k, even, odd, ahead[1], k + KB < whole);
            if (k + KB < whole) turn(k + KB, odd, even, ahead[0], k + 2 * KB < whole);
        }
    }
    if (whole < k1) {                                      // the last step, of fewer indices
        float raw[FRAGS][8];
        const int left = (int)(k1 - whole) - 16 * (wave & 1) - 8 * half;       // of this lane's eight, if less
#pragma unroll
        for (int i = 0; i < FRAGS; ++i) {
            const float *p = i < TM ? g.A + whole * g.M : g.B + whole * g.N;
#pragma unroll
            for (int j = 0; j < 8; ++j) raw[i][j] = j < left ? p[j * (long)(i < TM ? g.M : g.N) + at[i] / 4] : 0.f;
        }
        __syncthreads();
        put_parts(raw, even);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                half8 a[2][2], b[2][2];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    a[q / 2][q % 2] = *reinterpret_cast<const half8 *>(even + ((wm * TM + i) * 4 + q) * kFragBytes + lane * 16);
                    b[q / 2][q % 2] = *reinterpret_cast<const half8 *>(even + ((2 * TM + wn * TN + j) * 4 + q) * kFragBytes + lane * 16);
                }
                multiply(acc[i][j], a, b);
            }
    }
    float finite = 0.f;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) finite = fmaf(acc[i][j][v], 0.f, finite);
    const int m0 = (bm * 2 + wm) * TM * 32, n0 = (bn * 2 + wn) * TN * 32;
    const bool again = __any(finite != 0.f);               // 0 x (inf or NaN) is NaN
    if (again) {
        clear();
        for (long k = k0; k < k1; k += 2) {
            const bool in = k + half < k1;
            const long row = in ? k + half : k1 - 1;
            float x[TM], y[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) x[i] = in ? g.A[row * g.M + min(m0 + 32 * i + l, g.M - 1)] : 0.f;
#pragma unroll
            for (int j = 0; j < TN; ++j) y[j] = in ? g.B[row * g.N + min(n0 + 32 * j + l, g.N - 1)] : 0.f;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[j], acc[i][j], 0, 0, 0);
        }
    }
    float *part = g.part + (size_t)split * g.M * g.N;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int dm = 32 * i + 8 * (v / 4) + 4 * half + v % 4, m = m0 + dm;
            const int ea = again ? 0 : s_exp[wm * TM * 32 + dm];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int n = n0 + 32 * j + l, eb = again ? 0 : s_exp[64 * TM + (wn * TN + j) * 32 + l];
                if (m < g.M && n < g.N) part[(size_t)m * g.N + n] = ldexpf(acc[i][j][v], -(ea + eb));
            }
        }
    if (sums) {                                            // two instructions and two lane halves of a column
        float *s = reinterpret_cast<float *>(even);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TN; ++i) s[((wave / 2 + 2 * i) * 2 + (wave & 1)) * 64 + lane] = sum[i];
        __syncthreads();
        const int n = bn * 64 * TN + t, at = t / 32 * 128 + t % 32;
        if (t < 64 * TN && n < g.N) g.sums[(size_t)split * g.N + n] = (s[at] + s[at + 32]) + (s[at + 64] + s[at + 96]);
    }
}

// out[i] = sum over the chunks, in double and in a fixed order; the outputs of C, then the column sums.  32 VEC outputs a block,
// eight lanes each.
template <int VEC>
__global__ void __launch_bounds__(256)
tn_reduce_kernel(long count, int splits, const float *__restrict__ part, float *__restrict__ C, long count2,
                 const float *__restrict__ part2, float *__restrict__ sums) {
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
    if (sl == 0 && i < n)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            double t = 0.0;
            for (int k = 0; k < 8; ++k) t += red[k][o][v];
            (second ? sums : C)[i + v] = (float)t;
        }
}

// The same of fewer indices than kShortReduction, in float: a thread adds VEC columns of kShortRows rows of C.  B comes through the
// caches once per kShortRows rows, what bounds it is C.
constexpr int kShortRows = 4;

template <int VEC>
__global__ void __launch_bounds__(256)
tn_short_kernel(int M, int N, int K, int blocks_n, const float *__restrict__ A, const float *__restrict__ B, float *__restrict__ C,
                float *__restrict__ sums) {
    const int m0 = (int)(blockIdx.x / blocks_n) * kShortRows, n = ((int)(blockIdx.x % blocks_n) * 256 + threadIdx.x) * VEC;
    if (n >= N) return;
    float acc[kShortRows][VEC], sum[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        sum[v] = 0.f;
#pragma unroll
        for (int i = 0; i < kShortRows; ++i) acc[i][v] = 0.f;
    }
#pragma unroll 4
    for (int k = 0; k < K; ++k) {
        float b[VEC];
        if constexpr (VEC == 4) {
            const floatx4 x = *reinterpret_cast<const floatx4 *>(B + (size_t)k * N + n);
#pragma unroll
            for (int v = 0; v < 4; ++v) b[v] = x[v];
        } else {
            b[0] = B[(size_t)k * N + n];
        }
#pragma unroll
        for (int i = 0; i < kShortRows; ++i) {
            const float a = A[(size_t)k * M + min(m0 + i, M - 1)];
#pragma unroll
            for (int v = 0; v < VEC; ++v) acc[i][v] = fmaf(a, b[v], acc[i][v]);
        }
#pragma unroll
        for (int v = 0; v < VEC; ++v) sum[v] += b[v];
    }
#pragma unroll
    for (int i = 0; i < kShortRows; ++i) {
        if (m0 + i >= M) break;
        float *to = C + (size_t)(m0 + i) * N + n;
        if constexpr (VEC == 4) *reinterpret_cast<float4u *>(to) = float4u{acc[i][0], acc[i][1], acc[i][2], acc[i][3]};
        else *to = acc[i][0];
    }
    if (sums && m0 == 0)
#pragma unroll
        for (int v = 0; v < VEC; ++v) sums[n + v] = sum[v];
}

int tn_tile(int64_t extent) { return extent <= 64 ? 1 : 2; }

// Chunks: enough blocks for the chip, at least four steps each, at most kMostRows indices.
int64_t tn_chunks(int64_t M, int64_t N, int64_t K) {
    const int64_t tiles = ceil_div(M, 64 * tn_tile(M)) * ceil_div(N, 64 * tn_tile(N));
    int64_t chunks = ceil_div(512, tiles);
    const int64_t most = ceil_div(K, kChunkStep), least = ceil_div(K, kMostRows);
    if (chunks > most) chunks = most;
    if (chunks < least) chunks = least;
    return chunks < 1 ? 1 : chunks;
}

}  // namespace

// A grid has less than 2^32 threads: 2^24 blocks, of the product rounded up to a multiple of eight; of the last sums both those of
// C and those of the column sums.
bool gemm_half_tn_fits(int64_t M, int64_t N, int64_t K) {
    if (M > INT32_MAX / 4 || N > INT32_MAX / 4) return false;
    const int64_t blocks = ceil_div(M, 64) * ceil_div(N, 64), most = (int64_t)1 << 24;
    return blocks < most && blocks * tn_chunks(M, N, K) < most - 8 && ceil_div(M * N, 32) + ceil_div(N, 32) < most;
}

// no less for a larger K
size_t gemm_half_tn_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    const int64_t chunks = tn_chunks(M, N, K);
    return align_up((size_t)chunks * M * N * sizeof(float)) + align_up((size_t)chunks * N * sizeof(float));
}

gnn_status_t gemm_half_tn_launch(int64_t M, int64_t N, int64_t K, const float *A, const unsigned *a_tops, const float *B,
                                 const unsigned *b_tops, float *C, float *sums, void *workspace, hipStream_t st) {
    if (K < kShortReduction) {
        const int vec = N % 4 == 0 && aligned16(B) ? 4 : 1;
        const int64_t blocks_n = ceil_div(N, 256 * vec);
        hipLaunchKernelGGL(vec == 4 ? tn_short_kernel<4> : tn_short_kernel<1>, dim3((unsigned)(ceil_div(M, kShortRows) * blocks_n)),
                           dim3(256), 0, st, (int)M, (int)N, (int)K, (int)blocks_n, A, B, C, sums);
        return launch_status();
    }
    TnProduct g{};
    const int tm = tn_tile(M), tn = tn_tile(N);
    const int64_t chunks = tn_chunks(M, N, K);
    g.M = (int)M; g.N = (int)N; g.K = K;
    g.chunk = ceil_div(ceil_div(K, chunks), kChunkStep) * kChunkStep;
    g.splits = (int)ceil_div(K, g.chunk);
    g.A = A; g.B = B; g.a_tops = a_tops; g.b_tops = b_tops;
    g.tiles_m = (int)ceil_div(M, 64 * tm); g.tiles_n = (int)ceil_div(N, 64 * tn);
    Carver carve(workspace);
    g.part = carve.take<float>((size_t)chunks * M * N);
    float *part2 = carve.take<float>((size_t)chunks * N);
    g.sums = sums ? part2 : nullptr;
    const dim3 grid((unsigned)(8 * ceil_div((int64_t)g.tiles_m * g.tiles_n * g.splits, 8)));
    auto kernel = tm == 1 ? (tn == 1 ? gemm_half_tn_kernel<1, 1> : gemm_half_tn_kernel<1, 2>)
                          : (tn == 1 ? gemm_half_tn_kernel<2, 1> : gemm_half_tn_kernel<2, 2>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, g);
    GNN_TRY(launch_status());
    const long count = (long)M * N, count2 = sums ? N : 0;
    const int vec = N % 4 == 0 ? 4 : 1;                    // the chunks lie N and M N floats apart in an aligned workspace
    hipLaunchKernelGGL(vec == 4 ? tn_reduce_kernel<4> : tn_reduce_kernel<1>,
                       dim3((unsigned)(ceil_div(count, 32 * vec) + ceil_div(count2, 32 * vec))), dim3(256), 0, st, count, g.splits,
                       g.part, C, count2, part2, sums);
    return launch_status();
}

}  // namespace gnn
