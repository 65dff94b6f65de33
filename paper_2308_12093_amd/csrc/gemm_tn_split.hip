// C = A^T B, A [K][M], B [K][N] with K = all nodes, in float on the bf16 matrix instruction: the same six products of three
// parts of each operand as in gemm_split.hip (a third of the instruction time of the fp32 instruction, a quarter of that of the
// fp64 instruction that gemm.hip uses for X^T H).  A chunk of at most kMostRows indices is summed in float, every 32 of them
// with three roundings, and the chunks are added in double in their order.
// Operands whose parts are not finite (infinities, NaN, and what rounds to infinity) are taken again with the fp32 instruction,
// chunk by chunk and wavefront by wavefront; magnitudes below 2^-110 are held to 2^-134, the least that the parts resolve.
#include "split_parts.h"

namespace gnn {
namespace {

constexpr int KB = 32;                 // indices of a step: two instructions of 16, lane half h of each 8 h .. 8 h + 7
constexpr int64_t kMostRows = 4096;

struct TnProduct {
    int M, N;
    long K, chunk;
    const float *A, *B;
    int tiles_m, tiles_n, splits;
    float *part;                       // [split][M][N]
    float *sums;                       // [split][N]: column sums of B, or NULL
};

// A block of four wavefronts owns 64 TM x 64 TN outputs, a wavefront 32 TM x 32 TN, over one chunk.  Per step the block reads
// 32 rows of its columns (a lane eight rows of one column: rows of 128 bytes side by side), splits them in registers and shares
// the parts through LDS in the order of the instruction's lanes, 6 KB per 32 columns; the next step's rows are under way
// meanwhile.  One buffer and two barriers a step, three blocks a CU: one splits while another multiplies.
template <int TM, int TN>
__global__ void __launch_bounds__(256, 2)
gemm_tn_split_kernel(TnProduct g) {
    constexpr int TILES = 2 * (TM + TN), FRAGS = 2 * TILES / 4;     // 32-column tiles of the block; fragments of a wavefront
    __shared__ __align__(16) char lds[TILES * 6 * kFragBytes];
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t / 64), lane = t % 64, l = lane % 32, half = lane / 32;
    // each XCD takes a contiguous range of (chunk, tile), tiles of a chunk side by side: they read the same rows
    const long total = (long)g.tiles_m * g.tiles_n * g.splits, per = (total + 7) / 8;
    const long id = (long)(blockIdx.x % 8) * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || id >= total) return;
    const int split = (int)(id / (g.tiles_m * g.tiles_n)), tile = (int)(id % (g.tiles_m * g.tiles_n));
    const int bm = tile / g.tiles_n, bn = tile % g.tiles_n;
    const long k0 = split * g.chunk, k1 = min(g.K, k0 + g.chunk);

    // fragment i of the wavefront: number wave + 4 i, instruction (wave & 1) of 32-column tile wave / 2 + 2 i; tiles of A first
    const float *from[FRAGS];
    long ld[FRAGS];
#pragma unroll
    for (int i = 0; i < FRAGS; ++i) {
        const int tl = wave / 2 + 2 * i;
        const bool a = i < TM;                             // 2 TM tiles of A
        const int col = a ? (bm * 2 * TM + tl) * 32 + l : (bn * 2 * TN + tl - 2 * TM) * 32 + l;
        ld[i] = a ? g.M : g.N;
        // columns past the end re-read the last: their results are not stored
        from[i] = (a ? g.A : g.B) + min(col, (a ? g.M : g.N) - 1) + (k0 + 16 * (wave & 1) + 8 * half) * ld[i];
    }
    float raw[FRAGS][8], sum[TN];
#pragma unroll
    for (int i = 0; i < TN; ++i) sum[i] = 0.f;
    const bool sums = g.sums && bm == 0;                   // uniform
    auto load = [&](long k) __attribute__((always_inline)) {
        if (k + KB <= k1) {
#pragma unroll
            for (int i = 0; i < FRAGS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) raw[i][j] = from[i][j * ld[i]];
        } else {
            const long left = k1 - k - 16 * (wave & 1) - 8 * half;      // of this lane's eight, if less
#pragma unroll
            for (int i = 0; i < FRAGS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) raw[i][j] = j < left ? from[i][j * ld[i]] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < FRAGS; ++i) from[i] += KB * ld[i];
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
    load(k0);
    for (long k = k0; k < k1; k += KB) {
#pragma unroll
        for (int i = 0; i < FRAGS; ++i) {
            bf16x8 part[3];
            unsigned least;
            split8<false>(floatx4{raw[i][0], raw[i][1], raw[i][2], raw[i][3]}, floatx4{raw[i][4], raw[i][5], raw[i][6], raw[i][7]},
                          part, least);
            const int f = 2 * (wave / 2 + 2 * i) + (wave & 1);
#pragma unroll
            for (int p = 0; p < 3; ++p)
                *reinterpret_cast<bf16x8 *>(lds + (f * 3 + p) * kFragBytes + lane * 16) = part[p];
            if (i >= TM && sums)
                sum[i - TM] += ((raw[i][0] + raw[i][1]) + (raw[i][2] + raw[i][3])) + ((raw[i][4] + raw[i][5]) + (raw[i][6] + raw[i][7]));
        }
        __syncthreads();
        if (k + KB < k1) load(k + KB);
        bf16x8 a[TM][2][3];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int q = 0; q < 6; ++q)
                a[i][q / 3][q % 3] = *reinterpret_cast<const bf16x8 *>(lds + ((wm * TM + i) * 6 + q) * kFragBytes + lane * 16);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            bf16x8 b[2][3];
#pragma unroll
            for (int q = 0; q < 6; ++q)
                b[q / 3][q % 3] = *reinterpret_cast<const bf16x8 *>(lds + ((2 * TM + wn * TN + j) * 6 + q) * kFragBytes + lane * 16);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                floatx16 small;
#pragma unroll
                for (int v = 0; v < 16; ++v) small[v] = 0.f;
#pragma unroll
                for (int q = 0; q < kProducts - 1; ++q)
#pragma unroll
                    for (int ins = 0; ins < 2; ++ins)
                        small = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i][ins][kPartA[q]], b[ins][kPartB[q]], small, 0, 0, 0);
#pragma unroll
                for (int ins = 0; ins < 2; ++ins)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i][ins][0], b[ins][0], acc[i][j], 0, 0, 0);
                acc[i][j] += small;
            }
        }
        __syncthreads();
    }
    float finite = 0.f;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) finite = fmaf(acc[i][j][v], 0.f, finite);
    const int m0 = (bm * 2 + wm) * TM * 32, n0 = (bn * 2 + wn) * TN * 32;
    if (__any(finite != 0.f)) {                            // 0 x (inf or NaN) is NaN
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
    // accumulator register v of lane (half, l): row 8 (v / 4) + 4 half + v % 4, column l of its 32 x 32 tile
    float *part = g.part + (size_t)split * g.M * g.N;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int m = m0 + 32 * i + 8 * (v / 4) + 4 * half + v % 4;
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int n = n0 + 32 * j + l;
                if (m < g.M && n < g.N) part[(size_t)m * g.N + n] = acc[i][j][v];
            }
        }
    if (sums) {                                            // two instructions and two lane halves of a column
        float *s = reinterpret_cast<float *>(lds);
#pragma unroll
        for (int i = 0; i < TN; ++i) s[((wave / 2 + 2 * i) * 2 + (wave & 1)) * 64 + lane] = sum[i];
        __syncthreads();
        const int n = bn * 2 * TN * 32 + t, at = t / 32 * 128 + t % 32;
        if (t < 64 * TN && n < g.N) g.sums[(size_t)split * g.N + n] = (s[at] + s[at + 32]) + (s[at + 64] + s[at + 96]);
    }
}

// out[i] = sum over the chunks, in double and in a fixed order; the outputs of C, then the column sums.  32 outputs a block, eight
// lanes each.
__global__ void __launch_bounds__(256)
tn_reduce_kernel(long count, int splits, const float *__restrict__ part, float *__restrict__ C, long count2,
                 const float *__restrict__ part2, float *__restrict__ sums) {
    __shared__ double red[8][33];
    const int o = threadIdx.x % 32, sl = threadIdx.x / 32;
    const long blocks = (count + 31) / 32;
    const bool second = blockIdx.x >= blocks;
    const long i = (second ? blockIdx.x - blocks : blockIdx.x) * 32L + o, n = second ? count2 : count;
    const float *p = second ? part2 : part;
    double a0 = 0.0, a1 = 0.0;
    if (i < n) {
        int s = sl;
        for (; s + 8 < splits; s += 16) {
            a0 += p[s * n + i];
            a1 += p[(s + 8) * n + i];
        }
        if (s < splits) a0 += p[s * n + i];
    }
    red[sl][o] = a0 + a1;
    __syncthreads();
    if (sl == 0 && i < n) {
        double t = 0.0;
        for (int k = 0; k < 8; ++k) t += red[k][o];
        (second ? sums : C)[i] = (float)t;
    }
}

int tile_of(int64_t extent) { return extent <= 64 ? 1 : 2; }

// Chunks: enough blocks for the chip, at least four steps each, at most kMostRows indices.
int64_t tn_chunks(int64_t M, int64_t N, int64_t K) {
    const int64_t tiles = ceil_div(M, 64 * tile_of(M)) * ceil_div(N, 64 * tile_of(N));
    int64_t chunks = ceil_div(768, tiles);
    const int64_t most = ceil_div(K, 4 * KB), least = ceil_div(K, kMostRows);
    if (chunks > most) chunks = most;
    if (chunks < least) chunks = least;
    return chunks < 1 ? 1 : chunks;
}

}  // namespace

bool gemm_tn_split_fits(int64_t M, int64_t N, int64_t K) {
    if (M > INT32_MAX / 4 || N > INT32_MAX / 4) return false;
    const int64_t blocks = ceil_div(M, 64) * ceil_div(N, 64);
    return blocks < 1 << 24 && blocks * tn_chunks(M, N, K) < (int64_t)1 << 24 && ceil_div(M * N, 32) < (int64_t)1 << 24;
}

// no less for a larger K
size_t gemm_tn_split_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    const int64_t chunks = tn_chunks(M, N, K);
    return align_up((size_t)chunks * M * N * sizeof(float)) + align_up((size_t)chunks * N * sizeof(float));
}

// C [M][N] = A^T B, sums [N] = the column sums of B unless it is NULL; K >= 1 and gemm_tn_split_fits
gnn_status_t gemm_tn_split_launch(int64_t M, int64_t N, int64_t K, const float *A, const float *B, float *C, float *sums,
                                  void *workspace, hipStream_t st) {
    TnProduct g{};
    const int tm = tile_of(M), tn = tile_of(N);
    int64_t splits = tn_chunks(M, N, K);
    g.M = (int)M; g.N = (int)N; g.K = K;
    g.chunk = ceil_div(ceil_div(K, splits), KB) * KB;
    splits = ceil_div(K, g.chunk);
    g.A = A; g.B = B;
    g.tiles_m = (int)ceil_div(M, 64 * tm); g.tiles_n = (int)ceil_div(N, 64 * tn); g.splits = (int)splits;
    g.part = static_cast<float *>(workspace);
    float *part2 = reinterpret_cast<float *>(static_cast<char *>(workspace) + align_up((size_t)tn_chunks(M, N, K) * M * N * sizeof(float)));
    g.sums = sums ? part2 : nullptr;
    const dim3 grid((unsigned)(8 * ceil_div((int64_t)g.tiles_m * g.tiles_n * splits, 8)));
    auto kernel = tm == 1 ? (tn == 1 ? gemm_tn_split_kernel<1, 1> : gemm_tn_split_kernel<1, 2>)
                          : (tn == 1 ? gemm_tn_split_kernel<2, 1> : gemm_tn_split_kernel<2, 2>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, g);
    GNN_TRY(launch_status());
    const long count = (long)M * N, count2 = sums ? N : 0;
    hipLaunchKernelGGL(tn_reduce_kernel, dim3((unsigned)(ceil_div(count, 32) + ceil_div(count2, 32))), dim3(256), 0, st, count,
                       (int)splits, g.part, C, count2, part2, sums);
    return launch_status();
}

}  // namespace gnn
