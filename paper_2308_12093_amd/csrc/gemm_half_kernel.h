// The product of fp32 rows and weights on the fp16 matrix instruction (half_parts.h), and what becomes of it: the kernel, for the files that
// say what (gemm_half.hip, linear_half.hip).
#pragma once

#include <type_traits>

#include "activation.h"
#include "half_parts.h"

namespace gnn {
namespace half_parts {

// ---- rows times weights -----------------------------------------------------------------------------------
// What becomes of Z = X W + b where it is one array.
struct Linear {
    const float *R;                    // forward: Y = act(Z) + R, R or NULL; and Z itself unless NULL
    float *Y, *Z;
    const float *dY;                   // backward: D = dY .* act'(Z)
    float *D;
};

struct HalfProduct {
    int M, N, K, steps;
    const float *A;
    const unsigned *row_tops;          // [top_parts][M]
    int top_parts;
    HalfOperand B;
    const char *parts;                 // of B; neither they nor row_tops are read where the reduction is short
    const int *exps;
    float *C;
    int splits, split_steps;           // kPlain: the reduction's parts, C [split][M][N] then
    const float *bias;
    bool stream;                       // kPlain, kGateForward: outputs beyond the caches, non-temporal stores
    int tiles_m, tiles_n;
    Gated gated;
    Linear linear;
    Tops tops;                         // of D
};

// What becomes of a tile: C as it is, or [A | U] of a gated block (see Gated), the first half of whose tiles are columns of A
// and the other half the same columns of U, so that a lane has both of an element.
// kLinearForward, kLinearBackward: see Linear.
enum { kPlain, kGateForward, kGateBackward, kLinearForward, kLinearBackward };

// A block of four wavefronts owns 128 rows and 32 NT columns, a wavefront 32 rows of them.  Per step of 32 indices the block copies the
// parts of its columns to LDS and each wavefront its rows, without touching registers, a step ahead; one barrier a step.  A lane
// reads 16 consecutive floats of its row back and splits them.  A row's eight 16-byte pieces of a step lie in the order piece ^ (row / 2
// mod 8), so that the reads of sixteen rows fall on different banks; whole lines are copied.  Rows read by the lanes themselves,
// 16 bytes each, cost the L1 64 accesses an instruction instead of 8: 65536 x 512 x 2048 551 us, so 456, 300 TFLOP/s of the product and
// 0.90 PFLOP/s on the instruction (a library's bf16 product of these sizes: 0.82).  The clock falls to 1.66 GHz under it, where
// kernels bound by memory run at 2.3, and the instruction is busy for 52 % of the cycles.
// [A | U] of 65536 x 512 -> 1024, stored as well, 549 us; D of 2^17 x 128 -> 256 191 us, 0.47 GB in and out.
// Each buffer is an array of its own: the compiler then knows which copies a read has to wait for.
// GATE (gnn_gate_t, or gnn_act_t of kLinear..) is known to the compiler: with all three in it the epilogue of 32 elements a lane outgrew the instruction cache
// (2^17 x 128 -> 256 backward 213 us).
// ROWS: kCopied where K is a multiple of 4, below 2^24, and A 16-byte aligned; otherwise lanes read their rows themselves, kLoaded.
// kShort, not of kPlain, with K < kShortReduction: on the fp32 instruction, W's columns of the block through LDS.  A lane half takes
// 16 of the indices, 12 or 8.
enum { kLoaded, kCopied, kShort };

template <int NT, int OUT, int ROWS, int GATE>
__global__ void __launch_bounds__(256, OUT == kGateBackward || OUT == kLinearBackward ? 2 : 3)
gemm_half_kernel(HalfProduct g) {
    constexpr bool ALIGNED = ROWS == kCopied, GATED = OUT == kGateForward || OUT == kGateBackward;
    constexpr int STAGE = NT * kTileBytes;
    __shared__ __align__(16) char even[STAGE];
    __shared__ __align__(16) char odd[STAGE];
    __shared__ __align__(16) char rows[ALIGNED ? 4 * 4096 : 16];
    __shared__ int s_exp[4][32];
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t / 64), lane = t % 64, l = lane % 32, half = lane / 32;
    const long tiles = (long)g.tiles_m * g.tiles_n, id = xcd_tile(tiles * g.splits);
    if (id >= tiles * g.splits) return;
    const long tile = id % tiles;
    const int split = (int)(id / tiles), step0 = split * g.split_steps, step1 = min(g.steps, step0 + g.split_steps);
    const int ct0 = (int)(tile % g.tiles_n) * NT, row0 = ((int)(tile / g.tiles_n) * 4 + wave) * 32;
    auto column = [&](int c) __attribute__((always_inline)) {       // of this lane in tile c; N where there is none
        if constexpr (!GATED) return min((ct0 + c) * 32 + l, g.N);
        const int j = (ct0 / 2 + c % (NT / 2)) * 32 + l;
        return j < g.gated.half ? j + (c < NT / 2 ? 0 : g.gated.half) : g.N;
    };
    const size_t ro = (size_t)min(row0 + l, g.M - 1) * g.K;      // rows past the end re-read the last one

    // Four indices at a time, at any 4-byte aligned address; the ones that would run over the row's end are read from
    // its last four floats instead (K >= 4) and put in place by `settle`, so no load stands behind a branch.
    floatx4 raw[4];
    auto load = [&](int step) __attribute__((always_inline)) {
        const int k = min(step, step1 - 1) * KB + 16 * half;      // the last step again after the last: no branch, no use
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = *reinterpret_cast<const float4u *>(g.A + ro + min(k + 4 * i, g.K - 4));
    };
    auto settle_from = [&](int k0) __attribute__((always_inline)) {        // raw[i]: indices k0 + 4 i .. of this lane
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // floats past the end: 0 none .. 4 all; a shift by one, by two and by four places
            const int over = min(max(k0 + 4 * i + 4 - g.K, 0), 4);
            const bool one = over & 1, two = over & 2, all = over & 4;
            floatx4 v = raw[i];
            v = floatx4{one ? v.y : v.x, one ? v.z : v.y, one ? v.w : v.z, one ? 0.f : v.w};
            v = floatx4{two ? v.z : v.x, two ? v.w : v.y, two ? 0.f : v.z, two ? 0.f : v.w};
            raw[i] = floatx4{all ? 0.f : v.x, all ? 0.f : v.y, all ? 0.f : v.z, all ? 0.f : v.w};
        }
    };
    auto settle = [&](int step) __attribute__((always_inline)) {
        if ((step + 1) * KB > g.K) settle_from(step * KB + 16 * half);
    };
    // global -> LDS, 1 KB per wavefront and instruction, from a uniform base and a 32-bit offset
    auto copy = [](const void *base, unsigned offset, char *to) __attribute__((always_inline)) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)((const char *)base + offset),
                                         (__attribute__((address_space(3))) void *)to, 16, 0, 0);
    };
    // the 4 NT fragments of a step are dealt to the four wavefronts
    auto stage = [&](int step, char *buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int f = wave + 4 * i;
            copy(g.parts + ((size_t)(ct0 + f / 4) * g.steps + step) * kTileBytes + f % 4 * kFragBytes, lane * 16, buf + f * kFragBytes);
        }
    };
    // eight rows an instruction; pieces past the row's end re-read its last
    const int first = min(row0, g.M - 1);
    const float *base = g.A + (size_t)first * g.K;
    unsigned mine[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) mine[i] = (unsigned)min(8 * i + lane / 8, g.M - 1 - first) * (unsigned)g.K;
    auto stage_rows = [&](int step) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int piece = 4 * (lane % 8 ^ (4 * (i % 2) + lane / 16));
            copy(base + step * KB, 4 * (mine[i] + min(piece, g.K - 4 - step * KB)), rows + wave * 4096 + i * 1024);
        }
    };
    float scale = 1.f, scale2 = 1.f;
    if constexpr (ROWS != kShort) {
        stage(step0, even);
        if constexpr (ALIGNED) stage_rows(step0);
        else load(step0);
        unsigned top = 0;
        for (int p = 0; p < g.top_parts; ++p) top = max(top, g.row_tops[(size_t)p * g.M + min(row0 + l, g.M - 1)]);
        const int e = exponent_of(top);
        scale = power_of_two(e);
        scale2 = power_of_two(e + 11);
        if (half == 0) s_exp[wave][l] = e;
    }
    // what the epilogue of a backward pass reads, under way from the start: with short rows there is little else to wait beside
    float dh[OUT == kGateBackward ? NT / 2 : OUT == kLinearBackward ? 2 : 1][16];
    auto load_dy = [&](int c) __attribute__((always_inline)) {     // of tile c, two of which there is room for
#pragma unroll
        for (int v = 0; v < 16; ++v)
            dh[c % 2][v] = g.linear.dY[(size_t)min(row0 + 4 * half + 8 * (v / 4) + v % 4, g.M - 1) * g.N + min((ct0 + c) * 32 + l, g.N - 1)];
    };
    if constexpr (OUT == kLinearBackward) {
        load_dy(0);
        load_dy(1);
    }
    if constexpr (OUT == kGateBackward)
#pragma unroll
        for (int c = 0; c < NT / 2; ++c)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                dh[c][v] = g.gated.dH[(size_t)min(row0 + 4 * half + 8 * (v / 4) + v % 4, g.M - 1) * g.gated.half +
                                      min((ct0 / 2 + c) * 32 + l, g.gated.half - 1)];
    floatx16 acc[NT];
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[c][v] = 0.f;
    };
    clear();
    auto turn = [&](int step, const char *buf, char *next) __attribute__((always_inline)) {
        // this wavefront's copies of the step have arrived; after the barrier everyone's have, and the other buffer,
        // read in the step before, is free
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (step + 1 < step1) stage(step + 1, next);
        if constexpr (ALIGNED) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                raw[i] = *reinterpret_cast<const floatx4 *>(rows + wave * 4096 + l * 128 + ((4 * half + i) ^ (l / 2 % 8)) * 16);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // read before the next step's rows overwrite them
            if (step + 1 < step1) stage_rows(step + 1);
        }
        half8 a[2][2];
        settle(step);
#pragma unroll
        for (int ins = 0; ins < 2; ++ins) {
            const floatx4 u = raw[2 * ins], v = raw[2 * ins + 1];
            halves8({u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]}, scale, scale2, a[ins]);
        }
        if constexpr (!ALIGNED) load(step + 1);
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            half8 b[2][2];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                b[i / 2][i % 2] = *reinterpret_cast<const half8 *>(buf + (c * 4 + i) * kFragBytes + lane * 16);
            multiply(acc[c], a, b);
        }
    };
    bool again = ROWS == kShort;
    if constexpr (ROWS == kShort) {
        auto product = [&](auto each) __attribute__((always_inline)) {
            constexpr int P = decltype(each)::value;
            float *w = reinterpret_cast<float *>(even);            // [2 P indices][32 NT columns], zeros past the end
            for (int i = t; i < 2 * P * NT * 32; i += 256) {
                const int k = i / (NT * 32), c = i / 32 % NT, j = (GATED ? ct0 / 2 + c % (NT / 2) : ct0 + c) * 32 + i % 32;
                w[i] = k < g.K && j < (GATED ? g.gated.half : g.N) ? g.B.p[k * g.B.sk + j + (!GATED || c < NT / 2 ? 0 : g.gated.half)] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < P / 4; ++i) raw[i] = *reinterpret_cast<const float4u *>(g.A + ro + min(P * half + 4 * i, g.K - 4));
#pragma unroll
            for (int i = P / 4; i < 4; ++i) raw[i] = floatx4{0.f, 0.f, 0.f, 0.f};
            settle_from(P * half);
            __syncthreads();
#pragma unroll
            for (int j = 0; j < P; ++j)
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    acc[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(raw[j / 4][j % 4], w[((P * half + j) * NT + c) * 32 + l], acc[c], 0, 0, 0);
        };
        if (g.K > 24) product(std::integral_constant<int, 16>());
        else if (g.K > 16) product(std::integral_constant<int, 12>());
        else product(std::integral_constant<int, 8>());
    } else {
        for (int step = step0; step < step1; step += 2) {
            turn(step, even, odd);
            if (step + 1 < step1) turn(step + 1, odd, even);
        }
        float finite = 0.f;
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int v = 0; v < 16; ++v) finite = fmaf(acc[c][v], 0.f, finite);
        again = __any(finite != 0.f);                      // 0 x (inf or NaN) is NaN
        if (again) {
            clear();
            for (int step = step0; step < step1; ++step) {
                load(step);
                settle(step);
                const int k0 = step * KB + 16 * half;
#pragma unroll
                for (int j = 0; j < 16; ++j)
#pragma unroll
                    for (int c = 0; c < NT; ++c) {
                        const int n = column(c);
                        const float bv = k0 + j < g.K && n < g.N ? g.B.p[(k0 + j) * g.B.sk + n * g.B.sn] : 0.f;
                        acc[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(raw[j / 4][j % 4], bv, acc[c], 0, 0, 0);
                    }
            }
        }
    }
    int eb[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) eb[c] = again ? 0 : g.exps[(ct0 + c) * 32 + l];
    auto out = [&](float *at, float o) __attribute__((always_inline)) {
        if (g.stream) __builtin_nontemporal_store(o, at);
        else *at = o;
    };
    // accumulator register v of lane (half, l): row 8 (v / 4) + 4 half + v % 4, column l of its 32 x 32 tile
    auto value = [&](int c, int v) __attribute__((always_inline)) {
        const int ea = again ? 0 : s_exp[wave][8 * (v / 4) + 4 * half + v % 4];
        return ldexpf(acc[c][v], -(ea + eb[c]));
    };
    if constexpr (OUT == kPlain) {
        float *C = g.C + (size_t)split * g.M * g.N;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int row = row0 + 8 * (v / 4) + 4 * half + v % 4;
#pragma unroll
            for (int c = 0; c < NT; ++c) {                 // the columns of a row one after the other
                const int n = (ct0 + c) * 32 + l;
                if (row < g.M && n < g.N) out(C + (size_t)row * g.N + n, value(c, v));
            }
        }
    } else if constexpr (OUT == kLinearForward) {
        // Two tiles at a time, the part of R that they need under way at once.  Addresses are a scalar base and the lane's own 32-bit
        // offset.  Where columns end inside, lanes are off for a tile; where rows do, element by element.
        const size_t corner = (size_t)row0 * g.N + ct0 * 32;
        const unsigned mine = 4u * half * (unsigned)g.N + l;
        auto at = [&](int c, int v) __attribute__((always_inline)) { return corner + (size_t)(8 * (v / 4) + v % 4) * g.N + 32 * c; };
        auto put = [&](int c, int v, float bias, float r) __attribute__((always_inline)) {
            const float z = value(c, v) + bias;
            float y, slope;
            activate<GATE, false>(z, y, slope);
            if (g.linear.Z) (g.linear.Z + at(c, v))[mine] = z;
            (g.linear.Y + at(c, v))[mine] = y + r;
        };
        auto finish = [&](auto rows_inside, auto columns) __attribute__((always_inline)) {
            constexpr bool INSIDE = decltype(rows_inside)::value, COLUMNS = decltype(columns)::value;
#pragma unroll
            for (int c0 = 0; c0 < NT; c0 += 2) {
                float r[2][16], bias[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    bias[i] = g.bias ? g.bias[min((ct0 + c0 + i) * 32 + l, g.N - 1)] : 0.f;
#pragma unroll
                    for (int v = 0; v < 16; ++v) r[i][v] = 0.f;
                }
                if constexpr (INSIDE && COLUMNS) {
                    if (g.linear.R)
#pragma unroll
                        for (int v = 0; v < 16; ++v)
#pragma unroll
                            for (int i = 0; i < 2; ++i) r[i][v] = (g.linear.R + at(c0 + i, v))[mine];
#pragma unroll
                    for (int v = 0; v < 16; ++v)
#pragma unroll
                        for (int i = 0; i < 2; ++i) put(c0 + i, v, bias[i], r[i][v]);
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if ((ct0 + c0 + i) * 32 + l >= g.N) continue;
                        if constexpr (INSIDE) {
                            if (g.linear.R)
#pragma unroll
                                for (int v = 0; v < 16; ++v) r[i][v] = (g.linear.R + at(c0 + i, v))[mine];
#pragma unroll
                            for (int v = 0; v < 16; ++v) put(c0 + i, v, bias[i], r[i][v]);
                        } else {
#pragma unroll
                            for (int v = 0; v < 16; ++v)
                                if (row0 + 8 * (v / 4) + 4 * half + v % 4 < g.M)
                                    put(c0 + i, v, bias[i], g.linear.R ? (g.linear.R + at(c0 + i, v))[mine] : 0.f);
                        }
                    }
                }
            }
        };
        if (g.M - row0 < 32) finish(std::false_type(), std::false_type());
        else if (g.N - ct0 * 32 < 32 * NT) finish(std::true_type(), std::false_type());
        else finish(std::true_type(), std::true_type());
    } else {
        const int k = GATED ? g.gated.half : g.N, width = GATED ? 2 * k : k;   // of D
        unsigned col_top[NT], row_top[16];
#pragma unroll
        for (int c = 0; c < NT; ++c) col_top[c] = 0;
#pragma unroll
        for (int v = 0; v < 16; ++v) row_top[v] = 0;
        if constexpr (OUT == kLinearBackward) {
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                const int j = (ct0 + c) * 32 + l;
                const float bias = g.bias ? g.bias[min(j, k - 1)] : 0.f;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int row = row0 + 4 * half + 8 * (v / 4) + v % 4;
                    float act, slope;
                    activate<GATE, true>(value(c, v) + bias, act, slope);
                    const bool in = row < g.M && j < k;
                    const float d = in ? dh[c % 2][v] * slope : 0.f;
                    if (in) out(g.linear.D + (size_t)row * k + j, d);
                    row_top[v] = max(row_top[v], __float_as_uint(d) & 0x7fffffffu);
                    col_top[c] = max(col_top[c], __float_as_uint(d) & 0x7fffffffu);
                }
                if (c + 2 < NT) load_dy(c + 2);
            }
        } else
#pragma unroll
        for (int c = 0; c < NT / 2; ++c) {
            const int j = (ct0 / 2 + c) * 32 + l, jj = min(j, k - 1);
            const float ba = g.bias ? g.bias[jj] : 0.f, bu = g.bias ? g.bias[k + jj] : 0.f;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int row = row0 + 4 * half + 8 * (v / 4) + v % 4;
                const bool in = row < g.M && j < k;
                const float a = value(c, v) + ba, u = value(c + NT / 2, v) + bu;
                float act, slope = 0.f;
                gate_of<GATE, OUT == kGateBackward>(a, act, slope);
                if constexpr (OUT == kGateBackward) {
                    const float da = in ? dh[c][v] * u * slope : 0.f, du = in ? dh[c][v] * act : 0.f;
                    if (in) {
                        out(g.gated.D + (size_t)row * 2 * k + j, da);
                        out(g.gated.D + (size_t)row * 2 * k + k + j, du);
                    }
                    const unsigned ta = __float_as_uint(da) & 0x7fffffffu, tu = __float_as_uint(du) & 0x7fffffffu;
                    col_top[c] = max(col_top[c], ta);
                    col_top[c + NT / 2] = max(col_top[c + NT / 2], tu);
                    row_top[v] = max(row_top[v], max(ta, tu));
                } else if (in) {
                    out(g.gated.H + (size_t)row * k + j, act * u);
                    if (g.gated.Z) {
                        out(g.gated.Z + (size_t)row * 2 * k + j, a);
                        out(g.gated.Z + (size_t)row * 2 * k + k + j, u);
                    }
                }
            }
        }
        if constexpr (OUT == kGateBackward || OUT == kLinearBackward) {
            // over the 32 lanes of a row: each step a lane hands on half of its rows and keeps the other half; in the end lanes
            // 2 v and 2 v + 1 have row v
#pragma unroll
            for (int d = 16, rows = 8; rows >= 1; d >>= 1, rows >>= 1) {
                const bool upper = l & d;
#pragma unroll
                for (int v = 0; v < rows; ++v) {
                    const unsigned give = upper ? row_top[v] : row_top[v + rows], keep = upper ? row_top[v + rows] : row_top[v];
                    row_top[v] = max(keep, (unsigned)__shfl_xor((int)give, d, 64));
                }
            }
            row_top[0] = max(row_top[0], (unsigned)__shfl_xor((int)row_top[0], 1, 64));
            const int v = l / 2, row = row0 + 4 * half + 8 * (v / 4) + v % 4;
            if (l % 2 == 0 && row < g.M) g.tops.rows[(size_t)(ct0 / NT) * g.M + row] = row_top[0];
            unsigned *s = reinterpret_cast<unsigned *>(even);      // of the wavefronts, or of the block
            __syncthreads();
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                col_top[c] = max(col_top[c], (unsigned)__shfl_xor((int)col_top[c], 32, 64));
                if (half == 0) s[(wave * NT + c) * 32 + l] = col_top[c];
            }
            __syncthreads();
            const int each = top_rows(g.M) / 32;           // wavefronts to one
            for (int i = t; i < 4 / each * NT * 32; i += 256) {
                const int w = i / (NT * 32) * each, at = i % (NT * 32), c = at / 32;
                const int j = (GATED ? ct0 / 2 + c % (NT / 2) : ct0 + c) * 32 + at % 32;
                const long block = tile / g.tiles_n * (4 / each) + w / each;
                unsigned top = 0;
                for (int q = w; q < w + each; ++q) top = max(top, s[q * NT * 32 + at]);
                if (j < k && block * 32 * each < g.M) g.tops.cols[(size_t)block * width + (!GATED || c < NT / 2 ? 0 : k) + j] = top;
            }
        }
    }
}

// 32-column tiles of a block: four (a row is split once per block), or two where the columns are few or the blocks
inline int half_tiles(int64_t M, int64_t N) { return N <= 64 || ceil_div(M, 128) * ceil_div(N, 128) < 256 ? 2 : 4; }

inline size_t half_parts_bytes(int64_t N, int64_t K) { return align_up((size_t)ceil_div(N, 128) * 4 * ceil_div(K, KB) * kTileBytes); }
inline size_t half_exps_bytes(int64_t N) { return align_up((size_t)ceil_div(N, 128) * 128 * sizeof(int)); }

inline void set_product(HalfProduct &g, int64_t M, int64_t N, int64_t K, void *workspace) {
    const int w = half_tiles(M, N);
    g.M = (int)M; g.N = (int)N; g.K = (int)K;
    g.steps = (int)ceil_div(K, KB);
    g.tiles_m = (int)ceil_div(M, 128); g.tiles_n = (int)ceil_div(N, 32 * w);
    g.splits = 1;
    g.split_steps = g.steps;
    g.parts = static_cast<char *>(workspace);
    g.exps = reinterpret_cast<int *>(static_cast<char *>(workspace) + half_parts_bytes(N, K));
}

inline dim3 product_grid(const HalfProduct &g) { return dim3((unsigned)(8 * ceil_div((int64_t)g.tiles_m * g.tiles_n * g.splits, 8))); }

gnn_status_t split_weights(const HalfProduct &g, int tiles, int halves, hipStream_t st);

}  // namespace half_parts
}  // namespace gnn
