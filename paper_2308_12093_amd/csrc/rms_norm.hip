// Root-mean-square norm, on its own or behind a residual connection, forward and backward, and arrays put into 8 bits a row at a time.
#include "dropout.h"
#include "rows.h"
#include "rows8.h"

namespace gnn {
namespace {

using namespace rows;

struct RmsNorm {
    int n, f, lanes;
    const float *X, *R;                // R: H = R + dropout(X); without: H = X
    const float *gamma;                // kRows: what the columns are multiplied with before they are put into 8 bits
    float eps;
    Dropout drop;
    float *H, *Y, *rstd;               // Y, rstd: or NULL
    Rows8 held;                        // xhat, or kRows: X; q NULL: not wanted
};

// kRows: no norm, the array itself goes into 8 bits
enum { kRows, kNorm, kAddNorm };

// the largest of each of U values over the lanes of a row, in all of them
template <int U, bool WIDE>
__device__ __forceinline__ void row_largest(unsigned (&v)[U], int lanes, float *red) {
    for (int d = (WIDE ? 64 : lanes) >> 1; d > 0; d >>= 1)
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = max(v[u], (unsigned)__shfl_xor((int)v[u], d, 64));
    if constexpr (WIDE) {
        const int wave = threadIdx.x / 64, first = threadIdx.x / lanes * (lanes / 64);
        __syncthreads();
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int u = 0; u < U; ++u) red[4 * u + wave] = __uint_as_float(v[u]);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u)
            for (int k = 0; k < lanes / 64; ++k) v[u] = max(v[u], __float_as_uint(red[4 * u + first + k]));
    }
}

// A row lies in the registers of its lanes as in layer norm (norm.hip); sum of squares and largest magnitude come from one read.  The
// integers that xhat is held in are those of H: both differ by 1 / rms, which only the scale takes up, so that they do not depend on the
// order of a sum.  Bound by memory: 2^20 x 256 with residual and integers 4.6 GB in 824 us, 5.5 TB/s; 2^18 x 512 with residual 2.1 GB in
// 375, 5.7; 2^18 x 512 into 8 bits 0.67 GB in 117, 5.7; 30011 x 203, rows at any alignment from the caches, 49 MB in 10 to 12.
template <int R, int U, int KIND, int MEM, bool WIDE>
__global__ void __launch_bounds__(256)
rms_forward_kernel(RmsNorm a) {
    __shared__ float red[4 * U];
    const DropoutWords words(a.drop);
    const float inv_f = 1.f / (float)a.f;
    const int f = a.f, lanes = a.lanes, gl = threadIdx.x & (lanes - 1), grp = threadIdx.x / lanes, groups = 256 / lanes;
    const int64_t ld = rows8_stride(f);
    float4 ga[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
        ga[r] = a.gamma ? read4<MEM == kStreamed ? kAlignedRow : MEM>(a.gamma, 4 * (r * lanes + gl), f, true) : make_float4(1.f, 1.f, 1.f, 1.f);
    for (long base = (long)blockIdx.x * groups * U; base < a.n; base += (long)gridDim.x * groups * U) {
        float4 x[U][R];
        unsigned row[U], top[U];                           // rows are below 2^31 + 2^12
        float s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = (unsigned)base + u * groups + grp;
#pragma unroll
            for (int r = 0; r < R; ++r) x[u][r] = read4<MEM>(a.X + (size_t)row[u] * f, 4 * (r * lanes + gl), f, row[u] < (unsigned)a.n);
        }
        if constexpr (KIND == kAddNorm) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int g = r * lanes + gl;
                    const float4 o = read4<MEM>(a.R + (size_t)row[u] * f, 4 * g, f, row[u] < (unsigned)a.n);
                    float4 v = words.apply(x[u][r], row[u], g);
                    v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
                    x[u][r] = v;
                    if (row[u] < (unsigned)a.n) write4<MEM>(a.H + (size_t)row[u] * f, 4 * g, f, v);
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = 0.f;
            top[u] = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float4 &v = x[u][r];
                if constexpr (KIND == kRows) v = make_float4(v.x * ga[r].x, v.y * ga[r].y, v.z * ga[r].z, v.w * ga[r].w);
                else s[u] += fmaf(v.x, v.x, v.y * v.y) + fmaf(v.z, v.z, v.w * v.w);
                top[u] = max(top[u], largest(v));
            }
        }
        if constexpr (KIND != kRows) row_sums<U, WIDE>(s, lanes, red);
        if (a.held.q) row_largest<U, WIDE>(top, lanes, red);       // uniform
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row[u] >= (unsigned)a.n) continue;
            const float rstd = KIND == kRows ? 1.f : inverse_root(fmaf(s[u], inv_f, a.eps));
            if (gl == 0 && a.rstd) a.rstd[row[u]] = rstd;
            if (a.held.q) {
                const Held8 h(top[u]);
                if (gl == 0) a.held.scale[row[u]] = h.unit * rstd * (1.f / h.up);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int c = 4 * (r * lanes + gl);
                    if (c < f) *reinterpret_cast<unsigned *>(a.held.q + row[u] * ld + c) = h.four(x[u][r]);
                }
            }
            if (KIND == kRows || !a.Y) continue;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float4 v = x[u][r];
                write4<MEM>(a.Y + (size_t)row[u] * f, 4 * (r * lanes + gl), f,
                            make_float4(v.x * rstd * ga[r].x, v.y * rstd * ga[r].y, v.z * rstd * ga[r].z, v.w * rstd * ga[r].w));
            }
        }
    }
}

struct RmsBack {
    int n, f, lanes;
    const float *H;                    // NULL: xhat from `held`
    Rows8 held;
    const float *rstd, *gamma;
    Dropout drop;
    const float *dY, *dH;              // dH: or NULL
    float *dR, *dX;                    // either or both may be NULL
    float *part;                       // [block][f]: sums of dY xhat, or NULL
    int row_blocks;                    // few rows: the blocks behind these form dgamma, 64 columns each
    float *dgamma;
};

// four columns of xhat, not yet times the row's factor: H, or the integers; zeros past the row's end and the last row
template <int MEM, bool HELD>
__device__ __forceinline__ float4 rms_row(const RmsBack &a, long row, int c, bool valid) {
    if constexpr (!HELD) return read4<MEM>(a.H + row * a.f, c, a.f, valid);
    if (!valid || c >= a.f) return make_float4(0.f, 0.f, 0.f, 0.f);
    return integers(*reinterpret_cast<const unsigned *>(a.held.q + row * rows8_stride(a.f) + c));
}
// What lies behind a row's end in the last word of its integers is any integer, but dY is zero there.
template <bool HELD>
__device__ __forceinline__ float rms_factor(const RmsBack &a, long row) { return HELD ? a.held.scale[row] : a.rstd[row]; }

// 64 columns of dgamma over all rows, 16 groups of lanes every sixteenth row each: they need no more of a row than its factor, so that they
// go with the rows in one launch (28 x 29 forward and back 14.7 us in three).
template <bool HELD>
__device__ __forceinline__ void rms_columns(const RmsBack &a, int block, float4 *across) {
    const int c = block * 64 + 4 * (threadIdx.x % 16), group = threadIdx.x / 16;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < a.f) {
#pragma unroll 4
        for (long row = group; row < a.n; row += 16) {
            const float4 v = rms_row<kAnyRow, HELD>(a, row, c, true), d = load4(a.dY + row * a.f, c, a.f);
            const float k = rms_factor<HELD>(a, row);
            s = make_float4(fmaf(d.x, v.x * k, s.x), fmaf(d.y, v.y * k, s.y), fmaf(d.z, v.z * k, s.z), fmaf(d.w, v.w * k, s.w));
        }
    }
    across[threadIdx.x] = s;
    __syncthreads();
    if (group != 0 || c >= a.f) return;
    for (int k = 1; k < 16; ++k) {
        const float4 o = across[threadIdx.x + 16 * k];
        s = make_float4(s.x + o.x, s.y + o.y, s.z + o.z, s.w + o.w);
    }
    store4(a.dgamma, c, a.f, s);
}

// dR = dH + rstd (g - xhat mean(g xhat)) with g = gamma dY, dX = dropout(dR).  Bound by memory: 2^20 x 256 from 8 bits 3.5 GB in 634 us, 5.5
// TB/s (713 with dH loaded behind the sums); 2^18 x 512 from H 2.1 GB in 370, 5.8; 30011 x 203 73 MB in 17.
template <int R, int U, bool HELD, int MEM, bool WIDE>
__global__ void __launch_bounds__(256)
rms_backward_kernel(RmsBack a) {
    __shared__ float red[4 * U];
    __shared__ float4 across[256];
    if ((int)blockIdx.x >= a.row_blocks) {                 // uniform
        rms_columns<HELD>(a, blockIdx.x - a.row_blocks, across);
        return;
    }
    const DropoutWords words(a.drop);
    const float inv_f = 1.f / (float)a.f;
    const int f = a.f, lanes = a.lanes, gl = threadIdx.x & (lanes - 1), grp = threadIdx.x / lanes, groups = 256 / lanes;
    const bool write = a.dR || a.dX;                       // uniform
    float4 ga[R], dg[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        ga[r] = a.gamma ? read4<MEM == kStreamed ? kAlignedRow : MEM>(a.gamma, 4 * (r * lanes + gl), f, true) : make_float4(1.f, 1.f, 1.f, 1.f);
        dg[r] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (long base = (long)blockIdx.x * groups * U; base < a.n; base += (long)a.row_blocks * groups * U) {
        float4 x[U][R], d[U][R], h[U][R];
        long row[U];
        float rstd[U], s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = base + u * groups + grp;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int c = 4 * (r * lanes + gl);
                x[u][r] = rms_row<MEM, HELD>(a, row[u], c, row[u] < a.n);
                d[u][r] = read4<MEM>(a.dY + row[u] * f, c, f, row[u] < a.n);
                h[u][r] = a.dH && write ? read4<MEM>(a.dH + row[u] * f, c, f, row[u] < a.n) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float factor = row[u] < a.n ? rms_factor<HELD>(a, row[u]) : 0.f;
            rstd[u] = HELD && row[u] < a.n ? a.rstd[row[u]] : factor;
            s[u] = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float4 &v = x[u][r], &e = d[u][r];
                v = make_float4(v.x * factor, v.y * factor, v.z * factor, v.w * factor);
                dg[r] = make_float4(fmaf(e.x, v.x, dg[r].x), fmaf(e.y, v.y, dg[r].y), fmaf(e.z, v.z, dg[r].z), fmaf(e.w, v.w, dg[r].w));
                e = make_float4(e.x * ga[r].x, e.y * ga[r].y, e.z * ga[r].z, e.w * ga[r].w);
                s[u] += fmaf(e.x, v.x, e.y * v.y) + fmaf(e.z, v.z, e.w * v.w);
            }
        }
        if (!write) continue;
        row_sums<U, WIDE>(s, lanes, red);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row[u] >= a.n) continue;
            const float m = s[u] * inv_f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int g = r * lanes + gl;
                const float4 v = x[u][r], e = d[u][r], b = h[u][r];
                const float4 o = make_float4(fmaf(rstd[u], fmaf(-v.x, m, e.x), b.x), fmaf(rstd[u], fmaf(-v.y, m, e.y), b.y),
                                             fmaf(rstd[u], fmaf(-v.z, m, e.z), b.z), fmaf(rstd[u], fmaf(-v.w, m, e.w), b.w));
                if (a.dR) write4<MEM>(a.dR + row[u] * f, 4 * g, f, o);
                if (a.dX) write4<MEM>(a.dX + row[u] * f, 4 * g, f, words.apply(o, (uint32_t)row[u], g));
            }
        }
    }
    if (!a.part) return;
    // the block's rows: over the groups of a wavefront by shuffles, over the wavefronts through LDS
    float *part = a.part + (size_t)blockIdx.x * f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float4 v = dg[r];
        for (int k = lanes; k < 64; k <<= 1) {
            v.x += __shfl_xor(v.x, k, 64);
            v.y += __shfl_xor(v.y, k, 64);
            v.z += __shfl_xor(v.z, k, 64);
            v.w += __shfl_xor(v.w, k, 64);
        }
        if (lanes < 256) {
            __syncthreads();
            across[threadIdx.x] = v;
            __syncthreads();
            for (int k = lanes < 64 ? 64 : lanes; k < 256; k += lanes < 64 ? 64 : lanes)
                if ((int)threadIdx.x < lanes) {
                    const float4 o = across[threadIdx.x + k];
                    v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
                }
        }
        const int c = 4 * (r * lanes + gl);
        if ((int)threadIdx.x < lanes && c < f) store4(part, c, f, v);
    }
}

// Rows beyond kNormRow columns: a block per row, which it reads twice, the second time from the caches; for the columns' sums from
// memory again.  16384 x 8192 with residual: forward 410 us, 5.2 TB/s, backward 432 and 215 for the columns, from 8 bits 344 and 144; into 8
// bits 180.
template <int KIND>
__global__ void __launch_bounds__(256)
rms_forward_long_kernel(RmsNorm a) {
    __shared__ float red[4];
    const DropoutWords words(a.drop);
    const long row = blockIdx.x;
    const int f = a.f;
    const float *x = (KIND == kAddNorm ? a.H : a.X) + row * f;
    float s[1] = {0.f};
    unsigned top[1] = {0};
#pragma unroll 4
    for (int c = 4 * threadIdx.x; c < f; c += 1024) {
        float4 v = load4(a.X + row * f, c, f);
        if constexpr (KIND == kAddNorm) {
            const float4 r = load4(a.R + row * f, c, f);
            v = words.apply(v, (uint32_t)row, c / 4);
            v = make_float4(v.x + r.x, v.y + r.y, v.z + r.z, v.w + r.w);
            store4(a.H + row * f, c, f, v);
        }
        if (KIND == kRows && a.gamma) {
            const float4 g = load4(a.gamma, c, f);
            v = make_float4(v.x * g.x, v.y * g.y, v.z * g.z, v.w * g.w);
        }
        s[0] += fmaf(v.x, v.x, v.y * v.y) + fmaf(v.z, v.z, v.w * v.w);
        top[0] = max(top[0], largest(v));
    }
    if constexpr (KIND != kRows) s[0] = block_sum(s[0], red);
    if (a.held.q) row_largest<1, true>(top, 256, red);
    const float rstd = KIND == kRows ? 1.f : inverse_root(fmaf(s[0], 1.f / (float)f, a.eps));
    const Held8 h(top[0]);
    if (threadIdx.x == 0) {
        if (a.rstd) a.rstd[row] = rstd;
        if (a.held.q) a.held.scale[row] = h.unit * rstd * (1.f / h.up);
    }
#pragma unroll 2
    for (int c = 4 * threadIdx.x; c < f; c += 1024) {      // a thread reads back what it has written itself
        float4 v = load4(x, c, f);
        const float4 g = a.gamma ? load4(a.gamma, c, f) : make_float4(1.f, 1.f, 1.f, 1.f);
        if constexpr (KIND == kRows) v = make_float4(v.x * g.x, v.y * g.y, v.z * g.z, v.w * g.w);
        if (a.held.q) *reinterpret_cast<unsigned *>(a.held.q + row * rows8_stride(f) + c) = h.four(v);
        if (KIND != kRows && a.Y) store4(a.Y + row * f, c, f, make_float4(v.x * rstd * g.x, v.y * rstd * g.y, v.z * rstd * g.z, v.w * rstd * g.w));
    }
}

template <bool HELD>
__global__ void __launch_bounds__(256)
rms_backward_long_kernel(RmsBack a) {
    __shared__ float red[4];
    const DropoutWords words(a.drop);
    const long row = blockIdx.x;
    const int f = a.f;
    const float factor = rms_factor<HELD>(a, row), rstd = a.rstd[row];
    float s = 0.f;
#pragma unroll 2
    for (int c = 4 * threadIdx.x; c < f; c += 1024) {
        const float4 v = rms_row<kAnyRow, HELD>(a, row, c, true), d = load4(a.dY + row * f, c, f);
        const float4 g = a.gamma ? load4(a.gamma, c, f) : make_float4(1.f, 1.f, 1.f, 1.f);
        s += fmaf(d.x * g.x, v.x * factor, d.y * g.y * (v.y * factor)) + fmaf(d.z * g.z, v.z * factor, d.w * g.w * (v.w * factor));
    }
    const float m = block_sum(s, red) / (float)f * factor;
#pragma unroll 2
    for (int c = 4 * threadIdx.x; c < f; c += 1024) {
        const float4 v = rms_row<kAnyRow, HELD>(a, row, c, true), d = load4(a.dY + row * f, c, f);
        const float4 g = a.gamma ? load4(a.gamma, c, f) : make_float4(1.f, 1.f, 1.f, 1.f);
        float4 o = make_float4(rstd * fmaf(-v.x, m, d.x * g.x), rstd * fmaf(-v.y, m, d.y * g.y), rstd * fmaf(-v.z, m, d.z * g.z),
                               rstd * fmaf(-v.w, m, d.w * g.w));
        if (a.dH) {
            const float4 h = load4(a.dH + row * f, c, f);
            o = make_float4(o.x + h.x, o.y + h.y, o.z + h.z, o.w + h.w);
        }
        if (a.dR) store4(a.dR + row * f, c, f, o);
        if (a.dX) store4(a.dX + row * f, c, f, words.apply(o, (uint32_t)row, c / 4));
    }
}

// part[y] = sum dY xhat over every gridDim.y-th row, 1024 columns per block
template <bool HELD>
__global__ void __launch_bounds__(256)
rms_sums_long_kernel(RmsBack a) {
    const int f = a.f, c = 4 * ((int)blockIdx.x * 256 + threadIdx.x);
    if (c >= f) return;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (long row = blockIdx.y; row < a.n; row += gridDim.y) {
        const float4 v = rms_row<kAnyRow, HELD>(a, row, c, true), d = load4(a.dY + row * f, c, f);
        const float k = rms_factor<HELD>(a, row);
        s = make_float4(fmaf(d.x, v.x * k, s.x), fmaf(d.y, v.y * k, s.y), fmaf(d.z, v.z * k, s.z), fmaf(d.w, v.w * k, s.w));
    }
    store4(a.part + (size_t)blockIdx.y * f, c, f, s);
}

// the integers times the scale of their row, and of their column; four a thread.  Bound by memory: 2^18 x 512 0.67 GB in 125 us, 5.4 TB/s.
__global__ void __launch_bounds__(256)
dequantize_kernel(int n, int f, Rows8 in, float *__restrict__ Y) {
    const long groups = (f + 3) / 4, total = (long)n * groups;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long)gridDim.x * 256) {
        const long row = i / groups;
        const int c = 4 * (int)(i - row * groups);
        const float s = in.scale[row];
        float4 v = integers(*reinterpret_cast<const unsigned *>(in.q + row * rows8_stride(f) + c));
        v = make_float4(v.x * s, v.y * s, v.z * s, v.w * s);
        if (in.columns) {
            const float4 k = load4(in.columns, c, f);
            v = make_float4(v.x * k.x, v.y * k.y, v.z * k.z, v.w * k.w);
        }
        store4(Y + row * f, c, f, v);
    }
}

}  // namespace

// U_: rows at a time, and of streamed arrays, which take more loads under way
#define RMS_CASE(KERNEL_, KIND_, PER_, U_, STREAM_U_, WIDE_)                                                                          \
    if (shape.per == PER_ && shape.wide == WIDE_) {                                                                                   \
        if (mem == kStreamed) hipLaunchKernelGGL((KERNEL_<PER_, STREAM_U_, KIND_, kStreamed, WIDE_>), grid, dim3(256), 0, st, a);     \
        else if (mem == kAlignedRow) hipLaunchKernelGGL((KERNEL_<PER_, U_, KIND_, kAlignedRow, WIDE_>), grid, dim3(256), 0, st, a);   \
        else hipLaunchKernelGGL((KERNEL_<PER_, U_, KIND_, kAnyRow, WIDE_>), grid, dim3(256), 0, st, a);                               \
    }

template <int KIND>
static gnn_status_t forward(RmsNorm a, bool aligned, hipStream_t st) {
    if (a.f > kNormRow) {
        hipLaunchKernelGGL(rms_forward_long_kernel<KIND>, dim3((unsigned)a.n), dim3(256), 0, st, a);
        return launch_status();
    }
    const Shape shape = norm_shape(a.f);
    a.lanes = shape.lanes;
    const int u = shape.wide || shape.per == 4 ? 1 : shape.per == 2 ? 2 : 4, mem = norm_memory(a.n, a.f, aligned && a.f % 4 == 0);
    int64_t blocks = ceil_div(a.n, 256 / shape.lanes * u);
    if (blocks > 2048) blocks = 2048;
    const dim3 grid((unsigned)blocks);
    RMS_CASE(rms_forward_kernel, KIND, 1, 4, 4, false)
    RMS_CASE(rms_forward_kernel, KIND, 2, 2, 2, false)
    RMS_CASE(rms_forward_kernel, KIND, 4, 1, 1, false)
    RMS_CASE(rms_forward_kernel, KIND, 4, 1, 1, true)
    return launch_status();
}

gnn_status_t rms_norm_forward_launch(int n, int f, const float *X, const float *R, const Dropout &drop, const float *gamma, float eps,
                                     float *H, float *Y, const Rows8 &held, float *rstd, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    const RmsNorm a{n, f, 0, X, R, gamma, eps, drop, H, Y, rstd, held};
    const bool aligned = aligned16(X) && aligned16(Y) && aligned16(gamma) && aligned16(R) && aligned16(H);
    return R ? forward<kAddNorm>(a, aligned, st) : forward<kNorm>(a, aligned, st);
}

gnn_status_t quantize_rows_launch(int n, int f, const float *X, const float *columns, const Rows8 &out, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    const RmsNorm a{n, f, 0, X, nullptr, columns, 0.f, Dropout{nullptr, 0, 0, 1.f}, nullptr, nullptr, nullptr, out};
    return forward<kRows>(a, aligned16(X) && aligned16(columns), st);
}

gnn_status_t dequantize_rows_launch(int n, int f, const Rows8 &in, float *Y, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    int64_t blocks = ceil_div((int64_t)n * ((f + 3) / 4), 256);
    if (blocks > 1 << 20) blocks = 1 << 20;
    hipLaunchKernelGGL(dequantize_kernel, dim3((unsigned)blocks), dim3(256), 0, st, n, f, in, Y);
    return launch_status();
}

// not what this n takes, but what serves every smaller one as well
size_t rms_norm_workspace_bytes(int64_t n, int64_t f) {
    const int64_t blocks = norm_blocks(n, (int)f);
    return align_up((size_t)(blocks > 1024 ? blocks : 1024) * f * sizeof(float));
}

// Rows up to which dgamma comes from blocks of its own beside them instead of a launch of its own
constexpr int kFewRows = 512;

template <bool HELD>
static gnn_status_t rows_launch(const RmsBack &a, const Shape &shape, int mem, int64_t blocks, hipStream_t st) {
    const dim3 grid((unsigned)blocks);
    RMS_CASE(rms_backward_kernel, HELD, 1, 4, 4, false)
    RMS_CASE(rms_backward_kernel, HELD, 2, 1, 2, false)
    RMS_CASE(rms_backward_kernel, HELD, 4, 1, 1, false)
    RMS_CASE(rms_backward_kernel, HELD, 4, 1, 1, true)
    return launch_status();
}

template <bool HELD>
static gnn_status_t backward(RmsBack a, int64_t blocks, hipStream_t st) {
    if (a.f > kNormRow) {
        if (a.part) {                                      // before dR and dX, which may lie over dY
            hipLaunchKernelGGL(rms_sums_long_kernel<HELD>, dim3((unsigned)ceil_div(a.f, 1024), (unsigned)blocks), dim3(256), 0, st, a);
            GNN_TRY(launch_status());
        }
        if (a.dR || a.dX) hipLaunchKernelGGL(rms_backward_long_kernel<HELD>, dim3((unsigned)a.n), dim3(256), 0, st, a);
        return launch_status();
    }
    const Shape shape = norm_shape(a.f);
    a.lanes = shape.lanes;
    const bool aligned = a.f % 4 == 0 && aligned16(a.H) && aligned16(a.dY) && aligned16(a.gamma) && aligned16(a.dX) && aligned16(a.dR) &&
                         aligned16(a.dH);
    const int mem = norm_memory(a.n, a.f, aligned);
    a.row_blocks = (int)blocks;
    const int64_t columns = a.dgamma ? ceil_div(a.f, 64) : 0;
    if (columns && !a.dR && !a.dX) {
        a.row_blocks = 0;
        return rows_launch<HELD>(a, shape, mem, columns, st);
    }
    if (columns && (a.dR == a.dY || a.dX == a.dY)) {       // they read dY: before it is written
        a.row_blocks = 0;
        GNN_TRY((rows_launch<HELD>(a, shape, mem, columns, st)));
        a.dgamma = nullptr;
        a.row_blocks = (int)blocks;
        return rows_launch<HELD>(a, shape, mem, blocks, st);
    }
    return rows_launch<HELD>(a, shape, mem, blocks + columns, st);
}
#undef RMS_CASE

gnn_status_t rms_norm_backward_launch(int n, int f, const float *H, const Rows8 &held, const float *rstd, const float *gamma,
                                      const Dropout &drop, const float *dY, const float *dH, float *dR, float *dX, float *dgamma,
                                      void *workspace, hipStream_t st) {
    if (n <= 0) return dgamma ? fill_zero_launch(f, dgamma, st) : GNN_OK;
    if (!dgamma && !dX && !dR) return GNN_OK;
    const int64_t blocks = norm_blocks(n, f);
    const bool beside = n <= kFewRows && f <= kNormRow && dgamma;
    const RmsBack a{n, f, 0, H, held, rstd, gamma, drop, dY, dH, dR, dX, dgamma && !beside ? static_cast<float *>(workspace) : nullptr, 0,
                    beside ? dgamma : nullptr};
    GNN_TRY(H ? backward<false>(a, blocks, st) : backward<true>(a, blocks, st));
    return dgamma && !beside ? norm_sums_launch(f, f, blocks, a.part, dgamma, nullptr, st) : GNN_OK;
}

}  // namespace gnn
