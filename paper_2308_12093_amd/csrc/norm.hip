// Dropout, layer norm and the two around a residual connection, forward and backward.
#include "dropout.h"

namespace gnn {
namespace {

typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));

typedef float floatx2u __attribute__((ext_vector_type(2), aligned(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

typedef float floatx3u __attribute__((ext_vector_type(3), aligned(4)));

// Columns c .. c + 3 < f + 3 of a row of f, at any 4-byte aligned address; zeros past the row's end.  The one to three of the last
// lane are one access, too: f % 4 is the same for all.
__device__ __forceinline__ float4 load4(const float *row, int c, int f) {
    if (c + 4 <= f) {
        const float4u v = *reinterpret_cast<const float4u *>(row + c);
        return make_float4(v.x, v.y, v.z, v.w);
    }
    const int left = f & 3;
    if (left == 1) return make_float4(row[c], 0.f, 0.f, 0.f);
    if (left == 2) {
        const floatx2u v = *reinterpret_cast<const floatx2u *>(row + c);
        return make_float4(v.x, v.y, 0.f, 0.f);
    }
    const floatx3u v = *reinterpret_cast<const floatx3u *>(row + c);
    return make_float4(v.x, v.y, v.z, 0.f);
}

__device__ __forceinline__ void store4(float *row, int c, int f, float4 v) {
    if (c + 4 <= f) {
        *reinterpret_cast<float4u *>(row + c) = float4u{v.x, v.y, v.z, v.w};
        return;
    }
    const int left = f & 3;
    if (left == 1) row[c] = v.x;
    else if (left == 2) *reinterpret_cast<floatx2u *>(row + c) = floatx2u{v.x, v.y};
    else *reinterpret_cast<floatx3u *>(row + c) = floatx3u{v.x, v.y, v.z};
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// exp(x) for x <= 0: off by at most (1 + |x|) units in the last place, one instruction and a multiplication
__device__ __forceinline__ float exp_down(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// exp(x) - 1 for x <= 0: the series up to x^7 / 7! near zero (what it leaves out is below 2^-25 of the result), the difference
// where it keeps its digits
__device__ __forceinline__ float expm1_down(float x) {
    const float p = fmaf(fmaf(fmaf(fmaf(fmaf(1.f / 5040, x, 1.f / 720), x, 1.f / 120), x, 1.f / 24), x, 1.f / 6), x, 0.5f);
    return x > -0.35f ? fmaf(x * x, p, x) : exp_down(x) - 1.f;
}

template <int ACT>
__device__ __forceinline__ float activation(float z) {
    if constexpr (ACT == kActRelu) return z < 0.f ? 0.f : z;                // NaN stays
    if constexpr (ACT == kActElu) return z > 0.f ? z : expm1_down(z);
    return z;
}
template <int ACT>
__device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == kActRelu) return z > 0.f ? 1.f : 0.f;
    if constexpr (ACT == kActElu) return z > 0.f ? 1.f : exp_down(z);      // NaN stays
    return 1.f;
}
__device__ __forceinline__ float activation(float z, int act) {
    return act == kActRelu ? activation<kActRelu>(z) : act == kActElu ? activation<kActElu>(z) : z;
}
__device__ __forceinline__ float slope(float z, int act) {
    return act == kActRelu ? slope<kActRelu>(z) : act == kActElu ? slope<kActElu>(z) : 1.f;
}

// 1 / sqrt(x): the instruction's, and a Newton step (an IEEE division and root take thirty instructions, for each lane of a row)
__device__ __forceinline__ float inverse_root(float x) {
    const float y = __builtin_amdgcn_rsqf(x);
    const float r = fmaf(fmaf(-0.5f * x * y, y, 0.5f), y, y);
    return x > 0x1p-100f && x < 0x1p100f ? r : y;          // x y y keeps its range there; infinities and NaN as they are
}

// Four columns a thread, one generator's block each.  Bound by memory: 2^20 x 256 with a residual 3.2 GB in 525 us, 6.1 TB/s (a copy
// reaches 5.0, a sum of two arrays 5.9); the ten rounds of the generator, 40 multiplications for 48 bytes, hide behind it.
__global__ void __launch_bounds__(256)
dropout_kernel(int n, int f, const float *X, const float *R, Dropout drop, float *Y) {
    const DropoutWords words(drop);
    const long groups = (f + 3) / 4, total = (long)n * groups;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long)gridDim.x * 256) {
        const long row = i / groups;
        const int g = (int)(i - row * groups), c = 4 * g;
        float4 x = words.apply(load4(X + row * f, c, f), (uint32_t)row, g);
        if (R) {
            const float4 r = load4(R + row * f, c, f);
            x = make_float4(x.x + r.x, x.y + r.y, x.z + r.z, x.w + r.w);
        }
        store4(Y + row * f, c, f, x);
    }
}

// ---- layer norm -------------------------------------------------------------------------------------------
// A row is the work of `lanes` lanes (a power of two up to a block's 256), R times four columns each, and stays in their
// registers: mean and variance are sums over the same registers, so that the variance is one of differences.  Every array
// passes through memory once.  U rows at a time keep loads under way where a row is short; weights are loaded once per block.
struct Norm {
    int n, f, lanes;
    const float *X, *R;                // R: H = R + dropout(X), Y = norm(H); without: Y = dropout(act(norm(X)))
    const float *gamma, *beta;
    float eps;
    int act;
    Dropout drop;
    float *H, *Y, *stat;
};

// v: the sums of a wavefront's lanes of a row; then those of the row's wavefronts, two or four
template <int U>
__device__ __forceinline__ void wide_sums(float (&v)[U], int lanes, float *red) {
    const int wave = threadIdx.x / 64, first = threadIdx.x / lanes * (lanes / 64);
    __syncthreads();
    if (threadIdx.x % 64 == 0)
#pragma unroll
        for (int u = 0; u < U; ++u) red[4 * u + wave] = v[u];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float s = red[4 * u + first] + red[4 * u + first + 1];
        if (lanes == 256) s += red[4 * u + 2] + red[4 * u + 3];
        v[u] = s;
    }
}

// the sums of each of U values over the lanes of a row, in all of them
template <int U, bool WIDE>
__device__ __forceinline__ void row_sums(float (&v)[U], int lanes, float *red) {
    for (int d = (WIDE ? 64 : lanes) >> 1; d > 0; d >>= 1)
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] += __shfl_xor(v[u], d, 64);
    if constexpr (WIDE) wide_sums(v, lanes, red);
}
// The same of U pairs: each half of the lanes goes on with one value of a pair and hands it to the other in the end, two
// exchanges more than for one value.
template <int U, bool WIDE>
__device__ __forceinline__ void row_sums_of_pairs(float (&v)[2 * U], int lanes, float *red) {
    const int half = (WIDE ? 64 : lanes) >> 1;
    if (half > 0) {
        const bool upper = threadIdx.x & half;
        float s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) s[u] = (upper ? v[2 * u + 1] : v[2 * u]) + __shfl_xor(upper ? v[2 * u] : v[2 * u + 1], half, 64);
        for (int d = half >> 1; d > 0; d >>= 1)
#pragma unroll
            for (int u = 0; u < U; ++u) s[u] += __shfl_xor(s[u], d, 64);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float other = __shfl_xor(s[u], half, 64);
            v[2 * u] = upper ? other : s[u];
            v[2 * u + 1] = upper ? s[u] : other;
        }
    }
    if constexpr (WIDE) wide_sums(v, lanes, red);
}

// What the mean m of a row is off by, from the sum of the differences d to it, and its variance + eps, from the sum of their squares as
// well.  Far from zero one unit in the last place of m is as large as what rows of nearly equal values are normalised by, and
// a sum over lanes divided by f misses the value of a row of f equal ones in a third of all cases.  Such a row's d are a few
// units each, so the sums are exact; so is their quotient after the step behind the product with 1 / f: d - off and the variance
// are zero, and m + off is the value.  Forward forms xhat from d - off, backward from m + off rounded to a float, which is coarser far
// from zero; with ReLU forward takes the coarser one as well, so that both see the same signs.
__device__ __forceinline__ float rounded_mean(float sum, float inv_f) {
#pragma clang fp contract(off)
    return sum * inv_f;                                    // not one with the subtraction that follows: d is exact so
}
__device__ __forceinline__ float mean_off_by(float sum, float f, float inv_f) {
    const float off = sum * inv_f;
    return fmaf(fmaf(-off, f, sum), inv_f, off);
}
__device__ __forceinline__ float variance_and(float eps, float sum, float square, float off, float inv_f) {
    const float left = fmaf(-off, sum, square);
    return fmaf(left < 0.f ? 0.f : left, inv_f, eps);      // NaN stays
}

// How rows are read and written.  kStreamed: aligned rows of arrays beyond the caches, past them (2^20 x 256 backward 645 -> 600
// us, 2^18 x 512 around a residual connection 511 -> 488 and forward 398 -> 379; arrays that the caches hold would lose
// what the next kernel finds there).
enum { kAnyRow, kAlignedRow, kStreamed };

template <int MEM>
__device__ __forceinline__ float4 read4(const float *row, int c, int f, bool valid) {
    if (!valid || c >= f) return make_float4(0.f, 0.f, 0.f, 0.f);
    if constexpr (MEM == kAnyRow) return load4(row, c, f);
    else if constexpr (MEM == kAlignedRow) return *reinterpret_cast<const float4 *>(row + c);
    else {
        const floatx4 v = __builtin_nontemporal_load(reinterpret_cast<const floatx4 *>(row + c));
        return make_float4(v.x, v.y, v.z, v.w);
    }
}
template <int MEM>
__device__ __forceinline__ void write4(float *row, int c, int f, float4 v) {
    if (c >= f) return;
    if constexpr (MEM == kAnyRow) store4(row, c, f, v);
    else if constexpr (MEM == kAlignedRow) *reinterpret_cast<float4 *>(row + c) = v;
    else __builtin_nontemporal_store(floatx4{v.x, v.y, v.z, v.w}, reinterpret_cast<floatx4 *>(row + c));
}

// Bound by memory: 2^20 x 256 with ELU and dropout 2.1 GB in 409 us, 5.3 TB/s; 2^18 x 512 around a residual connection 2.1 GB in 344 to
// 377 us, 5.7 to 6.2 TB/s; 131072 x 47 from the caches 49 MB in 16 us.
template <int R, int U, int ACT, bool ADD, int MEM, bool WIDE>
__global__ void __launch_bounds__(256)
norm_forward_kernel(Norm a) {
    __shared__ float red[8 * U];
    const DropoutWords words(a.drop);
    const float inv_f = 1.f / (float)a.f;
    const int f = a.f, lanes = a.lanes, gl = threadIdx.x & (lanes - 1), grp = threadIdx.x / lanes, groups = 256 / lanes;
    float4 ga[R], be[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = 4 * (r * lanes + gl);
        ga[r] = a.gamma ? read4<MEM == kStreamed ? kAlignedRow : MEM>(a.gamma, c, f, true) : make_float4(1.f, 1.f, 1.f, 1.f);
        be[r] = a.beta ? read4<MEM == kStreamed ? kAlignedRow : MEM>(a.beta, c, f, true) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (long base = (long)blockIdx.x * groups * U; base < a.n; base += (long)gridDim.x * groups * U) {
        float4 x[U][R];
        unsigned row[U];                                   // below 2^31 + 2^12
        float mean[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = (unsigned)base + u * groups + grp;
#pragma unroll
            for (int r = 0; r < R; ++r) x[u][r] = read4<MEM>(a.X + (size_t)row[u] * f, 4 * (r * lanes + gl), f, row[u] < (unsigned)a.n);
        }
        if constexpr (ADD) {
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
            mean[u] = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) mean[u] += (x[u][r].x + x[u][r].y) + (x[u][r].z + x[u][r].w);
        }
        row_sums<U, WIDE>(mean, lanes, red);
        float s[2 * U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            mean[u] = rounded_mean(mean[u], inv_f);
            s[2 * u] = s[2 * u + 1] = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int c = 4 * (r * lanes + gl);
                const float4 v = x[u][r];
                const float d0 = c < f ? v.x - mean[u] : 0.f, d1 = c + 1 < f ? v.y - mean[u] : 0.f;
                const float d2 = c + 2 < f ? v.z - mean[u] : 0.f, d3 = c + 3 < f ? v.w - mean[u] : 0.f;
                if constexpr (ACT != kActRelu) x[u][r] = make_float4(d0, d1, d2, d3);
                s[2 * u] += (d0 + d1) + (d2 + d3);
                s[2 * u + 1] += fmaf(d0, d0, d1 * d1) + fmaf(d2, d2, d3 * d3);
            }
        }
        row_sums_of_pairs<U, WIDE>(s, lanes, red);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float off = mean_off_by(s[2 * u], (float)f, inv_f), whole = mean[u] + off;
            const float rstd = inverse_root(variance_and(a.eps, s[2 * u], s[2 * u + 1], off, inv_f));
            const float less = ACT == kActRelu ? whole : off;      // x[u] is d but for ReLU
            if (row[u] >= (unsigned)a.n) continue;
            if (gl == 0) *reinterpret_cast<floatx2u *>(a.stat + 2 * (size_t)row[u]) = floatx2u{whole, rstd};
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int g = r * lanes + gl;
                const float4 d = make_float4(x[u][r].x - less, x[u][r].y - less, x[u][r].z - less, x[u][r].w - less);
                float4 y = make_float4(fmaf(d.x * rstd, ga[r].x, be[r].x), fmaf(d.y * rstd, ga[r].y, be[r].y),
                                       fmaf(d.z * rstd, ga[r].z, be[r].z), fmaf(d.w * rstd, ga[r].w, be[r].w));
                if constexpr (!ADD) {
                    y = make_float4(activation<ACT>(y.x), activation<ACT>(y.y), activation<ACT>(y.z), activation<ACT>(y.w));
                    y = words.apply(y, row[u], g);
                }
                write4<MEM>(a.Y + (size_t)row[u] * f, 4 * g, f, y);
            }
        }
    }
}

struct NormBack {
    int n, f, lanes;
    const float *X, *stat, *gamma, *beta;
    int act;
    Dropout drop;
    const float *dY, *dH;
    float *dR, *dX;
    float *part;                       // [block][2 f]: sums of dZ xhat and of dZ, or NULL
};

// ADD: dR = dH + the norm's gradient, dX = dropout(dR); without: dX = the norm's gradient of act'(dropout(dY)).
// Bound by memory: 2^20 x 256 with ELU and dropout 3.2 GB in 590 us, 5.5 TB/s; 2^18 x 512 around a residual connection 2.7 GB in 475 us,
// 5.7 TB/s; 131072 x 47 74 MB in 18 us.
template <int R, int U, int ACT, bool ADD, int MEM, bool WIDE>
__global__ void __launch_bounds__(256)
norm_backward_kernel(NormBack a) {
    __shared__ float red[8 * U];
    __shared__ float4 across[256];
    const DropoutWords words(a.drop);
    const float inv_f = 1.f / (float)a.f;
    const int f = a.f, lanes = a.lanes, gl = threadIdx.x & (lanes - 1), grp = threadIdx.x / lanes, groups = 256 / lanes;
    const bool write = ADD || a.dX;                        // uniform
    float4 ga[R], be[R], dg[R], db[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = 4 * (r * lanes + gl);
        ga[r] = a.gamma ? read4<MEM == kStreamed ? kAlignedRow : MEM>(a.gamma, c, f, true) : make_float4(1.f, 1.f, 1.f, 1.f);
        be[r] = a.beta ? read4<MEM == kStreamed ? kAlignedRow : MEM>(a.beta, c, f, true) : make_float4(0.f, 0.f, 0.f, 0.f);
        dg[r] = db[r] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (long base = (long)blockIdx.x * groups * U; base < a.n; base += (long)gridDim.x * groups * U) {
        float4 x[U][R], d[U][R];
        long row[U];
        float rstd[U], s[2 * U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = base + u * groups + grp;
            const bool valid = row[u] < a.n;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int c = 4 * (r * lanes + gl);
                x[u][r] = read4<MEM>(a.X + row[u] * f, c, f, valid);
                d[u][r] = read4<MEM>(a.dY + row[u] * f, c, f, valid);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            floatx2u st = floatx2u{0.f, 0.f};
            if (row[u] < a.n) st = *reinterpret_cast<const floatx2u *>(a.stat + 2 * row[u]);
            rstd[u] = st.y;
            s[2 * u] = s[2 * u + 1] = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int g = r * lanes + gl, c = 4 * g;
                float4 &v = x[u][r], &e = d[u][r];
                // dY past the row's end is zero; so has to be xhat, for what it is multiplied with
                v = make_float4(c < f ? (v.x - st.x) * st.y : 0.f, c + 1 < f ? (v.y - st.x) * st.y : 0.f,
                                c + 2 < f ? (v.z - st.x) * st.y : 0.f, c + 3 < f ? (v.w - st.x) * st.y : 0.f);
                if constexpr (!ADD) {
                    e = words.apply(e, (uint32_t)row[u], g);
                    if constexpr (ACT != kActNone)
                        e = make_float4(e.x * slope<ACT>(fmaf(v.x, ga[r].x, be[r].x)), e.y * slope<ACT>(fmaf(v.y, ga[r].y, be[r].y)),
                                        e.z * slope<ACT>(fmaf(v.z, ga[r].z, be[r].z)), e.w * slope<ACT>(fmaf(v.w, ga[r].w, be[r].w)));
                }
                dg[r] = make_float4(fmaf(e.x, v.x, dg[r].x), fmaf(e.y, v.y, dg[r].y), fmaf(e.z, v.z, dg[r].z), fmaf(e.w, v.w, dg[r].w));
                db[r] = make_float4(db[r].x + e.x, db[r].y + e.y, db[r].z + e.z, db[r].w + e.w);
                e = make_float4(e.x * ga[r].x, e.y * ga[r].y, e.z * ga[r].z, e.w * ga[r].w);
                s[2 * u] += (e.x + e.y) + (e.z + e.w);
                s[2 * u + 1] += fmaf(e.x, v.x, e.y * v.y) + fmaf(e.z, v.z, e.w * v.w);
            }
        }
        if (!write) continue;
        row_sums_of_pairs<U, WIDE>(s, lanes, red);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row[u] >= a.n) continue;
            const float s1 = s[2 * u] * inv_f, s2 = s[2 * u + 1] * inv_f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int g = r * lanes + gl;
                const float4 v = x[u][r], e = d[u][r];
                float4 o = make_float4(rstd[u] * ((e.x - s1) - v.x * s2), rstd[u] * ((e.y - s1) - v.y * s2),
                                       rstd[u] * ((e.z - s1) - v.z * s2), rstd[u] * ((e.w - s1) - v.w * s2));
                if constexpr (ADD) {
                    if (a.dH) {
                        const float4 h = read4<MEM>(a.dH + row[u] * f, 4 * g, f, true);
                        o = make_float4(o.x + h.x, o.y + h.y, o.z + h.z, o.w + h.w);
                    }
                    write4<MEM>(a.dR + row[u] * f, 4 * g, f, o);
                    if (!a.dX) continue;
                    o = words.apply(o, (uint32_t)row[u], g);
                }
                write4<MEM>(a.dX + row[u] * f, 4 * g, f, o);
            }
        }
    }
    if (!a.part) return;
    // the block's rows: over the groups of a wavefront by shuffles, over the wavefronts through LDS
    float *part = a.part + (size_t)blockIdx.x * 2 * f;
#pragma unroll
    for (int i = 0; i < 2 * R; ++i) {
        float4 v = i < R ? dg[i] : db[i - R];
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
        const int c = 4 * ((i < R ? i : i - R) * lanes + gl);
        if ((int)threadIdx.x < lanes && c < f) {
            float *to = part + (i < R ? 0 : f) + c;
            to[0] = v.x;
            if (c + 1 < f) to[1] = v.y;
            if (c + 2 < f) to[2] = v.z;
            if (c + 3 < f) to[3] = v.w;
        }
    }
}

// Rows beyond 4096 columns: a block per row, which it reads several times (16 KB and more, from the caches; for the columns' sums
// from memory again).  16384 x 8192 forward 282 us, 3.8 TB/s, backward 648 us, 2.5 TB/s of X, dY and dX.
constexpr int kNormRow = 4096;

__device__ __forceinline__ float block_sum(float v, float *red) {
    v = wave_sum(v);
    __syncthreads();
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}
__device__ __forceinline__ void unpack(float4 v, float (&o)[4]) { o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w; }
__device__ __forceinline__ void weights4(const float *p, int c, int f, float without, float (&o)[4]) {
    unpack(p ? load4(p, c, f) : make_float4(without, without, without, without), o);
}

__global__ void __launch_bounds__(256)
norm_forward_long_kernel(Norm a) {
    __shared__ float red[4];
    const DropoutWords words(a.drop);
    const long row = blockIdx.x;
    const int f = a.f;
    const float *x = (a.R ? a.H : a.X) + row * f;
    float sum = 0.f;
#pragma unroll 4
    for (int c = 4 * threadIdx.x; c < f; c += 1024) {
        float4 v = load4(a.X + row * f, c, f);
        if (a.R) {
            const float4 r = load4(a.R + row * f, c, f);
            v = words.apply(v, (uint32_t)row, c / 4);
            v = make_float4(v.x + r.x, v.y + r.y, v.z + r.z, v.w + r.w);
            store4(a.H + row * f, c, f, v);
        }
        sum += (v.x + v.y) + (v.z + v.w);
    }
    const float inv_f = 1.f / (float)f, mean = rounded_mean(block_sum(sum, red), inv_f);
    float differences = 0.f, square = 0.f;
#pragma unroll 4
    for (int c = 4 * threadIdx.x; c < f; c += 1024) {      // a thread reads back what it has written itself
        float d[4];
        unpack(load4(x, c, f), d);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            d[j] = c + j < f ? d[j] - mean : 0.f;
            differences += d[j];
            square = fmaf(d[j], d[j], square);
        }
    }
    differences = block_sum(differences, red);
    square = block_sum(square, red);
    const float off = mean_off_by(differences, (float)f, inv_f), whole = mean + off;
    const float rstd = inverse_root(variance_and(a.eps, differences, square, off, inv_f));
    const float first = a.act == kActRelu ? whole : mean, then = a.act == kActRelu ? 0.f : off;
    if (threadIdx.x == 0) { a.stat[2 * row] = whole; a.stat[2 * row + 1] = rstd; }
#pragma unroll 2
    for (int c = 4 * threadIdx.x; c < f; c += 1024) {
        float z[4], ga[4], be[4];
        unpack(load4(x, c, f), z);
        weights4(a.gamma, c, f, 1.f, ga);
        weights4(a.beta, c, f, 0.f, be);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = activation(fmaf(((z[j] - first) - then) * rstd, ga[j], be[j]), a.act);
        float4 y = make_float4(z[0], z[1], z[2], z[3]);
        if (!a.R) y = words.apply(y, (uint32_t)row, c / 4);
        store4(a.Y + row * f, c, f, y);
    }
}

// xhat and dZ (dY through the dropout and the activation behind the norm) of four columns, and gamma of them; zeros past the row's end
__device__ __forceinline__ void norm_gradient(const NormBack &a, const DropoutWords &words, bool after, long row, int c,
                                              float mean, float rstd, float (&xhat)[4], float (&dz)[4], float (&ga)[4]) {
    float be[4];
    float4 d = load4(a.dY + row * a.f, c, a.f);
    if (after) d = words.apply(d, (uint32_t)row, c / 4);
    unpack(d, dz);
    unpack(load4(a.X + row * a.f, c, a.f), xhat);
    weights4(a.gamma, c, a.f, 1.f, ga);
    weights4(a.beta, c, a.f, 0.f, be);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool in = c + j < a.f;
        xhat[j] = in ? (xhat[j] - mean) * rstd : 0.f;
        dz[j] = in ? dz[j] * slope(fmaf(xhat[j], ga[j], be[j]), a.act) : 0.f;
    }
}

__global__ void __launch_bounds__(256)
norm_backward_long_kernel(NormBack a, bool before) {
    __shared__ float red[4];
    const DropoutWords words(a.drop);
    const long row = blockIdx.x;
    const int f = a.f;
    const float mean = a.stat[2 * row], rstd = a.stat[2 * row + 1];
    float s1 = 0.f, s2 = 0.f, xhat[4], dz[4], ga[4];
#pragma unroll 2
    for (int c = 4 * threadIdx.x; c < f; c += 1024) {
        norm_gradient(a, words, !before, row, c, mean, rstd, xhat, dz, ga);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s1 += dz[j] * ga[j];
            s2 = fmaf(dz[j] * ga[j], xhat[j], s2);
        }
    }
    s1 = block_sum(s1, red) / (float)f;
    s2 = block_sum(s2, red) / (float)f;
#pragma unroll 2
    for (int c = 4 * threadIdx.x; c < f; c += 1024) {
        norm_gradient(a, words, !before, row, c, mean, rstd, xhat, dz, ga);
        float o[4], h[4] = {0.f, 0.f, 0.f, 0.f};
        if (a.dH) unpack(load4(a.dH + row * f, c, f), h);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = rstd * ((dz[j] * ga[j] - s1) - xhat[j] * s2) + h[j];
        float4 v = make_float4(o[0], o[1], o[2], o[3]);
        if (a.dR) store4(a.dR + row * f, c, f, v);
        if (before) v = words.apply(v, (uint32_t)row, c / 4);
        if (a.dX) store4(a.dX + row * f, c, f, v);
    }
}

// part[y] = [sum dZ xhat | sum dZ] over every gridDim.y-th row, 1024 columns per block
__global__ void __launch_bounds__(256)
norm_sums_long_kernel(NormBack a, bool after) {
    const DropoutWords words(a.drop);
    const int f = a.f, c = 4 * ((int)blockIdx.x * 256 + threadIdx.x);
    if (c >= f) return;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (long row = blockIdx.y; row < a.n; row += gridDim.y) {
        float xhat[4], dz[4], ga[4];
        norm_gradient(a, words, after, row, c, a.stat[2 * row], a.stat[2 * row + 1], xhat, dz, ga);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s[j] = fmaf(dz[j], xhat[j], s[j]);
            s[4 + j] += dz[j];
        }
    }
    for (int j = 0; j < 4 && c + j < f; ++j) {
        a.part[(size_t)blockIdx.y * 2 * f + c + j] = s[j];
        a.part[(size_t)blockIdx.y * 2 * f + f + c + j] = s[4 + j];
    }
}

// dgamma, dbeta = the sums of the partial rows, in double and in a fixed order: 16 columns a block, 64 lanes each, four of them in a
// wavefront.  What it waits for is memory, four partial rows of a lane at a time: 1024 rows of 94 floats 4.0 us (16 lanes each: 6.7).
__global__ void __launch_bounds__(1024)
norm_sums_final_kernel(int f, int blocks, const float *__restrict__ part, float *dgamma, float *dbeta) {
    __shared__ double red[16][16];
    const int o = threadIdx.x % 16, sl = threadIdx.x / 16;
    const long c = (long)blockIdx.x * 16 + o, w = 2 * (long)f;
    double a0 = 0.0, a1 = 0.0, a2 = 0.0, a3 = 0.0;
    if (c < w) {
        long b = sl;
        for (; b + 192 < blocks; b += 256) {
            a0 += part[b * w + c];
            a1 += part[(b + 64) * w + c];
            a2 += part[(b + 128) * w + c];
            a3 += part[(b + 192) * w + c];
        }
        for (; b < blocks; b += 64) a0 += part[b * w + c];
    }
    double s = (a0 + a1) + (a2 + a3);
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    if (threadIdx.x % 64 < 16) red[threadIdx.x / 64][o] = s;
    __syncthreads();
    if (threadIdx.x < 16 && c < w) {
        double t = 0.0;
        for (int k = 0; k < 16; ++k) t += red[k][o];
        float *out = c < f ? dgamma : dbeta;
        if (out) out[c < f ? c : c - f] = (float)t;
    }
}

// How a row is dealt to lanes: as few of four columns as hold it, then more per lane.
struct Shape {
    int lanes, per;                    // lanes a row; times four columns of each
    bool wide;
};
Shape norm_shape(int f) {
    const int groups = (f + 3) / 4;
    int lanes = 1;
    while (lanes < 64 && lanes < groups) lanes <<= 1;
    int per = 1;
    while (per < 4 && lanes * per < groups) per <<= 1;
    while (lanes * per < groups) lanes <<= 1;              // up to kNormRow: 256 lanes
    return Shape{lanes, per, lanes > 64};
}
// Blocks of the backward pass, one partial row of sums each: a group of lanes adds at most 256 rows in float.
constexpr int kNormChain = 256;
int64_t norm_blocks(int64_t n, int f) {
    if (n <= 0) return 0;
    if (f > kNormRow) {                                    // a grid's y; more rows of this length no memory holds
        const int64_t blocks = ceil_div(n, kNormChain) > 64 ? ceil_div(n, kNormChain) : (n < 64 ? n : 64);
        return blocks < 65535 ? blocks : 65535;
    }
    const Shape s = norm_shape(f);
    const int64_t groups = 256 / s.lanes;
    const int64_t most = ceil_div(n, groups * 2);          // two rows a group at least
    int64_t blocks = ceil_div(n, groups * kNormChain);
    if (blocks < 1024) blocks = most < 1024 ? most : 1024;
    return blocks;
}

__global__ void rng_advance_kernel(uint64_t *state, uint64_t by) { state[1] += by; }

}  // namespace

gnn_status_t rng_advance_launch(uint64_t *state, uint64_t by, hipStream_t st) {
    hipLaunchKernelGGL(rng_advance_kernel, dim3(1), dim3(1), 0, st, state, by);
    return launch_status();
}

gnn_status_t dropout_launch(int n, int f, const float *X, const float *R, const Dropout &drop, float *Y, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    int64_t blocks = ceil_div((int64_t)n * ((f + 3) / 4), 256);
    if (blocks > 1 << 20) blocks = 1 << 20;
    hipLaunchKernelGGL(dropout_kernel, dim3((unsigned)blocks), dim3(256), 0, st, n, f, X, R, drop, Y);
    return launch_status();
}

// U_: rows at a time, and of streamed arrays, which take more loads under way
#define NORM_CASE(KERNEL_, PER_, U_, STREAM_U_, WIDE_)                                                       \
    if (shape.per == PER_ && shape.wide == WIDE_) {                                                              \
        if (mem == kStreamed) NORM_ACT(KERNEL_, PER_, STREAM_U_, kStreamed, WIDE_)                               \
        else if (mem == kAlignedRow) NORM_ACT(KERNEL_, PER_, U_, kAlignedRow, WIDE_)                             \
        else NORM_ACT(KERNEL_, PER_, U_, kAnyRow, WIDE_)                                                         \
    }
#define NORM_ACT(KERNEL_, PER_, U_, MEM_, WIDE_)                                                                 \
    {                                                                                                            \
        if (add) NORM_LAUNCH(KERNEL_, PER_, U_, kActNone, true, MEM_, WIDE_);                                    \
        else if (act == kActRelu) NORM_LAUNCH(KERNEL_, PER_, U_, kActRelu, false, MEM_, WIDE_);                  \
        else if (act == kActElu) NORM_LAUNCH(KERNEL_, PER_, U_, kActElu, false, MEM_, WIDE_);                    \
        else NORM_LAUNCH(KERNEL_, PER_, U_, kActNone, false, MEM_, WIDE_);                                       \
    }
#define NORM_LAUNCH(KERNEL_, PER_, U_, ACT_, ADD_, MEM_, WIDE_) \
    hipLaunchKernelGGL((KERNEL_<PER_, U_, ACT_, ADD_, MEM_, WIDE_>), grid, dim3(256), 0, st, a)

static int norm_memory(int64_t n, int f, bool aligned) {
    return !aligned ? kAnyRow : (size_t)n * f * sizeof(float) > kStreamBytes ? kStreamed : kAlignedRow;
}

gnn_status_t norm_forward_launch(int n, int f, const float *X, const float *R, const float *gamma, const float *beta,
                                 float eps, int act, const Dropout &drop, float *H, float *Y, float *stat, hipStream_t st) {
    if (n <= 0) return GNN_OK;
    Norm a{n, f, 0, X, R, gamma, beta, eps, act, drop, H, Y, stat};
    if (f > kNormRow) {
        hipLaunchKernelGGL(norm_forward_long_kernel, dim3((unsigned)n), dim3(256), 0, st, a);
        return launch_status();
    }
    const Shape shape = norm_shape(f);
    a.lanes = shape.lanes;
    const bool add = R != nullptr;
    const bool aligned = f % 4 == 0 && aligned16(X) && aligned16(Y) && aligned16(gamma) && aligned16(beta) &&
                         (!add || (aligned16(R) && aligned16(H)));
    const int u = shape.wide || shape.per == 4 ? 1 : shape.per == 2 ? 2 : 4, mem = norm_memory(n, f, aligned);
    int64_t blocks = ceil_div(n, 256 / shape.lanes * u);
    if (blocks > 2048) blocks = 2048;
    const dim3 grid((unsigned)blocks);
    NORM_CASE(norm_forward_kernel, 1, 4, 4, false)
    NORM_CASE(norm_forward_kernel, 2, 2, 2, false)
    NORM_CASE(norm_forward_kernel, 4, 1, 1, false)
    NORM_CASE(norm_forward_kernel, 4, 1, 1, true)
    return launch_status();
}

// not what this n takes, but what serves every smaller one as well
size_t norm_workspace_bytes(int64_t n, int64_t f) {
    const int64_t blocks = norm_blocks(n, (int)f);
    return align_up((size_t)(blocks > 1024 ? blocks : 1024) * 2 * f * sizeof(float));
}

gnn_status_t norm_backward_launch(int n, int f, const float *X, const float *stat, const float *gamma, const float *beta,
                                  int act, const Dropout &drop, bool before, const float *dY, const float *dH, float *dR,
                                  float *dX, float *dgamma, float *dbeta, void *workspace, hipStream_t st) {
    const bool sums = dgamma || dbeta, add = before;
    if (!sums && !dX && !dR) return GNN_OK;
    const int64_t blocks = norm_blocks(n, f);
    NormBack a{n, f, 0, X, stat, gamma, beta, act, drop, dY, dH, dR, dX, sums ? static_cast<float *>(workspace) : nullptr};
    if (n > 0 && f > kNormRow) {
        if (sums) {                                        // before dX, which may lie over dY
            hipLaunchKernelGGL(norm_sums_long_kernel, dim3((unsigned)ceil_div(f, 1024), (unsigned)blocks), dim3(256), 0, st, a, !before);
            GNN_TRY(launch_status());
        }
        if (dR || dX) hipLaunchKernelGGL(norm_backward_long_kernel, dim3((unsigned)n), dim3(256), 0, st, a, before);
    } else if (n > 0) {
        const Shape shape = norm_shape(f);
        a.lanes = shape.lanes;
        const bool aligned = f % 4 == 0 && aligned16(X) && aligned16(dY) && aligned16(gamma) && aligned16(beta) &&
                             aligned16(dX) && aligned16(dR) && aligned16(dH);
        const int mem = norm_memory(n, f, aligned);
        const dim3 grid((unsigned)blocks);
        NORM_CASE(norm_backward_kernel, 1, 2, 4, false)
        NORM_CASE(norm_backward_kernel, 2, 1, 2, false)
        NORM_CASE(norm_backward_kernel, 4, 1, 1, false)
        NORM_CASE(norm_backward_kernel, 4, 1, 1, true)
    }
    GNN_TRY(launch_status());
    if (!sums) return GNN_OK;
    hipLaunchKernelGGL(norm_sums_final_kernel, dim3((unsigned)ceil_div(2 * (int64_t)f, 16)), dim3(1024), 0, st, f, (int)blocks,
                       a.part, dgamma, dbeta);
    return launch_status();
}
#undef NORM_CASE
#undef NORM_ACT
#undef NORM_LAUNCH

}  // namespace gnn
