// Rows of fp32 arrays in the registers of a wavefront's or a block's lanes: how they are dealt, read, summed over and written.
#pragma once

#include "common.h"

namespace gnn {
namespace rows {

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

// 1 / sqrt(x): the instruction's, and a Newton step (an IEEE division and root take thirty instructions, for each lane of a row)
__device__ __forceinline__ float inverse_root(float x) {
    const float y = __builtin_amdgcn_rsqf(x);
    const float r = fmaf(fmaf(-0.5f * x * y, y, 0.5f), y, y);
    return x > 0x1p-100f && x < 0x1p100f ? r : y;          // x y y keeps its range there; infinities and NaN as they are
}

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

// columns of the longest row that stays in registers
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

// How a row is dealt to lanes: as few of four columns as hold it, then more per lane.
struct Shape {
    int lanes, per;                    // lanes a row; times four columns of each
    bool wide;
};
inline Shape norm_shape(int f) {
    const int groups = (f + 3) / 4;
    int lanes = 1;
    while (lanes < 64 && lanes < groups) lanes <<= 1;
    int per = 1;
    while (per < 4 && lanes * per < groups) per <<= 1;
    while (lanes * per < groups) lanes <<= 1;              // up to kNormRow: 256 lanes
    return Shape{lanes, per, lanes > 64};
}
// Blocks of a backward pass, one partial row of sums each: a group of lanes adds at most 256 rows in float.
constexpr int kNormChain = 256;
inline int64_t norm_blocks(int64_t n, int f) {
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

static inline int norm_memory(int64_t n, int f, bool aligned) {
    return !aligned ? kAnyRow : (size_t)n * f * sizeof(float) > kStreamBytes ? kStreamed : kAlignedRow;
}

}  // namespace rows
}  // namespace gnn
