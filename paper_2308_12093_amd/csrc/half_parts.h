// A float as the sum of two fp16 numbers, for the products of gemm_half.hip and gemm_half_tn.hip.
//
// A row of one operand and a column of the other are taken times a power of two each that brings their largest magnitude to
// 2^14 .. 2^15, and every element is then the sum of two fp16 numbers, h + 2^-11 l: h rounds it to 11 bits and l rounds the
// rest, times 2^11, to 11 bits.  What is left out is at most 2^-23 of the element, 2^-25.5 in the mean.  Products of two fp16
// numbers are exact in float; three of the four are formed (l l, at most 2^-22 of the whole, is not) and added in float:
// v_mfma_f32_32x32x16_f16 for h h, and for h l + l h into a sum of their own, which joins the other every 32 indices times 2^-11.
// That is three instructions of 32 cycles for 16 indices, half of what three bf16 parts take (gemm_split.hip), a sixth of the
// fp32 instruction's time.
//
// So a product is off by up to 8 u, 1.2 u in the root mean square, where one of floats is off by u = 2^-24 at most; sums of 32 and
// more make up for it by their fewer roundings (kShortReduction in gemm_half.h).
//
// Small elements are held to 2^-50 of their row's (column's) largest, where that is more: l is no finer than 2^-25, 2^-36 of what it
// stands for, beside 2^14 and more.  That begins at 2^-27 of the largest.  The power of two is taken back exactly.
// Infinities and NaN are taken as they are and come out as NaN, upon which a wavefront forms its tile again with the fp32
// instruction.
#pragma once

#include "gemm_half.h"

namespace gnn {
namespace half_parts {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

constexpr int KB = 32;                 // indices of a step: two instructions of 16
constexpr int kFragBytes = 64 * 16;    // eight fp16 per lane: one operand of one instruction
constexpr int kTileBytes = 4 * kFragBytes;       // [instruction][part] of 32 columns and a step

// e with 2^e times the magnitude in 2^14 .. 2^15; 0 for zero, infinities and NaN.  At most 115: 2^(e + 11) is a float as well.
__device__ __forceinline__ int exponent_of(unsigned top) {
    if (top == 0 || top >= 0x7f800000u) return 0;
    return min(14 + 127 - (int)(top >> 23), 115);
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }

// the two parts of two floats (i, i + 1 of eight) times s; s2 = 2^11 s.  x s is exact, so h is rounded once, and so is
// x s2 - 2^11 h.
__device__ __forceinline__ void halves2(const float (&x)[8], int i, float s, float s2, half8 (&part)[2]) {
    const floatx2 a = {x[i] * s, x[i + 1] * s};
    const half2v h = __builtin_convertvector(a, half2v);
    const floatx2 r = {fmaf((float)h[0], -2048.f, x[i] * s2), fmaf((float)h[1], -2048.f, x[i + 1] * s2)};
    const half2v q = __builtin_convertvector(r, half2v);
    part[0][i] = h[0];
    part[0][i + 1] = h[1];
    part[1][i] = q[0];
    part[1][i + 1] = q[1];
}
__device__ __forceinline__ void halves8(const float (&x)[8], float s, float s2, half8 (&part)[2]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) halves2(x, i, s, s2, part);
}

// a tile's products of 16 INS indices: acc += h h + 2^-11 (h l + l h)
template <int INS>
__device__ __forceinline__ void multiply(floatx16 &acc, const half8 (&a)[INS][2], const half8 (&b)[INS][2]) {
    floatx16 small;
#pragma unroll
    for (int v = 0; v < 16; ++v) small[v] = 0.f;
#pragma unroll
    for (int ins = 0; ins < INS; ++ins) {
        small = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[ins][1], b[ins][0], small, 0, 0, 0);
        small = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[ins][0], b[ins][1], small, 0, 0, 0);
    }
#pragma unroll
    for (int ins = 0; ins < INS; ++ins) acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[ins][0], b[ins][0], acc, 0, 0, 0);
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = fmaf(small[v], 0x1p-11f, acc[v]);
}

// a block's tile: each XCD (ids are dealt round-robin to eight) takes a contiguous range
__device__ __forceinline__ long xcd_tile(long total) {
    const long per = (total + 7) / 8;
    return blockIdx.x / 8 < per ? (long)(blockIdx.x % 8) * per + blockIdx.x / 8 : total;
}

}  // namespace half_parts
}  // namespace gnn
