// A float as the sum of two fp16 numbers in one scale, for the products of pair_product.hip and pair_tn.hip.
//
// A row of one operand and a column of the other are taken times a power of two each that brings their largest magnitude to
// 2^14 .. 2^15 (to 1 at least where it is below 2^-112 and no subnormal), and every element is then h + l: h rounds it to 11 bits and l
// rounds the rest to 11 bits.  What is left out is at most 2^-23 of the element, 2^-25.5 in the mean.  Three of the four products are
// formed (l l, at most 2^-22 of the whole, is not), all into one sum: v_mfma_f32_32x32x16_f16 three times for 16 indices.  half_parts.h,
// which takes l times 2^11 and needs a sum of its own for h l + l h, holds small elements to 2^-50 of the largest of their row (column);
// here it is 2^-40: l is no finer than 2^-25 beside 2^14, which begins at 2^-16 of the largest.  (Where that is below 2^-112 what is left
// out is at most 2^-151, a quarter of the least float.  The instruction and the conversions take subnormal fp16 numbers as they are.)
// X^T D over 4096 rows, eight of D's 2^16 times the others and met by zeros, emulated: 5.1e-7 off in the 2-norm, in two scales 4.8e-7, as a
// chain of floats 1.1e-6; 2^20 times 1.4e-6, 4.7e-7, 1.1e-6; 2^24 times 2.2e-5.  For that a step of 32 indices spares 32 of its 128
// vector instructions, and a wavefront the registers for twice the sums.
// Infinities and NaN are taken as they are and come out as NaN, upon which a wavefront forms its tiles again with the fp32
// instruction.
#pragma once

#include "half_parts.h"

namespace gnn {
namespace half_pair {

using half_parts::float4u;
using half_parts::floatx2;
using half_parts::floatx4;
using half_parts::floatx16;
using half_parts::half2v;
using half_parts::half8;
using half_parts::power_of_two;
using half_parts::xcd_tile;

constexpr int KP = 16;                 // indices of a step: one instruction
constexpr int kPairBytes = 2 * 64 * 16;          // [part][lane][8] of 32 columns and a step

// e with 2^e times the magnitude in 2^14 .. 2^15; 0 for zero, infinities and NaN.  At most 126: the least float comes to 2^-23, so that
// h + l is exact for subnormal rows.  (half_parts.h stops at 115, since it needs 2^(e + 11) as well: here a row of 2^-125 would come to
// 2^-10, and with l no finer than 2^-24 to fourteen bits.)
__device__ __forceinline__ int exponent_of(unsigned top) {
    if (top == 0 || top >= 0x7f800000u) return 0;
    return min(14 + 127 - (int)(top >> 23), 126);
}

// both parts of eight floats times s.  x s is exact, so h is rounded once, and so is x s - h.
__device__ __forceinline__ void pairs8(const float (&x)[8], float s, half8 (&part)[2]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const floatx2 a = {x[i] * s, x[i + 1] * s};
        const half2v h = __builtin_convertvector(a, half2v);
        const floatx2 r = {fmaf((float)h[0], -1.f, a[0]), fmaf((float)h[1], -1.f, a[1])};
        const half2v q = __builtin_convertvector(r, half2v);
        part[0][i] = h[0];
        part[0][i + 1] = h[1];
        part[1][i] = q[0];
        part[1][i + 1] = q[1];
    }
}

}  // namespace half_pair
}  // namespace gnn
