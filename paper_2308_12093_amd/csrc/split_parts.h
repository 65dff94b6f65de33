// A float as the exact sum of three bf16 numbers, for products on the bf16 matrix instruction (see gemm_split.hip).
#pragma once

#include "common.h"

namespace gnn {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
    return __builtin_bit_cast(unsigned, __builtin_convertvector((floatx2){a, b}, bf16x2));
}
__device__ __forceinline__ float low(unsigned u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float high(unsigned u) { return __uint_as_float(u & 0xffff0000u); }

// orders like the magnitude, except that zero comes last
__device__ __forceinline__ unsigned magnitude_code(float a) { return 2 * __float_as_uint(a) - 1; }

// three parts of eight floats; LEAST: `least` collects the smallest magnitude code
template <bool LEAST = true>
__device__ __forceinline__ void split8(const floatx4 &x, const floatx4 &y, bf16x8 (&part)[3], unsigned &least) {
    uintx4 u[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = i < 2 ? x[2 * i] : y[2 * i - 4], b = i < 2 ? x[2 * i + 1] : y[2 * i - 3];
        if constexpr (LEAST) least = min(least, min(magnitude_code(a), magnitude_code(b)));
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const unsigned h = pack_bf16(a, b);
            u[p][i] = h;
            if (p < 2) { a -= low(h); b -= high(h); }
        }
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) part[p] = __builtin_bit_cast(bf16x8, u[p]);
}

// the kept products, smallest first; the last, of the leading parts, goes to the sum itself
constexpr int kProducts = 6;
__device__ constexpr int kPartA[kProducts] = {1, 0, 2, 1, 0, 0}, kPartB[kProducts] = {1, 2, 0, 0, 1, 0};

constexpr int kFragBytes = 64 * 16;    // eight bf16 per lane: one operand of one instruction

}  // namespace gnn
