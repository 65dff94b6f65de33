// Rows of an array in 8 bits: integers of -127 .. 127 and a scale for each row.
#pragma once

#include "common.h"

namespace gnn {

// A gnn_rows8_t as the kernels take it, rows rows8_stride(f) bytes apart.
struct Rows8 {
    int8_t *q;
    float *scale;
    const float *columns;              // or NULL
};
static inline Rows8 no_rows8() { return Rows8{nullptr, nullptr, nullptr}; }
__host__ __device__ constexpr int64_t rows8_stride(int64_t f) { return (f + 15) / 16 * 16; }

// What a row's largest magnitude makes of it: x becomes round((x up) per_unit), each product rounded to a float, and stands for that
// times unit / up.  `up` brings the least floats to where their quotients are floats too, and is 1 for others.
struct Held8 {
    float up, per_unit, unit;
    bool lost;                         // an infinity or a NaN among them: integers 0, unit NaN
    __device__ __forceinline__ explicit Held8(unsigned top) {
        lost = top >= 0x7f800000u;
        up = top < 0x0d800000u ? 0x1p64f : 1.f;            // below 2^-100
        const float a = __uint_as_float(top) * up;
        per_unit = top ? 127.f / a : 0.f;
        unit = lost ? __uint_as_float(0x7fc00000u) : a / 127.f;
    }
    __device__ __forceinline__ unsigned one(float x) const {
#pragma clang fp contract(off)
        const float t = x * up * per_unit;                 // at most 127 (1 + 2^-23)
        return __float_as_uint(t + 12582912.f) & 255u;     // 1.5 2^23: the sum's last bits are t, rounded, ties to even
    }
    __device__ __forceinline__ unsigned four(float4 v) const {
        return lost ? 0u : one(v.x) | one(v.y) << 8 | one(v.z) << 16 | one(v.w) << 24;
    }
};
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ unsigned largest(float4 v) {
    return max(max(magnitude(v.x), magnitude(v.y)), max(magnitude(v.z), magnitude(v.w)));
}
// the four integers of a word
__device__ __forceinline__ float4 integers(unsigned w) {
    return make_float4((float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24));
}

}  // namespace gnn
