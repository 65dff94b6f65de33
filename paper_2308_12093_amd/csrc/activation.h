// Activations and their derivatives.
#pragma once

#include "gated.h"

namespace gnn {

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

// Every gnn_act_t, and its derivative where that is asked for.
template <int ACT, bool SLOPE>
__device__ __forceinline__ void activate(float z, float &y, float &dy) {
    if constexpr (ACT == GNN_ACT_SIGMOID || ACT == GNN_ACT_SILU || ACT == GNN_ACT_GELU) {
        gate_of<ACT == GNN_ACT_SIGMOID ? GNN_GATE_SIGMOID : ACT == GNN_ACT_SILU ? GNN_GATE_SILU : GNN_GATE_GELU, SLOPE>(z, y, dy);
    } else {
        y = activation<ACT>(z);
        if constexpr (SLOPE) dy = slope<ACT>(z);
    }
}

}  // namespace gnn
