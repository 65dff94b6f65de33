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
    if constexpr (ACT == kActRelu) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;       // NaN stays
    if constexpr (ACT == kActElu) return z > 0.f ? 1.f : exp_down(z);      // NaN stays
    return 1.f;
}
__device__ __forceinline__ float activation(float z, int act) {
    return act == kActRelu ? activation<kActRelu>(z) : act == kActElu ? activation<kActElu>(z) : z;
}
__device__ __forceinline__ float slope(float z, int act) {
    return act == kActRelu ? slope<kActRelu>(z) : act == kActElu ? slope<kActElu>(z) : 1.f;
}

// Phi(z) of the normal distribution, and exp(-z^2 / 2).  Below zero Phi(-a) = exp(-a^2 / 2) Q(t) with t = 1 / (1 + 0.345 a), and Q is t
// times a polynomial of degree 8 (found by reweighted least squares on Chebyshev points over 0 <= a <= 14: largest relative error 2.0e-8, and
// 5.7e-8, 0.95 x 2^-24, with the coefficients rounded to floats).  In units of 2^-24 of it Phi is off by at most 15 + 1.5 z^2 below zero,
// of which 1.5 z^2 are three roundings of -z^2 / 2, 7 those of t and 7 the other steps', and above zero by 16.  Measured, z Phi(z): 7.3 near
// zero on either side, 14 at -3.5, 128 at -12.4, 3.4 from 0.5 on and 2.2 from 1 on.
__device__ __forceinline__ void normal_integral(float z, float &phi, float &bell) {
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.345f, 1.f));
    float q = fmaf(-0.02838203945231031f, t, 0.14528229325785152f);
    q = fmaf(q, t, -0.2711736111261439f);
    q = fmaf(q, t, 0.18719713317870015f);
    q = fmaf(q, t, -0.03760189167020016f);
    q = fmaf(q, t, 0.11179965379086171f);
    q = fmaf(q, t, 0.11723827857890808f);
    q = fmaf(q, t, 0.13802088561997014f);
    q = fmaf(q, t, 0.1376192904176441f);
    bell = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    const float below = q * t * bell;
    phi = z > 0.f ? 1.f - below : below;
}

// Every gnn_act_t, and its derivative where that is asked for.  The sigmoid is off by (2 + |z|) units in the last place, as if z were off by
// one, and Phi likewise: four and eighteen instructions, where those of gate_of, exact where the gate shuts, take nineteen and fifty.  In
// the epilogue of a product such instructions count: they are not hidden behind the loads and stores of an element.
template <int ACT, bool SLOPE>
__device__ __forceinline__ void activate(float z, float &y, float &dy) {
    if constexpr (ACT == GNN_ACT_SIGMOID || ACT == GNN_ACT_SILU) {
        const float e = __builtin_amdgcn_exp2f(z * -1.44269504088896341f), s = __builtin_amdgcn_rcpf(1.f + e);
        y = ACT == GNN_ACT_SILU ? z * s : s;
        if constexpr (SLOPE) {
            const float shut = z > 0.f ? e * s : 1.f - s;  // s(-z); e may be infinite below zero
            dy = ACT == GNN_ACT_SILU ? s * fmaf(z, shut, 1.f) : s * shut;
        }
    } else if constexpr (ACT == GNN_ACT_GELU) {
        float phi, bell;
        normal_integral(z, phi, bell);
        y = z * phi;
        if constexpr (SLOPE) dy = fmaf(z * 0.39894228040143268f, bell, phi);
    } else {
        y = activation<ACT>(z);
        if constexpr (SLOPE) dy = slope<ACT>(z);
    }
}

}  // namespace gnn
