// The activation of a gated block, for the kernels that form [A | U] and those that read it.
#pragma once

#include "common.h"

namespace gnn {

// What becomes of [A | U] = X W + b, n rows of 2 half columns, in the kernel that forms it.
struct Gated {
    int half;
    int gate;                          // gnn_gate_t
    float *H, *Z;                      // forward: H = act(A) .* U, and [A | U] itself unless NULL
    const float *dH;                   // backward: D = [dH .* U .* act'(A) | dH .* act(A)]
    float *D;
};

// act(a) and, where asked for, act'(a).  Phi by erfc, which keeps its relative precision where the gate shuts.
template <int GATE, bool SLOPE>
__device__ __forceinline__ void gate_of(float a, float &g, float &dg) {
    if constexpr (GATE == GNN_GATE_GELU) {
        const float below = 0.5f * erfcf(a * -0.70710678118654752f);
        g = a * below;
        if constexpr (SLOPE) dg = fmaf(a * 0.39894228040143268f, expf(-0.5f * a * a), below);
    } else {
        // one exponential for s(a) = 1 / (1 + exp(-a)) and s(-a) = 1 - s(a), neither of which loses its precision then
        const float e = expf(-fabsf(a)), t = __builtin_amdgcn_rcpf(1.f + e), r = e * t;
        const float s = a > 0.f ? t : r, shut = a > 0.f ? r : t;
        g = GATE == GNN_GATE_SILU ? a * s : s;
        if constexpr (SLOPE) dg = GATE == GNN_GATE_SILU ? s * fmaf(a, shut, 1.f) : s * shut;
    }
}

}  // namespace gnn
