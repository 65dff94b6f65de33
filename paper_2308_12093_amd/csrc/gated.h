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
template <bool SLOPE>
__device__ __forceinline__ void gate_of(int gate, float a, float &g, float &dg) {
    if (gate == GNN_GATE_GELU) {
        const float below = 0.5f * erfcf(a * -0.70710678118654752f);
        g = a * below;
        if constexpr (SLOPE) dg = fmaf(a * 0.39894228040143268f, expf(-0.5f * a * a), below);
        return;
    }
    const float s = 1.f / (1.f + expf(-a));
    const float t = gate == GNN_GATE_SILU ? a : 1.f;
    g = t * s;
    // s' = s (1 - s); 1 - s would lose what is left of an open gate, so exp(-a) s takes its place where a > 0
    if constexpr (SLOPE) {
        const float shut = a > 0.f ? 1.f / (1.f + expf(a)) : 1.f - s;
        dg = gate == GNN_GATE_SILU ? s * fmaf(a, shut, 1.f) : s * shut;
    }
}

}  // namespace gnn
