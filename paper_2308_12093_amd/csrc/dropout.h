// Dropout whose mask is a function of (seed, step, site, row, column), computed where it is used and stored nowhere.
#pragma once

#include "common.h"

namespace gnn {

// A gnn_dropout_t as the kernels take it.  below = 0: nothing is dropped, and the state is not read.
struct Dropout {
    const uint64_t *state;             // device: {seed, step}
    uint32_t site;
    uint32_t below;                    // an element stays where its word is at least this: p 2^32
    float scale;                       // 1 / (1 - p)
};

// Philox4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): a
// bijection of the 128-bit counter for each 64-bit key.  A round is two 32 x 32 -> 64 bit multiplications, whose high halves
// go through an exclusive or with the other two words and the round's key.
__device__ __forceinline__ uint4 philox4x32(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

// The words of a launch: one block of four per four columns of a row, so that rows of any length begin with a block.
struct DropoutWords {
    uint32_t k0, k1, step, site, below;
    float scale;
    __device__ __forceinline__ explicit DropoutWords(const Dropout &d)
        : k0(0), k1(0), step(0), site(d.site), below(d.below), scale(d.scale) {
        if (!below) return;                                // uniform
        const uint64_t seed = d.state[0];
        k0 = (uint32_t)seed;
        k1 = (uint32_t)(seed >> 32);
        step = (uint32_t)d.state[1];
    }
    // columns 4 group .. 4 group + 3 of a row, dropped or scaled.  A dropped infinity or NaN is zero too.
    __device__ __forceinline__ float4 apply(float4 x, uint32_t row, uint32_t group) const {
        if (!below) return x;
        const uint4 u = philox4x32(make_uint4(group, row, site, step), k0, k1);
        return make_float4(u.x < below ? 0.f : x.x * scale, u.y < below ? 0.f : x.y * scale, u.z < below ? 0.f : x.z * scale,
                           u.w < below ? 0.f : x.w * scale);
    }
};

}  // namespace gnn
