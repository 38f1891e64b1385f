// What stands behind a product in a layer: activations in fp32, and the types that select them.
#pragma once

#include "common.cuh"

namespace cmpq {

inline bool act_ok(cmpq_act a) { return a >= CMPQ_ACT_NONE && a <= CMPQ_ACT_GELU_TANH; }

// z / (1 + e^-w).  The fast exponential is off by 2 + 1.173 |w| units of 2^-23, relative to e^-w, of which the quotient takes
// over at most e^-w / (1 + e^-w), and the fast quotient by 2: far inside the rounding to 16 bits behind it.  Where e^-w
// passes 2^126 the quotient is 0.
__device__ __forceinline__ float gate_by(float z, float w) { return __fdividef(z, 1.0f + __expf(-w)); }

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if (ACT == CMPQ_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == CMPQ_ACT_SILU) return gate_by(z, z);
    // z Phi(z): by the complement, which keeps its relative accuracy where Phi is small
    if (ACT == CMPQ_ACT_GELU) return 0.5f * z * erfcf(-0.707106781f * z);
    // 0.5 z (1 + tanh(w / 2)) = z / (1 + e^-w), w = sqrt(8/pi) (z + 0.044715 z^3)
    if (ACT == CMPQ_ACT_GELU_TANH) return gate_by(z, 1.59576912f * (z + 0.044715f * z * z * z));
    return z;
}

template <int A>
struct ActIs {
    static constexpr int value = A;
};
// f(ActIs<ACT>()) for the activation of a launch: one branch around a loop instead of one in it.
template <class F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case CMPQ_ACT_RELU: return f(ActIs<CMPQ_ACT_RELU>());
        case CMPQ_ACT_SILU: return f(ActIs<CMPQ_ACT_SILU>());
        case CMPQ_ACT_GELU: return f(ActIs<CMPQ_ACT_GELU>());
        case CMPQ_ACT_GELU_TANH: return f(ActIs<CMPQ_ACT_GELU_TANH>());
        default: return f(ActIs<CMPQ_ACT_NONE>());
    }
}

}  // namespace cmpq
