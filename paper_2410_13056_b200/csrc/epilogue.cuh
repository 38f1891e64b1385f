// What stands behind a product in a layer: activations in fp32, and the types that select them.
#pragma once

#include "common.cuh"

namespace cmpq {

inline bool act_ok(cmpq_act a) { return a >= CMPQ_ACT_NONE && a <= CMPQ_ACT_GELU_TANH; }

// z / (1 + e^-w).  The fast exponential is off by 2 + 1.173 |w| units of 2^-23, relative to e^-w, of which the quotient takes
// over at most e^-w / (1 + e^-w), and the fast quotient by 2: far inside the rounding to 16 bits behind it.  Where e^-w
// passes 2^126 the quotient is 0.
__device__ __forceinline__ float gate_by(float z, float w) { return __fdividef(z, 1.0f + __expf(-w)); }

// z Phi(z).  With t = |z| and s = 1 / (1 + t / sqrt(8)), Phi(-t) = s P(s) e^(-t^2/2), P a polynomial of degree 8 fitted to
// erfcx(t / sqrt(2)) / (2 s) for t up to 14, by least squares with weights raised where it was worst: with the coefficients as
// they stand here, off by 9.3e-8 of its value, and with the roundings of float32 3.1e-7.  Relative accuracy is kept where Phi is
// small, for which a library call takes three times as long: a layer of 53 tokens 4096 -> 11008 took 15.1 us with it, 13.4 so, 12.0
// with silu; 4000 tokens 201, 172 and 145.  Infinity stays so, and t is held where its square is finite.
__device__ __forceinline__ float by_normal(float z) {
    const float t = fminf(fabsf(z), 1e18f), s = __fdividef(1.0f, __fmaf_rn(0.353553385f, t, 1.0f));
    float p = -0.0295344833f;
    p = __fmaf_rn(p, s, 0.142287493f);
    p = __fmaf_rn(p, s, -0.243599981f);
    p = __fmaf_rn(p, s, 0.139033601f);
    p = __fmaf_rn(p, s, -0.0133128483f);
    p = __fmaf_rn(p, s, 0.101343438f);
    p = __fmaf_rn(p, s, 0.121551879f);
    p = __fmaf_rn(p, s, 0.141187653f);
    p = __fmaf_rn(p, s, 0.141043216f);
    const float tail = t * (p * s * __expf(-0.5f * t * t));
    return z < 0.0f ? -tail : z - tail;
}

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if (ACT == CMPQ_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == CMPQ_ACT_SILU) return gate_by(z, z);
    if (ACT == CMPQ_ACT_GELU) return by_normal(z);
    // 0.5 z (1 + tanh(w / 2)) = z / (1 + e^-w), w = sqrt(8/pi) (z + 0.044715 z^3)
    if (ACT == CMPQ_ACT_GELU_TANH) return gate_by(z, z * __fmaf_rn(0.0713548163f, z * z, 1.59576912f));
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
