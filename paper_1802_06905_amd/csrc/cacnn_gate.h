// The activations of the gated projection, in 32 bits.
#ifndef CACNN_GATE_H
#define CACNN_GATE_H

#include <hip/hip_runtime.h>

namespace cacnn {

enum { GATE_SILU = 0, GATE_GELU = 1, GATE_GELU_TANH = 2 };

// 1 / (1 + e^-x) from the hardware's power of two and reciprocal, each within an ulp: 0 where it is below 2^-126 (x < -87.3; the reciprocal has no
// subnormal results), 1 where e^-x vanishes
__device__ __forceinline__ float gate_sigmoid(float x) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.44269504088896f));
}

// 0.5 (1 + tanh y) = sigmoid(2 y), y = sqrt(2 / pi) (x + 0.044715 x^3)
__device__ __forceinline__ float gate_tanh_share(float x) { return gate_sigmoid(1.59576912160573f * x * (1.f + 0.044715f * x * x)); }

// Phi(x), the normal distribution's integral, from the complement: 1 + erf(x / sqrt 2) cancels for negative gates, 4 % off at -5 and nothing at -5.5
__device__ __forceinline__ float gate_normal_share(float x) { return 0.5f * erfcf(x * -0.70710678118655f); }

__device__ __forceinline__ float gate_value(int activation, float x) {
    if (activation == GATE_SILU) return x * gate_sigmoid(x);
    if (activation == GATE_GELU) return x * gate_normal_share(x);
    return x * gate_tanh_share(x);
}

// d/dgate and d/dup of act(gate) * up, times `out`'s gradient
__device__ __forceinline__ void gate_grad(int activation, float x, float up, float out, float& grad_gate, float& grad_up) {
    float share, slope;    // act(x) = x * share, act'(x) = share + slope
    if (activation == GATE_SILU) {
        share = gate_sigmoid(x);
        slope = x * (share * (1.f - share));
    } else if (activation == GATE_GELU) {
        share = gate_normal_share(x);
        slope = x * (0.398942280401433f * __builtin_amdgcn_exp2f(x * x * -0.72134752044448f));
    } else {
        share = gate_tanh_share(x);
        const float s = share * (1.f - share);
        // (far out s is 0 and the square infinite)
        slope = s == 0.f ? 0.f : x * s * (1.59576912160573f * (1.f + 0.134145f * x * x));
    }
    grad_gate = out * up * (share + slope);
    grad_up = out * (x * share);
}

}  // namespace cacnn
#endif
