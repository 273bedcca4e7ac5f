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

// Phi(x), the normal distribution's integral, and e^(-x^2 / 2), sqrt(2 pi) times its density.  1 + erf(x / sqrt 2) cancels for negative gates (4 % off at -5 and
// nothing at -5.5), so the tail is computed, Phi(-|x|) = e^(-x^2 / 2) q(t) with t = 1 / (1 + 0.4 |x|): q, of degree 8, was fitted to the least relative error of
// e^(x^2 / 2) Phi(-x) from 0 to 14 (0.7 of an ulp, 3.1 with its roundings in fp32; its last coefficient such that Phi(0) is
// 1/2), and the exponential is the slope's too.  bf16 gated (2048, 2048, 4096) takes 71.0 us with it,
// 73.5 with the device library's erf, and 2.7 % more than that with its complementary error function.
__device__ __forceinline__ float gate_normal_share(float x, float& density) {
    density = __builtin_amdgcn_exp2f(x * x * -0.72134752044448f);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.4f, __builtin_fabsf(x), 1.f));
    constexpr float q[9] = {-1.19876985e-5f, 0.159904182f, 0.155786574f, 0.158416808f, -0.0123865642f, 0.250974923f, -0.373684853f, 0.200602099f, -0.0396011882f};
    float p = q[8];
#pragma unroll
    for (int i = 7; i >= 0; --i) p = __builtin_fmaf(p, t, q[i]);
    const float tail = density * p;
    return x < 0.f ? tail : 1.f - tail;
}

__device__ __forceinline__ float gate_value(int activation, float x) {
    if (activation == GATE_SILU) return x * gate_sigmoid(x);
    float density;
    if (activation == GATE_GELU) return x * gate_normal_share(x, density);
    return x * gate_tanh_share(x);
}

// d/dgate and d/dup of act(gate) * up, times `out`'s gradient
__device__ __forceinline__ void gate_grad(int activation, float x, float up, float out, float& grad_gate, float& grad_up) {
    float share, slope;    // act(x) = x * share, act'(x) = share + slope
    if (activation == GATE_SILU) {
        share = gate_sigmoid(x);
        slope = x * (share * (1.f - share));
    } else if (activation == GATE_GELU) {
        float density;
        share = gate_normal_share(x, density);
        slope = x * (0.398942280401433f * density);
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
