// Activations of the products' epilogues and their slopes, in fp32.  The numbers are terra.h's TERRA_ACT_*.
#pragma once
#include "../../include/terra.h"
#include "swin_common.cuh"

namespace terra {

__device__ __forceinline__ float fast_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sigmoid(float x) { return fast_rcp(1.f + fast_exp2(-kLog2e * x)); }

// exp(-x^2 / 2) and the normal distribution's lower tail beyond |x|, half erfc(|x| / sqrt 2): erfc(z) exp(z^2) as a polynomial of
// t = 1 / (1 + 0.65 z), the form of Abramowitz and Stegun 7.1.26 with the coefficients fitted here (linear programming over z = 0 .. 12) for the least
// relative error, 9e-6: a fiftieth of fp16's half step, far into the tail.  (Their own, with an absolute bound, lose the tail.)
__device__ __forceinline__ void normal_tail(float x, float& bell, float& tail) {
    const float t = fast_rcp(fmaf(fabsf(x), 0.65f * 0.70710678f, 1.f));
    bell = fast_exp2(x * x * (-0.5f * kLog2e));
    float g = 0.5f * 0.14364023f;
    g = fmaf(g, t, 0.5f * -0.47167895f);
    g = fmaf(g, t, 0.5f * 0.35566068f);
    g = fmaf(g, t, 0.5f * 0.23218703f);
    g = fmaf(g, t, 0.5f * 0.37380508f);
    g = fmaf(g, t, 0.5f * 0.36639139f);
    tail = g * t * bell;
}

constexpr float kGeluTanhA = 0.7978845608028654f;      // sqrt(2 / pi)
constexpr float kGeluTanhB = 0.044715f;

template <int ACT>
__device__ __forceinline__ float act(float z) {
    if (ACT == TERRA_ACT_RELU) return z < 0.f ? 0.f : z;
    if (ACT == TERRA_ACT_SILU) return z * sigmoid(z);
    if (ACT == TERRA_ACT_GELU) {
        float bell, tail;
        normal_tail(z, bell, tail);
        return z * (z < 0.f ? tail : 1.f - tail);
    }
    // 0.5 z (1 + tanh u) = z sigmoid(2 u)
    if (ACT == TERRA_ACT_GELU_TANH) return z * sigmoid(2.f * kGeluTanhA * z * fmaf(kGeluTanhB, z * z, 1.f));
    return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if (ACT == TERRA_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    if (ACT == TERRA_ACT_SILU) {
        const float s = sigmoid(z), c = fminf(fmaxf(z, -100.f), 100.f);      // beyond, s (1 - s) is 0 and z may be infinite
        return s + c * s * (1.f - s);
    }
    if (ACT == TERRA_ACT_GELU) {
        float bell, tail;
        normal_tail(z, bell, tail);
        const float c = fminf(fmaxf(z, -100.f), 100.f);
        return fmaf(c * 0.3989422804f, bell, z < 0.f ? tail : 1.f - tail);
    }
    if (ACT == TERRA_ACT_GELU_TANH) {
        const float s = sigmoid(2.f * kGeluTanhA * z * fmaf(kGeluTanhB, z * z, 1.f)), c = fminf(fmaxf(z, -100.f), 100.f);
        return s + c * s * (1.f - s) * (2.f * kGeluTanhA) * fmaf(3.f * kGeluTanhB, c * c, 1.f);
    }
    return 1.f;
}

// f(integral constant of the activation)
template <int N> struct ActTag { static constexpr int value = N; };
template <class F>
__device__ __forceinline__ void with_act(int activation, F f) {
    switch (activation) {
        case TERRA_ACT_RELU: f(ActTag<TERRA_ACT_RELU>()); break;
        case TERRA_ACT_SILU: f(ActTag<TERRA_ACT_SILU>()); break;
        case TERRA_ACT_GELU: f(ActTag<TERRA_ACT_GELU>()); break;
        case TERRA_ACT_GELU_TANH: f(ActTag<TERRA_ACT_GELU_TANH>()); break;
        default: f(ActTag<TERRA_ACT_NONE>()); break;
    }
}

}  // namespace terra
