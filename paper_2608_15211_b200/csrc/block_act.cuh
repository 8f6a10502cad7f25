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
constexpr float kGeluTanhA = 0.7978845608028654f;      // sqrt(2 / pi)
constexpr float kGeluTanhB = 0.044715f;

// (lo, hi) += the two elements of v, one instruction each (sm_100)
__device__ __forceinline__ void add_elems(float& lo, float& hi, uint32_t v) {
#ifdef TERRA_ELEM_F16
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.f16 %0, l, %0;\n\tadd.rn.f32.f16 %1, h, %1;\n\t}\n" : "+f"(lo), "+f"(hi) : "r"(v));
#else
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.bf16 %0, l, %0;\n\tadd.rn.f32.bf16 %1, h, %1;\n\t}\n" : "+f"(lo), "+f"(hi) : "r"(v));
#endif
}

// Two values at a time: one instruction for a pair of additions or products (sm_100).
typedef unsigned long long Pair;                       // two fp32
__device__ __forceinline__ Pair pair_of(float a, float b) { Pair p; asm("mov.b64 %0, {%1, %2};\n" : "=l"(p) : "f"(a), "f"(b)); return p; }
__device__ __forceinline__ Pair both(float a) { return pair_of(a, a); }
__device__ __forceinline__ void split_pair(Pair p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;\n" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ Pair pfma(Pair a, Pair b, Pair c) { Pair d; asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ Pair padd(Pair a, Pair b) { Pair d; asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ Pair pmul(Pair a, Pair b) { Pair d; asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ Pair prcp(Pair p) { float a, b; split_pair(p, a, b); return pair_of(fast_rcp(a), fast_rcp(b)); }
__device__ __forceinline__ Pair pexp2(Pair p) { float a, b; split_pair(p, a, b); return pair_of(fast_exp2(a), fast_exp2(b)); }
// |x| up to `most`, a NaN stays one
__device__ __forceinline__ float abs_upto(float x, float most) { float y; asm("min.NaN.f32 %0, %1, %2;\n" : "=f"(y) : "f"(fabsf(x)), "f"(most)); return y; }
__device__ __forceinline__ float clamp_nan(float x, float most) {
    float y;
    asm("{\n\t.reg .f32 t;\n\tmin.NaN.f32 t, %1, %2;\n\tmax.NaN.f32 %0, t, %3;\n\t}\n" : "=f"(y) : "f"(x), "f"(most), "f"(-most));
    return y;
}

// For a = |x| <= 100: exp(-x^2 / 2), and the normal distribution's lower tail beyond |x|, half erfc(|x| / sqrt 2), negative: that is what is needed of it.
// erfc(z) exp(z^2) as a polynomial of
// t = 1 / (1 + 0.65 z), the form of Abramowitz and Stegun 7.1.26 with the coefficients fitted here (linear programming over z = 0 .. 12) for the least
// relative error, 9e-6: a fiftieth of fp16's half step, far into the tail.  (Their own, with an absolute bound, lose the tail.)
__device__ __forceinline__ void normal_tail2(Pair a, Pair& bell, Pair& minus_tail) {
    const Pair t = prcp(pfma(a, both(0.65f * 0.70710678f), both(1.f)));
    bell = pexp2(pmul(pmul(a, both(-0.5f * kLog2e)), a));
    Pair g = pfma(both(-0.5f * 0.14364023f), t, both(0.5f * 0.47167895f));
    g = pfma(g, t, both(-0.5f * 0.35566068f));
    g = pfma(g, t, both(-0.5f * 0.23218703f));
    g = pfma(g, t, both(-0.5f * 0.37380508f));
    g = pfma(g, t, both(-0.5f * 0.36639139f));
    minus_tail = pmul(pmul(g, t), bell);
}
__device__ __forceinline__ Pair sigmoid2(Pair log2e_x) {           // of x, given x log2(e)
    float a, b;
    split_pair(log2e_x, a, b);
    return prcp(padd(both(1.f), pair_of(fast_exp2(-a), fast_exp2(-b))));
}

template <int ACT>
__device__ __forceinline__ Pair act2(Pair z) {
    float a, b;
    split_pair(z, a, b);
    if (ACT == TERRA_ACT_RELU) return pair_of(a < 0.f ? 0.f : a, b < 0.f ? 0.f : b);
    if (ACT == TERRA_ACT_SILU) return pmul(z, sigmoid2(pmul(z, both(kLog2e))));
    if (ACT == TERRA_ACT_GELU) {       // max(z, 0) - |z| tail; beyond 100 the tail is 0 in fp32, and |z| may be infinite
        const Pair m = pair_of(abs_upto(a, 100.f), abs_upto(b, 100.f));
        Pair bell, minus_tail;
        normal_tail2(m, bell, minus_tail);
        return pfma(m, minus_tail, pair_of(fmaxf(a, 0.f), fmaxf(b, 0.f)));
    }
    if (ACT == TERRA_ACT_GELU_TANH)
        return pmul(z, sigmoid2(pmul(z, pfma(pmul(z, z), both(2.f * kGeluTanhA * kLog2e * kGeluTanhB), both(2.f * kGeluTanhA * kLog2e)))));
    return z;
}

template <int ACT>
__device__ __forceinline__ Pair act_slope2(Pair z) {
    float a, b;
    split_pair(z, a, b);
    if (ACT == TERRA_ACT_RELU) return pair_of(a > 0.f ? 1.f : 0.f, b > 0.f ? 1.f : 0.f);
    if (ACT == TERRA_ACT_GELU) {
        const Pair m = pair_of(abs_upto(a, 100.f), abs_upto(b, 100.f));
        Pair bell, minus_tail;
        normal_tail2(m, bell, minus_tail);
        // Phi(z) + z phi(z): tail - |z| phi below 0, 1 less that above
        float u, v;
        split_pair(pfma(pmul(m, both(0.3989422804f)), bell, minus_tail), u, v);
        return pair_of(a < 0.f ? -u : 1.f + u, b < 0.f ? -v : 1.f + v);
    }
    if (ACT == TERRA_ACT_SILU || ACT == TERRA_ACT_GELU_TANH) {     // beyond 100 (30 for the cube) s (1 - s) is 0 in fp32
        const Pair c = pair_of(clamp_nan(a, 100.f), clamp_nan(b, 100.f)), cc = pmul(c, c);
        const float k = 2.f * kGeluTanhA;
        const Pair s = ACT == TERRA_ACT_SILU ? sigmoid2(pmul(c, both(kLog2e)))
                                             : sigmoid2(pmul(c, pfma(cc, both(k * kLog2e * kGeluTanhB), both(k * kLog2e))));
        const Pair rest = pmul(pmul(c, s), pfma(s, both(-1.f), both(1.f)));
        return ACT == TERRA_ACT_SILU ? padd(s, rest) : pfma(rest, pfma(cc, both(3.f * k * kGeluTanhB), both(k)), s);
    }
    return both(1.f);
}

// The same for one value: every call computes an activation and its slope by the same instructions, whatever the number of rows.
template <int ACT>
__device__ __forceinline__ float act(float z) { float a, b; split_pair(act2<ACT>(both(z)), a, b); return a; }
template <int ACT>
__device__ __forceinline__ float act_slope(float z) { float a, b; split_pair(act_slope2<ACT>(both(z)), a, b); return a; }

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
