// Activations of the gated linears and their derivatives, in fp32.
//
//   silu       g s(g), s(x) = 1 / (1 + e^-x)
//   gelu_tanh  .5 g (1 + tanh(c (g + .044715 g^3))), c = sqrt(2 / pi): since .5 (1 + tanh x) = s(2 x) this is g s(g (2 c + 2 c .044715 g^2)),
//              silu with another argument, so that the two share one path
//   gelu       g Phi(g), Phi(-|g|) = .5 erfc(x) with x = |g| / sqrt 2, and erfc(x) e^(x^2) as a polynomial in t = 1 / (1 + .33 x) without a constant, the form of
//              7.1.26 in Abramowitz and Stegun's Handbook, whose five terms are off by 7e-4 of themselves at x = 3 and by 4e-2 at 9.5. These eight are
//              fitted, in 64 bits, to the least largest error relative to the value over 0 <= x <= 9.5 (2e-7 with their rounding to fp32), behind which e^(-x^2)
//              is below 2^-126: as a product Phi keeps its relative accuracy where it is small. (The three terms more: [4096, 8192, 128] with G and U 56.8 -> 58.7 us,
//              unseen in longer contractions and in the elementwise backward pass.)
// 1 / x is the hardware's (an fp32 unit), e^x too, whose argument's roundings make it off by up to 3 |x| units; all of it is rounded to bf16 afterwards, whose half step
// is up to 2^-8 of the value.
#pragma once
#include <hip/hip_runtime.h>
#include "rtlynx.h"

namespace rtl {
namespace {

__device__ __forceinline__ float gate_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
__device__ __forceinline__ float gate_sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + gate_exp(-x)); }

// What an activation of the first path makes of g before the logistic function: g (a + b g^2).
struct GateForm {
    float a, b;
};
__device__ __forceinline__ GateForm gate_form(int act) {
    const float c2 = 1.59576912f;                                             // 2 sqrt(2 / pi)
    return act == RTL_ACT_SILU ? GateForm{1.0f, 0.0f} : GateForm{c2, c2 * 0.044715f};
}

// Phi(g); e = exp(-g^2 / 2) comes out too, the derivative needs it.
__device__ __forceinline__ float gate_phi(float g, float& e) {
    const float x = fabsf(g) * 0.70710678f;
    e = gate_exp(-0.5f * g * g);
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.33f * x);
    const float p = t * (0.186366311f + t * (0.182834496f + t * (0.201939305f + t * (0.0449638905f +
                    t * (0.412623469f + t * (-0.355522237f + t * (0.462733941f - t * 0.135939258f)))))));
    const float half = 0.5f * p * e;
    return g < 0.0f ? half : 1.0f - half;
}

// g^2, cut where it no longer matters: a factor of zero (silu), and the slope's 1 - s, stay zero beside it for gates up to infinity.
__device__ __forceinline__ float gate_square(float g) { return fminf(g * g, 1e30f); }

template <bool ERF>
__device__ __forceinline__ float gate_value(float g, GateForm f) {
    if constexpr (ERF) {
        float e;
        return g * gate_phi(g, e);
    } else {
        return g * gate_sigmoid(g * (f.a + f.b * gate_square(g)));
    }
}

// value and derivative. x = g (a + b g^2): (g s(x))' = s + g s (1 - s) x', x' = a + 3 b g^2; (g Phi)' = Phi + g phi(g).
template <bool ERF>
__device__ __forceinline__ void gate_both(float g, GateForm f, float& value, float& slope) {
    if constexpr (ERF) {
        float e;
        const float phi = gate_phi(g, e);
        value = g * phi;
        slope = phi + 0.39894228f * g * e;
    } else {
        const float g2 = gate_square(g), s = gate_sigmoid(g * (f.a + f.b * g2));
        value = g * s;
        slope = s + value * (1.0f - s) * (f.a + 3.0f * f.b * g2);
    }
}

}  // namespace
}  // namespace rtl
