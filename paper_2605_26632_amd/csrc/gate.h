// Activations of the gated linears and their derivatives, in fp32.
//
//   silu       g s(g), s(x) = 1 / (1 + e^-x)
//   gelu_tanh  .5 g (1 + tanh(c (g + .044715 g^3))), c = sqrt(2 / pi): since .5 (1 + tanh x) = s(2 x) this is g s(g (2 c + 2 c .044715 g^2)),
//              silu with another argument, so that the two share one path
//   gelu       g Phi(g), Phi(g) = .5 erfc(-g / sqrt 2) by the rational approximation 7.1.26 of Abramowitz and Stegun's Handbook: erfc(x) = (a1 t + ..
//              + a5 t^5) e^-x^2, t = 1 / (1 + p x), x >= 0, off by at most 1.5e-7. As a product it keeps its relative accuracy where Phi is small.
// e^x and 1 / x are the hardware's (an fp32 unit or two); all of it is rounded to bf16 afterwards, whose half step is up to 2^-8 of the value.
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
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * x);
    const float p = t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
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
