// Activations of the gated feed-forward and their derivatives.
#pragma once

#include "../../include/pcpp.h"
#include "common.h"

namespace pcpp {

// act(g), and in `grad` its derivative.
//
// SiLU: g s and s (1 + g (1 - s)) with s = 1 / (1 + e^-g).
//
// GELU: g Phi(g) and Phi(g) + g phi(g).  The normal distribution's tail
// Phi(-|g|) = erfc(|g| / sqrt 2) / 2 by Abramowitz and Stegun, Handbook of
// Mathematical Functions, formula 7.1.26, (a1 t + ... + a5 t^5) exp(-g^2 / 2)
// with t = 1 / (1 + p |g| / sqrt 2), its coefficients halved: absolute error at
// most 7.5e-8 by the formula, about 3e-7 with the float32 roundings of its terms
// (2.6e-7 for the tail, 2.7e-7 for 1 - tail, 3.0e-7 for g Phi(g), over |g| <= 9
// with the hardware's reciprocal and exponential taken as exact).  The density
// takes the same exponential.
template <int ACT>
__device__ __forceinline__ float ff_act(float g, float* grad = nullptr) {
    if constexpr (ACT == PCPP_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g));
        const float y = g * s;
        if (grad) *grad = __builtin_fmaf(y, 1.f - s, s);
        return y;
    } else {
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.70710678118654752f, fabsf(g), 1.0f));
        float y = __builtin_fmaf(0.5f * 1.061405429f, t, 0.5f * -1.453152027f);
        y = __builtin_fmaf(y, t, 0.5f * 1.421413741f);
        y = __builtin_fmaf(y, t, 0.5f * -0.284496736f);
        y = __builtin_fmaf(y, t, 0.5f * 0.254829592f);
        const float e = __builtin_amdgcn_exp2f(g * g * -0.72134752044448170f);
        const float tail = y * t * e;
        const float cdf = g < 0.f ? tail : 1.f - tail;
        if (grad) *grad = __builtin_fmaf(g * e, 0.39894228040143268f, cdf);
        return g * cdf;
    }
}

}  // namespace pcpp
