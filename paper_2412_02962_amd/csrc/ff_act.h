// Activations of the gated feed-forward and their derivatives.
#pragma once

#include "../../include/pcpp.h"
#include "gelu.h"

namespace pcpp {

// act(g), and in `grad` its derivative.  GELU: g Phi(g), Phi(g) + g phi(g);
// SiLU: g s, s (1 + g (1 - s)) with s = 1 / (1 + e^-g).
__device__ __forceinline__ float ff_act(int act, float g, float* grad = nullptr) {
    if (act == PCPP_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g));
        const float y = g * s;
        if (grad) *grad = __builtin_fmaf(y, 1.f - s, s);
        return y;
    }
    const float cdf = 0.5f * (1.f + erf_as(g * 0.70710678118654752f));
    if (grad) {
        const float pdf = 0.39894228040143268f * __builtin_amdgcn_exp2f(g * g * -0.72134752044448170f);
        *grad = __builtin_fmaf(g, pdf, cdf);
    }
    return g * cdf;
}

}  // namespace pcpp
