// Activations and their derivatives in fp32 (include/fpdt_tokenwise.h: FPDT_TW_ACT_*), for the kernels that have them behind a
// product or in front of a gradient.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/fpdt_tokenwise.h"

namespace fpdt_tw {

// exp(a^2 / 2) Phi(-a) = t P(t) with t = 1 / (1 + 0.3 a), for a >= 0; Phi(-a): the share of the normal distribution below -a.  P: eight
// terms fitted to the relative error over 0 .. 14 (1.5e-7; 4e-7 as computed here), so that the tail keeps its value where 1 + erf has
// nothing left of it.
__device__ __forceinline__ float tail_over_exp(float a)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, a, 1.f));
    float p = 0.03567545542148818f;
    p = fmaf(p, t, -0.15720593913611508f);
    p = fmaf(p, t, 0.2063584413658594f);
    p = fmaf(p, t, -0.053688180413640665f);
    p = fmaf(p, t, 0.1285640129536115f);
    p = fmaf(p, t, 0.09991277616585857f);
    p = fmaf(p, t, 0.12075406915047618f);
    p = fmaf(p, t, 0.1196292915805715f);
    return p * t;
}
__device__ __forceinline__ float exp_half_square(float a) { return __builtin_amdgcn_exp2f(a * -0.72134752044448170f * a); }
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.4426950408889634f)); }

// x Phi(x) = max(x, 0) - |x| Phi(-|x|): infinities keep their value (20 Phi(-20) is nothing next to any of them), NaN stays NaN.  (fmaxf would be two
// instructions.)
__device__ __forceinline__ float gelu_of(float x, float a, float below)
{
    float top;
    asm("v_max_f32 %0, 0, %1" : "=v"(top) : "v"(x));
    return fmaf(-__builtin_amdgcn_fmed3f(a, 0.f, 20.f), below, top);
}
template <int ACT> __device__ __forceinline__ float act_of(float x)
{
    if constexpr (ACT == FPDT_TW_ACT_GELU) {
        const float a = fabsf(x);
        return gelu_of(x, a, tail_over_exp(a) * exp_half_square(a));
    } else if constexpr (ACT == FPDT_TW_ACT_SILU) {
        return x * logistic(x);
    } else {
        return x;
    }
}

// The activation and its derivative
template <int ACT> __device__ __forceinline__ float slope_of(float x, float& y)
{
    if constexpr (ACT == FPDT_TW_ACT_GELU) {
        // Phi(x) + x phi(x), phi the density: what it is below 0 is one less what it is above
        const float a = fabsf(x), e = exp_half_square(a), tail = tail_over_exp(a), low = fmaf(-0.3989422804014327f, a, tail) * e;
        y = gelu_of(x, a, tail * e);
        return x > 0.f ? 1.f - low : low;
    } else if constexpr (ACT == FPDT_TW_ACT_SILU) {
        const float s = logistic(x);
        y = x * s;
        return s * fmaf(x, 1.f - s, 1.f);
    } else {
        y = x;
        return 1.f;
    }
}

}  // namespace fpdt_tw
