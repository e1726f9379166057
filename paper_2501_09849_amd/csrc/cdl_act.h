// Activations and their derivatives in fp32 (CDL_ACT_*).
#pragma once

#include "cdl_types.h"

namespace cdl {

// 2^(-x^2 / (2 ln 2)) and the normal distribution's upper tail at x = |z|, as the first times a polynomial in t = 1 / (1 + 0.375 x) without a constant term:
// exp(x^2 / 2) (1 - Phi(x)) has such an expansion, as it is smooth and falls as 1 / x.  Its nine coefficients are a fit of the smallest largest relative error over
// x >= 0 (2.2e-7, against values of erfcx in double); in fp32 the tail is right to 1.1e-6 of itself for x < 4 and to 4e-6 at 9 (the square's rounding), Phi to 2.5e-7.  One exponential and one reciprocal serve the value
// and the derivative; the library's erf takes twice the instructions, and a branch.
struct Normal { float below, bell; };      // Phi(z), exp(-z^2 / 2)
__device__ __forceinline__ Normal normal(float z)
{
    const float x = fabsf(z), t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.375f, x, 1.0f));
    float w = -0.032910119742155075f;
    w = __builtin_fmaf(w, t, 0.13687631487846375f);
    w = __builtin_fmaf(w, t, -0.1865154653787613f);
    w = __builtin_fmaf(w, t, 0.05062757432460785f);
    w = __builtin_fmaf(w, t, 0.015630224719643593f);
    w = __builtin_fmaf(w, t, 0.08863760530948639f);
    w = __builtin_fmaf(w, t, 0.1284457892179489f);
    w = __builtin_fmaf(w, t, 0.14960457384586334f);
    w = __builtin_fmaf(w, t, 0.14960338175296783f);
    const float bell = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f), tail = w * t * bell;
    return {z < 0.0f ? tail : 1.0f - tail, bell};
}

// 1 / (1 + exp(-z)); 0 where exp(-z) passes the largest float
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f)); }

// NaN stays NaN in all of them.
template <int ACT>
__device__ __forceinline__ float act_value(float z)
{
    if (ACT == CDL_ACT_RELU) return z <= 0.0f ? 0.0f : z;
    if (ACT == CDL_ACT_GELU) return z * normal(z).below;
    if (ACT == CDL_ACT_SILU) return z * sigmoid(z);
    return z;
}
struct ValueSlope { float value, slope; };
template <int ACT>
__device__ __forceinline__ ValueSlope act_both(float z)
{
    if (ACT == CDL_ACT_RELU) return {z <= 0.0f ? 0.0f : z, z <= 0.0f ? 0.0f : z == z ? 1.0f : z};
    if (ACT == CDL_ACT_GELU) {
        const Normal n = normal(z);
        return {z * n.below, __builtin_fmaf(z * 0.3989422804014327f, n.bell, n.below)};
    }
    if (ACT == CDL_ACT_SILU) {
        const float s = sigmoid(z);
        return {z * s, s * __builtin_fmaf(z, 1.0f - s, 1.0f)};
    }
    return {z, 1.0f};
}

}  // namespace cdl
