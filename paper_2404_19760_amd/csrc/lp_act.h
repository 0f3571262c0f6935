// The activations of the operators next to the path (lp_act), their slopes, and the types their tensors come in.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "lightplane.h"

namespace lp {
namespace act {

constexpr float kInvSqrt2Pi = 0.39894228040143268f;

// 1 / (1 + exp(-z)) from the hardware's exponential and reciprocal (a few units in the last place)
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// The normal distribution's integral up to z and its density.  For |z| < 1 the integral is 1/2 + z P(z^2), elsewhere the tail beyond
// |z| is t Q(t) exp(-z^2 / 2), t = 1 / (1 + 0.35 |z|) (0 at infinity, where t Q(t) goes like 1 / |z| as the tail does).  P and Q are fits
// of least largest relative error to the error function and its scaled complement in 64 bits, of 4.1e-8 and 1.1e-7.  With fp32 rounding, which
// enters the exponential's argument as 1.2e-7 z^2: relative error of the integral 4e-7 at z = -1, 1.4e-6 at -5, 5.2e-6 at -10.  The value and
// slope of the GELU are off by 2.3e-8 and 2.6e-8 (root mean square over a normal distribution), by the formula in fp32 torch by 2.5e-8 and 2.7e-8.
// (One polynomial for all z would be shorter and 4.4e-8 off in the slope.)
__device__ __forceinline__ void normal(float z, float& integral, float& density)
{
    const float a = fabsf(z), s = z * z, e = __builtin_amdgcn_exp2f(s * -0.72134752f), t = __builtin_amdgcn_rcpf(fmaf(0.35f, a, 1.0f));
    float tail = fmaf(t, 0.0431161788f, -0.109335177f);
    tail = fmaf(t, tail, 0.0433747092f);
    tail = fmaf(t, tail, 0.0312121292f);
    tail = fmaf(t, tail, 0.0901153928f);
    tail = fmaf(t, tail, 0.122394714f);
    tail = fmaf(t, tail, 0.139633358f);
    tail = fmaf(t, tail, 0.13962978f);
    tail *= t * e;
    float near = fmaf(s, 9.42352438e-05f, -0.0011693537f);
    near = fmaf(s, near, 0.00996719686f);
    near = fmaf(s, near, -0.0664895827f);
    near = fmaf(s, near, 0.398942264f);
    near = fmaf(z, near, 0.5f);
    asm("" : "+v"(near), "+v"(tail));   // (both are computed: branches around them took 24 registers more, of all activations' kernels)
    integral = a < 1.0f ? near : z < 0.0f ? tail : 1.0f - tail;
    density = e * kInvSqrt2Pi;
}

template <int ACT>
__device__ __forceinline__ float activate(float z)
{
    if (ACT == LP_ACT_RELU) return z < 0.0f ? 0.0f : z;   // (a NaN stays one)
    if (ACT == LP_ACT_SILU) return z * sigmoid(z);
    if (ACT == LP_ACT_GELU) {
        float i, d;
        normal(z, i, d);
        return z * i;
    }
    return z;
}

template <int ACT>
__device__ __forceinline__ float slope(float z)
{
    if (ACT == LP_ACT_RELU) return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    if (ACT == LP_ACT_SILU) {
        const float s = sigmoid(z);
        return fmaf(z * s, 1.0f - s, s);
    }
    if (ACT == LP_ACT_GELU) {
        float i, d;
        normal(z, i, d);
        return fmaf(z, d, i);
    }
    return 1.0f;
}

// Calls f with the activation as a constant: the choice stands outside the loops.
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f)
{
    switch (act) {
        case LP_ACT_RELU: f(std::integral_constant<int, LP_ACT_RELU>()); break;
        case LP_ACT_SILU: f(std::integral_constant<int, LP_ACT_SILU>()); break;
        case LP_ACT_GELU: f(std::integral_constant<int, LP_ACT_GELU>()); break;
        default: f(std::integral_constant<int, LP_ACT_NONE>());
    }
}

}  // namespace act
}  // namespace lp
