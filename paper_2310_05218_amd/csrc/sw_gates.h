// The terms of the gated recurrence of one token and channel, from its two gates:
//     s = sigmoid(r), L = log_decay s, a = e^L, w = sqrt(1 - a^2), p = sigmoid(i).
// e^x is 2^(x log2 e): the product's rounding is an error of |x| units of the result's last place, which fp32 tensors get back from its remainder.
// 1 - a^2 = -(e^u - 1), u = 2 L, loses its leading digits to the subtraction where a is near 1: there it is the series of e^u - 1.
#pragma once

#include "sw_layers.h"

namespace swconv {

// e^x; EXACT: within two units in the last place for any x, infinities and NaN included
template <bool EXACT>
__device__ __forceinline__ float exp_of(float x)
{
    constexpr float kLog2e = 1.44269502f, kLog2eLow = 1.92596303e-8f, kLn2 = 0.693147182f;
    const float t = x * kLog2e, e = __builtin_amdgcn_exp2f(t);
    if constexpr (!EXACT) return e;
    const float low = __builtin_fmaf(x, kLog2eLow, __builtin_fmaf(x, kLog2e, -t));
    return fabsf(t) < 128.f ? __builtin_fmaf(e * kLn2, low, e) : e;
}

// -(e^u - 1) for u <= 0, where a2 = e^u.  The series' first term that is left out is below 2^-25 of the sum at either border, the subtraction's
// error below 2^-18 (half a step of 16-bit formats is 2^-12 at least), EXACT below 2^-22.
template <bool EXACT>
__device__ __forceinline__ float one_minus(float u, float a2)
{
    constexpr float kBorder = EXACT ? -0.5f : -0.03125f;
    float q;
    if constexpr (EXACT) {
        q = 2.48015873e-5f;                             // 1/8!
        q = __builtin_fmaf(q, u, 1.98412698e-4f);
        q = __builtin_fmaf(q, u, 1.38888889e-3f);
        q = __builtin_fmaf(q, u, 8.33333333e-3f);
        q = __builtin_fmaf(q, u, 4.16666667e-2f);
    } else {
        q = 4.16666667e-2f;                             // 1/4!
    }
    q = __builtin_fmaf(q, u, 0.166666667f);
    q = __builtin_fmaf(q, u, 0.5f);
    q = __builtin_fmaf(q, u, 1.f);
    return u > kBorder ? -u * q : 1.f - a2;
}

template <int EK>
struct Gate {
    static constexpr bool EXACT = EK == kElemF32;
    float s, L, a, w, p;                // as above
    float es, ep;                       // e^-r, e^-i
    __device__ __forceinline__ Gate(float log_decay, float r, float i)
    {
        es = exp_of<EXACT>(-r), ep = exp_of<EXACT>(-i);
        s = __builtin_amdgcn_rcpf(1.f + es), p = __builtin_amdgcn_rcpf(1.f + ep);
        L = log_decay * s;
        a = exp_of<EXACT>(L);
        w = __builtin_amdgcn_sqrtf(one_minus<EXACT>(2.f * L, a * a));
    }
    // 1 - s and 1 - p, to fp32's bits at both ends
    __device__ __forceinline__ float shut_s(float r) const { return r > 0.f ? es * s : 1.f - s; }
    __device__ __forceinline__ float shut_p(float i) const { return i > 0.f ? ep * p : 1.f - p; }
};

// (-infinity times a gate that is shut would be NaN)
__device__ __forceinline__ float finite_decay(float log_decay) { return log_decay < -3e38f ? -3e38f : log_decay; }

}  // namespace swconv
