// Activations of the gated feed-forward layer and their derivatives, in fp32.
#pragma once

#include <cuda_runtime.h>

#include <type_traits>

#include "bdr.h"

namespace bdr {
namespace act {

inline bool known(int a) { return a == MX_ACT_SILU || a == MX_ACT_GELU || a == MX_ACT_GELU_TANH || a == MX_ACT_RELU; }

// The exponentials and the quotient are single instructions, without a range reduction of their own.  With t = exp(-|x|) off by |x| 2^-23 of
// itself, 1 / (1 + t) in (1/2, 1] is off by at most max(|x| exp(-|x|)) 2^-23, less than its own last bit, and the smaller of the two values,
// t / (1 + t), by |x| 2^-23 of itself: |x| 2^-23 exp(-|x|) beside results of size |x|.
__device__ __forceinline__ float exp_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.4426950408889634f));
    return y;
}
__device__ __forceinline__ float inverse(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// p = sigmoid(x), q = sigmoid(-x)
__device__ __forceinline__ void sigmoids(float x, float& p, float& q) {
    const float t = exp_of(-fabsf(x)), r = inverse(1.f + t), s = t * r;
    p = x < 0.f ? s : r;
    q = x < 0.f ? r : s;
}
__device__ __forceinline__ float sigmoid(float x) {
    const float t = exp_of(-fabsf(x)), r = inverse(1.f + t);
    return x < 0.f ? t * r : r;
}
// Phi(x) from the error function: off by 2^-24 or so, beside which tails below it are lost
__device__ __forceinline__ float normal_cdf(float x) { return fmaf(0.5f, erff(x * 0.7071067811865476f), 0.5f); }

// y = act(g)
template <int ACT>
__device__ __forceinline__ float of(float g) {
    if constexpr (ACT == MX_ACT_SILU) return g * sigmoid(g);
    if constexpr (ACT == MX_ACT_GELU) return g * normal_cdf(g);
    if constexpr (ACT == MX_ACT_GELU_TANH) return g * sigmoid(1.5957691216057308f * (g + 0.044715f * g * g * g));  // (1 + tanh x) / 2 = sigmoid(2 x)
    return g < 0.f ? 0.f : g;
}
// y = act(g), slope = act'(g)
template <int ACT>
__device__ __forceinline__ void both(float g, float& y, float& slope) {
    if constexpr (ACT == MX_ACT_SILU) {
        float p, q;
        sigmoids(g, p, q);
        y = g * p;
        slope = p + y * q;
    } else if constexpr (ACT == MX_ACT_GELU) {
        const float p = normal_cdf(g);
        y = g * p;
        slope = p + g * (0.3989422804014327f * exp_of(-0.5f * g * g));
    } else if constexpr (ACT == MX_ACT_GELU_TANH) {
        float p, q;
        sigmoids(1.5957691216057308f * (g + 0.044715f * g * g * g), p, q);
        q *= p;
        y = g * p;
        slope = q == 0.f ? p : p + g * q * (1.5957691216057308f * (1.f + 0.134145f * g * g));  // (far out the square overflows)
    } else {
        y = g < 0.f ? 0.f : g;
        slope = g > 0.f ? 1.f : 0.f;
    }
}
template <typename F>
__device__ __forceinline__ void with(int act, F&& f) {
    switch (act) {
        case MX_ACT_SILU: f(std::integral_constant<int, MX_ACT_SILU>()); break;
        case MX_ACT_GELU: f(std::integral_constant<int, MX_ACT_GELU>()); break;
        case MX_ACT_GELU_TANH: f(std::integral_constant<int, MX_ACT_GELU_TANH>()); break;
        default: f(std::integral_constant<int, MX_ACT_RELU>()); break;
    }
}

}  // namespace act
}  // namespace bdr
