// Activations of the gated feed-forward layer and their derivatives, in fp32.
#pragma once

#include <cuda_runtime.h>

#include <type_traits>

#include "bdr.h"

namespace bdr {
namespace act {

inline bool known(int a) { return a == MX_ACT_SILU || a == MX_ACT_GELU || a == MX_ACT_GELU_TANH || a == MX_ACT_RELU; }

__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + expf(-x)); }

// y = act(g)
template <int ACT>
__device__ __forceinline__ float of(float g) {
    if constexpr (ACT == MX_ACT_SILU) return g * sigmoid(g);
    if constexpr (ACT == MX_ACT_GELU) return g * normcdff(g);
    if constexpr (ACT == MX_ACT_GELU_TANH) return g * sigmoid(1.5957691216057308f * (g + 0.044715f * g * g * g));  // (1 + tanh x) / 2 = sigmoid(2 x)
    return g < 0.f ? 0.f : g;
}
// y = act(g), slope = act'(g)
template <int ACT>
__device__ __forceinline__ void both(float g, float& y, float& slope) {
    if constexpr (ACT == MX_ACT_SILU) {
        const float t = expf(-fabsf(g)), r = __fdividef(1.f, 1.f + t), s = t * r;  // the sigmoid of |g| and what it lacks to one
        const float p = g < 0.f ? s : r, q = g < 0.f ? r : s;
        y = g * p;
        slope = p + y * q;
    } else if constexpr (ACT == MX_ACT_GELU) {
        const float p = normcdff(g);
        y = g * p;
        slope = p + g * (0.3989422804014327f * expf(-0.5f * g * g));
    } else if constexpr (ACT == MX_ACT_GELU_TANH) {
        const float x = 1.5957691216057308f * (g + 0.044715f * g * g * g), p = sigmoid(x), q = p * sigmoid(-x);
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
