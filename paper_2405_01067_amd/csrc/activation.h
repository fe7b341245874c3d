// Activations and their slopes in fp32, two evaluations of the transcendental unit each.
#pragma once

#include <type_traits>

#include "common.h"

namespace abt {

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }

// The normal distribution below -|z|, and its density times sqrt(2 pi).  Their ratio R is a polynomial in t = 1 / (1 + 0.3 |z|) without a constant term, as R falls with 1 / |z|: the one of degree 8
// whose largest relative error from 0 to 15 is least, 1.7e-7 (fitted for this; degree 7 8e-7, 9 2e-8), 5e-7 of R as it is evaluated.  exp(-z^2 / 2) is off by z^2 2^-24 of itself beside that, as
// much as half a unit of z's last place makes.
__device__ __forceinline__ float normal_tail(float z, float& density) {
    const float t = rcp_fast(1.0f + 0.3f * __builtin_fabsf(z));
    density = exp2_fast(z * z * -0.72134752f);                                     // log2(e) / 2
    return (((((((0.03542370477f * t - 0.1561583277f) * t + 0.2045565902f) * t - 0.05203385004f) * t + 0.1276916903f) * t + 0.1001759705f) * t + 0.1207121328f) * t + 0.1196320074f) *
           (t * density);
}
// 1 / (1 + exp(-2 c (z + 0.044715 z^3))), c = sqrt(2 / pi): the sigmoid by which gelu_tanh multiplies (the tanh form is the same number)
__device__ __forceinline__ float tanh_gate(float z) {
    return rcp_fast(1.0f + exp2_fast(z * (-2.30220819f - 0.10294324f * z * z)));   // -2 c log2(e), and 0.044715 times it
}
__device__ __forceinline__ float sigmoid(float z) { return rcp_fast(1.0f + exp2_fast(z * -1.44269504f)); }

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == ABT_ACT_RELU) return z < 0.0f ? 0.0f : z;                 // (NaN stays)
    if constexpr (ACT == ABT_ACT_GELU) {
        float density;
        const float tail = normal_tail(z, density);
        return __builtin_fmaxf(z, 0.0f) - __builtin_fminf(__builtin_fabsf(z), 16.0f) * tail;       // (beyond 16 the tail is 0, also at infinity; a NaN is in it)
    }
    if constexpr (ACT == ABT_ACT_GELU_TANH) return z * tanh_gate(z);
    if constexpr (ACT == ABT_ACT_SILU) return z * sigmoid(z);
    return z;
}
template <int ACT>                                        // of the smooth ones
__device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == ABT_ACT_GELU) {
        float density;
        const float tail = normal_tail(z, density);
        return (z > 0.0f ? 1.0f - tail : tail) + z * density * 0.39894228f;
    }
    if constexpr (ACT == ABT_ACT_GELU_TANH) {
        z = z > 30.0f ? 30.0f : z < -30.0f ? -30.0f : z;                           // the gate is 0 or 1 long before; z^2 stays finite
        const float s = tanh_gate(z);
        return s + z * s * (1.0f - s) * (1.59576912f + 0.21406445f * z * z);      // 2 c, and 3 * 0.044715 times it
    }
    if constexpr (ACT == ABT_ACT_SILU) {
        const float s = sigmoid(z);
        return s + z * s * (1.0f - s);
    }
}

// the gradient d behind the activation, in front of it
template <int ACT>
__device__ __forceinline__ float through(float z, float d) {
    if constexpr (ACT == ABT_ACT_NONE) return d;
    else if constexpr (ACT == ABT_ACT_RELU) return z > 0.0f ? d : 0.0f;
    else return d * slope<ACT>(z);
}

// f(std::integral_constant<int, ACT>) for the activation of a launch, which is the same for all its threads: one branch around what f does
template <class F>
__device__ __forceinline__ void with_activation(int act, F&& f) {
    switch (act) {
        case ABT_ACT_RELU: f(std::integral_constant<int, ABT_ACT_RELU>{}); break;
        case ABT_ACT_GELU: f(std::integral_constant<int, ABT_ACT_GELU>{}); break;
        case ABT_ACT_GELU_TANH: f(std::integral_constant<int, ABT_ACT_GELU_TANH>{}); break;
        case ABT_ACT_SILU: f(std::integral_constant<int, ABT_ACT_SILU>{}); break;
        default: f(std::integral_constant<int, ABT_ACT_NONE>{});
    }
}

}  // namespace abt
