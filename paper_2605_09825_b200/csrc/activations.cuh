// Activations of a gate and their derivatives, in fp32.  Sigmoid and tanh come from the exponential of the
// hardware (2 + 1.17 |x| units in the last place, and |x| is at most 103 where a result is not 0) and one division: below
// 2^-16 of a value, far below the 2^-9 of a bf16 result.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/mxfp4.h"

namespace mxfp4 {

// 1 / (1 + exp(-x)), from e = exp(-|x|): e / (1 + e) for a negative x, so that the exponential never overflows and results
// below 2^-126 are not lost (times x, or the other projection, they are normal numbers).
__device__ __forceinline__ float logistic(float x)
{
    const float e = __expf(-fabsf(x)), r = __fdividef(1.0f, 1.0f + e);
    return x < 0.0f ? e * r : r;
}

constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kGeluC = 0.79788456080286536f;       // sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;

template <int ACT>
__device__ __forceinline__ float act_value(float g)
{
    if constexpr (ACT == MXFP4_GATE_SIGMOID) return logistic(g);
    if constexpr (ACT == MXFP4_GATE_SILU) return g * logistic(g);
    if constexpr (ACT == MXFP4_GATE_GELU) return 0.5f * g * erfcf(-g * kSqrtHalf);
    // (1 + tanh y) / 2 = 1 / (1 + exp(-2 y))
    if constexpr (ACT == MXFP4_GATE_GELU_TANH) return g * logistic(2.0f * kGeluC * (g + kGeluCubic * g * g * g));
    if constexpr (ACT == MXFP4_GATE_RELU) return g < 0.0f ? 0.0f : g;         // NaN stays
    return g;
}

// value and derivative
template <int ACT>
__device__ __forceinline__ float2 act_both(float g)
{
    if constexpr (ACT == MXFP4_GATE_SIGMOID) {
        // s (1 - s) = e / (1 + e)^2: 1 - s itself would have lost its bits from g = 10 on
        const float e = __expf(-fabsf(g)), r = __fdividef(1.0f, 1.0f + e);
        return make_float2(g < 0.0f ? e * r : r, e * r * r);
    }
    if constexpr (ACT == MXFP4_GATE_SILU) {
        const float s = logistic(g);
        return make_float2(g * s, s * (1.0f + g * (1.0f - s)));
    }
    if constexpr (ACT == MXFP4_GATE_GELU) {
        const float cdf = 0.5f * erfcf(-g * kSqrtHalf);
        return make_float2(g * cdf, cdf + g * kInvSqrt2Pi * __expf(-0.5f * g * g));
    }
    if constexpr (ACT == MXFP4_GATE_GELU_TANH) {
        const float s = logistic(2.0f * kGeluC * (g + kGeluCubic * g * g * g));
        const float bend = s * (1.0f - s);            // 0 far from the origin, where the slope's square may overflow
        const float slope = kGeluC * (1.0f + 3.0f * kGeluCubic * g * g);
        return make_float2(g * s, bend > 0.0f ? s + 2.0f * g * bend * slope : s);
    }
    if constexpr (ACT == MXFP4_GATE_RELU) return make_float2(g < 0.0f ? 0.0f : g, g > 0.0f ? 1.0f : g <= 0.0f ? 0.0f : g);
    return make_float2(g, 1.0f);
}

// Calls f with the activation as a compile-time constant: one uniform branch for a stretch of elements.
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f)
{
    switch (act) {
        case MXFP4_GATE_SIGMOID: f(std::integral_constant<int, MXFP4_GATE_SIGMOID>{}); break;
        case MXFP4_GATE_SILU: f(std::integral_constant<int, MXFP4_GATE_SILU>{}); break;
        case MXFP4_GATE_GELU: f(std::integral_constant<int, MXFP4_GATE_GELU>{}); break;
        case MXFP4_GATE_GELU_TANH: f(std::integral_constant<int, MXFP4_GATE_GELU_TANH>{}); break;
        case MXFP4_GATE_RELU: f(std::integral_constant<int, MXFP4_GATE_RELU>{}); break;
        default: f(std::integral_constant<int, MXFP4_GATE_LINEAR>{}); break;
    }
}

}  // namespace mxfp4
