// The gated projection's activations and their derivatives, in binary32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/fedhybrid.h"

namespace fh {

inline bool is_activation(int a) { return a == FH_SILU || a == FH_GELU || a == FH_GELU_TANH; }

struct Activated { float value, slope; };

// g times a factor s that goes from 0 to 1 (silu: 1/(1 + e^-g); gelu: the normal distribution's, by erfc; gelu_tanh:
// (1 + tanh z)/2 = 1/(1 + e^-2z), z = sqrt(2/pi) (g + 0.044715 g^3)), each in a form that loses nothing where s is small.
constexpr float kSqrtHalf = 0.70710678118654752f, kInvSqrt2Pi = 0.39894228040143268f, kTwoSqrt2OverPi = 1.5957691216057308f, kCubic = 0.044715f;

__device__ __forceinline__ float sigmoid(float z) { return 1.0f / (1.0f + expf(-z)); }

__device__ __forceinline__ float activated(float g, int act)
{
    if (act == FH_SILU) return g * sigmoid(g);
    if (act == FH_GELU) return g * (0.5f * erfcf(-g * kSqrtHalf));
    return g * sigmoid(kTwoSqrt2OverPi * (g + kCubic * g * g * g));
}
// d(g s)/dg = s + g s'; for the two of a sigmoid s' = s (1 - s) z'.
__device__ __forceinline__ Activated activated_both(float g, int act)
{
    if (act == FH_GELU) {
        const float s = 0.5f * erfcf(-g * kSqrtHalf);
        return {g * s, s + g * (kInvSqrt2Pi * expf(-0.5f * g * g))};
    }
    const bool silu = act == FH_SILU;
    const float z = silu ? g : kTwoSqrt2OverPi * (g + kCubic * g * g * g), turn = silu ? 1.0f : kTwoSqrt2OverPi * (1.0f + 3.0f * kCubic * g * g);
    const float s = sigmoid(z);
    return {g * s, s + g * turn * s * (1.0f - s)};
}

}  // namespace fh
