// The gated projection's activations and their derivatives, in binary32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/fedhybrid.h"

namespace fh {

inline bool is_activation(int a) { return a == FH_SILU || a == FH_GELU || a == FH_GELU_TANH; }

// g times a factor s that goes from 0 to 1, each in a form whose error goes by the size of s where that is small:
//   silu        s = 1/(1 + e^-g)
//   gelu_tanh   s = (1 + tanh z)/2 = 1/(1 + e^-2z), z = sqrt(2/pi) (g + 0.044715 g^3)
//   gelu        s = the normal distribution function.  Its tail at x = |g| is e^(-x^2/2) R(x), and R(x), which goes from 1/2 to 1/(sqrt(2 pi) x), is a
//               polynomial in t = 1/(1 + 0.348 x): a minimax fit weighted for the relative error, 2.7e-7 at most where the power is not 0 yet (x <= 13.4), 3.2e-7
//               with its constants in binary32.  A coefficient less leaves 1.9e-6, one more 4e-8, which the roundings cover.  The derivative needs the same power.
// Powers and reciprocals are the hardware's, a unit in the last place off.  The power's argument a is off by 2, 8 and 3 half units of its own, as many of the
// power's times |a|: a multiple of what g's own rounding costs it.  Below 2^-126 (g beyond -87, -10, -13) powers and reciprocals are 0 to the hardware.
// An epilogue of 256 x 128 pairs is bound by these instructions: with the library's expf, erfcf and correctly rounded divisions 8192 tokens of
// 768 -> 2048 took 3 us of 66 longer (silu).
constexpr float kLog2E = 1.4426950408889634f, kInvSqrt2Pi = 0.39894228040143268f, kTwoSqrt2OverPi = 1.5957691216057308f,
                kCubic = 0.044715f;

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -kLog2E)); }
// s of gelu, and e^(-g^2/2).
__device__ __forceinline__ float normal_distribution(float g, float& power)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(g), 0.348f, 1.0f));
    power = __builtin_amdgcn_exp2f(g * g * (-0.5f * kLog2E));
    constexpr float kTail[8] = {-3.38016544e-05f, 0.139593884f, 0.131631389f, 0.15915966f, -0.0252088439f, 0.25113973f, -0.205177411f, 0.0488954782f};
    float tail = kTail[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) tail = __builtin_fmaf(t, tail, kTail[i]);
    const float beyond = tail * power;                           // |g|
    return g > 0.0f ? 1.0f - beyond : beyond;
}

// act(g) of N values, and its derivative where `slopes` is not null: d(g s)/dg = s + g s'; for the two of a sigmoid s' = s (1 - s) z'.  The choice stands outside
// the loops: within them it made every value wait for the one before (a pair's tile of 256 x 128 spent 10 us on its outputs).
template <int N>
__device__ __forceinline__ void activate(const float (&g)[N], int act, float (&values)[N], float* slopes = nullptr)
{
    if (act == FH_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float s = sigmoid(g[i]);
            values[i] = g[i] * s;
            if (slopes) slopes[i] = __builtin_fmaf(g[i] * (1.0f - s), s, s);
        }
    } else if (act == FH_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float power;
            const float s = normal_distribution(g[i], power);
            values[i] = g[i] * s;
            if (slopes) slopes[i] = __builtin_fmaf(g[i] * kInvSqrt2Pi, power, s);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float square = g[i] * g[i], s = sigmoid(kTwoSqrt2OverPi * __builtin_fmaf(kCubic * g[i], square, g[i]));
            values[i] = g[i] * s;
            // z' stays finite where g^2 leaves the range: s (1 - s) is 0 there
            if (slopes) slopes[i] = __builtin_fmaf(g[i] * (s * (1.0f - s)), kTwoSqrt2OverPi * __builtin_fmaf(3.0f * kCubic, __builtin_fminf(square, 0x1p60f), 1.0f), s);
        }
    }
}

}  // namespace fh
