// The gated projection's activations and their derivatives, in binary32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/fedhybrid.h"

namespace fh {

inline bool is_activation(int a) { return a == FH_SILU || a == FH_GELU || a == FH_GELU_TANH; }

// g times a factor s that goes from 0 to 1, each in a form that loses nothing where s is small:
//   silu        s = 1/(1 + e^-g)
//   gelu_tanh   s = (1 + tanh z)/2 = 1/(1 + e^-2z), z = sqrt(2/pi) (g + 0.044715 g^3)
//   gelu        s = the normal distribution function = erfc(-g/sqrt 2)/2.  For x = |g|/sqrt 2, erfc x = (a1 t + ... + a5 t^5) e^(-x^2), t = 1/(1 + p x)
//               (Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26: within 1.5e-7 of it everywhere, and since the power
//               multiplies the error too, within some 1e-6 of its size); the derivative needs the same power.
// Powers and reciprocals are the hardware's, a unit in the last place off.  The power's argument is rounded, which is |z| units of the power: what g's own
// rounding costs it too.  An epilogue of 256 x 128 pairs is bound by these instructions: with the library's expf, erfcf and
// correctly rounded divisions 8192 tokens of 768 -> 2048 took 3 us of 66 longer (silu).
constexpr float kLog2E = 1.4426950408889634f, kSqrtHalf = 0.70710678118654752f, kInvSqrt2Pi = 0.39894228040143268f, kTwoSqrt2OverPi = 1.5957691216057308f,
                kCubic = 0.044715f;

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -kLog2E)); }
// s of gelu, and e^(-g^2/2).
__device__ __forceinline__ float normal_distribution(float g, float& power)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(g), 0.3275911f * kSqrtHalf, 1.0f));
    power = __builtin_amdgcn_exp2f(g * g * (-0.5f * kLog2E));
    float sum = __builtin_fmaf(t, 1.061405429f, -1.453152027f);
    sum = __builtin_fmaf(t, sum, 1.421413741f);
    sum = __builtin_fmaf(t, sum, -0.284496736f);
    sum = __builtin_fmaf(t, sum, 0.254829592f);
    const float beyond = 0.5f * (t * sum) * power;               // of |g|
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
            // g s (1 - s) first: it is 0 where g^3 leaves the range
            if (slopes) slopes[i] = __builtin_fmaf(g[i] * (s * (1.0f - s)), kTwoSqrt2OverPi * __builtin_fmaf(3.0f * kCubic, square, 1.0f), s);
        }
    }
}

}  // namespace fh
