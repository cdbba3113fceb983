// Activations of the linear layer and their derivatives, in fp32.
//
//   relu       v < 0 ? 0 : v
//   gelu       v Phi(v), Phi the normal distribution: (1 + erf(v / sqrt 2)) / 2
//   gelu_tanh  v (1 + tanh u) / 2 with u = sqrt(2/pi) (v + 0.044715 v^3), taken as v / (1 + e^-2u): no cancellation
//   silu       v / (1 + e^-v)
//
// e^x is 2^(x log2 e) on the instruction for it: the product's rounding makes it |x| 2^-24
// of itself off, where |x| is large enough to matter e^-x next to 1 is not.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/xtc.h"

namespace xtc {

__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504f); }
// 1 / (1 + e^-v)
__device__ __forceinline__ float logistic(float v) { return __builtin_amdgcn_rcpf(1.f + exp_of(-v)); }

constexpr float kTanhScale = 1.59576912f, kTanhCube = 0.044715f;   // (2 sqrt(2/pi))

// Phi(v), and e^(-v^2 / 2) in `density`.  Left of zero it is that times t P(t), t = 1 / (1 + 0.35 |v|), right of zero 1 less
// as much: no sum cancels on the left (1 + erf is 4 % off at -5 and zero from -6 on, where Phi is 1e-9).  P is of degree 8,
// fitted for the least relative error up to |v| = 13.5, 2^-25; with the roundings Phi is within (1.5 v^2 + 16) 2^-24 of itself.
// (gelu behind a product, 8192 x 4096 to 4096, 220 us, by erff 227, by erfcf 237; its derivative 48 us, 55 and 65.)
__device__ __forceinline__ float normal_cdf(float v, float &density) {
    const float t = __builtin_amdgcn_rcpf(1.f + 0.35f * __builtin_fabsf(v));
    float p = __builtin_fmaf(t, -0.0291259643f, 0.143872693f);
    p = __builtin_fmaf(t, p, -0.255505472f);
    p = __builtin_fmaf(t, p, 0.158930287f);
    p = __builtin_fmaf(t, p, -0.0229377821f);
    p = __builtin_fmaf(t, p, 0.105433188f);
    p = __builtin_fmaf(t, p, 0.119852379f);
    p = __builtin_fmaf(t, p, 0.139859095f);
    p = __builtin_fmaf(t, p, 0.139621571f);
    density = exp_of(-0.5f * v * v);
    const float left = density * (t * p);
    return v > 0.f ? 1.f - left : left;
}

template <int ACT>
__device__ __forceinline__ float activated(float v) {
    if constexpr (ACT == XTC_RELU) return v < 0.f ? 0.f : v;
    else if constexpr (ACT == XTC_GELU) {
        float density;
        return v * normal_cdf(v, density);
    } else if constexpr (ACT == XTC_GELU_TANH) return v * logistic(kTanhScale * v * (1.f + kTanhCube * v * v));
    else if constexpr (ACT == XTC_SILU) return v * logistic(v);
    else return v;
}

// The derivative (relu's at 0 is 0).  Beyond 100 either way it is 1 or 0 to the last bit; there v
// is cut, before its powers leave fp32 and meet zeros.
template <int ACT>
__device__ __forceinline__ float slope(float v) {
    if constexpr (ACT == XTC_RELU) return v > 0.f ? 1.f : v <= 0.f ? 0.f : v;      // (a NaN stays one)
    v = v > 100.f ? 100.f : v < -100.f ? -100.f : v;
    if constexpr (ACT == XTC_GELU) {
        float density;
        const float cdf = normal_cdf(v, density);
        return cdf + v * 0.39894228f * density;
    } else if constexpr (ACT == XTC_GELU_TANH) {
        // q + v q (1 - q) u', u' = 2 sqrt(2/pi) (1 + 3 * 0.044715 v^2)
        const float s = kTanhCube * v * v, q = logistic(kTanhScale * v * (1.f + s));
        return q + v * q * (1.f - q) * kTanhScale * (1.f + 3.f * s);
    } else if constexpr (ACT == XTC_SILU) {
        const float q = logistic(v);
        return q + v * q * (1.f - q);
    } else return 1.f;
}

// f(activation's code as a constant)
template <typename F>
__device__ __forceinline__ void with_activation(int act, F &&f) {
    switch (act) {
        case XTC_RELU: return f(std::integral_constant<int, XTC_RELU>());
        case XTC_GELU: return f(std::integral_constant<int, XTC_GELU>());
        case XTC_GELU_TANH: return f(std::integral_constant<int, XTC_GELU_TANH>());
        case XTC_SILU: return f(std::integral_constant<int, XTC_SILU>());
        default: return f(std::integral_constant<int, XTC_NO_ACTIVATION>());
    }
}

}  // namespace xtc
