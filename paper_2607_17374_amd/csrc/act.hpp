// Activations and their slopes in fp32 (norm.hip, linear.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../include/taurus.h"

namespace taurus {

// 1 / (1 + exp(-z)) for |z| <= SIGMOID_END by the chip's power of two and
// reciprocal (one unit in the last place each): with t = -z and h = t log2(e)
// rounded, exp(t) is 2^h times the exponential of t - h ln 2, taken linearly
// (ln 2 in two parts).  Right to about three units in the last place above z =
// -87.3; below, where it passes under the least normal value, it may be 0.
// (The library's exponential and division take three times the steps; SiLU is
// then bound by them.)
constexpr float SIGMOID_END = 88.7f;
__device__ inline float sigmoid(float z) {
    const float t = -z, h = t * 1.44269502f;  // |h| < 128: the power is finite
    const float rest = __builtin_fmaf(h, 1.90465421e-9f, __builtin_fmaf(h, -0.693147182f, t));
    const float e = __builtin_amdgcn_exp2f(h);
    return __builtin_amdgcn_rcpf(1.f + __builtin_fmaf(e, rest, e));
}
// Arguments past its ends are held there (NaN stays): above, the sigmoid is 1
// and SiLU's slope too; below, SiLU and its slope are less than 2^-119 from 0.
__device__ inline float silu(float z) {
    const float c = __builtin_elementwise_maximum(z, -SIGMOID_END);
    return c * sigmoid(__builtin_elementwise_minimum(c, SIGMOID_END));
}
__device__ inline float silu_slope(float z) {
    const float c = __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, -SIGMOID_END), SIGMOID_END);
    const float q = sigmoid(c);
    return q * (1.f + c * (1.f - q));
}
// exp(t) for t <= 0 (as the sigmoid's); 0 below about -87.3, NaN stays.  t is
// finite.
__device__ inline float exp_of(float t) {
    const float h = t * 1.44269502f;
    const float rest = __builtin_fmaf(h, 1.90465421e-9f, __builtin_fmaf(h, -0.693147182f, t));
    const float e = __builtin_amdgcn_exp2f(h);
    return __builtin_fmaf(e, rest, e);
}

// GELU, z times the normal distribution function Phi, and its slope Phi(z) +
// z phi(z).  Phi(-x) = exp(-x^2 / 2) t P(t) for x >= 0, t = 1 / (1 + 0.28 x), with
// P fitted to the scaled tail erfcx(x / sqrt(2)) / 2 for equal relative error
// over [0, 15] (5.8e-8 before, 3.3e-7 after rounding in fp32; the power adds
// x^2 1e-7), so that the negative tail keeps its digits.  A library erf takes
// about three times the steps, and none of that.  Arguments are held at
// +-GELU_END (NaN stays): there Phi is 0 or 1 in fp32 and z phi(z) is 0, and
// infinities give the limits.
constexpr float GELU_END = 15.f;
struct Normal {
    float cdf, density;
};
__device__ inline Normal normal(float z) {
    const float x = fabsf(z), e = __builtin_amdgcn_exp2f(-0.721347520f * (x * x));
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.28f, x, 1.f));
    float p = 0.0232955366f;
    p = __builtin_fmaf(p, t, -0.0858391151f);
    p = __builtin_fmaf(p, t, 0.0749406517f);
    p = __builtin_fmaf(p, t, 0.0148789166f);
    p = __builtin_fmaf(p, t, 0.0574233681f);
    p = __builtin_fmaf(p, t, 0.0902868807f);
    p = __builtin_fmaf(p, t, 0.10139332f);
    p = __builtin_fmaf(p, t, 0.11192932f);
    p = __builtin_fmaf(p, t, 0.111691147f);
    const float tail = e * (t * p);
    return {z < 0.f ? tail : 1.f - tail, 0.398942280f * e};
}
__device__ inline float gelu(float z) {
    const float c = __builtin_elementwise_maximum(z, -GELU_END);
    return c * normal(__builtin_elementwise_minimum(c, GELU_END)).cdf;
}
__device__ inline float gelu_slope(float z) {
    const float c = __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, -GELU_END), GELU_END);
    const Normal n = normal(c);
    return __builtin_fmaf(c, n.density, n.cdf);
}
// The same with Phi replaced by (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2,
// which is a sigmoid of twice the argument: at +-15 that is +-265, held at the
// sigmoid's ends, where it is 0 or 1 to 2^-127.
__device__ inline float tanh_sigmoid(float c) {
    const float u = c * __builtin_fmaf(0.0713548163f, c * c, 1.59576912f);
    return sigmoid(__builtin_elementwise_minimum(__builtin_elementwise_maximum(u, -SIGMOID_END), SIGMOID_END));
}
__device__ inline float gelu_tanh(float z) {
    const float c = __builtin_elementwise_maximum(z, -GELU_END);
    return c * tanh_sigmoid(__builtin_elementwise_minimum(c, GELU_END));
}
__device__ inline float gelu_tanh_slope(float z) {
    const float c = __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, -GELU_END), GELU_END);
    const float q = tanh_sigmoid(c);
    return q * (1.f + c * (1.f - q) * __builtin_fmaf(0.214064449f, c * c, 1.59576912f));
}

inline bool known_act(int act) { return act >= TAURUS_ACT_NONE && act <= TAURUS_ACT_GELU_TANH; }
template <int ACT>
__device__ inline float activation(float z) {
    if constexpr (ACT == TAURUS_ACT_RELU) return fmaxf(z, 0.f);
    else if constexpr (ACT == TAURUS_ACT_SILU) return silu(z);
    else if constexpr (ACT == TAURUS_ACT_GELU) return gelu(z);
    else if constexpr (ACT == TAURUS_ACT_GELU_TANH) return gelu_tanh(z);
    else return z;
}
template <int ACT>
__device__ inline float activation_slope(float z) {
    if constexpr (ACT == TAURUS_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    else if constexpr (ACT == TAURUS_ACT_SILU) return silu_slope(z);
    else if constexpr (ACT == TAURUS_ACT_GELU) return gelu_slope(z);
    else if constexpr (ACT == TAURUS_ACT_GELU_TANH) return gelu_tanh_slope(z);
    else return 1.f;
}
// f(integral_constant<int, act>) for an activation known at run time
template <typename F>
inline void with_act(int act, F&& f) {
    switch (act) {
        case TAURUS_ACT_RELU: return f(std::integral_constant<int, TAURUS_ACT_RELU>{});
        case TAURUS_ACT_SILU: return f(std::integral_constant<int, TAURUS_ACT_SILU>{});
        case TAURUS_ACT_GELU: return f(std::integral_constant<int, TAURUS_ACT_GELU>{});
        case TAURUS_ACT_GELU_TANH: return f(std::integral_constant<int, TAURUS_ACT_GELU_TANH>{});
        default: return f(std::integral_constant<int, TAURUS_ACT_NONE>{});
    }
}

}  // namespace taurus
