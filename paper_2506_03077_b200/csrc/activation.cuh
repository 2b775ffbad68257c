// Activations of the product epilogue and their slopes, in fp32.
//   FAST: through ex2.approx and rcp.approx (relative error below 1e-6, for results that are rounded to bf16);
//   otherwise CUDA's expf / tanhf and IEEE division (fp32 results).
// tanh is taken as 2 sigmoid(2x) - 1, so that GELU's tanh form is z sigmoid(2a): one exponential and one reciprocal.
#pragma once

#include "common.cuh"

namespace sbp {

constexpr float kGeluA = 0.7978845608028654f;       // sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;
constexpr float kSqrtHalf = 0.7071067811865476f;
constexpr float kInvSqrt2Pi = 0.3989422804014327f;

// 1 / (1 + exp(-x)): 0 and 1 at the ends of the range, no overflow into NaN
template <bool FAST>
__device__ __forceinline__ float sigmoid(float x) {
    if constexpr (FAST) {
        float e, r;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-1.4426950408889634f * x));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
        return r;
    } else {
        return 1.f / (1.f + expf(-x));
    }
}

// The normal distribution function of z and exp(-z^2 / 2) on the way, to 1e-7 absolute: erfc by formula 7.1.26 of
// Abramowitz and Stegun, Handbook of Mathematical Functions (t = 1 / (1 + 0.3275911 x), a polynomial of degree 5 in t times
// exp(-x^2), error below 1.5e-7).  A dozen operations instead of the forty of erff: the epilogue of a product with a short K
// and this activation is bound by them (8192 x 8192 x 512: 192 us with erff).
__device__ __forceinline__ float normal_cdf(float z, float &bell) {
    const float x = fabsf(z) * kSqrtHalf;
    float t;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(bell) : "f"(-0.7213475204444817f * z * z));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(0.3275911f, x, 1.f)));
    const float q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    const float tail = 0.5f * q * bell;                  // of |z|
    return z < 0.f ? tail : 1.f - tail;
}

template <int ACT, bool FAST>
__device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == STREAMBP_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
    else if constexpr (ACT == STREAMBP_ACT_GELU) {
        if constexpr (FAST) {
            float bell;
            return z * normal_cdf(z, bell);
        } else return 0.5f * z * (1.f + erff(z * kSqrtHalf));
    } else if constexpr (ACT == STREAMBP_ACT_GELU_TANH) {
        const float a = kGeluA * fmaf(kGeluB * z * z, z, z);
        if constexpr (FAST) return z * sigmoid<true>(2.f * a);
        else return 0.5f * z * (1.f + tanhf(a));
    } else if constexpr (ACT == STREAMBP_ACT_SILU) return z * sigmoid<FAST>(z);
    else return z;
}

// d activate(z) / dz
template <int ACT, bool FAST>
__device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == STREAMBP_ACT_RELU) return z > 0.f ? 1.f : (z != z ? z : 0.f);
    else if constexpr (ACT == STREAMBP_ACT_GELU) {
        if constexpr (FAST) {
            float bell;
            const float c = normal_cdf(z, bell);
            return fmaf(z * kInvSqrt2Pi, bell, c);
        } else return fmaf(z * kInvSqrt2Pi, expf(-0.5f * z * z), 0.5f * (1.f + erff(z * kSqrtHalf)));
    } else if constexpr (ACT == STREAMBP_ACT_GELU_TANH) {
        // with s = sigmoid(2a): 0.5 (1 + tanh a) = s and 0.5 (1 - tanh^2 a) = 2 s (1 - s).  The factors z of z^2 are applied to
        // z s (1 - s) one by one: that is zero long before z^2 overflows, and zero times infinity is not.
        const float a = kGeluA * fmaf(kGeluB * z * z, z, z);
        const float s = sigmoid<FAST>(2.f * a), w = z * s * (1.f - s);
        return fmaf(2.f * kGeluA, fmaf(3.f * kGeluB * z, z * w, w), s);
    } else if constexpr (ACT == STREAMBP_ACT_SILU) {
        const float s = sigmoid<FAST>(z);
        return s * fmaf(z, 1.f - s, 1.f);
    } else return 1.f;
}

}  // namespace sbp
