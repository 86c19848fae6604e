// The activations of a linear layer and their derivatives, in fp32.
#pragma once

#include "acrl_device.cuh"

namespace acrl {
namespace {

constexpr float kTanhK = 1.5957691216057308f;   // 2 sqrt(2 / pi): (1 + tanh z) / 2 is the logistic function of 2 z
constexpr float kTanhC = 0.044715f;
constexpr float kNormal = 0.3989422804014327f;  // 1 / sqrt(2 pi)

// 1 / x, to 2^-23 of it; 0 for x beyond 2^126.
__device__ __forceinline__ float fast_recip(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 1 / (1 + e^-x).
__device__ __forceinline__ float logistic(float x) { return fast_recip(1.f + ex2(-kLog2e * x)); }

// Phi(u), and e^(-u^2 / 2) beside it: erfc by Abramowitz and Stegun's formula 7.1.26 (absolute error 1.5e-7), which takes one
// exponential and one reciprocal.  CUDA's normcdff, more exact in the tail than a rounding to bf16 shows, cost a product of
// 4,096 x 16,384 x 4,096 with its pre-activation 80 us of 380.
__device__ __forceinline__ float normal_cdf(float u, float& bell) {
    const float t = fast_recip(fmaf(0.3275911f * 0.70710678f, fabsf(u), 1.f));
    bell = ex2(-0.5f * kLog2e * u * u);
    const float tail = 0.5f * bell * t *
                       fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    return u < 0.f ? tail : 1.f - tail;
}

template <int ACT>
__device__ __forceinline__ float act(float u) {
    if (ACT == ACRL_ACT_RELU) return u > 0.f || u != u ? u : 0.f;
    if (ACT == ACRL_ACT_GELU) {
        float bell;
        return u * normal_cdf(u, bell);
    }
    if (ACT == ACRL_ACT_GELU_TANH) return u * logistic(kTanhK * fmaf(kTanhC * u * u, u, u));
    if (ACT == ACRL_ACT_SILU) return u * logistic(u);
    return u;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float u) {
    if (ACT == ACRL_ACT_RELU) return u > 0.f ? 1.f : u != u ? u : 0.f;
    if (ACT == ACRL_ACT_GELU) {
        float bell;
        const float p = normal_cdf(u, bell);
        return fmaf(u * kNormal, bell, p);
    }
    if (ACT == ACRL_ACT_GELU_TANH) {
        // beyond 30 the logistic function is 0 or 1, and u^2 could leave fp32's range
        const float v = u > 30.f ? 30.f : u < -30.f ? -30.f : u, v2 = v * v;
        const float p = logistic(kTanhK * fmaf(kTanhC * v2, v, v));
        return fmaf(v * p * (1.f - p), kTanhK * fmaf(3.f * kTanhC, v2, 1.f), p);
    }
    if (ACT == ACRL_ACT_SILU) {
        const float p = logistic(u);
        return p == 0.f ? 0.f : p * fmaf(u, 1.f - p, 1.f);
    }
    return 1.f;
}

__device__ __forceinline__ float load_float(const void* p, bool f32, int64_t i) {
    return f32 ? static_cast<const float*>(p)[i] : bf16_to_float(static_cast<const acrl_bf16*>(p)[i]);
}

__device__ __forceinline__ acrl_bf16 to_bf16(float v) { return acrl_bf16(pack_bf16x2(v, 0.f) & 0xffffu); }

}  // namespace
}  // namespace acrl
