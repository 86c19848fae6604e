// The activations of a linear layer and their derivatives, in fp32.
#pragma once

#include "acrl_device.cuh"

namespace acrl {
namespace {

constexpr float kTanhK = 1.5957691216057308f;   // 2 sqrt(2 / pi): (1 + tanh z) / 2 is the logistic function of 2 z
constexpr float kTanhC = 0.044715f;
constexpr float kNormal = 0.3989422804014327f;  // 1 / sqrt(2 pi)

template <int ACT>
__device__ __forceinline__ float act(float u) {
    if (ACT == ACRL_ACT_RELU) return u > 0.f || u != u ? u : 0.f;
    if (ACT == ACRL_ACT_GELU) return u * normcdff(u);
    if (ACT == ACRL_ACT_GELU_TANH) return u / (1.f + expf(-kTanhK * fmaf(kTanhC * u * u, u, u)));
    if (ACT == ACRL_ACT_SILU) return u / (1.f + expf(-u));
    return u;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float u) {
    if (ACT == ACRL_ACT_RELU) return u > 0.f ? 1.f : u != u ? u : 0.f;
    if (ACT == ACRL_ACT_GELU) return fmaf(u * kNormal, expf(-0.5f * u * u), normcdff(u));
    if (ACT == ACRL_ACT_GELU_TANH) {
        // beyond 30 the logistic function is 0 or 1, and u^2 could leave fp32's range
        const float v = u > 30.f ? 30.f : u < -30.f ? -30.f : u, v2 = v * v;
        const float p = 1.f / (1.f + expf(-kTanhK * fmaf(kTanhC * v2, v, v)));
        return fmaf(v * p * (1.f - p), kTanhK * fmaf(3.f * kTanhC, v2, 1.f), p);
    }
    if (ACT == ACRL_ACT_SILU) {
        const float p = 1.f / (1.f + expf(-u));
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
