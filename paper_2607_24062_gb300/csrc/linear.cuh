// What the ways to make a layer's product share: what follows the sum, and loads and stores of both types.
#pragma once

#include <cstdint>
#include <type_traits>

#include "acrl_host.h"
#include "activation.cuh"

namespace acrl {

// What follows the sum: out = f(sum + bias) + residual.
struct Finish {
    const void *bias, *residual;
    void* out;
    acrl_bf16* pre;
    int64_t ldr, ldp, ldo;
    int act;
    bool bias_f32, residual_f32, out_f32;
};

// A layer of a few rows (linear_few.cu), where it is faster than the tensor memory's way.
bool linear_few_rows(int64_t M, int64_t N, int64_t K);
acrl_status linear_few(const acrl_bf16* x, int64_t M, int64_t K, int64_t ldx, const acrl_bf16* w, int64_t N, int64_t ldw, const Finish& f,
                       cudaStream_t s);

namespace {

template <typename F>
__host__ __device__ __forceinline__ acrl_status by_act(int a, F f) {
    switch (a) {
        case ACRL_ACT_NONE: return f(std::integral_constant<int, ACRL_ACT_NONE>{});
        case ACRL_ACT_RELU: return f(std::integral_constant<int, ACRL_ACT_RELU>{});
        case ACRL_ACT_GELU: return f(std::integral_constant<int, ACRL_ACT_GELU>{});
        case ACRL_ACT_GELU_TANH: return f(std::integral_constant<int, ACRL_ACT_GELU_TANH>{});
        case ACRL_ACT_SILU: return f(std::integral_constant<int, ACRL_ACT_SILU>{});
    }
    return ACRL_ERR_INVALID_ARG;
}

__device__ __forceinline__ void store_float(void* p, bool f32, int64_t i, float v) {
    if (f32)
        static_cast<float*>(p)[i] = v;
    else
        static_cast<acrl_bf16*>(p)[i] = to_bf16(v);
}

template <int N>
__device__ __forceinline__ void apply(int which, float (&v)[N]) {
    by_act(which, [&](auto a) {
        if constexpr (a != ACRL_ACT_NONE && N == 1) {
            v[0] = act<a>(v[0]);
        } else if constexpr (a != ACRL_ACT_NONE) {
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                float u[2] = {v[j], v[j + 1]};
                act2<a>(u);
                v[j] = u[0];
                v[j + 1] = u[1];
            }
        }
        return ACRL_OK;
    });
}

// N values of a row from column c on, as fp32; N and c multiples of four.
template <int N>
__device__ __forceinline__ void load_row(const void* p, bool f32, int64_t row, int c, int cols, float (&v)[N]) {
    if (c + N > cols) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = c + j < cols ? load_float(p, f32, row + c + j) : 0.f;
    } else if (f32) {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + row + c);
#pragma unroll
        for (int j = 0; j < N / 4; ++j) {
            const float4 x = q[j];
            v[4 * j] = x.x;
            v[4 * j + 1] = x.y;
            v[4 * j + 2] = x.z;
            v[4 * j + 3] = x.w;
        }
    } else {
        const uint2* q = reinterpret_cast<const uint2*>(static_cast<const acrl_bf16*>(p) + row + c);
#pragma unroll
        for (int j = 0; j < N / 4; ++j) {
            const uint2 x = q[j];
            v[4 * j] = bf16_lo(x.x);
            v[4 * j + 1] = bf16_hi(x.x);
            v[4 * j + 2] = bf16_lo(x.y);
            v[4 * j + 3] = bf16_hi(x.y);
        }
    }
}

}  // namespace
}  // namespace acrl
