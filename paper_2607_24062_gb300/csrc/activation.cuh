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

// Two fp32 numbers in the pipe's packed instructions, which round as the single ones do.
using Two = unsigned long long;
__device__ __forceinline__ Two two(float a, float b) {
    Two v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ Two both(float c) { return two(c, c); }
__device__ __forceinline__ void part(Two v, float (&u)[2]) { asm("mov.b64 {%0, %1}, %2;" : "=f"(u[0]), "=f"(u[1]) : "l"(v)); }
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two v;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
    return v;
}

// The logistic function of two numbers, p = 1 / (1 + e^-z), and q = 1 - p.  The exponential is the square of its root, taken down
// by 2^-32 before: 2^-64 + 2^-64 e^-z stays a normal number down to z = -131, where p is zero in fp32, and p and q keep their
// digits where they are small (1 / (1 + e^-z) as it stands is zero below -87.3, where silu is still -1e-36).  Below -131 q is no
// number.
__device__ __forceinline__ void logistic(Two z, Two& p, Two& q) {
    float a[2], d[2];
    part(mul2(z, both(-0.5f * kLog2e)), a);
    const Two root = mul2(two(ex2(a[0]), ex2(a[1])), both(0x1p-32f));
    part(fma2(root, root, both(0x1p-64f)), d);
    const Two r = two(fast_recip(d[0]), fast_recip(d[1]));
    p = mul2(r, both(0x1p-64f));
    q = mul2(mul2(root, root), r);
}

// Phi(-|u|) of two numbers, and e^(-u^2 / 2) beside it.  With x = |u| and t = 1 / (1 + 0.31 x), e^(x^2 / 2) Phi(-x) is t times a
// polynomial in t of degree seven, fitted by linear programming for the least relative error from x = 0 to 15.5: 1.7e-7, and
// 4.6e-7 as evaluated in fp32.  So the tail keeps its digits as far down as fp32 goes: gelu(-10) to 2^-17 of itself, by the square's
// rounding in the exponent.  (Abramowitz and Stegun's 7.1.26, fitted for its absolute error, was off by 1.6e-3 at -5 and 2e-2 at
// -10.)  The exponential is a square, so that it does not vanish before its product with u does.  One exponential and one
// reciprocal each, the rest in packed instructions: 4,096 x 16,384 x 1,024 89.6 us, of which the product alone takes 79.4; with single
// ones 104, with 7.1.26 in single ones 96.
__device__ __forceinline__ void normal_tail(const float (&u)[2], Two& tail, Two& bell) {
    const Two v = two(u[0], u[1]);
    const Two t = two(fast_recip(fmaf(0.31f, fabsf(u[0]), 1.f)), fast_recip(fmaf(0.31f, fabsf(u[1]), 1.f)));
    float e[2];
    part(mul2(mul2(v, both(-0.25f * kLog2e)), v), e);
    const Two root = two(ex2(e[0]), ex2(e[1]));
    bell = mul2(root, root);
    constexpr float c[] = {0.0359040648f, -0.141878068f, 0.15556632f, -0.0153910015f, 0.11038553f, 0.107681662f, 0.124075733f, 0.123655833f};
    Two p = both(c[0]);
#pragma unroll
    for (int k = 1; k < 8; ++k) p = fma2(p, t, both(c[k]));
    tail = mul2(mul2(bell, t), p);
}

// u Phi(u): u less, or beyond 0 nothing but, its part of the tail.  (100 keeps infinity from the tail's zero.)
__device__ __forceinline__ void gelu(float (&u)[2]) {
    Two tail, bell;
    normal_tail(u, tail, bell);
    float t[2];
    part(tail, t);
#pragma unroll
    for (int j = 0; j < 2; ++j) u[j] = fmaf(-fabsf(fminf(u[j], 100.f)), t[j], fmaxf(u[j], 0.f));
}

// Phi(u) + u phi(u).
__device__ __forceinline__ void gelu_slope(float (&u)[2]) {
    Two tail, bell;
    normal_tail(u, tail, bell);
    float p[2];
    part(tail, p);
#pragma unroll
    for (int j = 0; j < 2; ++j) p[j] = u[j] < 0.f ? p[j] : 1.f - p[j];
    part(fma2(mul2(two(u[0], u[1]), both(kNormal)), bell, two(p[0], p[1])), u);
}

__device__ __forceinline__ float relu(float u) { return u > 0.f || u != u ? u : 0.f; }
__device__ __forceinline__ float step(float u) { return u > 0.f ? 1.f : u != u ? u : 0.f; }

// u at least `least` and, with BOTH, at most -least; a NaN stays one.
template <bool BOTH>
__device__ __forceinline__ float within(float u, float least) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(u) : "f"(least));
    if (BOTH) asm("min.NaN.f32 %0, %0, %1;" : "+f"(u) : "f"(-least));
    return u;
}

// f of two numbers.
template <int ACT>
__device__ __forceinline__ void act2(float (&u)[2]) {
    if (ACT == ACRL_ACT_RELU) {
        u[0] = relu(u[0]);
        u[1] = relu(u[1]);
    }
    if (ACT == ACRL_ACT_GELU) gelu(u);
    if (ACT == ACRL_ACT_GELU_TANH || ACT == ACRL_ACT_SILU) {
        const Two v = two(u[0], u[1]);
        Two p, q;
        logistic(ACT == ACRL_ACT_SILU ? v : mul2(fma2(mul2(mul2(v, v), both(kTanhC)), v, v), both(kTanhK)), p, q);
        part(mul2(v, p), u);
    }
}

// f' of two numbers.  Of the logistic function's, numbers so small that p is zero are taken to ones where q is a number.
template <int ACT>
__device__ __forceinline__ void act_slope2(float (&u)[2]) {
    if (ACT == ACRL_ACT_RELU) {
        u[0] = step(u[0]);
        u[1] = step(u[1]);
    }
    if (ACT == ACRL_ACT_GELU) gelu_slope(u);
    if (ACT == ACRL_ACT_GELU_TANH) {   // beyond 11.5 p is 0 or 1, and u^2 could leave fp32's range
        const Two v = two(within<true>(u[0], -11.5f), within<true>(u[1], -11.5f)), square = mul2(v, v);
        Two p, q;
        logistic(mul2(fma2(mul2(square, both(kTanhC)), v, v), both(kTanhK)), p, q);
        part(fma2(mul2(v, mul2(p, q)), fma2(square, both(3.f * kTanhC * kTanhK), both(kTanhK)), p), u);
    }
    if (ACT == ACRL_ACT_SILU) {   // p (1 + u (1 - p))
        const Two v = two(within<false>(u[0], -130.f), within<false>(u[1], -130.f));
        Two p, q;
        logistic(v, p, q);
        part(mul2(p, fma2(v, q, both(1.f))), u);
    }
}

template <int ACT>
__device__ __forceinline__ float act(float u) {
    float v[2] = {u, 0.f};
    act2<ACT>(v);
    return v[0];
}

__device__ __forceinline__ float load_float(const void* p, bool f32, int64_t i) {
    return f32 ? static_cast<const float*>(p)[i] : bf16_to_float(static_cast<const acrl_bf16*>(p)[i]);
}

__device__ __forceinline__ acrl_bf16 to_bf16(float v) { return acrl_bf16(pack_bf16x2(v, 0.f) & 0xffffu); }

}  // namespace
}  // namespace acrl
