// 8-bit matrices with power-of-two scales: what the kernels that make them and the
// kernels that multiply them share.
#pragma once

#include <algorithm>

#include "acrl_device.cuh"
#include "acrl_host.h"

namespace acrl {

struct Matrix {   // one operand of a product, as the entry points take it
    const uint8_t* q;
    int64_t rows, ld;
    acrl_fp8_format format;
    const uint8_t* scale;
    int64_t lds;
    acrl_fp8_block block;
};

inline bool matrix_ok(const Matrix& m, int64_t K) {
    if (m.rows < 0 || m.rows > kMaxGrid - 256 || m.ld < K || (m.ld & 15) || m.lds < (K + 127) / 128) return false;
    if (m.format != ACRL_FP8_E4M3 && m.format != ACRL_FP8_E5M2) return false;
    return m.block == ACRL_FP8_ROW || m.block == ACRL_FP8_TILE;
}

// out = A B^T of one row of A and a matrix of moderate size, in fp8_few.cu: `a`, or bf16 activations `x` quantised in the kernel.
// kFewNot: these sizes are not its.
constexpr acrl_status kFewNot = ACRL_ERR_NOT_IMPLEMENTED;
bool few_rows(int64_t M, int64_t N, int64_t K);
acrl_status matmul_few(const Matrix& a, const acrl_bf16* x, const Matrix& b, int64_t K, void* out, acrl_dtype out_dtype, int32_t* flags,
                       cudaStream_t s);

// Where a quantised matrix goes.
struct Quantised {
    uint8_t* q;
    int64_t ldq;
    uint8_t* scale;
    int64_t lds;
};

// For a layer's backward: dy [M, N] by rows (`as`) and its transpose by rows (`turned`), dy read once, and the transpose of x
// [M, K] by rows; checked arguments.
acrl_status quantize_backward(const acrl_bf16* dy, int64_t M, int64_t N, int64_t lddy, acrl_fp8_format format, const Quantised& as,
                              const Quantised& turned, const acrl_bf16* x, int64_t K, int64_t ldx, acrl_fp8_format x_format,
                              const Quantised& x_turned, int32_t* flags, cudaStream_t s);

namespace {

constexpr int kTopExp[2] = {8, 15};        // of 448 and 57344, by acrl_fp8_format

// 8 consecutive elements of a row in registers, as fp32 bit patterns.
template <typename T>
__device__ __forceinline__ void load8(const T* __restrict__ p, int n, float (&f)[8]);

template <>
__device__ __forceinline__ void load8<acrl_bf16>(const acrl_bf16* __restrict__ p, int n, float (&f)[8]) {
    if (n >= 8) {
        const uint4 v = ld_stream(reinterpret_cast<const uint4*>(p));
        f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x);
        f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
        f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z);
        f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = j < n ? bf16_to_float(p[j]) : 0.f;
}

template <>
__device__ __forceinline__ void load8<float>(const float* __restrict__ p, int n, float (&f)[8]) {
    if (n >= 8) {
        const uint4 a = ld_stream(reinterpret_cast<const uint4*>(p)), b = ld_stream(reinterpret_cast<const uint4*>(p) + 1);
        f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y); f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
        f[4] = __uint_as_float(b.x); f[5] = __uint_as_float(b.y); f[6] = __uint_as_float(b.z); f[7] = __uint_as_float(b.w);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = j < n ? p[j] : 0.f;
}

// Bits of |f|: they order as unsigned integers, with an infinity and then NaN above every number.
__device__ __forceinline__ uint32_t abs_bits(float f) { return __float_as_uint(f) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t max8(const float (&f)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, abs_bits(f[j]));
    return m;
}

// A block's scale from the bits of its maximum: the stored byte, and the factor 2^-e.
struct Scale {
    uint32_t byte;   // e + 127; 255 (NaN) for a block with an infinity or a NaN
    float inv;       // NaN for such a block: every element becomes one
};

template <int FMT>
__device__ __forceinline__ Scale block_scale(uint32_t m) {
    if (m == 0u) return Scale{127u, 1.f};
    if (m >= 0x7f800000u) return Scale{255u, __int_as_float(0x7fc00000)};
    // a below 2^-126 is stored without its leading one; its e is below -127 whatever its bits, and is raised to that
    const int e = max(int(m >> 23) - 127 - kTopExp[FMT] + ((m & 0x7fffffu) > 0x600000u ? 1 : 0), -127);
    return Scale{uint32_t(e + 127), __uint_as_float(uint32_t(127 - e) << 23)};
}

// Two fp32 numbers times a power of two to a pair of 8-bit numbers, `lo` in the low byte.
template <int FMT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi, float inv) {
    uint16_t r;
    if (FMT == ACRL_FP8_E4M3)
        asm("{\n .reg .b64 v, s;\n .reg .f32 a, b;\n mov.b64 v, {%1, %2};\n mov.b64 s, {%3, %3};\n mul.rn.f32x2 v, v, s;\n"
            " mov.b64 {a, b}, v;\n cvt.rn.satfinite.e4m3x2.f32 %0, b, a;\n}" : "=h"(r) : "f"(lo), "f"(hi), "f"(inv));
    else
        asm("{\n .reg .b64 v, s;\n .reg .f32 a, b;\n mov.b64 v, {%1, %2};\n mov.b64 s, {%3, %3};\n mul.rn.f32x2 v, v, s;\n"
            " mov.b64 {a, b}, v;\n cvt.rn.satfinite.e5m2x2.f32 %0, b, a;\n}" : "=h"(r) : "f"(lo), "f"(hi), "f"(inv));
    return r;
}

template <int FMT>
__device__ __forceinline__ uint2 pack8(const float (&f)[8], float inv) {
    uint2 o;
    o.x = pack2<FMT>(f[0], f[1], inv) | pack2<FMT>(f[2], f[3], inv) << 16;
    o.y = pack2<FMT>(f[4], f[5], inv) | pack2<FMT>(f[6], f[7], inv) << 16;
    return o;
}

}  // namespace
}  // namespace acrl
