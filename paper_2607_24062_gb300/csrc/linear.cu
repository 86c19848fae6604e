// acrl_linear and acrl_linear_backward: a bf16 layer with bias, activation and residual, and its gradients.
#include <algorithm>

#include "acrl_host.h"
#include "activation.cuh"
#include "simple_product.cuh"
#include "tma_host.h"

namespace acrl {
namespace {

constexpr int64_t kMostSize = kMaxGrid - 512;

struct Epilogue {
    const void *bias, *residual;
    bool bias_f32, residual_f32, out_f32;
    int64_t ldr, ldp, ldo;
    acrl_bf16* pre;
    void* out;
};

template <int ACT>
__global__ void __launch_bounds__(256) product_kernel(View A, View B, int M, int N, int K, Epilogue e) {
    grid_begin();
    const int tiles = (N + 63) / 64, m0 = int(blockIdx.x) / tiles * 64, n0 = int(blockIdx.x) % tiles * 64;
    simple_product(A, B, M, N, K, m0, n0, [&](int64_t m, int64_t n, float u) {
        if (e.bias) u += load_float(e.bias, e.bias_f32, n);
        if (e.pre) e.pre[m * e.ldp + n] = to_bf16(u);
        u = act<ACT>(u);
        if (e.residual) u += load_float(e.residual, e.residual_f32, m * e.ldr + n);
        if (e.out_f32)
            static_cast<float*>(e.out)[m * e.ldo + n] = u;
        else
            static_cast<acrl_bf16*>(e.out)[m * e.ldo + n] = to_bf16(u);
    });
}

template <int ACT>
acrl_status product(const View& A, const View& B, int64_t M, int64_t N, int64_t K, const Epilogue& e, cudaStream_t s) {
    const int64_t tiles = ((M + 63) / 64) * ((N + 63) / 64);
    if (tiles > kMaxGrid) return ACRL_ERR_INVALID_ARG;
    return launch(product_kernel<ACT>, tiles, 256, 0, 0, s, A, B, int(M), int(N), int(K), e);
}

// g = dy f'(u), rounded, and the columns' sums of the unrounded.
constexpr int kSlopeRows = 256;   // of a CTA

template <int ACT>
__global__ void __launch_bounds__(256) slope_kernel(const acrl_bf16* dy, int64_t lddy, const acrl_bf16* pre, int64_t ldp, int M,
                                                    int N, acrl_bf16* g, int64_t ldg, float* sums) {
    grid_begin();
    const int tiles = (N + 255) / 256, n = int(blockIdx.x) % tiles * 256 + threadIdx.x, part = int(blockIdx.x) / tiles;
    const int m0 = part * kSlopeRows;
    if (n >= N) return;
    float sum = 0.f;
    for (int64_t m = m0; m < min(M, m0 + kSlopeRows); ++m) {
        float v = bf16_to_float(dy[m * lddy + n]);
        if (ACT != ACRL_ACT_NONE) {
            v = __fmul_rn(v, act_slope<ACT>(bf16_to_float(pre[m * ldp + n])));   // the same with and without g: no fma into the sum
            if (g) g[m * ldg + n] = to_bf16(v);
        }
        sum += v;
    }
    if (sums) sums[int64_t(part) * N + n] = sum;
}

__global__ void __launch_bounds__(256) sums_kernel(const float* sums, int parts, int N, float* dbias) {
    grid_begin();
    const int n = int(blockIdx.x) * 256 + threadIdx.x;
    if (n >= N) return;
    float sum = 0.f;
    for (int p = 0; p < parts; ++p) sum += sums[int64_t(p) * N + n];
    dbias[n] = sum;
}

template <typename F>
acrl_status by_act(acrl_activation a, F f) {
    switch (a) {
        case ACRL_ACT_NONE: return f(std::integral_constant<int, ACRL_ACT_NONE>{});
        case ACRL_ACT_RELU: return f(std::integral_constant<int, ACRL_ACT_RELU>{});
        case ACRL_ACT_GELU: return f(std::integral_constant<int, ACRL_ACT_GELU>{});
        case ACRL_ACT_GELU_TANH: return f(std::integral_constant<int, ACRL_ACT_GELU_TANH>{});
        case ACRL_ACT_SILU: return f(std::integral_constant<int, ACRL_ACT_SILU>{});
    }
    return ACRL_ERR_INVALID_ARG;
}

bool dtype_ok(acrl_dtype d) { return d == ACRL_BF16 || d == ACRL_F32; }
bool matrix_ok(const void* p, int64_t cols, int64_t ld) { return p && aligned16(p) && ld >= cols && (ld & 7) == 0; }

struct BackwardParts {
    int64_t ldg, g, sums, end;   // bytes
    BackwardParts(int64_t M, int64_t N, int64_t K) {
        ldg = (N + 7) / 8 * 8;
        g = 0;
        sums = M * ldg * 2;
        end = sums + (M + kSlopeRows - 1) / kSlopeRows * ldg * 4;
    }
};

}  // namespace
}  // namespace acrl

using namespace acrl;

extern "C" int64_t acrl_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) { return M < 0 || N < 0 || K < 0 ? -1 : 0; }

extern "C" acrl_status acrl_linear(const acrl_bf16* x, int64_t M, int64_t K, int64_t ldx, const acrl_bf16* w, int64_t N, int64_t ldw,
                                   const void* bias, acrl_dtype bias_dtype, acrl_activation act, const void* residual,
                                   acrl_dtype residual_dtype, int64_t ldr, acrl_bf16* pre, int64_t ldp, void* out,
                                   acrl_dtype out_dtype, int64_t ldo, void* workspace, int64_t workspace_bytes, int32_t* dev_flags,
                                   acrl_stream stream) {
    if (M < 0 || N < 0 || K < 0 || M > kMostSize || N > kMostSize || K > kMostSize) return ACRL_ERR_INVALID_ARG;
    if (act < ACRL_ACT_NONE || act > ACRL_ACT_SILU || !dtype_ok(out_dtype) || (bias && !dtype_ok(bias_dtype)) ||
        (residual && !dtype_ok(residual_dtype)))
        return ACRL_ERR_INVALID_ARG;
    if (workspace_bytes < acrl_linear_workspace_bytes(M, N, K)) return ACRL_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return ACRL_OK;
    if (!matrix_ok(out, N, ldo) || (residual && !matrix_ok(residual, N, ldr)) || (pre && !matrix_ok(pre, N, ldp)))
        return ACRL_ERR_INVALID_ARG;
    if (K > 0 && (!matrix_ok(x, K, ldx) || !matrix_ok(w, K, ldw) || !operands_on_current_device({x, w, out})))
        return ACRL_ERR_INVALID_ARG;
    const Epilogue e{bias, residual, bias_dtype == ACRL_F32, residual_dtype == ACRL_F32, out_dtype == ACRL_F32, ldr, ldp, ldo, pre,
                     out};
    return by_act(act, [&](auto a) {
        return product<a>(View{x, false, ldx, 1}, View{w, false, ldw, 1}, M, N, K, e, reinterpret_cast<cudaStream_t>(stream));
    });
}

extern "C" int64_t acrl_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    return M < 0 || N < 0 || K < 0 ? -1 : BackwardParts(M, N, K).end;
}

extern "C" acrl_status acrl_linear_backward(const acrl_bf16* dy, int64_t M, int64_t N, int64_t lddy, const acrl_bf16* x, int64_t K,
                                            int64_t ldx, const acrl_bf16* w, int64_t ldw, acrl_activation act,
                                            const acrl_bf16* pre, int64_t ldp, void* dx, acrl_dtype dx_dtype, int64_t lddx, void* dw,
                                            acrl_dtype dw_dtype, int64_t lddw, float* dbias, void* workspace,
                                            int64_t workspace_bytes, int32_t* dev_flags, acrl_stream stream) {
    if (M < 0 || N < 0 || K < 0 || M > kMostSize || N > kMostSize || K > kMostSize) return ACRL_ERR_INVALID_ARG;
    if (act < ACRL_ACT_NONE || act > ACRL_ACT_SILU || (dx && !dtype_ok(dx_dtype)) || (dw && !dtype_ok(dw_dtype)))
        return ACRL_ERR_INVALID_ARG;
    const BackwardParts parts(M, N, K);
    if (workspace_bytes < parts.end) return ACRL_ERR_INVALID_ARG;
    const bool has_dx = dx && M > 0 && K > 0, has_dw = dw && N > 0 && K > 0, has_g = M > 0 && N > 0;
    if ((has_dx && !matrix_ok(dx, K, lddx)) || (has_dw && !matrix_ok(dw, K, lddw))) return ACRL_ERR_INVALID_ARG;
    if (has_g && (!matrix_ok(dy, N, lddy) || (act != ACRL_ACT_NONE && !matrix_ok(pre, N, ldp)))) return ACRL_ERR_INVALID_ARG;
    if (act == ACRL_ACT_NONE && pre) return ACRL_ERR_INVALID_ARG;
    if (has_g && ((has_dx && !matrix_ok(w, K, ldw)) || (has_dw && !matrix_ok(x, K, ldx)))) return ACRL_ERR_INVALID_ARG;
    if (!has_dx && !has_dw && !(dbias && N > 0)) return ACRL_OK;
    if (has_g && parts.end > 0 && (!workspace || !aligned16(workspace))) return ACRL_ERR_INVALID_ARG;
    if (has_g && !operands_on_current_device({dy, workspace})) return ACRL_ERR_INVALID_ARG;
    if ((has_dx && has_g && !operands_on_current_device({w, dx})) || (has_dw && has_g && !operands_on_current_device({x, dw})))
        return ACRL_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    uint8_t* base = static_cast<uint8_t*>(workspace);
    const acrl_bf16* g = dy;
    int64_t ldg = lddy;
    acrl_status st = ACRL_OK;
    if (has_g && (act != ACRL_ACT_NONE || dbias)) {
        acrl_bf16* to = act == ACRL_ACT_NONE || !(has_dx || has_dw) ? nullptr : reinterpret_cast<acrl_bf16*>(base + parts.g);
        float* sums = dbias ? reinterpret_cast<float*>(base + parts.sums) : nullptr;
        const int64_t rows = (M + kSlopeRows - 1) / kSlopeRows, tiles = (N + 255) / 256;
        if (rows * tiles > kMaxGrid) return ACRL_ERR_INVALID_ARG;
        st = by_act(act, [&](auto a) {
            return launch(slope_kernel<a>, rows * tiles, 256, 0, 0, s, dy, lddy, pre, ldp, int(M), int(N), to, parts.ldg, sums);
        });
        if (st != ACRL_OK) return st;
        if (to) {
            g = to;
            ldg = parts.ldg;
        }
        if (dbias) st = launch(sums_kernel, tiles, 256, 0, 0, s, static_cast<const float*>(sums), int(rows), int(N), dbias);
        if (st != ACRL_OK) return st;
    } else if (dbias && N > 0) {
        if (cudaMemsetAsync(dbias, 0, size_t(N) * 4, s) != cudaSuccess) return launch_status();
    }
    // without rows, or without columns of dy, the sums are empty: K = 0 below
    if (has_dx) {
        const Epilogue e{nullptr, nullptr, false, false, dx_dtype == ACRL_F32, 0, 0, lddx, nullptr, dx};
        st = product<ACRL_ACT_NONE>(View{g, false, ldg, 1}, View{w, false, 1, ldw}, M, K, has_g ? N : 0, e, s);
        if (st != ACRL_OK) return st;
    }
    if (has_dw) {
        const Epilogue e{nullptr, nullptr, false, false, dw_dtype == ACRL_F32, 0, 0, lddw, nullptr, dw};
        st = product<ACRL_ACT_NONE>(View{g, false, 1, ldg}, View{x, false, 1, ldx}, N, K, has_g ? M : 0, e, s);
    }
    return st;
}
