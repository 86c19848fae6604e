// acrl_orthogonalize: Newton-Schulz steps on an update.  With X (m x n, m <= n; a tall matrix's transpose) a step is
//     A = X X^T,   Q = a I + b A + c A^2,   X <- Q X,
// so the polynomial in the Gram matrix is made on its m x m elements, and X is read and written once.
#include <algorithm>

#include "acrl_host.h"
#include "simple_product.cuh"
#include "tma_host.h"

namespace acrl {
namespace {

constexpr int kMostSteps = 64;

// 1 / (|G| + eps) of each matrix; NaN, and the flag, where an element is none.
__global__ void __launch_bounds__(1024) norm_kernel(View g, int64_t stride, int m, int n, float eps, double* inv, int32_t* flags) {
    __shared__ double part[32];
    grid_begin();
    const int64_t at = int64_t(blockIdx.x) * stride;
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < int64_t(m) * n; i += 1024) {
        const double v = load_float(g.p, g.f32, at + i / n * g.row + i % n);
        sum += v * v;
    }
    sum = warp_sum(sum);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int i = 0; i < 32; ++i) sum += part[i];
        const bool bad = !(sum <= 1.7e308);
        if (bad) raise_flag(flags, ACRL_FLAG_NONFINITE);
        const double d = sqrt(sum) + double(eps);
        inv[blockIdx.x] = bad ? nan("") : d > 0.0 ? 1.0 / d : 0.0;
    }
}

__global__ void __launch_bounds__(256) first_kernel(View g, int64_t stride, int m, int n, bool tall, const double* inv, float* x) {
    grid_begin();
    const int64_t b = blockIdx.y, size = int64_t(m) * n;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < size; i += int64_t(gridDim.x) * 256) {
        const int64_t r = i / n, c = i % n;
        const float v = load_float(g.p, g.f32, b * stride + r * g.row + c);
        x[b * size + (tall ? c * m + r : i)] = float(double(v) * inv[b]);
    }
}

// MODE 0: A = X X^T; 1: Q = a I + b A + c A A^T; 2: X' = Q X; 3: the same to `out`, scaled.
struct Step {
    float a, b, c, scale;
    const float *x, *gram, *q;
    float* to;
    acrl_bf16* out;
    int64_t ldo, out_stride;
    int m, n;
    bool tall;
};

template <int MODE>
__global__ void __launch_bounds__(256) step_kernel(Step s) {
    grid_begin();
    const int64_t b = blockIdx.y, mm = int64_t(s.m) * s.m, mn = int64_t(s.m) * s.n;
    const int N = MODE < 2 ? s.m : s.n, K = MODE == 0 ? s.n : s.m;
    const int tiles = (N + 63) / 64, m0 = int(blockIdx.x) / tiles * 64, n0 = int(blockIdx.x) % tiles * 64;
    const View X{s.x + b * mn, true, s.n, 1}, XT{s.x + b * mn, true, 1, s.n};
    const View A{s.gram + b * mm, true, s.m, 1}, Q{s.q + b * mm, true, s.m, 1};
    simple_product(MODE == 0 ? X : MODE == 1 ? A : Q, MODE == 0 ? X : MODE == 1 ? A : XT, s.m, N, K, m0, n0,
                   [&](int64_t i, int64_t j, float v) {
                       if (MODE == 1) v = fmaf(s.c, v, fmaf(s.b, A.at(i, j), i == j ? s.a : 0.f));
                       if (MODE < 3)
                           s.to[b * (MODE < 2 ? mm : mn) + i * N + j] = v;
                       else
                           s.out[b * s.out_stride + (s.tall ? j * s.ldo + i : i * s.ldo + j)] = to_bf16(s.scale * v);
                   });
}

struct Parts {
    int64_t inv, x[2], gram, q, end;
    Parts(int64_t batch, int64_t m, int64_t n) {
        const int64_t k = std::min(m, n);
        inv = 0;
        x[0] = (batch * 8 + 15) / 16 * 16;
        x[1] = x[0] + (batch * m * n * 4 + 15) / 16 * 16;
        gram = x[1] + (batch * m * n * 4 + 15) / 16 * 16;
        q = gram + (batch * k * k * 4 + 15) / 16 * 16;
        end = q + (batch * k * k * 4 + 15) / 16 * 16;
    }
};

}  // namespace
}  // namespace acrl

using namespace acrl;

extern "C" int64_t acrl_orthogonalize_workspace_bytes(int64_t batch, int64_t m, int64_t n) {
    return batch < 0 || m < 0 || n < 0 ? -1 : batch == 0 || m == 0 || n == 0 ? 0 : Parts(batch, m, n).end;
}

extern "C" acrl_status acrl_orthogonalize(const void* g, acrl_dtype g_dtype, int64_t batch, int64_t m, int64_t n, int64_t ldg,
                                          int64_t g_stride, const float* coeffs, int32_t steps, float eps, float scale,
                                          acrl_bf16* out, int64_t ldo, int64_t out_stride, void* workspace, int64_t workspace_bytes,
                                          int32_t* dev_flags, acrl_stream stream) {
    if (batch < 0 || m < 0 || n < 0 || batch > 65535 || m > kMaxGrid - 512 || n > kMaxGrid - 512) return ACRL_ERR_INVALID_ARG;
    if ((g_dtype != ACRL_BF16 && g_dtype != ACRL_F32) || steps < 1 || steps > kMostSteps || !coeffs) return ACRL_ERR_INVALID_ARG;
    if (!(eps >= 0.f && eps < INFINITY) || !(scale > -INFINITY && scale < INFINITY)) return ACRL_ERR_INVALID_ARG;
    for (int i = 0; i < 3 * steps; ++i)
        if (!(coeffs[i] > -INFINITY && coeffs[i] < INFINITY)) return ACRL_ERR_INVALID_ARG;
    if (workspace_bytes < acrl_orthogonalize_workspace_bytes(batch, m, n)) return ACRL_ERR_INVALID_ARG;
    if (batch == 0 || m == 0 || n == 0) return ACRL_OK;
    const int64_t to = g_dtype == ACRL_BF16 ? 7 : 3;
    if (!g || !aligned16(g) || ldg < n || (ldg & to) || (g_stride & to) || !out || !aligned16(out) || ldo < n || (ldo & 7) ||
        (out_stride & 7) || !workspace || !aligned16(workspace))
        return ACRL_ERR_INVALID_ARG;
    if (batch > 1 && (g_stride < (m - 1) * ldg + n || out_stride < (m - 1) * ldo + n)) return ACRL_ERR_INVALID_ARG;
    if (!operands_on_current_device({g, out, workspace})) return ACRL_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const Parts p(batch, m, n);
    uint8_t* base = static_cast<uint8_t*>(workspace);
    const bool tall = m > n;
    const View G{g, g_dtype == ACRL_F32, ldg, 1};
    double* inv = reinterpret_cast<double*>(base + p.inv);
    float* x[2] = {reinterpret_cast<float*>(base + p.x[0]), reinterpret_cast<float*>(base + p.x[1])};
    norm_kernel<<<unsigned(batch), 1024, 0, s>>>(G, g_stride, int(m), int(n), eps, inv, dev_flags);
    first_kernel<<<dim3(unsigned(std::min<int64_t>(1024, (m * n + 255) / 256)), unsigned(batch)), 256, 0, s>>>(G, g_stride, int(m), int(n), tall, inv, x[0]);
    Step t = {};
    t.m = int(std::min(m, n));
    t.n = int(std::max(m, n));
    t.tall = tall;
    t.scale = scale;
    t.out = out;
    t.ldo = ldo;
    t.out_stride = out_stride;
    float* gram = reinterpret_cast<float*>(base + p.gram);
    float* q = reinterpret_cast<float*>(base + p.q);
    t.gram = gram;
    t.q = q;
    const int64_t tm = (t.m + 63) / 64, tn = (t.n + 63) / 64;
    if (tm * tn > kMaxGrid) return ACRL_ERR_INVALID_ARG;
    const dim3 small(unsigned(tm * tm), unsigned(batch)), large(unsigned(tm * tn), unsigned(batch));
    for (int i = 0; i < steps; ++i) {
        t.a = coeffs[3 * i];
        t.b = coeffs[3 * i + 1];
        t.c = coeffs[3 * i + 2];
        t.x = x[i & 1];
        t.to = gram;
        step_kernel<0><<<small, 256, 0, s>>>(t);
        t.to = q;
        step_kernel<1><<<small, 256, 0, s>>>(t);
        t.to = x[1 - (i & 1)];
        if (i + 1 < steps)
            step_kernel<2><<<large, 256, 0, s>>>(t);
        else
            step_kernel<3><<<large, 256, 0, s>>>(t);
    }
    return launch_status();
}
