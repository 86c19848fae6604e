// The product of one row, a token, with an 8-bit matrix: every byte of the matrix is used once, so HBM would bound it; at the
// sizes of one layer the latency of a launch and of a warp's loads does (of 9.0 us at 4,096 x 4,096 some 6.4 bring 15.7 MB, 2.5 TB/s: a
// lane has four loads of 16 bytes in flight, and 4,096 columns are four round trips one after another).  No tensor cores: their pipeline's start and end (tensor memory,
// barriers, the split of the sum) and the launch that quantises the row take longer than a small product: 1,024 x 1,024 2.6 us
// against 6.6, 4,096 x 4,096 9.0 against 9.1, and 16 against 25 as a call; from there on the tensor cores' way is faster (8,192 x
// 4,096 14.7 against 11.5).  A warp takes kW rows of the matrix at a time: each lane loads 16 bytes of each,
// 512 columns a step, two steps ahead, converts them to fp32 through half precision (exact for both formats) and multiplies
// them with the row, whose 8-bit numbers lie in shared memory as fp32; the 16 products' sum takes both blocks' scales at once, as
// each alone could carry it out of fp32's range where the product stays within (a row of 2^120 and a matrix of 2^-120).
// Then the lanes' sums meet in a fixed order.  The row may come as bf16 activations: every CTA then quantises it itself (8 KB for
// 4,096 columns, from L2), while its first loads of the matrix are under way.
#include <cuda_fp16.h>

#include "fp8.cuh"

namespace acrl {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kStep = 512;                      // columns of a warp's step
constexpr int kW = 2;                           // rows of the matrix a warp takes at a time
constexpr int kMostBytes = 64 * 1024 + 128;     // of the row in shared memory: 16,384 columns
constexpr int64_t kFewBytes = 16 << 20;

int64_t few_cols(int64_t K) { return (K + 2 * kStep - 1) / (2 * kStep) * (2 * kStep); }
int64_t few_bytes(int64_t K) { return few_cols(K) * 4 + few_cols(K) / 128; }

struct FewArgs {
    Matrix a, b;          // a: the one row
    const acrl_bf16* x;   // the row as activations, or null
    int K, cols;          // columns, and those that the steps cover
    void* out;
    int32_t* flags;
};

// part 2^(sa + sb - 254) + acc of two scale bytes; NaN where one of them is 255.  The power goes in two factors, the second 1 for
// exponents that one can hold.
__device__ __forceinline__ float add_scaled(float part, uint32_t sa, uint32_t sb, float acc) {
    const int e = int(sa + sb) - 254, first = max(-126, min(127, e)), second = max(-126, e - first);
    const float by = sa == 255u || sb == 255u ? __int_as_float(0x7fc00000) : __uint_as_float(uint32_t(first + 127) << 23);
    return fmaf(part * by, __uint_as_float(uint32_t(second + 127) << 23), acc);
}

// Four 8-bit numbers of a word to fp32.
template <int FMT>
__device__ __forceinline__ void widen4(uint32_t w, float* f) {
    uint32_t lo, hi;
    if (FMT == ACRL_FP8_E4M3) {
        asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}\n"
            : "=r"(lo), "=r"(hi)
            : "r"(w));
    } else {
        asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e5m2x2 %0, a;\n cvt.rn.f16x2.e5m2x2 %1, b;\n}\n"
            : "=r"(lo), "=r"(hi)
            : "r"(w));
    }
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    f[0] = a.x;
    f[1] = a.y;
    f[2] = b.x;
    f[3] = b.y;
}

template <int FMT>
__device__ __forceinline__ void widen16(const uint4& v, float (&f)[16]) {
    widen4<FMT>(v.x, f);
    widen4<FMT>(v.y, f + 4);
    widen4<FMT>(v.z, f + 8);
    widen4<FMT>(v.w, f + 12);
}

// 16 bytes of a row, zeros beyond its end.
__device__ __forceinline__ uint4 load16(const uint8_t* row, int c, int K) {
    if (c + 16 <= K) return ld_stream(reinterpret_cast<const uint4*>(row + c));
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    uint8_t* b = reinterpret_cast<uint8_t*>(&v);
#pragma unroll
    for (int j = 0; j < 16; ++j)
        if (c + j < K) b[j] = row[c + j];
    return v;
}

// The row's 8-bit numbers as fp32, zeros beyond K, and its blocks' scale bytes: sixteen lanes a block of 128 columns.
template <int FMT>
__device__ __forceinline__ void quantise_into(const FewArgs& A, float* xs, uint8_t* scales) {
    const int l = threadIdx.x & 15;
    for (int u = threadIdx.x >> 4; u < A.cols / 128; u += kThreads / 16) {   // whole half-warps
        const int c = u * 128 + l * 8;
        float f[8];
        load8<acrl_bf16>(A.x + min(c, A.K), max(0, A.K - c), f);
        uint32_t top = max8(f);
        const uint32_t mask = 0xffffu << (threadIdx.x & 16);
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) top = max(top, __shfl_xor_sync(mask, top, d));
        const Scale s = block_scale<FMT>(top);
        if (s.byte == 255u && l == 0 && blockIdx.x == 0) raise_flag(A.flags, ACRL_FLAG_NONFINITE);
        const uint2 q = pack8<FMT>(f, s.inv);
        if (l == 0) scales[u] = uint8_t(s.byte);
        float w[8];
        widen4<FMT>(q.x, w);
        widen4<FMT>(q.y, w + 4);
        float4* to = reinterpret_cast<float4*>(xs + c);
        to[0] = make_float4(w[0], w[1], w[2], w[3]);
        to[1] = make_float4(w[4], w[5], w[6], w[7]);
    }
}

template <int FMT>
__device__ __forceinline__ void widen_into(const FewArgs& A, float* xs, uint8_t* scales) {
    for (int c = threadIdx.x * 16; c < A.cols; c += kThreads * 16) {
        float w[16];
        widen16<FMT>(load16(A.a.q, c, A.K), w);
        if ((c & 127) == 0) scales[c >> 7] = c < A.K ? A.a.scale[c >> 7] : 127;
        float4* to = reinterpret_cast<float4*>(xs + c);
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = make_float4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
    }
}

template <int FMT>
__device__ __forceinline__ void dot_step(const float* xs, uint32_t scale, const uint4 (&v)[kW], const uint32_t (&by)[kW],
                                         float (&acc)[kW]) {
    float part[kW] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float4 x = *reinterpret_cast<const float4*>(xs + 4 * j);
#pragma unroll
        for (int r = 0; r < kW; ++r) {
            float w[4];
            widen4<FMT>(j == 0 ? v[r].x : j == 1 ? v[r].y : j == 2 ? v[r].z : v[r].w, w);
            part[r] = fmaf(w[3], x.w, fmaf(w[2], x.z, fmaf(w[1], x.y, fmaf(w[0], x.x, part[r]))));
        }
    }
#pragma unroll
    for (int r = 0; r < kW; ++r) acc[r] = add_scaled(part[r], scale, by[r], acc[r]);
}

template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads, 2) few_kernel(const __grid_constant__ FewArgs A) {
    extern __shared__ __align__(16) float xs[];   // the row, then its scale bytes
    uint8_t* scales = reinterpret_cast<uint8_t*>(xs + A.cols);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int N = int(A.b.rows), shift = A.b.block == ACRL_FP8_TILE ? 7 : 0, step = int(gridDim.x) * kWarps * kW;
    grid_begin();
    auto load = [&](int n0, int c, uint4 (&v)[kW], uint32_t (&by)[kW]) {
#pragma unroll
        for (int r = 0; r < kW; ++r) {
            const int n = min(n0 + r, N - 1);
            v[r] = load16(A.b.q + n * A.b.ld, min(c, A.K), A.K);
            by[r] = c < A.K ? __ldg(A.b.scale + int64_t(n >> shift) * A.b.lds + (c >> 7)) : 127u;
        }
    };
    int n0 = (int(blockIdx.x) * kWarps + warp) * kW;
    uint4 v[2][kW];
    uint32_t by[2][kW];
    if (n0 < N) {   // under way while the row is made
        load(n0, lane * 16, v[0], by[0]);
        load(n0, lane * 16 + kStep, v[1], by[1]);
    }
    if (A.x) {
        if (A.a.format == ACRL_FP8_E4M3) quantise_into<ACRL_FP8_E4M3>(A, xs, scales);
        else quantise_into<ACRL_FP8_E5M2>(A, xs, scales);
    } else {
        if (A.a.format == ACRL_FP8_E4M3) widen_into<ACRL_FP8_E4M3>(A, xs, scales);
        else widen_into<ACRL_FP8_E5M2>(A, xs, scales);
    }
    __syncthreads();
    for (; n0 < N; n0 += step) {
        float acc[kW] = {};
        // two steps in flight: those to come of these rows, then the first ones of the warp's next
        for (int c = lane * 16; c < A.cols; c += 2 * kStep) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int at = c + k * kStep, ahead = at + 2 * kStep;
                dot_step<FMT>(xs + at, scales[at >> 7], v[k], by[k], acc);
                if (ahead < A.cols) load(n0, ahead, v[k], by[k]);
                else if (n0 + step < N) load(n0 + step, lane * 16 + k * kStep, v[k], by[k]);
            }
        }
#pragma unroll
        for (int r = 0; r < kW; ++r) {
            const float sum = warp_sum(acc[r]);
            if (lane == 0 && n0 + r < N) {
                if constexpr (sizeof(T) == 2)
                    static_cast<acrl_bf16*>(A.out)[n0 + r] = acrl_bf16(pack_bf16x2(sum, 0.f) & 0xffffu);
                else
                    static_cast<float*>(A.out)[n0 + r] = sum;
            }
        }
    }
}

template <typename T, int FMT>
acrl_status launch_few(const FewArgs& A, cudaStream_t s) {
    const size_t smem = size_t(few_bytes(A.K));
    auto* kernel = few_kernel<T, FMT>;
    if (smem > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostBytes) != cudaSuccess)
        return launch_status();
    const int64_t tasks = (A.b.rows + kW * kWarps - 1) / (kW * kWarps);
    return launch(kernel, std::min<int64_t>(tasks, 152 * 2), kThreads, smem, 0, s, A);
}

}  // namespace

// Matrices of up to kFewBytes only: beyond, the latency is a small part, and the tensor cores' path streams a matrix faster
// (1 x 4,096 x 151,936: 100 us against 142).
bool few_rows(int64_t M, int64_t N, int64_t K) { return M == 1 && K > 0 && N * K <= kFewBytes && few_bytes(K) <= kMostBytes; }

acrl_status matmul_few(const Matrix& a, const acrl_bf16* x, const Matrix& b, int64_t K, void* out, acrl_dtype out_dtype, int32_t* flags,
                       cudaStream_t s) {
    if (!few_rows(a.rows, b.rows, K)) return kFewNot;
    const int64_t cols = few_cols(K);
    FewArgs A = {};
    A.a = a;
    A.b = b;
    A.x = x;
    A.K = int(K);
    A.cols = int(cols);
    A.out = out;
    A.flags = flags;
    const bool bf16 = out_dtype == ACRL_BF16;
    if (b.format == ACRL_FP8_E4M3) return bf16 ? launch_few<acrl_bf16, 0>(A, s) : launch_few<float, 0>(A, s);
    return bf16 ? launch_few<acrl_bf16, 1>(A, s) : launch_few<float, 1>(A, s);
}

}  // namespace acrl
