// A product of two matrices of any strides on the fp32 pipes: 64 x 64 results a CTA, 16 of the sum at a time in shared memory.
#pragma once

#include "activation.cuh"

namespace acrl {
namespace {

struct View {
    const void* p;
    bool f32;
    int64_t row, col;   // strides
    __device__ __forceinline__ float at(int64_t r, int64_t c) const { return load_float(p, f32, r * row + c * col); }
};

// emit(m, n, sum) for every element of A B^T, A [M, K] and B [N, K].
template <class Emit>
__device__ void simple_product(const View& A, const View& B, int M, int N, int K, int m0, int n0, Emit emit) {
    __shared__ float as[16][65], bs[16][65];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += 16) {
        for (int i = threadIdx.x; i < 1024; i += 256) {
            const int k = i & 15, r = i >> 4;
            as[k][r] = m0 + r < M && k0 + k < K ? A.at(m0 + r, k0 + k) : 0.f;
            bs[k][r] = n0 + r < N && k0 + k < K ? B.at(n0 + r, k0 + k) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(as[k][ty + 16 * i], bs[k][tx + 16 * j], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m < M && n < N) emit(m, n, acc[i][j]);
        }
}

}  // namespace
}  // namespace acrl
