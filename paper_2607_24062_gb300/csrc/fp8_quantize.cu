// acrl_fp8_quantize: a matrix (or its transpose) to 8-bit floating point with
// one power-of-two scale for each block of 128 columns of a row, or of 128 x 128.
//
//     a = max |x| of the block,  2^e the smallest power of two with a <= MAX 2^e
//     q = x 2^-e rounded to nearest even,  scale byte = e + 127
//
// MAX is 1.75 times a power of two in both formats (448 = 1.75 2^8, 57344 = 1.75 2^15),
// so e follows from a's exponent and one comparison of its fraction, and x 2^-e
// is exact: the only rounding is the one to the 8-bit format.
//
// HBM bounds it (2 or 4 bytes in, 1 out): every element is loaded once, 16 bytes a
// load, stays in registers while its block's maximum is found, and is stored 8 or 16
// bytes at a time.
#include "acrl_device.cuh"
#include "acrl_host.h"
#include "fp8.cuh"

namespace acrl {
namespace {

// The first n (of 8) bytes; p is 8-byte aligned.
__device__ __forceinline__ void store8(uint8_t* p, const uint2& v, int n) {
    if (n >= 8) {
        *reinterpret_cast<uint2*>(p) = v;
        return;
    }
    const uint8_t* b = reinterpret_cast<const uint8_t*>(&v);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) p[j] = b[j];
}

// Rows as they are: sixteen lanes a block of 128 columns, kRowUnroll blocks of a row in flight per lane.
constexpr int kRowThreads = 256, kRowUnroll = 4;

template <typename T, int FMT>
__global__ void __launch_bounds__(kRowThreads)
    quantize_rows(const T* __restrict__ x, int64_t R, int C, int64_t ldx, int KB, int chunks, uint8_t* __restrict__ q,
                  int64_t ldq, uint8_t* __restrict__ scale, int64_t lds, int32_t* flags) {
    grid_begin();
    const int team = threadIdx.x >> 4, l = threadIdx.x & 15;
    // a unit is kRowUnroll consecutive blocks of one row; a CTA's teams take consecutive units
    const int64_t unit = int64_t(blockIdx.x) * (kRowThreads / 16) + team;
    const int64_t row = unit >> 32 ? unit / chunks : int64_t(uint32_t(unit) / uint32_t(chunks));
    const int kb0 = int(unit - row * chunks) * kRowUnroll;
    const bool in = row < R;
    const T* xr = x + (in ? row : 0) * ldx;
    float f[kRowUnroll][8];
    uint32_t m[kRowUnroll];
    // whole units without a test between their loads, so that all of them are in flight together
    if (in && (kb0 + kRowUnroll) * 128 <= C) {
#pragma unroll
        for (int k = 0; k < kRowUnroll; ++k) load8<T>(xr + (kb0 + k) * 128 + l * 8, 8, f[k]);
    } else {
#pragma unroll
        for (int k = 0; k < kRowUnroll; ++k) {
            const int c = (kb0 + k) * 128 + l * 8;
            load8<T>(xr + c, in ? C - c : 0, f[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < kRowUnroll; ++k) {
        m[k] = max8(f[k]);
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) m[k] = max(m[k], __shfl_xor_sync(0xffffffffu, m[k], d));
    }
    if (!in) return;
#pragma unroll
    for (int k = 0; k < kRowUnroll; ++k) {
        const int kb = kb0 + k, c = kb * 128 + l * 8;
        if (kb >= KB) break;
        const Scale s = block_scale<FMT>(m[k]);
        if (l == 0) {
            scale[row * lds + kb] = uint8_t(s.byte);
            if (s.byte == 255u) raise_flag(flags, ACRL_FLAG_NONFINITE);
        }
        if (c < C) store8(q + row * ldq + c, pack8<FMT>(f[k], s), C - c);
    }
}

// 128 x 128 elements of x a CTA: a thread holds eight consecutive rows of eight columns.  TILE: one scale, else (the
// transpose of x, by rows) one per column.  TR: the result is the transpose, turned in shared memory: 8-byte pieces,
// piece g of a column at g ^ (column / 8), so that neither side meets a bank twice.
constexpr int kTileThreads = 256;

// The tile's result, turned, in rows of 128 bytes.
template <int FMT, bool TILE>
__device__ __forceinline__ void turn_and_store(const float (&f)[8][8], const Scale* s, uint8_t* turned, uint8_t* q,
                                               int64_t ldq, int64_t rb, int64_t cb, int64_t R, int64_t C) {
    const int g = threadIdx.x >> 4, cl = threadIdx.x & 15;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float col[8] = {f[0][j], f[1][j], f[2][j], f[3][j], f[4][j], f[5][j], f[6][j], f[7][j]};
        *reinterpret_cast<uint2*>(turned + (8 * cl + j) * 128 + 8 * (g ^ cl)) = pack8<FMT>(col, s[TILE ? 0 : j]);
    }
    __syncthreads();
    // eight lanes a column of x (128 bytes of the result's row)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = k * 32 + (threadIdx.x >> 3), p = 2 * (threadIdx.x & 7);
        const int64_t col = cb * 128 + c, row = rb * 128 + 8 * p;
        if (col >= C || row >= R) continue;
        const uint2 a = *reinterpret_cast<const uint2*>(turned + c * 128 + 8 * (p ^ (c >> 3)));
        const uint2 b = *reinterpret_cast<const uint2*>(turned + c * 128 + 8 * ((p + 1) ^ (c >> 3)));
        uint8_t* to = q + col * ldq + row;
        if (row + 16 <= R) {
            *reinterpret_cast<uint4*>(to) = make_uint4(a.x, a.y, b.x, b.y);
        } else {
            store8(to, a, int(R - row));
            if (row + 8 < R) store8(to + 8, b, int(R - row - 8));
        }
    }
}

template <typename T, int FMT, bool TILE, bool TR>
__global__ void __launch_bounds__(kTileThreads)
    quantize_tiles(const T* __restrict__ x, int64_t R, int64_t C, int64_t ldx, int col_blocks, uint8_t* __restrict__ q,
                   int64_t ldq, uint8_t* __restrict__ scale, int64_t lds, int32_t* flags) {
    static_assert(TILE || TR, "rows as they are have a kernel of their own");
    __shared__ uint32_t sh_max[TILE ? 8 : 8 * 128];
    __shared__ __align__(16) uint8_t turned[TR ? 128 * 128 : 16];
    grid_begin();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int g = threadIdx.x >> 4, cl = threadIdx.x & 15;        // rows 8 g .., columns 8 cl ..
    const int64_t rb = blockIdx.x / col_blocks, cb = blockIdx.x % col_blocks;
    const int64_t r0 = rb * 128 + 8 * g, c0 = cb * 128 + 8 * cl;
    const int nc = int(min(int64_t(8), C - c0));
    float f[8][8];
    if (r0 + 8 <= R && nc == 8) {   // no test between the loads: all eight in flight
#pragma unroll
        for (int i = 0; i < 8; ++i) load8<T>(x + (r0 + i) * ldx + c0, 8, f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) load8<T>(x + (r0 + i < R && nc > 0 ? (r0 + i) * ldx + c0 : 0), r0 + i < R ? nc : 0, f[i]);
    }
    Scale s[TILE ? 1 : 8];
    if constexpr (TILE) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, max8(f[i]));
        m = __reduce_max_sync(0xffffffffu, m);
        if (lane == 0) sh_max[wid] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) m = max(m, sh_max[w]);
        s[0] = block_scale<FMT>(m);
        if (threadIdx.x == 0) {
            scale[TR ? cb * lds + rb : rb * lds + cb] = uint8_t(s[0].byte);
            if (s[0].byte == 255u) raise_flag(flags, ACRL_FLAG_NONFINITE);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, abs_bits(f[i][j]));
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 16));
            if (lane < 16) sh_max[wid * 128 + 8 * cl + j] = m;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) m = max(m, sh_max[w * 128 + 8 * cl + j]);
            s[j] = block_scale<FMT>(m);
            if (g == 0 && c0 + j < C) {
                scale[(c0 + j) * lds + rb] = uint8_t(s[j].byte);
                if (s[j].byte == 255u) raise_flag(flags, ACRL_FLAG_NONFINITE);
            }
        }
    }
    if constexpr (!TR) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (r0 + i < R && nc > 0) store8(q + (r0 + i) * ldq + c0, pack8<FMT>(f[i], s[0]), nc);
    } else {
        turn_and_store<FMT, TILE>(f, s, turned, q, ldq, rb, cb, R, C);
    }
}

template <typename T, int FMT>
acrl_status launch_quantize(const T* x, int64_t R, int64_t C, int64_t ldx, bool tile, bool transpose, uint8_t* q,
                            int64_t ldq, uint8_t* scale, int64_t lds, int32_t* flags, cudaStream_t s) {
    if (!tile && !transpose) {
        const int KB = int((C + 127) / 128), chunks = (KB + kRowUnroll - 1) / kRowUnroll;
        const int64_t units = R * chunks, grid = (units + kRowThreads / 16 - 1) / (kRowThreads / 16);
        if (grid > kMaxGrid) return ACRL_ERR_INVALID_ARG;
        return launch(quantize_rows<T, FMT>, grid, kRowThreads, 0, 0, s, x, R, int(C), ldx, KB, chunks, q, ldq, scale, lds,
                      flags);
    }
    const int64_t cb = (C + 127) / 128, grid = (R + 127) / 128 * cb;
    if (grid > kMaxGrid) return ACRL_ERR_INVALID_ARG;
    auto* kernel = !transpose ? quantize_tiles<T, FMT, true, false>
                   : tile     ? quantize_tiles<T, FMT, true, true>
                              : quantize_tiles<T, FMT, false, true>;
    return launch(kernel, grid, kTileThreads, 0, 0, s, x, R, C, ldx, int(cb), q, ldq, scale, lds, flags);
}

}  // namespace
}  // namespace acrl

using namespace acrl;

extern "C" acrl_status acrl_fp8_quantize(const void* x, acrl_dtype x_dtype, int64_t R, int64_t C, int64_t ldx,
                                         acrl_fp8_format format, acrl_fp8_block block, int32_t transpose, uint8_t* q,
                                         int64_t ldq, uint8_t* scale, int64_t lds, int32_t* dev_flags,
                                         acrl_stream stream) {
    if (R < 0 || C < 0 || R > kMaxGrid || C > kMaxGrid) return ACRL_ERR_INVALID_ARG;
    if (x_dtype != ACRL_BF16 && x_dtype != ACRL_F32) return ACRL_ERR_INVALID_ARG;
    if (format != ACRL_FP8_E4M3 && format != ACRL_FP8_E5M2) return ACRL_ERR_INVALID_ARG;
    if (block != ACRL_FP8_ROW && block != ACRL_FP8_TILE) return ACRL_ERR_INVALID_ARG;
    const int64_t cols = transpose ? R : C;   // of the result
    if (ldx < C || (ldx & (x_dtype == ACRL_BF16 ? 7 : 3)) || ldq < cols || (ldq & 15) || lds < (cols + 127) / 128)
        return ACRL_ERR_INVALID_ARG;
    if (R == 0 || C == 0) return ACRL_OK;
    if (!x || !q || !scale || !aligned16(x) || !aligned16(q)) return ACRL_ERR_INVALID_ARG;
    const bool tile = block == ACRL_FP8_TILE, tr = transpose != 0;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (x_dtype == ACRL_BF16) {
        auto* p = static_cast<const acrl_bf16*>(x);
        return format == ACRL_FP8_E4M3 ? launch_quantize<acrl_bf16, 0>(p, R, C, ldx, tile, tr, q, ldq, scale, lds, dev_flags, s)
                                       : launch_quantize<acrl_bf16, 1>(p, R, C, ldx, tile, tr, q, ldq, scale, lds, dev_flags, s);
    }
    auto* p = static_cast<const float*>(x);
    return format == ACRL_FP8_E4M3 ? launch_quantize<float, 0>(p, R, C, ldx, tile, tr, q, ldq, scale, lds, dev_flags, s)
                                   : launch_quantize<float, 1>(p, R, C, ldx, tile, tr, q, ldq, scale, lds, dev_flags, s);
}
