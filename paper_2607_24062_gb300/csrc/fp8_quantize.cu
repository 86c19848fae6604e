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
// HBM bounds it (2 or 4 bytes in, 1 out; 4,096 x 4,096 by rows in 11.7 us, of which some 4 are a launch's): every element is loaded once, 16 bytes a
// load, stays in registers while its block's maximum is found, and is stored 8 or 16
// bytes at a time.
#include "acrl_device.cuh"
#include "acrl_host.h"
#include "fp8.cuh"

namespace acrl {
namespace {

// Maxima are found in the bits of |x|, which order as unsigned integers: of bf16 two in a word (one instruction for both; as fp32
// numbers one at a time, 2,507 x 8,200 both ways took 27 us, the ALUs more than half busy), of fp32 one.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Eight elements as they were loaded: a bf16 tile's registers are half of what its fp32 numbers would take.
template <typename T>
struct Eight;
template <>
struct Eight<acrl_bf16> {
    static constexpr int kKeys = 4;       // words of the elements' keys
    uint32_t w[4];
    __device__ __forceinline__ void load(const acrl_bf16* p, int n) {
        if (n >= 8) {
            const uint4 v = ld_stream(reinterpret_cast<const uint4*>(p));
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            return;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = (2 * j < n ? uint32_t(p[2 * j]) : 0u) | (2 * j + 1 < n ? uint32_t(p[2 * j + 1]) << 16 : 0u);
    }
    __device__ __forceinline__ float at(int j) const { return j & 1 ? bf16_hi(w[j >> 1]) : bf16_lo(w[j >> 1]); }
    __device__ __forceinline__ uint32_t key(int k) const { return w[k] & 0x7fff7fffu; }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max_u16x2(a, b); }
    // The keys' maximum as bits of an fp32 number.
    static __device__ __forceinline__ uint32_t most(const uint32_t (&k)[4]) {
        const uint32_t m = larger(larger(k[0], k[1]), larger(k[2], k[3]));
        return max(m << 16, m & 0xffff0000u);
    }
};
template <>
struct Eight<float> {
    static constexpr int kKeys = 8;
    float f[8];
    __device__ __forceinline__ void load(const float* p, int n) { load8<float>(p, n, f); }
    __device__ __forceinline__ float at(int j) const { return f[j]; }
    __device__ __forceinline__ uint32_t key(int k) const { return abs_bits(f[k]); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }
    static __device__ __forceinline__ uint32_t most(const uint32_t (&k)[8]) {
        return max(max(max(k[0], k[1]), max(k[2], k[3])), max(max(k[4], k[5]), max(k[6], k[7])));
    }
};

// The largest of the eights of sixteen lanes, U of them, as bits of fp32 in every lane; bf16's go through the lanes in pairs.
template <typename T, int U>
__device__ __forceinline__ void most_of_sixteen(const Eight<T> (&f)[U], uint32_t (&m)[U]) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
        uint32_t k[Eight<T>::kKeys];
#pragma unroll
        for (int j = 0; j < Eight<T>::kKeys; ++j) k[j] = f[i].key(j);
        m[i] = Eight<T>::most(k);
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < U; i += 2) {
            uint32_t v = m[i] >> 16 | m[i + 1];
#pragma unroll
            for (int d = 8; d >= 1; d >>= 1) v = max_u16x2(v, __shfl_xor_sync(0xffffffffu, v, d));
            m[i] = v << 16;
            m[i + 1] = v & 0xffff0000u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int d = 8; d >= 1; d >>= 1) m[i] = max(m[i], __shfl_xor_sync(0xffffffffu, m[i], d));
    }
}

// The scales of U (a power of two) maxima that sixteen lanes share: each lane works one out, that of m[lane % U], which it
// returns, and `inv` has all.
template <int FMT, int U>
__device__ __forceinline__ Scale scales_of(const uint32_t (&m)[U], float (&inv)[U]) {
    const int lane = threadIdx.x & 31;
    uint32_t mine = m[0];
#pragma unroll
    for (int i = 1; i < U; ++i) mine = (lane & (U - 1)) == i ? m[i] : mine;
    const Scale s = block_scale<FMT>(mine);
#pragma unroll
    for (int i = 0; i < U; ++i) inv[i] = __shfl_sync(0xffffffffu, s.inv, (lane & 16) + i);
    return s;
}

template <int FMT, typename T>
__device__ __forceinline__ uint2 pack8(const Eight<T>& f, float inv) {
    uint2 o;
    o.x = pack2<FMT>(f.at(0), f.at(1), inv) | pack2<FMT>(f.at(2), f.at(3), inv) << 16;
    o.y = pack2<FMT>(f.at(4), f.at(5), inv) | pack2<FMT>(f.at(6), f.at(7), inv) << 16;
    return o;
}

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
    Eight<T> f[kRowUnroll];
    // whole units without a test between their loads, so that all of them are in flight together
    if (in && kb0 + kRowUnroll <= C >> 7) {   // in blocks: their columns' number may pass 32 bits
#pragma unroll
        for (int k = 0; k < kRowUnroll; ++k) f[k].load(xr + (kb0 + k) * 128 + l * 8, 8);
    } else {
#pragma unroll
        for (int k = 0; k < kRowUnroll; ++k) {
            const int c = (kb0 + k) * 128 + l * 8;
            f[k].load(xr + c, in ? C - c : 0);
        }
    }
    uint32_t m[kRowUnroll];
    float inv[kRowUnroll];
    most_of_sixteen<T, kRowUnroll>(f, m);
    const Scale s = scales_of<FMT, kRowUnroll>(m, inv);
    if (!in) return;
    if (l < kRowUnroll && kb0 + l < KB) {
        scale[row * lds + kb0 + l] = uint8_t(s.byte);
        if (s.byte == 255u) raise_flag(flags, ACRL_FLAG_NONFINITE);
    }
#pragma unroll
    for (int k = 0; k < kRowUnroll; ++k) {
        const int c = (kb0 + k) * 128 + l * 8;
        if (c < C) store8(q + row * ldq + c, pack8<FMT>(f[k], inv[k]), C - c);
    }
}

// 128 x 128 elements of x a CTA, loaded once into registers: eight consecutive rows of eight columns a thread for what is stored as
// it is (151,936 x 4,096 in 266 us, 1.05 of the copy rate; when compared 284, and 357 with four rows in twice the threads), four for
// what is turned (the transpose of 5,003 x 2,056 in 12.3 us; when compared 15, and 18.7 with eight).  What is made of them:
//   kTile    one scale, the elements as they are          kTileT  one scale, the transpose
//   kRowT    a scale per column, the transpose            kBoth   a scale per row, the elements as they are, and kRowT's
// The transpose is turned in shared memory: 8-byte pieces, piece p of a column at p ^ (column / 8), so that neither side meets a
// bank twice; a thread writes half a piece.
enum Make { kTile, kTileT, kRowT, kBoth };
template <Make MAKE>
constexpr int kTileRows = MAKE == kTile ? 8 : 4;
template <Make MAKE>
constexpr int kTileThreads = 2048 / kTileRows<MAKE>;

template <typename T>
struct Tiled {
    const T* x;
    int64_t R, C, ldx;
    int col_blocks;
    Quantised as, turned;
};

template <typename T, int FMT, Make MAKE>
__device__ __forceinline__ void quantize_tile(const Tiled<T>& job, int64_t block, int32_t* flags) {
    const T* __restrict__ x = job.x;
    const int64_t R = job.R, C = job.C, ldx = job.ldx;
    const int col_blocks = job.col_blocks;
    const Quantised &as = job.as, &turned = job.turned;
    constexpr int U = kTileRows<MAKE>, kThreads = kTileThreads<MAKE>;
    constexpr int kWarps = kThreads / 32, kKeys = Eight<T>::kKeys;
    constexpr bool kOne = MAKE == kTile || MAKE == kTileT;
    __shared__ uint32_t top[kWarps];                    // kOne: the warps' maxima
    __shared__ __align__(16) float inverse[kOne ? 4 : 128];   // else each column's 2^-e
    __shared__ __align__(16) uint8_t turn[MAKE == kTile ? 16 : 128 * 128];
    const int lane = threadIdx.x & 31;
    const int g = threadIdx.x >> 4, cl = threadIdx.x & 15;        // rows U g .., columns 8 cl ..
    const int64_t rb = block / col_blocks, cb = block - rb * col_blocks;
    const int64_t r0 = rb * 128 + U * g, c0 = cb * 128 + 8 * cl;
    const int nc = int(min(int64_t(8), C - c0));
    grid_begin();
    Eight<T> f[U];
    if (r0 + U <= R && nc == 8) {   // no test between the loads: all in flight
#pragma unroll
        for (int i = 0; i < U; ++i) f[i].load(x + (r0 + i) * ldx + c0, 8);
    } else {
#pragma unroll
        for (int i = 0; i < U; ++i) f[i].load(x + (r0 + i < R && nc > 0 ? (r0 + i) * ldx + c0 : 0), r0 + i < R ? nc : 0);
    }
    auto store_as = [&](int i, float inv) {
        if (r0 + i < R && nc > 0) store8(as.q + (r0 + i) * as.ldq + c0, pack8<FMT>(f[i], inv), nc);
    };
    if constexpr (MAKE == kBoth) {   // sixteen lanes hold a row's 128 columns
        uint32_t m[U];
        float inv[U];
        most_of_sixteen<T, U>(f, m);
        const Scale s = scales_of<FMT, U>(m, inv);
        if (cl < U && r0 + cl < R) as.scale[(r0 + cl) * as.lds + cb] = uint8_t(s.byte);
#pragma unroll
        for (int i = 0; i < U; ++i) store_as(i, inv[i]);
    }
    uint32_t k[kKeys];               // the largest of this thread's rows
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
        k[j] = f[0].key(j);
#pragma unroll
        for (int i = 1; i < U; ++i) k[j] = Eight<T>::larger(k[j], f[i].key(j));
    }
    float inv[kOne ? 1 : 8];
    if constexpr (kOne) {
        const uint32_t m = __reduce_max_sync(0xffffffffu, Eight<T>::most(k));
        if (lane == 0) top[threadIdx.x >> 5] = m;
        __syncthreads();
        const Scale s = block_scale<FMT>(__reduce_max_sync(0xffffffffu, lane < kWarps ? top[lane] : 0u));
        inv[0] = s.inv;
        if (threadIdx.x == 0) {
            if (MAKE == kTileT) turned.scale[cb * turned.lds + rb] = uint8_t(s.byte);
            else as.scale[rb * as.lds + cb] = uint8_t(s.byte);
            if (s.byte == 255u) raise_flag(flags, ACRL_FLAG_NONFINITE);
        }
    } else {
        // each warp's maxima of the columns, where the turned elements will be; then a thread a column
        uint32_t* parts = reinterpret_cast<uint32_t*>(turn);
#pragma unroll
        for (int j = 0; j < kKeys; ++j) {
            k[j] = Eight<T>::larger(k[j], __shfl_xor_sync(0xffffffffu, k[j], 16));
            if (lane < 16) parts[((threadIdx.x >> 5) * kKeys + j) * 16 + cl] = k[j];
        }
        __syncthreads();
        if (threadIdx.x < 128) {
            // thread t: column 8 (t % 16) + t / 16
            const int l = threadIdx.x & 15, j = threadIdx.x >> 4, word = j * kKeys / 8;
            uint32_t most = 0u;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) most = Eight<T>::larger(most, parts[(i * kKeys + word) * 16 + l]);
            if (kKeys == 4) most = j & 1 ? most & 0xffff0000u : most << 16;
            const Scale mine = block_scale<FMT>(most);
            inverse[8 * l + j] = mine.inv;
            const int64_t c = cb * 128 + 8 * l + j;
            if (c < C) {
                turned.scale[c * turned.lds + rb] = uint8_t(mine.byte);
                if (mine.byte == 255u) raise_flag(flags, ACRL_FLAG_NONFINITE);
            }
        }
        __syncthreads();
        const float4 a = *reinterpret_cast<const float4*>(inverse + 8 * cl), b = *reinterpret_cast<const float4*>(inverse + 8 * cl + 4);
        inv[0] = a.x; inv[1] = a.y; inv[2] = a.z; inv[3] = a.w;
        inv[4] = b.x; inv[5] = b.y; inv[6] = b.z; inv[7] = b.w;
    }
    if constexpr (MAKE == kTile) {
#pragma unroll
        for (int i = 0; i < U; ++i) store_as(i, inv[0]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float by = inv[MAKE == kTileT ? 0 : j];
            const uint32_t w = pack2<FMT>(f[0].at(j), f[1].at(j), by) | pack2<FMT>(f[2].at(j), f[3].at(j), by) << 16;
            *reinterpret_cast<uint32_t*>(turn + (8 * cl + j) * 128 + 8 * ((g >> 1) ^ cl) + 4 * (g & 1)) = w;
        }
        __syncthreads();
        // eight lanes a column of x (128 bytes of the result's row)
#pragma unroll
        for (int k = 0; k < 128 / (kThreads / 8); ++k) {
            const int c = k * (kThreads / 8) + (threadIdx.x >> 3), p = 2 * (threadIdx.x & 7);
            const int64_t col = cb * 128 + c, row = rb * 128 + 8 * p;
            if (col >= C || row >= R) continue;
            const uint2 a = *reinterpret_cast<const uint2*>(turn + c * 128 + 8 * (p ^ (c >> 3)));
            const uint2 b = *reinterpret_cast<const uint2*>(turn + c * 128 + 8 * ((p + 1) ^ (c >> 3)));
            uint8_t* to = turned.q + col * turned.ldq + row;
            if (row + 16 <= R) {
                *reinterpret_cast<uint4*>(to) = make_uint4(a.x, a.y, b.x, b.y);
            } else {
                store8(to, a, int(R - row));
                if (row + 8 < R) store8(to + 8, b, int(R - row - 8));
            }
        }
    }
}

// (fp32 as it is: 64 registers of elements a thread, and two CTAs an SM have 128 KB of loads in flight)
template <typename T, int FMT, Make MAKE>
__global__ void __launch_bounds__(kTileThreads<MAKE>, MAKE == kTile && sizeof(T) == 2 ? 3 : 2)
    quantize_tiles(const __grid_constant__ Tiled<T> job, int32_t* flags) {
    quantize_tile<T, FMT, MAKE>(job, int64_t(blockIdx.x), flags);
}

// What a layer's backward needs: `dy` both ways, then `x` turned, in one launch (two: 2.5 us more on the GPU, 4 on the host).
template <int FMT, int X_FMT>
__global__ void __launch_bounds__(kTileThreads<kBoth>, 2)
    quantize_backward_tiles(const __grid_constant__ Tiled<acrl_bf16> dy, const __grid_constant__ Tiled<acrl_bf16> x,
                            int64_t dy_tiles, int32_t* flags) {
    if (int64_t(blockIdx.x) < dy_tiles)
        quantize_tile<acrl_bf16, FMT, kBoth>(dy, int64_t(blockIdx.x), flags);
    else
        quantize_tile<acrl_bf16, X_FMT, kRowT>(x, int64_t(blockIdx.x) - dy_tiles, flags);
}

template <typename T>
Tiled<T> tiled(const T* x, int64_t R, int64_t C, int64_t ldx, const Quantised& as, const Quantised& turned) {
    return Tiled<T>{x, R, C, ldx, int((C + 127) / 128), as, turned};
}
template <typename T>
int64_t tiles_of(const Tiled<T>& t) { return (t.R + 127) / 128 * t.col_blocks; }

template <typename T, int FMT, Make MAKE>
acrl_status launch_tiles(const T* x, int64_t R, int64_t C, int64_t ldx, const Quantised& as, const Quantised& turned,
                         int32_t* flags, cudaStream_t s) {
    const Tiled<T> job = tiled(x, R, C, ldx, as, turned);
    if (tiles_of(job) > kMaxGrid) return ACRL_ERR_INVALID_ARG;
    return launch(quantize_tiles<T, FMT, MAKE>, tiles_of(job), kTileThreads<MAKE>, 0, 0, s, job, flags);
}

template <typename T, int FMT>
acrl_status launch_quantize(const T* x, int64_t R, int64_t C, int64_t ldx, bool tile, bool transpose, const Quantised& out,
                            int32_t* flags, cudaStream_t s) {
    if (transpose)
        return tile ? launch_tiles<T, FMT, kTileT>(x, R, C, ldx, out, out, flags, s)
                    : launch_tiles<T, FMT, kRowT>(x, R, C, ldx, out, out, flags, s);
    if (tile) return launch_tiles<T, FMT, kTile>(x, R, C, ldx, out, out, flags, s);
    const int KB = int((C + 127) / 128), chunks = (KB + kRowUnroll - 1) / kRowUnroll;
    const int64_t units = R * chunks, grid = (units + kRowThreads / 16 - 1) / (kRowThreads / 16);
    if (grid > kMaxGrid) return ACRL_ERR_INVALID_ARG;
    return launch(quantize_rows<T, FMT>, grid, kRowThreads, 0, 0, s, x, R, int(C), ldx, KB, chunks, out.q, out.ldq, out.scale,
                  out.lds, flags);
}

}  // namespace

acrl_status quantize_backward(const acrl_bf16* dy, int64_t M, int64_t N, int64_t lddy, acrl_fp8_format format, const Quantised& as,
                              const Quantised& turned, const acrl_bf16* x, int64_t K, int64_t ldx, acrl_fp8_format x_format,
                              const Quantised& x_turned, int32_t* flags, cudaStream_t s) {
    const Tiled<acrl_bf16> a = tiled(dy, M, N, lddy, as, turned), b = tiled(x, M, K, ldx, x_turned, x_turned);
    const int64_t tiles = tiles_of(a), grid = tiles + tiles_of(b);
    if (grid > kMaxGrid) return ACRL_ERR_INVALID_ARG;
    auto run = [&](auto* kernel) { return launch(kernel, grid, kTileThreads<kBoth>, 0, 0, s, a, b, tiles, flags); };
    if (format == ACRL_FP8_E4M3)
        return x_format == ACRL_FP8_E4M3 ? run(quantize_backward_tiles<0, 0>) : run(quantize_backward_tiles<0, 1>);
    return x_format == ACRL_FP8_E4M3 ? run(quantize_backward_tiles<1, 0>) : run(quantize_backward_tiles<1, 1>);
}

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
    const Quantised out{q, ldq, scale, lds};
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (x_dtype == ACRL_BF16) {
        auto* p = static_cast<const acrl_bf16*>(x);
        return format == ACRL_FP8_E4M3 ? launch_quantize<acrl_bf16, 0>(p, R, C, ldx, tile, tr, out, dev_flags, s)
                                       : launch_quantize<acrl_bf16, 1>(p, R, C, ldx, tile, tr, out, dev_flags, s);
    }
    auto* p = static_cast<const float*>(x);
    return format == ACRL_FP8_E4M3 ? launch_quantize<float, 0>(p, R, C, ldx, tile, tr, out, dev_flags, s)
                                   : launch_quantize<float, 1>(p, R, C, ldx, tile, tr, out, dev_flags, s);
}
