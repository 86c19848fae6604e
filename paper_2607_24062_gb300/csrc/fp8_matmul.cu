// acrl_fp8_matmul: out = A B^T of two 8-bit matrices whose blocks of 128 columns (of
// one row, or of 128 rows) carry power-of-two scales:
//
//     out[m, n] = sum_k 2^(sa[m, k/128] - 127) a[m, k] 2^(sb[n, k/128] - 127) b[n, k]
//
// The tensor cores apply the scales themselves: tcgen05.mma kind::mxf8f6f4 with
// block scaling multiplies every 32 products of a row and a column by one scale
// byte of each, read from tensor memory, and accumulates in fp32 there.  A block
// of 128 is four such groups with the same byte, so a 32-bit word per row holds
// the scales of four blocks (512 columns), and the MMA's scale id picks the byte.
//
// One CTA per SM, warp-specialised:
//   warp 0     one thread issues the TMA loads of the operands' 128-byte slabs
//              (128-byte swizzle) into a ring of stages;
//   warp 1     one thread issues the MMAs, four of K = 32 per slab;
//   warps 2-5  load the scales of four slabs at a time and write them to tensor
//              memory (each warp its own quarter of the lanes: the MMA wants the
//              32 lanes' words in every quarter);
//   warps 6-9  the epilogue: accumulator rows out of tensor memory, rounded once,
//              stored.
// The operand whose rows become the MMA's 128 rows is "P", the other, whose rows
// become its columns, is "Q".
#include <algorithm>

#include "acrl_device.cuh"
#include "acrl_host.h"
#include "mbarrier.cuh"
#include "tcgen05.cuh"
#include "tma_host.h"

namespace acrl {
namespace {

constexpr int kRows = 128;             // rows of P per tile
constexpr int kSlab = 128;             // columns of a slab: 128 bytes, one row of the 128-byte swizzle
constexpr int kGroup = 4;              // slabs whose scales share a word
constexpr int kThreads = 320;
constexpr int kMaxStages = 12, kScaleSlots = 4;
constexpr uint32_t kTmemCols = 512;
// Tensor memory: accumulators from column 0, scale slots of 16 columns at the end (P's words in the first four of
// them, Q's, up to 256 rows, in the last eight).
constexpr uint32_t kScaleCols = 16, kScaleBase = kTmemCols - kScaleSlots * kScaleCols;
constexpr int kRingBytes = 216 * 1024;

struct Barriers {
    uint64_t full[kMaxStages];      // the copies of a stage have landed
    uint64_t empty[kMaxStages];     // the MMAs that read it are done
    uint64_t sfull[kScaleSlots];    // the four warps have written a slot's scales
    uint64_t sempty[kScaleSlots];   // the MMAs that read them are done
    uint64_t tfull[2];              // an accumulator is complete
    uint64_t tempty[2];             // the epilogue has read it
    uint64_t mma_done;
    uint32_t tmem_base;
    int32_t abort;
};
constexpr int kSmemBytes = 1024 + kRingBytes + int(sizeof(Barriers));
static_assert(kSmemBytes <= 227 * 1024, "shared memory per CTA");

struct Operand {
    const uint8_t* scale;
    int64_t lds;
    int rows;
    int shift;       // row >> shift is the scale's row: 0 for rows, 7 for tiles
    int words;       // scales may be read four at a time
};

struct Problem {
    Operand p, q;
    int slabs;             // ceil(K / 128)
    int cols;              // columns of a tile (rows of Q), a multiple of 16, at most 256
    int p_tiles, q_tiles;
    int stages;
    int accs;              // 2 where two accumulators fit, else 1
    uint32_t idesc;
    void* out;
    int64_t ldo;
    int32_t* flags;
};

// tcgen05.mma kind::mxf8f6f4 instruction descriptor: scale type E8M0 (bit 23), formats of A (bits 7-9) and B (10-12),
// both K-major, N / 8 at bit 17, M / 128 at bit 27; the scale ids (A's at bit 29, B's at 4) are added per slab.
constexpr uint32_t kIdescBase = (1u << 23) | (1u << 27);

__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sa,
                                           uint32_t sb, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate));
}

__device__ __forceinline__ void commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void tma_load(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_u32(bar))
        : "memory");
}

// Tiles in bands of kBand row tiles, all column tiles of a band in turn, so that the tiles in flight share operands in L2.
constexpr int kBand = 16;
__device__ __forceinline__ void tile_at(int t, const Problem& pr, int& tp, int& tq) {
    const int per_band = kBand * pr.q_tiles;
    const int band = t / per_band, r = t - band * per_band;
    const int h = min(kBand, pr.p_tiles - band * kBand);
    tp = band * kBand + r % h;
    tq = r / h;
}

__device__ void produce(const CUtensorMap* tmP, const CUtensorMap* tmQ, uint8_t* ring, Barriers* bars, const Problem& pr) {
    volatile int32_t* abort = &bars->abort;
    const int bytes = (kRows + pr.cols) * kSlab;
    int stage = 0;
    uint32_t phase = 0;
    long issued = 0;
    for (int t = blockIdx.x; t < pr.p_tiles * pr.q_tiles; t += gridDim.x) {
        int tp, tq;
        tile_at(t, pr, tp, tq);
        for (int kb = 0; kb < pr.slabs; ++kb) {
            if (!mbar_try_wait(&bars->empty[stage], phase ^ 1u) && !wait_phase(&bars->empty[stage], phase ^ 1u, abort)) {
                give_up(abort, pr.flags);
                // the copies that were started land before the CTA can exit
                for (long j = issued - 1; j >= 0 && j >= issued - pr.stages; --j)
                    wait_phase(&bars->full[j % pr.stages], uint32_t((j / pr.stages) & 1), nullptr);
                return;
            }
            uint8_t* s = ring + stage * bytes;
            mbar_expect_tx(&bars->full[stage], bytes);
            tma_load(s, tmP, &bars->full[stage], kb * kSlab, tp * kRows);
            tma_load(s + kRows * kSlab, tmQ, &bars->full[stage], kb * kSlab, tq * pr.cols);
            ++issued;
            if (++stage == pr.stages) {
                stage = 0;
                phase ^= 1u;
            }
        }
    }
}

__device__ void issue_mmas(uint8_t* ring, Barriers* bars, uint32_t tmem, const Problem& pr) {
    volatile int32_t* abort = &bars->abort;
    const int bytes = (kRows + pr.cols) * kSlab;
    const uint64_t pdesc0 = smem_desc(smem_u32(ring)), qdesc0 = smem_desc(smem_u32(ring + kRows * kSlab));
    int stage = 0, slot = 0, acc = 0;
    uint32_t phase = 0, sphase = 0, aphase = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < pr.p_tiles * pr.q_tiles && ok; t += gridDim.x) {
        if (!wait_phase(&bars->tempty[acc], aphase ^ 1u, abort)) {
            give_up(abort, pr.flags);
            break;
        }
        tc_fence_after();
        const uint32_t d = tmem + uint32_t(acc * pr.cols);
        for (int kb = 0; kb < pr.slabs; ++kb) {
            const uint32_t id = uint32_t(kb % kGroup);
            if ((id == 0 && !wait_phase(&bars->sfull[slot], sphase, abort)) ||
                (!mbar_try_wait(&bars->full[stage], phase) && !wait_phase(&bars->full[stage], phase, abort))) {
                give_up(abort, pr.flags);
                ok = false;
                break;
            }
            tc_fence_after();
            const uint64_t pd = pdesc0 + uint64_t((stage * bytes) >> 4), qd = qdesc0 + uint64_t((stage * bytes) >> 4);
            const uint32_t sc = tmem + kScaleBase + uint32_t(slot) * kScaleCols;
#pragma unroll
            for (int k = 0; k < kSlab / 32; ++k)   // 32 columns = 32 bytes = 2 descriptor units
                mma_scaled(d, pd + uint64_t(2 * k), qd + uint64_t(2 * k), pr.idesc | id << 29 | id << 4, sc, sc + 8,
                           (kb | k) != 0);
            commit(&bars->empty[stage]);
            if (++stage == pr.stages) {
                stage = 0;
                phase ^= 1u;
            }
            if (id == kGroup - 1 || kb == pr.slabs - 1) {
                commit(&bars->sempty[slot]);
                if (++slot == kScaleSlots) {
                    slot = 0;
                    sphase ^= 1u;
                }
            }
        }
        if (!ok) break;
        commit(&bars->tfull[acc]);
        if (++acc == pr.accs) {
            acc = 0;
            aphase ^= 1u;
        }
    }
    commit(&bars->mma_done);   // every MMA has finished before the CTA moves on
    wait_phase(&bars->mma_done, 0, nullptr);
}

// The scales of slabs kb .. kb+3 of one row, one a byte; 127 (2^0) beyond the matrix, where the operands are zeros.
__device__ __forceinline__ uint32_t scale_word(const Operand& o, int row, int kb, int slabs) {
    if (row >= o.rows) return 0x7f7f7f7fu;
    const uint8_t* p = o.scale + int64_t(row >> o.shift) * o.lds + kb;
    if (o.words && kb + kGroup <= slabs) return __ldg(reinterpret_cast<const uint32_t*>(p));
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < kGroup; ++i) w |= (kb + i < slabs ? uint32_t(__ldg(p + i)) : 127u) << (8 * i);
    return w;
}

__device__ void write_scales(Barriers* bars, uint32_t tmem, const Problem& pr) {
    volatile int32_t* abort = &bars->abort;
    const int lane = threadIdx.x & 31;
    const uint32_t lanes = uint32_t((threadIdx.x >> 5) & 3) << 21;   // this warp's quarter, 32 lanes each
    int slot = 0;
    uint32_t phase = 0;
    for (int t = blockIdx.x; t < pr.p_tiles * pr.q_tiles; t += gridDim.x) {
        int tp, tq;
        tile_at(t, pr, tp, tq);
        const int p0 = tp * kRows + lane, q0 = tq * pr.cols + lane;
        for (int kb = 0; kb < pr.slabs; kb += kGroup) {
            uint32_t w[12];
#pragma unroll
            for (int c = 0; c < 4; ++c) w[c] = scale_word(pr.p, p0 + 32 * c, kb, pr.slabs);
#pragma unroll
            for (int c = 0; c < 8; ++c) w[4 + c] = 32 * c < pr.cols ? scale_word(pr.q, q0 + 32 * c, kb, pr.slabs) : 0x7f7f7f7fu;
            const bool free = wait_phase(&bars->sempty[slot], phase ^ 1u, abort);
            if (!__all_sync(0xffffffffu, free)) {
                give_up(abort, pr.flags);
                return;
            }
            tc_fence_after();
            const uint32_t at = tmem + lanes + kScaleBase + uint32_t(slot) * kScaleCols;
            asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]),
                         "r"(w[2]), "r"(w[3])
                         : "memory");
            asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at + 8),
                         "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"(w[8]), "r"(w[9]), "r"(w[10]), "r"(w[11])
                         : "memory");
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->sfull[slot]);
            if (++slot == kScaleSlots) {
                slot = 0;
                phase ^= 1u;
            }
        }
    }
}

// 32 accumulators of one row of P, as columns q0 .. q0+31 of `out` row `row` (SWAP: as rows q0 .. of column `row`).
template <typename T>
__device__ __forceinline__ T round_to(float v);
template <>
__device__ __forceinline__ float round_to<float>(float v) { return v; }
template <>
__device__ __forceinline__ acrl_bf16 round_to<acrl_bf16>(float v) { return acrl_bf16(pack_bf16x2(v, 0.f) & 0xffffu); }

template <typename T, bool SWAP>
__device__ __forceinline__ void store_chunk(T* out, int64_t ldo, int row, int q0, int n, const uint32_t (&r)[32]) {
    if constexpr (SWAP) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < n) out[int64_t(q0 + j) * ldo + row] = round_to<T>(__uint_as_float(r[j]));
    } else {
        T* p = out + int64_t(row) * ldo + q0;
        if (n >= 32) {
            uint4* v = reinterpret_cast<uint4*>(p);
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        w[i] = pack_bf16x2(__uint_as_float(r[8 * j + 2 * i]), __uint_as_float(r[8 * j + 2 * i + 1]));
                    v[j] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < n) p[j] = round_to<T>(__uint_as_float(r[j]));
    }
}

template <typename T, bool SWAP>
__device__ void epilogue(Barriers* bars, uint32_t tmem, const Problem& pr) {
    volatile int32_t* abort = &bars->abort;
    const int lane = threadIdx.x & 31, quarter = (threadIdx.x >> 5) & 3;
    int acc = 0;
    uint32_t phase = 0;
    for (int t = blockIdx.x; t < pr.p_tiles * pr.q_tiles; t += gridDim.x) {
        int tp, tq;
        tile_at(t, pr, tp, tq);
        const bool ready = wait_phase(&bars->tfull[acc], phase, abort);
        if (!__all_sync(0xffffffffu, ready)) {
            give_up(abort, pr.flags);
            return;
        }
        tc_fence_after();
        const int row = tp * kRows + quarter * 32 + lane;
#pragma unroll 1
        for (int c = 0; c < pr.cols; c += 32) {
            uint32_t r[32];
            __syncwarp();
            tmem_ld32(tmem + uint32_t(acc * pr.cols + c) + (uint32_t(quarter * 32) << 16), r);
            const int q0 = tq * pr.cols + c;
            const int n = min(min(32, pr.cols - c), pr.q.rows - q0);
            if (row < pr.p.rows && n > 0) store_chunk<T, SWAP>(static_cast<T*>(pr.out), pr.ldo, row, q0, n, r);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->tempty[acc]);
        if (++acc == pr.accs) {
            acc = 0;
            phase ^= 1u;
        }
    }
}

template <typename T, bool SWAP>
__global__ void __launch_bounds__(kThreads, 1)
    fp8_matmul_kernel(const __grid_constant__ CUtensorMap tmP, const __grid_constant__ CUtensorMap tmQ,
                      const __grid_constant__ Problem pr) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Barriers* bars = reinterpret_cast<Barriers*>(ring + kRingBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            mbar_init(&bars->full[s], 1);
            mbar_init(&bars->empty[s], 1);
        }
        for (int s = 0; s < kScaleSlots; ++s) {
            mbar_init(&bars->sfull[s], 4);
            mbar_init(&bars->sempty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&bars->tfull[b], 1);
            mbar_init(&bars->tempty[b], 4);
        }
        mbar_init(&bars->mma_done, 1);
        bars->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmP)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmQ)) : "memory");
    }
    grid_begin();
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;
    if (warp == 0) {
        if (lane == 0) produce(&tmP, &tmQ, ring, bars, pr);
    } else if (warp == 1) {
        if (lane == 0) issue_mmas(ring, bars, tmem, pr);
    } else if (warp < 6) {
        write_scales(bars, tmem, pr);
    } else {
        epilogue<T, SWAP>(bars, tmem, pr);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

struct Matrix {   // one operand of a product, as the entry points take it
    const uint8_t* q;
    int64_t rows, ld;
    acrl_fp8_format format;
    const uint8_t* scale;
    int64_t lds;
    acrl_fp8_block block;
};

bool matrix_ok(const Matrix& m, int64_t K) {
    if (m.rows < 0 || m.rows > kMaxGrid - 256 || m.ld < K || (m.ld & 15) || m.lds < (K + 127) / 128) return false;
    if (m.format != ACRL_FP8_E4M3 && m.format != ACRL_FP8_E5M2) return false;
    return m.block == ACRL_FP8_ROW || m.block == ACRL_FP8_TILE;
}

Operand operand(const Matrix& m) {
    return Operand{m.scale, m.lds, int(m.rows), m.block == ACRL_FP8_TILE ? 7 : 0,
                   (m.lds & 3) == 0 && (reinterpret_cast<uintptr_t>(m.scale) & 3) == 0};
}

// Tokens up to this many become the MMA's columns, so that a tile has no more of them than there are.
constexpr int64_t kSwapRows = 128;

template <typename T>
acrl_status launch_matmul(const Matrix& a, const Matrix& b, int64_t K, void* out, int64_t ldo, int32_t* flags,
                          cudaStream_t s) {
    const bool swap = a.rows <= kSwapRows;
    const Matrix &p = swap ? b : a, &q = swap ? a : b;
    Problem pr = {};
    pr.p = operand(p);
    pr.q = operand(q);
    pr.slabs = int((K + kSlab - 1) / kSlab);
    pr.cols = int(q.rows < 256 ? (q.rows + 15) / 16 * 16 : 256);
    pr.p_tiles = int((p.rows + kRows - 1) / kRows);
    pr.q_tiles = int((q.rows + pr.cols - 1) / pr.cols);
    const int64_t total = int64_t(pr.p_tiles) * pr.q_tiles;
    if (total > kMaxGrid) return ACRL_ERR_INVALID_ARG;
    pr.stages = std::min(kMaxStages, kRingBytes / ((kRows + pr.cols) * kSlab));
    pr.accs = 2 * pr.cols <= int(kScaleBase) ? 2 : 1;
    pr.idesc = kIdescBase | uint32_t(p.format) << 7 | uint32_t(q.format) << 10 | uint32_t(pr.cols >> 3) << 17;
    pr.out = out;
    pr.ldo = ldo;
    pr.flags = flags;
    CUtensorMap tmP, tmQ;
    auto map = [&](CUtensorMap* m, const Matrix& x, int box_rows) {
        return encode_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, x.q, uint64_t(x.rows), uint64_t(K), uint64_t(x.ld), box_rows,
                          kSlab, CU_TENSOR_MAP_SWIZZLE_128B);
    };
    if (!map(&tmP, p, kRows) || !map(&tmQ, q, pr.cols)) return ACRL_ERR_CUDA;
    auto* kernel = swap ? fp8_matmul_kernel<T, true> : fp8_matmul_kernel<T, false>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess)
        return launch_status();
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return launch_status();
    return launch(kernel, std::min<int64_t>(total, sms), kThreads, kSmemBytes, 0, s, tmP, tmQ, pr);
}

acrl_status matmul(const Matrix& a, const Matrix& b, int64_t K, void* out, acrl_dtype out_dtype, int64_t ldo,
                   int32_t* flags, cudaStream_t s) {
    if (K < 0 || K > kMaxGrid - 512 || !matrix_ok(a, K) || !matrix_ok(b, K) || !flags) return ACRL_ERR_INVALID_ARG;
    if ((out_dtype != ACRL_BF16 && out_dtype != ACRL_F32) || ldo < b.rows || (ldo & 7)) return ACRL_ERR_INVALID_ARG;
    if (a.rows == 0 || b.rows == 0) return ACRL_OK;
    if (!out || !aligned16(out)) return ACRL_ERR_INVALID_ARG;
    if (K == 0)   // an empty sum
        return cudaMemset2DAsync(out, size_t(ldo) * (out_dtype == ACRL_BF16 ? 2 : 4), 0,
                                 size_t(b.rows) * (out_dtype == ACRL_BF16 ? 2 : 4), size_t(a.rows), s) == cudaSuccess
                   ? ACRL_OK
                   : launch_status();
    if (!a.q || !b.q || !a.scale || !b.scale || !aligned16(a.q) || !aligned16(b.q)) return ACRL_ERR_INVALID_ARG;
    if (!operands_on_current_device({a.q, b.q})) return ACRL_ERR_INVALID_ARG;
    return out_dtype == ACRL_BF16 ? launch_matmul<acrl_bf16>(a, b, K, out, ldo, flags, s)
                                  : launch_matmul<float>(a, b, K, out, ldo, flags, s);
}

}  // namespace
}  // namespace acrl

using namespace acrl;

extern "C" acrl_status acrl_fp8_matmul(const uint8_t* a, int64_t M, int64_t K, int64_t lda, acrl_fp8_format a_format,
                                       const uint8_t* a_scale, int64_t ldas, acrl_fp8_block a_block, const uint8_t* b,
                                       int64_t N, int64_t ldb, acrl_fp8_format b_format, const uint8_t* b_scale,
                                       int64_t ldbs, acrl_fp8_block b_block, void* out, acrl_dtype out_dtype, int64_t ldo,
                                       int32_t* dev_flags, acrl_stream stream) {
    return matmul(Matrix{a, M, lda, a_format, a_scale, ldas, a_block}, Matrix{b, N, ldb, b_format, b_scale, ldbs, b_block}, K,
                  out, out_dtype, ldo, dev_flags, reinterpret_cast<cudaStream_t>(stream));
}

// Rows of quantised activations at a stride of 16 bytes, then their scales at one of four.
extern "C" int64_t acrl_fp8_linear_workspace_bytes(int64_t M, int64_t K) {
    if (M < 0 || K < 0) return -1;
    return M * ((K + 15) / 16 * 16 + ((K + 127) / 128 + 3) / 4 * 4);
}

extern "C" acrl_status acrl_fp8_linear(const acrl_bf16* x, int64_t M, int64_t K, int64_t ldx, acrl_fp8_format x_format,
                                       const uint8_t* w, int64_t N, int64_t ldw, acrl_fp8_format w_format,
                                       const uint8_t* w_scale, int64_t ldws, acrl_fp8_block w_block, void* out,
                                       acrl_dtype out_dtype, int64_t ldo, void* workspace, int64_t workspace_bytes,
                                       int32_t* dev_flags, acrl_stream stream) {
    if (M < 0 || K < 0 || workspace_bytes < acrl_fp8_linear_workspace_bytes(M, K)) return ACRL_ERR_INVALID_ARG;
    const int64_t ldq = (K + 15) / 16 * 16, lds = ((K + 127) / 128 + 3) / 4 * 4;
    if (M > 0 && K > 0 && (!workspace || !aligned16(workspace))) return ACRL_ERR_INVALID_ARG;
    uint8_t* q = static_cast<uint8_t*>(workspace);
    const Matrix a{q, M, ldq, x_format, q + M * ldq, lds, ACRL_FP8_ROW};
    const Matrix b{w, N, ldw, w_format, w_scale, ldws, w_block};
    // the product's arguments are checked before anything is launched
    if (!dev_flags || !matrix_ok(a, K) || !matrix_ok(b, K) || (out_dtype != ACRL_BF16 && out_dtype != ACRL_F32) || ldo < N ||
        (ldo & 7) || (M > 0 && N > 0 && (!out || !aligned16(out))) ||
        (M > 0 && N > 0 && K > 0 && (!w || !w_scale || !aligned16(w) || !operands_on_current_device({w, q}))))
        return ACRL_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return ACRL_OK;
    const acrl_status st = acrl_fp8_quantize(x, ACRL_BF16, M, K, ldx, x_format, ACRL_FP8_ROW, 0, q, ldq, q + M * ldq, lds,
                                             dev_flags, stream);
    if (st != ACRL_OK) return st;
    return matmul(a, b, K, out, out_dtype, ldo, dev_flags, reinterpret_cast<cudaStream_t>(stream));
}
