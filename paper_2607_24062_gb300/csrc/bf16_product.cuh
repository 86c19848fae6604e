// The tensor-core product that the bf16 layer and the orthogonalised update share: sums of bf16 products
//
//     acc[i, j] = sum_k p[i, k] q[j, k]
//
// in fp32, handed to an epilogue of the caller's.  Either operand may lie with the sum's index along its rows ([rows, K]:
// "K-major", a layer's forward) or along its columns ([K, rows]: its gradients, which contract over rows of what they
// read); the copies then fetch 64 x 64 blocks and the MMA takes them transposed, so nothing is turned beforehand.
//
// One CTA per SM, warp-specialised: warp 0 issues the TMA loads of slabs of 64 along the sum (128-byte swizzle) into a ring
// of stages; warp 1 issues tcgen05.mma, four of K = 16 a slab; warps 4-11 are the epilogue, which reads one of two
// accumulators in tensor memory while the MMAs fill the other.  Persistent over the tiles.  Two ways:
//
// Pairs: two CTAs (cta_group::2) share a tile of 256 rows x up to 256 columns, each staging its 128 rows of p and half of q's.
// Alone: a CTA has 128 rows of p or fewer and up to 128 columns.  For few rows of a layer's input, which then are the columns: p is
//   the weight, so that no product is made and nothing is loaded for rows that are not there.
//
// Where tiles are few their sums are split: the parts' accumulators go to a workspace in fp32, and the caller joins them in
// order.  (Joining them in a cluster through distributed shared memory instead saved a launch, but clusters of four CTAs that
// each take an SM do not all find a place at once: 48 x 16,384 x 4,096 33.4 us against 30.3.  Splitting only the tiles of a
// part-filled last round, so that it fills up, gained less than its join takes: 24 x 1,024 x 1,024 in three rounds and a sixth
// 61 us and 9 for the join, in four 66; at the power cap a round that leaves SMs idle runs at a higher clock anyway.)
//
// The tensor cores cut partial sums off where they should round them: an error toward zero that grows with the length of a run
// (relative to the result's norm, of normal numbers: 0.7e-6 for a sum of 1,027, 1.7e-6 for 2,507).  bf16 hides it; for an fp32
// result the sum is taken in runs of kRun slabs, whose accumulators the epilogue's warps add up in registers, rounding, while
// the MMAs fill the next (LONG).  No accumulator takes more than kLongest slabs, whatever the result's type.
//
// TERMS = 3: each operand is two bf16 matrices, p = p0 + p1, and acc takes p0 q0 + p0 q1 + p1 q0 (Dekker's split product
// without its smallest term): four tiles in shared memory feed three MMAs.  One copy brings both halves of an operand: a copy
// takes 75 ns to issue, and of a short sum the first four slabs' sixteen took longer than its MMAs.
#pragma once

#include <cuda.h>

#include <algorithm>

#include "acrl_device.cuh"
#include "acrl_host.h"
#include "mbarrier.cuh"
#include "tcgen05.cuh"
#include "tma_host.h"

namespace acrl {
namespace {

constexpr int kRows = 128;           // rows of p per CTA and tile
constexpr int kSlab = 64;            // of the sum: 128 bytes, one row of the 128-byte swizzle
constexpr int kRowBytes = kSlab * 2;
constexpr int kMaxStages = 12;
constexpr int kDrain = 8;            // epilogue warps
constexpr int kProductThreads = (4 + kDrain) * 32;
constexpr uint32_t kTmemCols = 512;
constexpr int kAccCols = 256;        // of each accumulator
constexpr int kWarpStaging = 4096;   // bytes of an epilogue warp: a block of 32 x 32 in fp32
constexpr int kProductSmem = 227 * 1024;
constexpr int kRun = 8;              // slabs of a run
constexpr int kLongest = 512;        // slabs of a run of any result: 32,768 columns

struct ProductBarriers {
    uint64_t full[kMaxStages];    // the copies of a stage have landed (pair: the even CTA's counts both CTAs')
    uint64_t empty[kMaxStages];   // the MMAs that read it are done
    uint64_t tfull[2];            // an accumulator is complete
    uint64_t tempty[2];           // the epilogue warps (pair: of both CTAs, on the even one) have read it
    uint64_t mma_done;
    uint32_t tmem_base;
    int32_t abort;
};
constexpr int kRingBytes = (kProductSmem - 1024 - kDrain * kWarpStaging - int(sizeof(ProductBarriers))) / 1024 * 1024;

struct Problem {
    int rows, cols_all;      // of the result
    int slabs;               // ceil(K / 64)
    int batch;
    int cols;                // of a tile: a multiple of 32 (pair; of 128 where q is not K-major) or of 16 (alone)
    int p_tiles, q_tiles;
    int parts, per;          // of the sum, of so many slabs
    int run;                 // slabs that one accumulator takes
    int lower;               // p and q are the same, the result symmetric: tiles above the diagonal's are left out
    int p_turned, q_turned;  // the operand lies with the sum along its columns
    uint32_t idesc;
    int tiles, units;        // tiles of one matrix; parts of all
    int pair;
    int high;                // rows of a tile of p: both CTAs' 256, or alone 128 or fewer, a multiple of eight

    // The result's rows and columns of a tile: alone, the rows of q are the result's.
    __host__ __device__ int tile_rows() const { return pair ? 2 * kRows : cols; }
    __host__ __device__ int tile_cols() const { return pair ? cols : high; }
};

// What a CTA or pair works on at a time.
struct Unit {
    int tp, tq, z, part, lo, hi;
    int all;   // the tile among all matrices'
};

// Sums over rows of a matrix's columns, from sums of parts of them ([part][ldparts]), which a warp that is idle otherwise adds up
// beside the products.  The parts go to eight sums in turn, and those are added up in order.
struct ColumnSums {
    const float* parts;
    int64_t ldparts;   // a multiple of 32
    int count, cols;
    float* out;        // or null

    __device__ __forceinline__ void run(int warp, int warps) const {
        const int64_t step = int64_t(warps) * 32;   // as wide as a grid of its own: an int would pass 2^31 beside the most columns
        for (int64_t c = int64_t(warp) * 32 + int(threadIdx.x & 31); c < cols; c += step) {
            float sum[8] = {};
            for (int p = 0; p < count; p += 8) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (p + k < count) sum[k] += parts[(p + k) * ldparts + c];
            }
            float total = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) total += sum[k];
            out[c] = total;
        }
    }
};

template <int NP, int TERMS, class Epi>
struct ProductLaunch {
    CUtensorMap p[NP], q[NP];
    Problem pr[NP];
    Epi epi[NP];
    ColumnSums sums;
    int stages, stage_bytes;
    int32_t* flags;
};

// A tile of 256 x 256 on a symmetric result's diagonal: a CTA's rows of p are its share of q as well, and are loaded once (10 %
// of all loads where there are four tiles to a side; of L2's bandwidth, which bounds 24 x 1,024 x 1,024).
__device__ __forceinline__ bool on_diagonal(const Problem& pr, const Unit& t) {
    return pr.lower && pr.cols == 2 * kRows && t.tp == t.tq;
}

// Tiles in bands of kBand row tiles, all column tiles of a band in turn, so that the tiles in flight share operands in L2.
constexpr int kBand = 16;

// Tile `all` of all matrices'.
__device__ __forceinline__ Unit tile_at(const Problem& pr, int all) {
    Unit w;
    w.all = all;
    w.z = all / pr.tiles;
    const int t = all - w.z * pr.tiles;
    if (pr.lower) {
        // row tile i has min(q_tiles, (i + 1) r) column tiles, r of them as wide as a row tile is high: r i (i + 1) / 2 before it
        const int r = 2 * kRows / pr.cols;
        int i = int((sqrtf(8.f * float(t / r) + 1.f) - 1.f) * 0.5f);
        while (r * i * (i + 1) / 2 > t) --i;
        while (r * (i + 1) * (i + 2) / 2 <= t) ++i;
        w.tp = i;
        w.tq = t - r * i * (i + 1) / 2;
    } else {
        const int per_band = kBand * pr.q_tiles, band = t / per_band, k = t - band * per_band;
        const int h = min(kBand, pr.p_tiles - band * kBand);
        w.tp = band * kBand + k % h;
        w.tq = k / h;
    }
    return w;
}

__device__ __forceinline__ Unit unit_at(const Problem& pr, int u) {
    Unit w = tile_at(pr, u / pr.parts);
    w.part = u - w.all * pr.parts;
    w.lo = w.part * pr.per;
    w.hi = min(pr.slabs, w.lo + pr.per);
    return w;
}

// The units that this CTA or pair takes, of all problems in turn.
template <bool PAIR, int NP, class L>
struct Units {
    const L& l;
    int u, step, which = 0;
    __device__ Units(const L& launch) : l(launch) {
        u = int(blockIdx.x) >> (PAIR ? 1 : 0);
        step = int(gridDim.x) >> (PAIR ? 1 : 0);
        turn();
    }
    __device__ __forceinline__ void turn() {
        if (NP == 2 && which == 0 && u >= l.pr[0].units) {
            which = 1;
            u -= l.pr[0].units;
        }
    }
    __device__ __forceinline__ bool more() const { return u < l.pr[NP == 2 ? which : 0].units; }
    __device__ __forceinline__ void next() {
        u += step;
        turn();
    }
    __device__ __forceinline__ const Problem& problem() const { return l.pr[NP == 2 ? which : 0]; }
    __device__ __forceinline__ Unit unit() const { return unit_at(problem(), u); }
};

// The descriptor of an operand's tile: rows of 128 bytes along the sum, or 64 x 64 blocks in which the sum runs from row to row:
// 64 of the operand's rows are the 128 bytes, eight of the sum are 1,024, and the next 64 rows are a block further (two
// blocks, where each half has its own).
template <int MATS>
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, int turned) {
    return smem_desc(addr) | (turned ? uint64_t(MATS * kSlab * kRowBytes >> 4) << 16 : 0);
}

// What the roles have in common: the ring of stages, its barriers, and how they give up.
struct Ring {
    uint8_t* at;
    ProductBarriers* bars;
    int stages, stage_bytes;
    uint32_t rank;
    int32_t* flags;
};

// The producer warp's loops, and the MMA warp's, run in the whole warp, and one lane is elected for each batch of copies or
// MMAs.  Each role goes through the units that it is given; false: it has given up.
template <bool PAIR, int TERMS>
struct Producer {
    static constexpr int kMats = TERMS == 3 ? 2 : 1;
    const Ring& ring;
    int stage = 0;
    uint32_t phase = 0;
    long issued = 0;

    // The copies that were started land before the CTA can exit: the even CTA's barriers count both CTAs', the odd one gives its
    // own time to land.
    __device__ void land() {
        ProductBarriers* bars = ring.bars;
        if (!PAIR || ring.rank == 0) {
            for (long j = issued - 1; j >= 0 && j >= issued - ring.stages; --j)
                wait_phase(&bars->full[j % ring.stages], uint32_t((j / ring.stages) & 1), nullptr);
        } else {
            const uint64_t t0 = global_ns();
            while (global_ns() - t0 < 100000ull) {
            }
        }
    }

    // p and q: the operands' maps.
    __device__ __forceinline__ bool unit(const Problem& pr, const Unit& t, const CUtensorMap* p, const CUtensorMap* q) {
        ProductBarriers* bars = ring.bars;
        volatile int32_t* abort = &bars->abort;
        const int q_rows = PAIR ? pr.cols / 2 : pr.cols, q_bytes = q_rows * kRowBytes;
        const bool once = PAIR && on_diagonal(pr, t);
        const int bytes = kMats * ((PAIR ? kRows : pr.high) * kRowBytes + (once ? 0 : q_bytes));
        const int p0 = PAIR ? (2 * t.tp + int(ring.rank)) * kRows : t.tp * pr.high;
        const int q0 = t.tq * pr.cols + (PAIR ? int(ring.rank) * q_rows : 0);
        const bool p_turned = pr.p_turned, q_turned = pr.q_turned;
        for (int kb = t.lo; kb < t.hi; ++kb) {
            if (!warp_wait(&bars->empty[stage], phase ^ 1u, abort)) {
                give_up(abort, ring.flags);
                land();
                return false;
            }
            uint8_t* s = ring.at + stage * ring.stage_bytes;
            const uint32_t bar = PAIR ? peer_addr(&bars->full[stage], 0) : smem_u32(&bars->full[stage]);
            if (elect_one()) {
                if (!PAIR || ring.rank == 0) mbar_expect_tx(&bars->full[stage], uint32_t((PAIR ? 2 : 1) * bytes));
                // 64 x 64 blocks of a turned operand, rows of the other kind
                auto copy = [&](uint8_t* to, const CUtensorMap* map, bool turned, int row, int rows) {
                    for (int j = 0; j < (turned ? rows : 1); j += kSlab) {
                        uint8_t* at = to + kMats * j * kRowBytes;
                        const int x = turned ? row + j : kb * kSlab, y = turned ? kb * kSlab : row;
                        if constexpr (kMats == 2) tma_load_4d<PAIR>(at, map, bar, x, y, t.z);
                        else tma_load_3d<PAIR>(at, map, bar, x, y, t.z);
                    }
                };
                copy(s, p, p_turned, p0, kRows);
                if (!once) copy(s + kMats * kRows * kRowBytes, q, q_turned, q0, q_rows);
            }
            ++issued;
            if (++stage == ring.stages) {
                stage = 0;
                phase ^= 1u;
            }
        }
        return true;
    }
};

template <bool PAIR>
__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t pdesc, uint64_t qdesc, uint32_t idesc, uint32_t accumulate) {
    if (PAIR)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
            "l"(pdesc), "l"(qdesc), "r"(idesc), "r"(accumulate));
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
            "l"(pdesc), "l"(qdesc), "r"(idesc), "r"(accumulate));
}

template <bool PAIR, int TERMS>
struct Multiplier {
    static constexpr int kMats = TERMS == 3 ? 2 : 1;
    const Ring& ring;
    uint32_t tmem;
    int stage = 0, acc = 0;
    uint32_t phase = 0, aphase = 0;

    __device__ __forceinline__ bool unit(const Problem& pr, const Unit& t) {
        ProductBarriers* bars = ring.bars;
        volatile int32_t* abort = &bars->abort;
        const uint32_t base = smem_u32(ring.at), units = uint32_t(ring.stage_bytes) >> 4;   // of a stage, in descriptors
        const uint64_t pdesc0 = tile_desc<kMats>(base, pr.p_turned);
        const uint64_t qdesc0 = PAIR && on_diagonal(pr, t) ? pdesc0 : tile_desc<kMats>(base + kMats * kRows * kRowBytes, pr.q_turned);
        // from one K = 16 to the next: 32 bytes of a row, or sixteen rows
        const uint32_t pstep = pr.p_turned ? 16 * kRowBytes >> 4 : 2, qstep = pr.q_turned ? 16 * kRowBytes >> 4 : 2;
        // from a half to the other
        const uint32_t plow = uint32_t((pr.p_turned ? kSlab : kRows) * kRowBytes) >> 4;
        const uint32_t qlow = uint32_t((pr.q_turned ? kSlab : PAIR ? pr.cols / 2 : pr.cols) * kRowBytes) >> 4;
        for (int run = t.lo; run < t.hi; run += pr.run) {
            if (!warp_wait(&bars->tempty[acc], aphase ^ 1u, abort)) {
                give_up(abort, ring.flags);
                return false;
            }
            tc_fence_after();
            const uint32_t d = tmem + uint32_t(acc * kAccCols);
            const int end = min(t.hi, run + pr.run);
            for (int kb = run; kb < end; ++kb) {
                if (!warp_wait(&bars->full[stage], phase, abort)) {
                    give_up(abort, ring.flags);
                    return false;
                }
                tc_fence_after();
                const uint64_t pd = pdesc0 + stage * units, qd = qdesc0 + stage * units;
                const uint32_t more = kb > run;
                if (elect_one()) {
#pragma unroll
                    for (int i = 0; i < TERMS; ++i) {
                        const uint64_t a = pd + (i == 2 ? plow : 0u), b = qd + (i == 1 ? qlow : 0u);
#pragma unroll
                        for (uint32_t k = 0; k < kSlab / 16; ++k)
                            mma_bf16<PAIR>(d, a + k * pstep, b + k * qstep, pr.idesc, i > 0 || k > 0 ? 1u : more);
                    }
                    commit<PAIR>(&bars->empty[stage]);
                }
                if (++stage == ring.stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            if (elect_one()) commit<PAIR>(&bars->tfull[acc]);
            if (++acc == 2) {
                acc = 0;
                aphase ^= 1u;
            }
        }
        return true;
    }

    // Every MMA has finished before the CTA moves on.
    __device__ void finish() {
        if (elect_one()) {
            if (PAIR)
                asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                                 peer_addr(&ring.bars->mma_done, 0))
                             : "memory");
            else
                commit<false>(&ring.bars->mma_done);
        }
        wait_phase(&ring.bars->mma_done, 0, nullptr);
        __syncwarp();
    }
};

__device__ __forceinline__ void ld_shared16(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr));
}

// An epilogue warp's way out: through its block of shared memory, so that neighbouring lanes store neighbouring pieces of 16
// bytes, four or eight to a row.  (TMA stores of the blocks took longer: a copy keeps its block for about 1,000 cycles, and the
// next 32 columns waited for it.  256 x 256 x 256, alone: 4.3 us, now 3.3.)
struct WarpOut {
    uint8_t* staging;
    int lane;

    // What was staged, 32 rows of T, to rows row0 .. and columns col0 .. of a matrix of rows x cols at a stride of ld.  Every lane
    // of the warp.  `wide`: the pieces start on 16 bytes.
    template <typename T>
    __device__ __forceinline__ void send(T* to, int64_t ld, int rows, int cols, int row0, int col0, bool wide) const {
        constexpr int kPieces = 32 * int(sizeof(T)) / 16, kEach = 16 / int(sizeof(T)), kRowsAtOnce = 32 / kPieces;
        const uint32_t base = smem_u32(staging);
        __syncwarp();
        const int piece = lane & (kPieces - 1), c = col0 + piece * kEach, r0 = lane / kPieces;
        uint32_t v[kPieces][4];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int r = i * kRowsAtOnce + r0;
            const uint32_t swz = kPieces == 4 ? uint32_t((r >> 1) & 3) : uint32_t(r & 7);
            ld_shared16(base + uint32_t(r * 32 * int(sizeof(T))) + ((uint32_t(piece) ^ swz) << 4), v[i]);
        }
        T* p = to + (row0 + r0) * ld + c;
        const int64_t step = kRowsAtOnce * ld;
        if (c + kEach <= cols && wide) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                if (row0 + r0 + i * kRowsAtOnce < rows)
                    *reinterpret_cast<uint4*>(p + i * step) = make_uint4(v[i][0], v[i][1], v[i][2], v[i][3]);
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#pragma unroll
                for (int k = 0; k < kEach; ++k)
                    if (c + k < cols && row0 + r0 + i * kRowsAtOnce < rows) {
                        if constexpr (sizeof(T) == 2) p[i * step + k] = T(v[i][k >> 1] >> (k & 1) * 16);
                        else p[i * step + k] = __uint_as_float(v[i][k]);
                    }
        }
        __syncwarp();   // the block may be written again
    }

    // Lane i has row row0 + i and its columns col0 .. col0 + 31.
    template <typename T>
    __device__ __forceinline__ void store(T* to, int64_t ld, int rows, int cols, const float (&v)[32], int row0, int col0,
                                          bool wide = true) const {
        constexpr int kPieces = 32 * int(sizeof(T)) / 16;
        const uint32_t swz = kPieces == 4 ? uint32_t((lane >> 1) & 3) : uint32_t(lane & 7);
        const uint32_t at = smem_u32(staging) + uint32_t(lane * 32 * int(sizeof(T)));
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            uint4 x;
            if constexpr (sizeof(T) == 2)
                x = make_uint4(pack_bf16x2(v[8 * k], v[8 * k + 1]), pack_bf16x2(v[8 * k + 2], v[8 * k + 3]),
                               pack_bf16x2(v[8 * k + 4], v[8 * k + 5]), pack_bf16x2(v[8 * k + 6], v[8 * k + 7]));
            else
                x = make_uint4(__float_as_uint(v[4 * k]), __float_as_uint(v[4 * k + 1]), __float_as_uint(v[4 * k + 2]),
                               __float_as_uint(v[4 * k + 3]));
            st_shared16(at + ((uint32_t(k) ^ swz) << 4), x);
        }
        send(to, ld, rows, cols, row0, col0, wide);
    }

    // The values as two bf16 numbers each, h their roundings and l those of what is left, to two matrices; as store, or turned:
    // lane i has column col0 + i and its rows row0 .. row0 + 31.  Both go through shared memory at once, turned ones as words of
    // both halves: one after the other, with 16-bit words, a tile of 256 x 256 and its mirror image took 9 us.
    __device__ __forceinline__ void store_halves(acrl_bf16* hi, acrl_bf16* lo, int64_t ld, int rows, int cols, const uint32_t (&h)[16],
                                                 const uint32_t (&l)[16], int row0, int col0) const {
        const uint32_t base = smem_u32(staging), swz = uint32_t((lane >> 1) & 3), at = base + uint32_t(lane * 64);
        constexpr uint32_t kHalf = kWarpStaging / 2;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t to = at + ((uint32_t(k) ^ swz) << 4);
            st_shared16(to, make_uint4(h[4 * k], h[4 * k + 1], h[4 * k + 2], h[4 * k + 3]));
            st_shared16(to + kHalf, make_uint4(l[4 * k], l[4 * k + 1], l[4 * k + 2], l[4 * k + 3]));
        }
        __syncwarp();
        const int piece = lane & 3, c = col0 + 8 * piece, r0 = lane >> 2;
        uint32_t v[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = (i & 3) * 8 + r0;
            ld_shared16(base + (i >> 2) * kHalf + uint32_t(r * 64) + ((uint32_t(piece) ^ uint32_t((r >> 1) & 3)) << 4), v[i]);
        }
        const int64_t to = (row0 + r0) * ld + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            acrl_bf16* p = (i < 4 ? hi : lo) + to + (i & 3) * 8 * ld;
            if (row0 + r0 + (i & 3) * 8 >= rows) continue;
            if (c + 8 <= cols) {
                *reinterpret_cast<uint4*>(p) = make_uint4(v[i][0], v[i][1], v[i][2], v[i][3]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < cols) p[k] = acrl_bf16(v[i][k >> 1] >> (k & 1) * 16);
            }
        }
        __syncwarp();
    }

    __device__ __forceinline__ void store_halves_turned(acrl_bf16* hi, acrl_bf16* lo, int64_t ld, int rows, int cols, const uint32_t (&h)[16],
                                                        const uint32_t (&l)[16], int row0, int col0) const {
        const uint32_t base = smem_u32(staging), at = base + uint32_t((lane & 3) * 4);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const uint32_t word = __byte_perm(h[j >> 1], l[j >> 1], j & 1 ? 0x7632 : 0x5410);
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(at + uint32_t(j * 128) + ((uint32_t(lane >> 2) ^ uint32_t(j & 7)) << 4)), "r"(word)
                         : "memory");
        }
        __syncwarp();
        const int piece = lane & 7, c = col0 + 4 * piece, r0 = lane >> 3;
        uint32_t v[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = i * 4 + r0;
            ld_shared16(base + uint32_t(r * 128) + ((uint32_t(piece) ^ uint32_t(r & 7)) << 4), v[i]);
        }
        const int64_t to = (row0 + r0) * ld + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (row0 + r0 + i * 4 >= rows) continue;
            acrl_bf16 *p = hi + to + i * 4 * ld, *q = lo + to + i * 4 * ld;
            if (c + 4 <= cols) {
                *reinterpret_cast<uint2*>(p) = make_uint2(__byte_perm(v[i][0], v[i][1], 0x5410), __byte_perm(v[i][2], v[i][3], 0x5410));
                *reinterpret_cast<uint2*>(q) = make_uint2(__byte_perm(v[i][0], v[i][1], 0x7632), __byte_perm(v[i][2], v[i][3], 0x7632));
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < cols) {
                        p[k] = acrl_bf16(v[i][k]);
                        q[k] = acrl_bf16(v[i][k] >> 16);
                    }
            }
        }
        __syncwarp();
    }

    // The same values turned, rounded to bf16: lane i has column col0 + i and its rows row0 .. row0 + 31.
    __device__ __forceinline__ void store_turned(acrl_bf16* to, int64_t ld, int rows, int cols, const float (&v)[32], int row0,
                                                 int col0, bool wide) const {
        const uint32_t at = smem_u32(staging) + uint32_t((lane & 7) * 2);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const uint32_t piece = uint32_t(lane >> 3) ^ uint32_t((j >> 1) & 3);
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(at + uint32_t(j * 64) + (piece << 4)),
                         "h"(acrl_bf16(pack_bf16x2(v[j], 0.f) & 0xffffu))
                         : "memory");
        }
        send(to, ld, rows, cols, row0, col0, wide);
    }
};

// Eight columns of a warp's 32 lanes, added to v.  (Sixteen at a time would not fit beside a long sum.)
__device__ __forceinline__ void tmem_add8(uint32_t taddr, float* v) {
    uint32_t r[8];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += __uint_as_float(r[j]);
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]),
        "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
        : "memory");
}

template <bool PAIR, bool LONG>
struct Drain {
    const Ring& ring;
    uint32_t tmem;
    WarpOut out;
    int lane, quarter, first;   // the two warps of a quarter take 32 columns in turn
    int acc = 0;
    uint32_t phase = 0;
    // The first unit's first columns are gone through twice, before its products are there with a matrix of no rows and no
    // columns, which loads and stores nothing: what follows a sum is then in the instruction cache when it is waited for (from
    // there its 1,100 cycles were mostly misses; a layer of 256 x 256 x 256 3.9 us, now 3.4).
    bool dry = true;

    __device__ Drain(const Ring& r, uint32_t t, uint8_t* staging) : ring(r), tmem(t) {
        const int warp = int(threadIdx.x >> 5) - 4;
        lane = threadIdx.x & 31;
        quarter = warp & 3;
        first = 32 * (warp >> 2);
        out = WarpOut{staging + warp * kWarpStaging, lane};
    }

    // The accumulator is read out: the MMA warp may fill it again.  The fence orders the reads of tensor memory; the arrival has
    // nothing else to release, and one that releases to the whole cluster waits for the stores under way, 1,000 cycles.
    __device__ __forceinline__ void release() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
            if (PAIR)
                asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(peer_addr(&ring.bars->tempty[acc], 0)) : "memory");
            else
                mbar_arrive(&ring.bars->tempty[acc]);
        }
    }
    __device__ __forceinline__ void turn() {
        if (++acc == 2) {
            acc = 0;
            phase ^= 1u;
        }
    }

    // The sums of a unit, once their accumulator holds them whole.
    __device__ __forceinline__ bool ready(const Problem& pr, const Unit& t) {
        volatile int32_t* abort = &ring.bars->abort;
        if constexpr (!LONG) {
            const bool ok = warp_wait(&ring.bars->tfull[acc], phase, abort);
            tc_fence_after();
            return ok;
        }
        constexpr int kMost = PAIR ? 4 : 2;   // chunks of a warp
        const uint32_t lanes = uint32_t(quarter * 32) << 16;
        float sum[kMost * 32] = {};
        const int runs = (t.hi - t.lo + pr.run - 1) / pr.run;
        bool ok = true;
        for (int i = 0; i < runs && ok; ++i) {
            // a call would spill the sums
            ok = __all_sync(0xffffffffu, wait_phase_inline(&ring.bars->tfull[acc], phase, abort));
            if (!ok) break;
            tc_fence_after();
            if (runs == 1) break;
            const bool last = i + 1 == runs;
            const uint32_t at = tmem + uint32_t(acc * kAccCols + first) + lanes;   // beyond the tile's columns, too
#pragma unroll
            for (int k = 0; k < 4 * kMost; ++k) tmem_add8(at + 64 * (k >> 2) + 8 * (k & 3), sum + 8 * k);
            if (last) {   // what follows reads the whole sum as it would read one run's
#pragma unroll
                for (int k = 0; k < 2 * kMost; ++k) tmem_st16(at + 64 * (k >> 1) + 16 * (k & 1), sum + 16 * k);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            } else {
                release();
                turn();
            }
        }
        return ok;
    }

    // The unit numbered u.
    template <class Epi>
    __device__ __forceinline__ bool unit(const Problem& pr, int u, const Epi& epi) {
        Unit t = unit_at(pr, u);
#pragma unroll 1
        for (int pass = dry ? 0 : 1; pass < 2; ++pass) {
            const bool live = pass == 1;
            if (live && !ready(pr, t)) {
                give_up(&ring.bars->abort, ring.flags);
                return false;
            }
            if constexpr (LONG) {   // worked out again: kept beside a long sum it would take registers that the sum needs
                asm volatile("" : "+r"(u));
                t = unit_at(pr, u);
            }
            const int row0 = (PAIR ? (2 * t.tp + int(ring.rank)) * kRows : t.tp * pr.high) + quarter * 32;
            const int rows = PAIR ? pr.rows : min(pr.rows, (t.tp + 1) * pr.high);   // of the result, as far as the tile goes
            if (live && first >= pr.cols) release();   // a tile of 32 columns has none for this warp
#pragma unroll 1
            for (int c = first; c < pr.cols; c += 64) {
                uint32_t r[32];
                __syncwarp();
                tmem_ld32(tmem + uint32_t(acc * kAccCols + c) + (uint32_t(quarter * 32) << 16), r);
                if (live && c + 64 >= pr.cols) release();
                const int col0 = t.tq * pr.cols + c;
                if (row0 < rows && col0 < pr.cols_all)   // the same for the whole warp
                    epi.chunk(pr, t, r, row0, col0, live ? rows : 0, live ? pr.cols_all : 0, out);
                if (!live) break;
            }
            __syncwarp();
        }
        dry = false;
        turn();
        return true;
    }
};

// What a kernel of products does before its roles begin, and after they have ended.
struct Begun {
    Ring ring;
    uint8_t* staging;
    uint32_t tmem;
};

template <bool PAIR>
__device__ __forceinline__ Begun begin_products(uint8_t* smem, int stages, int stage_bytes, const CUtensorMap* p, const CUtensorMap* q,
                                                int32_t* flags) {
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem) + 1023) & ~uintptr_t(1023));
    uint8_t* staging = ring + kRingBytes;
    ProductBarriers* bars = reinterpret_cast<ProductBarriers*>(staging + kDrain * kWarpStaging);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            mbar_init(&bars->full[s], 1);
            mbar_init(&bars->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&bars->tfull[b], 1);
            mbar_init(&bars->tempty[b], (PAIR ? 2 : 1) * kDrain);
        }
        mbar_init(&bars->mma_done, 1);
        bars->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(p)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(q)) : "memory");
    }
    // Before the grid's wait, while the launch before this one ends: nothing here touches memory, and with all of an SM's shared
    // memory a CTA shares its tensor memory with no other.
    if (threadIdx.x >> 5 == 2) {
        if (PAIR) {   // one warp of each CTA of the pair, together
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)),
                         "r"(kTmemCols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)),
                         "r"(kTmemCols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();   // the other's barriers are initialised, and it runs
    tc_fence_after();
    const Begun b{Ring{ring, bars, stages, stage_bytes, PAIR ? cluster_rank() : 0u, flags}, staging, bars->tmem_base};
    grid_begin();
    return b;
}

template <bool PAIR>
__device__ __forceinline__ void end_products(uint32_t tmem) {
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();   // no CTA frees its TMEM or leaves while the other may still touch it
    if (threadIdx.x >> 5 == 2) {
        tc_fence_after();
        if (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

template <bool PAIR, bool LONG, int NP, int TERMS, class Epi>
__global__ void __launch_bounds__(kProductThreads, 1)
    product_kernel(const __grid_constant__ ProductLaunch<NP, TERMS, Epi> l) {
    using L = ProductLaunch<NP, TERMS, Epi>;
    extern __shared__ uint8_t smem_raw[];
    const Begun b = begin_products<PAIR>(smem_raw, l.stages, l.stage_bytes, &l.p[0], &l.q[0], l.flags);
    const int warp = threadIdx.x >> 5;
    if (warp < 4) {
        if (warp == 0) {
            Producer<PAIR, TERMS> role{b.ring};
            for (Units<PAIR, NP, L> w(l); w.more(); w.next())
                if (!role.unit(w.problem(), w.unit(), &l.p[NP == 2 ? w.which : 0], &l.q[NP == 2 ? w.which : 0])) break;
        }
        if (warp == 1 && b.ring.rank == 0) {
            Multiplier<PAIR, TERMS> role{b.ring, b.tmem};
            for (Units<PAIR, NP, L> w(l); w.more(); w.next())
                if (!role.unit(w.problem(), w.unit())) break;
            role.finish();
        }
        if (warp == 3 && l.sums.out) l.sums.run(int(blockIdx.x), int(gridDim.x));
    } else {
        Drain<PAIR, LONG> role(b.ring, b.tmem, b.staging);
        for (Units<PAIR, NP, L> w(l); w.more(); w.next())
            if (!role.unit(w.problem(), w.u, l.epi[NP == 2 ? w.which : 0])) break;
    }
    end_products<PAIR>(b.tmem);
}

// ---------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------

// An operand of a product: [rows, K], or with `turned` [K, rows]; `count` of them `apart` elements from one another, and with
// `halves` > 0 two such lots, that many from one another.
struct Matrix {
    const acrl_bf16* at;
    int64_t rows, ld;
    bool turned;
    int64_t count, apart, halves;
};

inline bool operand_map(CUtensorMap* map, const Matrix& m, int64_t K, int box_rows) {
    return encode_map_3d(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m.at, uint64_t(m.count), uint64_t(m.turned ? K : m.rows),
                         uint64_t(m.turned ? m.rows : K), uint64_t(m.ld), uint64_t(m.apart), uint64_t(m.halves),
                         uint32_t(m.turned ? kSlab : box_rows), kSlab, CU_TENSOR_MAP_SWIZZLE_128B);
}

// How a product is cut: columns of a tile, tiles of all matrices, and the sum's parts of `per` slabs.
struct Cut {
    int cols;
    int64_t tiles;
    int parts, per;

    int64_t units() const { return tiles * parts; }
};

// What is cut.  cols from `widest` down to `least` in steps of `step`, or halves for 0.
struct Shape {
    bool pair;
    int64_t rows, cols_all, K, batch;
    bool lower;
    int terms, widest, least, step;
    int high;   // rows of a tile

    int64_t slabs() const { return std::max<int64_t>(1, (K + kSlab - 1) / kSlab); }
    int64_t lanes() const { return pair ? 76 : 152; }   // what a GPU of 152 SMs runs at once (another one is served, by these estimates)
    int64_t tiles(int cols) const {
        const int64_t p = (rows + high - 1) / high, q = (cols_all + cols - 1) / cols, r = high / cols;
        // of a symmetric matrix, each row tile but the last has r columns more than the one before
        return batch * (lower && p > 0 ? r * (p - 1) * p / 2 + q : p * q);
    }
    // Cycles of a slab: the MMAs, or the copies at 52 bytes a cycle of an SM; alone, where they come from HBM, no less than 3,800
    // a turn of the ring (48 x 4,096 x 4,096 whole: 64 slabs 16 us, whether the tiles have 64 or 128 rows of p), and of pairs, whose
    // rings are deeper, no less than 450.
    int64_t slab(int cols) const {
        const int64_t mats = terms == 3 ? 2 : 1, mine = pair ? cols / 2 : cols, bytes = mats * (kRows + mine) * kRowBytes;
        const int64_t work = std::max<int64_t>(terms * (pair ? 2 : 4) * int64_t(cols), bytes / 52);
        return pair ? std::max<int64_t>(work, 450) : std::max(work, 3800 / std::min<int64_t>(kMaxStages, kRingBytes / bytes));
    }
    int64_t tile_bytes(int cols) const { return int64_t(high) * cols * 4; }
    int next(int cols) const { return step > 0 ? cols - step : cols / 2; }
};

constexpr int64_t kTileCycles = 500;                             // of a tile in a run of them
constexpr int64_t kJoinCycles = 5000, kJoinBytes = 3000;         // of a join's launch; bytes a cycle
constexpr int64_t kPartCycles = 1500;                            // of a part of pairs' sums: a join reads one after another
// (with 450 cycles a slab and these: 768 x 4,096 x 1,024 18.4 -> 15.0 us, 2,048 x 8,192 x 256 20.5 -> 16.9, 200 x 4,096 x 4,096 18.5 ->
// 17.2; 256 x 2,048 x 2,048 11.3 -> 11.9)
constexpr int kPartChoices[] = {2, 3, 4, 5, 6, 8, 10, 12, 16};

// Parts of equal length, none of them empty: false where `parts` is no such number.
inline bool part_length(int64_t slabs, int64_t parts, int64_t& per) {
    if (parts > slabs) return false;
    per = (slabs + parts - 1) / parts;
    return (slabs + per - 1) / per == parts;
}

inline int64_t join_cycles(const Shape& s, const Cut& c) {
    return c.parts == 1 ? 0 : kJoinCycles + (s.pair && s.terms == 1 ? c.parts * kPartCycles : 0) +
                                  c.tiles * (c.parts + 1) * s.tile_bytes(c.cols) / kJoinBytes;
}
inline int64_t unit_cycles(const Shape& s, const Cut& c) { return c.per * s.slab(c.cols) + kTileCycles; }

// Rounds of units, the last of them part-filled, and the joining of parts.  Alone, HBM bounds a round that is full.
constexpr int64_t kHbmBytes = 3100;   // a cycle
inline int64_t cut_cycles(const Shape& s, const Cut& c) {
    const int64_t lanes = s.lanes(), units = c.units(), unit = unit_cycles(s, c);
    const int64_t bytes = s.pair ? 0 : int64_t(c.per) * s.high * kRowBytes;
    auto round = [&](int64_t n) { return std::max(unit, n * bytes / kHbmBytes); };
    return units / lanes * round(lanes) + (units % lanes > 0 ? round(units % lanes) : 0) + join_cycles(s, c);
}

// consider(cut) for the whole sums of tiles of `cols` columns and, where there are no more than `few` tiles, for parts of them.
template <typename F>
void each_cut(const Shape& s, int cols, int64_t few, F consider) {
    const int64_t tiles = s.tiles(cols), slabs = s.slabs();
    // products of two halves each have no runs: a very long sum is split wherever it is
    const int64_t least = s.terms == 3 ? (slabs + kLongest - 1) / kLongest : 1, longest = (slabs + least - 1) / least;
    consider(Cut{cols, tiles, int((slabs + longest - 1) / longest), int(longest)});
    for (int64_t parts : kPartChoices) {
        int64_t per;
        if (tiles > few || tiles * (parts - 1) >= 2 * s.lanes()) break;
        if (parts > least && part_length(slabs, parts, per)) consider(Cut{cols, tiles, int(parts), int(per)});
    }
}

// The cut with the least estimated time: rounds of units, and the joining of parts.
inline Cut best_cut(const Shape& s) {
    const int64_t lanes = s.lanes();
    Cut best = {};
    int64_t least = -1;
    for (int cols = s.widest; cols >= s.least; cols = s.next(cols))
        each_cut(s, cols, 2 * lanes, [&](const Cut& c) {
            const int64_t cost = cut_cycles(s, c);
            if (least >= 0 && cost >= least) return;
            least = cost;
            best = c;
        });
    return best;
}

// Two products in one launch, the second's units after the first's: the cycles of the busiest lane, whose units are every
// lanes-th.
inline int64_t two_cycles(const Shape& s0, const Cut& c0, const Shape& s1, const Cut& c1) {
    const int64_t lanes = s0.lanes(), a = c0.units(), b = a + c1.units();
    auto upto = [&](int64_t x, int64_t lane) { return x > lane ? (x - lane + lanes - 1) / lanes : 0; };
    int64_t most = 0;
    for (int64_t lane : {int64_t(0), a % lanes, b % lanes}) {   // where the counts change
        const int64_t n = upto(a, lane);
        most = std::max(most, n * unit_cycles(s0, c0) + (upto(b, lane) - n) * unit_cycles(s1, c1));
    }
    return most + join_cycles(s0, c0) + join_cycles(s1, c1);
}

// Cuts both for one launch.
inline void best_cuts(const Shape& s0, const Shape& s1, Cut& best0, Cut& best1) {
    int64_t least = -1;
    for (int cols = s0.widest; cols >= s0.least; cols = s0.next(cols))
        each_cut(s0, cols, s0.lanes(), [&](const Cut& c0) {
            each_cut(s1, cols, s0.lanes(), [&](const Cut& c1) {
                const int64_t cost = two_cycles(s0, c0, s1, c1);
                if (least >= 0 && cost >= least) return;
                least = cost;
                best0 = c0;
                best1 = c1;
            });
        });
}

// The parts' workspace: [tile][part][row of the tile][column of it].
inline int64_t parts_bytes(const Shape& s, const Cut& c) { return c.parts == 1 ? 0 : c.units() * s.tile_bytes(c.cols); }

// tcgen05.mma kind::f16: D f32 (bits 4-5 = 1), A and B bf16 (bits 7-9, 10-12 = 1), A and B transposed (bits 15, 16),
// N / 8 at bit 17, M / 16 at bit 24.
inline Problem problem_of(const Shape& s, const Cut& cut, bool p_turned, bool q_turned, bool runs) {
    Problem pr = {};
    pr.rows = int(s.rows);
    pr.cols_all = int(s.cols_all);
    pr.slabs = int(s.slabs());
    pr.batch = int(s.batch);
    pr.cols = cut.cols;
    pr.pair = s.pair;
    pr.high = s.high;
    pr.p_tiles = int((s.rows + s.high - 1) / s.high);
    pr.q_tiles = int((s.cols_all + cut.cols - 1) / cut.cols);
    pr.parts = cut.parts;
    pr.per = cut.per;
    pr.run = runs ? kRun : pr.slabs;
    pr.lower = s.lower;
    pr.p_turned = p_turned;
    pr.q_turned = q_turned;
    pr.idesc = 1u << 4 | 1u << 7 | 1u << 10 | uint32_t(p_turned) << 15 | uint32_t(q_turned) << 16 |
               uint32_t(cut.cols >> 3) << 17 | uint32_t((s.pair ? 2 * kRows : kRows) >> 4) << 24;
    pr.tiles = int(cut.tiles / std::max<int64_t>(1, s.batch));
    pr.units = int(cut.units());
    return pr;
}

// More units than an int counts are refused by the caller.
inline bool units_fit(const Cut& cut) { return cut.tiles < (1 << 30) && cut.units() < (1 << 30); }

// Allows the kernel its shared memory; the pairs, or CTAs alone, that can be resident at once: kept for the device that the
// calling thread used last.
template <bool PAIR, bool LONG, int NP, int TERMS, class Epi>
int64_t resident_products() {
    static thread_local int known = -1;
    static thread_local int64_t most = 0;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    if (dev == known) return most;
    auto* kernel = product_kernel<PAIR, LONG, NP, TERMS, Epi>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kProductSmem) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    most = PAIR ? resident_clusters(reinterpret_cast<const void*>(kernel), kProductThreads, kProductSmem, 2) : sms;
    if (most > 0) known = dev;
    return most;
}

template <bool PAIR, bool LONG, int NP, int TERMS, class Epi>
acrl_status launch_product(ProductLaunch<NP, TERMS, Epi>& l, int32_t* flags, cudaStream_t s) {
    constexpr int kMats = TERMS == 3 ? 2 : 1;
    l.stage_bytes = 0;
    int64_t units = 0;
    for (int i = 0; i < NP; ++i) {
        const int bytes = kMats * (kRows + (PAIR ? l.pr[i].cols / 2 : l.pr[i].cols)) * kRowBytes;
        l.stage_bytes = std::max(l.stage_bytes, bytes);
        units += l.pr[i].units;
    }
    l.stages = std::min(kMaxStages, kRingBytes / l.stage_bytes);
    l.flags = flags;
    const int64_t most = resident_products<PAIR, LONG, NP, TERMS, Epi>();
    if (most < 1) return ACRL_ERR_CUDA;
    return launch(product_kernel<PAIR, LONG, NP, TERMS, Epi>, std::min(units, most) * (PAIR ? 2 : 1), kProductThreads, kProductSmem,
                  PAIR ? 2 : 0, s, l);
}

}  // namespace
}  // namespace acrl
