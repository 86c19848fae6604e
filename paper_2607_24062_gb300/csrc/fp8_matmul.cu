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
//   warp 0     issues the TMA loads of the operands' 128-byte slabs (128-byte swizzle) into a ring of stages;
//   warp 1     issues the MMAs, four of K = 32 per slab;
//   warps 2-5  load the scales of four slabs at a time and write them to tensor
//              memory (each warp its own quarter of the lanes: the MMA wants the
//              32 lanes' words in every quarter);
//   the rest   the epilogue: accumulator rows out of tensor memory, rounded once,
//              stored, while the MMAs fill the other accumulator.
// The operand whose rows become the MMA's rows is "P", the other, whose rows
// become its columns, is "Q".  Two ways:
//
// Pairs (many rows): two CTAs share a tile of 256 rows (cta_group::2), each staging
//   its 128 rows of P and half of Q's, so that an SM loads 240 bytes per
//   256 x 224 x 1 products where a CTA alone would load 352: the way from L2 into shared
//   memory (12 TB/s) bounds the product.  The even CTA issues the MMAs, which read
//   both CTAs' shared memory and each CTA's own tensor memory (accumulator, the
//   scales of its own rows and of all columns).  Persistent over the tiles.  Where there
//   are tiles enough, or K is long, a tile has 320 to 448 columns: 176 bytes for as many products,
//   in two parts of one accumulator, each drained by the epilogue while the other's MMAs run.  4,096 x 16,384 x
//   8,192 in 309 us, 3.6 PFLOP/s; 4,096 x 151,936 x 4,096 in 1,515 us, and 1,718 in a loop at the power cap.
// Alone (few rows): P is the wide operand, the weight, and the few rows are the
//   MMA's columns, so that nothing is computed or loaded for rows that are not there;
//   HBM bounds it (48 x 151,936 x 4,096 in 101 us, 6.3 TB/s).  Where there are fewer tiles than SMs, a cluster shares a tile by
//   columns of the sum (K), exchanges its accumulators through distributed shared
//   memory and adds them in rank order, each CTA a share of them (16 x 4,096 x 4,096 in 7.8 us).
#include <algorithm>

#include "acrl_device.cuh"
#include "acrl_host.h"
#include "fp8.cuh"
#include "mbarrier.cuh"
#include "tcgen05.cuh"
#include "tma_host.h"

namespace acrl {
namespace {

constexpr int kRows = 128;             // rows of P per CTA and tile
constexpr int kSlab = 128;             // columns of a slab: 128 bytes, one row of the 128-byte swizzle
constexpr int kGroup = 4;              // slabs whose scales share a word
constexpr int kMaxStages = 12, kScaleSlots = 4;
constexpr int kMaxSplit = 8;           // CTAs that share a tile's sum; 16 columns are eight's shares
constexpr uint32_t kTmemCols = 512;
// Tensor memory: accumulators from column 0, scale slots of 16 columns at the end (P's words in the first four of
// them, Q's, up to 256 rows, in the last eight).
constexpr uint32_t kScaleCols = 16, kScaleBase = kTmemCols - kScaleSlots * kScaleCols;
constexpr int kPairCols = int(kScaleBase) / 2;   // 224: two accumulators beside the scales

// How a tile is made: kAlone and kPair as above; kWide, a pair's tile of up to 448 columns in two parts, the first of 256
// (the most columns of an MMA), with two slots of scales of twice the width.
enum Mode { kAlone, kPair, kWide };
constexpr int kPart = 256;
template <int MODE>
constexpr int kSlots = MODE == kWide ? 2 : kScaleSlots;
template <int MODE>
constexpr int kSlotCols = (kTmemCols - kScaleBase) / kSlots<MODE>;
// Epilogue warps: four, or eight that share the columns of a wide tile, whose drain the next tile's MMAs wait for.
template <int MODE>
constexpr int kDrain = MODE == kWide ? 8 : 4;
template <int MODE>
constexpr int kThreads = (6 + kDrain<MODE>) * 32;

// A CTA of a wide tile holds half of the columns in one piece, 32 h of them, and an MMA takes equal shares of both CTAs':
// where the j-th 32 columns of the accumulator are in the tile.
__device__ __forceinline__ int wide_chunk(int j, int h) { return j < 4 ? j : j < 8 ? h + j - 4 : j < 4 + h ? j - 4 : j; }

struct Barriers {
    uint64_t full[kMaxStages];      // the copies of a stage have landed (pair: the even CTA's counts both CTAs')
    uint64_t empty[kMaxStages];     // the MMAs that read it are done
    uint64_t sfull[kScaleSlots];    // the scale warps (pair: of both CTAs, on the even one) have written a slot
    uint64_t sempty[kScaleSlots];   // the MMAs that read it are done
    uint64_t tfull[2];              // an accumulator is complete
    uint64_t tempty[2];             // the epilogue warps (pair: of both CTAs, on the even one) have read it
    uint64_t mma_done;
    uint32_t tmem_base;
    int32_t abort;
};
// Staging of the pair's output: blocks of 32 x 32, two per epilogue warp, one of fp32 where there are eight warps.
template <typename T>
constexpr int kOutBlock = 32 * 32 * int(sizeof(T));
template <typename T, int MODE>
constexpr int kBlocks = MODE == kWide && sizeof(T) == 4 ? 1 : 2;   // a warp's blocks
template <typename T, int MODE>
constexpr int kStaging = MODE == kAlone ? 0 : kDrain<MODE> * kBlocks<T, MODE> * kOutBlock<T>;
constexpr int kSmemBytes = 227 * 1024;
template <typename T, int MODE>
constexpr int kRingBytes = (kSmemBytes - 1024 - kStaging<T, MODE> - int(sizeof(Barriers))) / 1024 * 1024;

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
    int cols;              // columns of a tile (rows of Q): a multiple of 32 (pair) or 16
    int p_tiles, q_tiles;
    uint32_t idesc, idesc2;   // idesc2: of a wide tile's second part
    void* out;
    int64_t ldo;
    bool f32;              // the output's type, where a launch has both
};

// One launch: one problem, or two whose tiles share the pairs.
template <int N>
struct Launch {
    CUtensorMap p[N], q[N], o[N];
    Problem pr[N];
    int stages, stage_bytes;
    int acc_cols;          // of an accumulator
    int more_first, most_else, extra;   // N == 2: tiles of the second problem, see Tiles
    int32_t* flags;
};

// tcgen05.mma kind::mxf8f6f4 instruction descriptor: scale type E8M0 (bit 23), formats of A (bits 7-9) and B (10-12),
// both K-major, N / 8 at bit 17, M / 128 at bit 27; the scale ids (A's at bit 29, B's at 4) are added per slab.
constexpr uint32_t kIdescBase = 1u << 23;

template <bool PAIR>
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sa,
                                           uint32_t sb, uint32_t accumulate) {
    if (PAIR)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
            "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate));
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
            "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate));
}

// What a CTA works on.  Pairs take tiles in turn, all slabs of each; of two problems the first one's, and then consecutive tiles of
// the second, as many as even out what the first left unequal (share_out): `more_first` for a pair that has one tile more of
// the first, `most_else` or one more for the others.  Alone, a cluster of CTAs splits one tile's slabs.
template <int MODE, int N>
struct Tiles {
    int tile, step, count;
    int second, end;       // N == 2: the second problem's tiles
    int which = 0;
    int lo = 0, hi;        // slabs
    __device__ Tiles(const Launch<N>& L, uint32_t rank) {
        count = L.pr[0].p_tiles * L.pr[0].q_tiles;
        hi = L.pr[0].slabs;
        second = end = 0;
        if (MODE != kAlone) {
            tile = int(blockIdx.x >> 1);
            step = int(gridDim.x >> 1);
            if (N == 2) {
                const int full = count % step, i = tile - full;   // pairs below `full` have a tile more of the first problem
                second = i < 0 ? tile * L.more_first : full * L.more_first + i * L.most_else + min(i, L.extra);
                end = second + (i < 0 ? L.more_first : L.most_else + (i < L.extra ? 1 : 0));
            }
        } else {
            const int parts = int(cluster_size());
            tile = int(blockIdx.x) / parts;
            step = int(gridDim.x) / parts;
            // whole groups of slabs, so that a word of scales is one CTA's
            const int groups = (hi + kGroup - 1) / kGroup, per = (groups + parts - 1) / parts * kGroup, slabs = hi;
            lo = min(slabs, int(rank) * per);
            hi = min(slabs, lo + per);
        }
        turn(L);
    }
    __device__ __forceinline__ void turn(const Launch<N>& L) {
        if (N == 2 && which == 0 && tile >= count) {
            which = 1;
            tile = second;
            count = end;
            hi = L.pr[N - 1].slabs;
        }
    }
    __device__ __forceinline__ bool more() const { return tile < count; }
    __device__ __forceinline__ void next(const Launch<N>& L) {
        tile += which ? 1 : step;
        turn(L);
    }
    __device__ __forceinline__ const Problem& problem(const Launch<N>& L) const { return L.pr[N == 2 ? which : 0]; }
};

// Tiles in bands of kBand row tiles, all column tiles of a band in turn, so that the tiles in flight share operands in L2.
constexpr int kBand = 16;
__device__ __forceinline__ void tile_at(int t, const Problem& pr, int& tp, int& tq) {
    const int per_band = kBand * pr.q_tiles;
    const int band = t / per_band, r = t - band * per_band;
    const int h = min(kBand, pr.p_tiles - band * kBand);
    tp = band * kBand + r % h;
    tq = r / h;
}

// The producer's and the MMA warp's loops run in the whole warp, and one lane is elected for each batch of copies or MMAs:
// stage, descriptors and coordinates are then the same for the warp and live in the uniform registers that those
// instructions take.  Run by one lane of a diverged warp, the MMA loop took 900 cycles a slab, twice the MMAs' time.
template <int MODE, int N>
__device__ void produce(const Launch<N>& L, uint8_t* ring, Barriers* bars, uint32_t rank) {
    constexpr bool PAIR = MODE != kAlone;
    volatile int32_t* abort = &bars->abort;
    int stage = 0;
    uint32_t phase = 0;
    long issued = 0;
    for (Tiles<MODE, N> w(L, rank); w.more(); w.next(L)) {
        const Problem& pr = w.problem(L);
        const CUtensorMap *tmP = &L.p[N == 2 ? w.which : 0], *tmQ = &L.q[N == 2 ? w.which : 0];
        const int q_rows = PAIR ? pr.cols / 2 : pr.cols, bytes = (kRows + q_rows) * kSlab;
        int tp, tq;
        tile_at(w.tile, pr, tp, tq);
        const int p0 = PAIR ? (2 * tp + int(rank)) * kRows : tp * kRows;
        const int q0 = tq * pr.cols + (PAIR ? int(rank) * q_rows : 0);
        for (int kb = w.lo; kb < w.hi; ++kb) {
            if (!warp_wait(&bars->empty[stage], phase ^ 1u, abort)) {
                give_up(abort, L.flags);
                // the copies that were started land before the CTA can exit: the even CTA's barriers count both CTAs',
                // the odd one gives its own time to land
                if (!PAIR || rank == 0) {
                    for (long j = issued - 1; j >= 0 && j >= issued - L.stages; --j)
                        wait_phase(&bars->full[j % L.stages], uint32_t((j / L.stages) & 1), nullptr);
                } else {
                    const uint64_t t0 = global_ns();
                    while (global_ns() - t0 < 100000ull) {
                    }
                }
                return;
            }
            uint8_t* s = ring + stage * L.stage_bytes;
            const uint32_t bar = PAIR ? peer_addr(&bars->full[stage], 0) : smem_u32(&bars->full[stage]);
            if (elect_one()) {
                if (!PAIR || rank == 0) mbar_expect_tx(&bars->full[stage], (PAIR ? 2 : 1) * bytes);
                tma_load<PAIR>(s, tmP, bar, kb * kSlab, p0);
                tma_load<PAIR>(s + kRows * kSlab, tmQ, bar, kb * kSlab, q0);
            }
            ++issued;
            if (++stage == L.stages) {
                stage = 0;
                phase ^= 1u;
            }
        }
    }
}

template <int MODE, int N>
__device__ void issue_mmas(const Launch<N>& L, uint8_t* ring, Barriers* bars, uint32_t tmem, uint32_t rank) {
    constexpr bool PAIR = MODE != kAlone;
    volatile int32_t* abort = &bars->abort;
    const uint32_t units = uint32_t(L.stage_bytes) >> 4;   // of a stage, in descriptors
    const uint64_t pdesc0 = smem_desc(smem_u32(ring)), qdesc0 = smem_desc(smem_u32(ring + kRows * kSlab));
    int stage = 0, slot = 0, acc = 0;
    uint32_t phase = 0, sphase = 0, aphase = 0;
    bool ok = true;
    for (Tiles<MODE, N> w(L, rank); w.more() && ok; w.next(L)) {
        const Problem& pr = w.problem(L);
        if (!warp_wait(&bars->tempty[acc], aphase ^ 1u, abort)) {
            give_up(abort, L.flags);
            break;
        }
        tc_fence_after();
        const uint32_t d = tmem + uint32_t(acc * L.acc_cols);
        for (int kb = w.lo; kb < w.hi && ok; kb += kGroup) {
            ok = warp_wait(&bars->sfull[slot], sphase, abort);
            const uint32_t sc = tmem + kScaleBase + uint32_t(slot) * kSlotCols<MODE>;
#pragma unroll
            for (int i = 0; i < kGroup; ++i) {     // the slab's scales are byte i of the group's words
                if (kb + i >= w.hi || !ok) break;
                ok = warp_wait(&bars->full[stage], phase, abort);
                if (!ok) break;
                tc_fence_after();
                const uint64_t pd = pdesc0 + stage * units, qd = qdesc0 + stage * units;
                const uint32_t more = kb + i > w.lo, id = uint32_t(i) << 29 | uint32_t(i) << 4;
                auto mmas = [&](uint32_t to, uint64_t q, uint32_t idesc, uint32_t sq) {
#pragma unroll
                    for (int k = 0; k < kSlab / 32; ++k)   // 32 columns = 32 bytes = 2 descriptor units
                        mma_scaled<PAIR>(to, pd + uint64_t(2 * k), q + uint64_t(2 * k), idesc | id, sc, sq, k > 0 ? 1u : more);
                };
                if constexpr (MODE == kWide) {
                    if (elect_one()) {
                        mmas(d, qd, pr.idesc, sc + 8);
                        if (kb + i + 1 == w.hi) commit<true>(&bars->tfull[0]);
                    }
                    if (more == 0) {
                        ok = warp_wait(&bars->tempty[1], aphase ^ 1u, abort);
                        if (!ok) break;
                        tc_fence_after();
                    }
                    if (elect_one()) {
                        mmas(d + kPart, qd + (kPart / 2 * kSlab >> 4), pr.idesc2, sc + 16);
                        commit<true>(&bars->empty[stage]);
                    }
                } else if (elect_one()) {
                    mmas(d, qd, pr.idesc, sc + 8);
                    commit<PAIR>(&bars->empty[stage]);
                }
                if (++stage == L.stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            if (!ok) break;
            if (elect_one()) commit<PAIR>(&bars->sempty[slot]);
            if (++slot == kSlots<MODE>) {
                slot = 0;
                sphase ^= 1u;
            }
        }
        if (!ok) {
            give_up(abort, L.flags);
            break;
        }
        if (elect_one()) commit<PAIR>(&bars->tfull[MODE == kWide ? 1 : acc]);
        if (MODE == kWide) {
            aphase ^= 1u;
        } else if (++acc == 2) {
            acc = 0;
            aphase ^= 1u;
        }
    }
    // every MMA has finished before the CTA moves on
    if (elect_one()) {
        if (PAIR)
            asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                             peer_addr(&bars->mma_done, 0))
                         : "memory");
        else
            commit<false>(&bars->mma_done);
    }
    wait_phase(&bars->mma_done, 0, nullptr);
    __syncwarp();
}

// The scales of slabs kb .. kb+3 of N rows 32 apart, one a byte.  Rows and slabs beyond the matrix take the last one's: what
// they scale is zeros, or is not stored.  There is no test around a load, so that all of them are in flight together (a
// test for each, and they came one after the other: 4,096 x 16,384 x 16,384 in 952 us, the tensor cores half idle).
// `h`: the order of a wide tile, from its word `j0`; 0 for the matrix's.
template <int N>
__device__ __forceinline__ void scale_words(const Operand& o, int row, int kb, int slabs, int h, int j0, uint32_t* v) {
    const uint8_t* p[N];
#pragma unroll
    for (int c = 0; c < N; ++c)
        p[c] = o.scale + int64_t(min(row + 32 * (h > 0 ? wide_chunk(j0 + c, h) : c), o.rows - 1) >> o.shift) * o.lds;
    if (o.words && kb + kGroup <= slabs) {
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] = __ldg(reinterpret_cast<const uint32_t*>(p[c] + kb));
        return;
    }
    uint32_t b[N][kGroup];
#pragma unroll
    for (int i = 0; i < kGroup; ++i) {
        const int at = min(kb + i, slabs - 1);
#pragma unroll
        for (int c = 0; c < N; ++c) b[c][i] = __ldg(p[c] + at);
    }
#pragma unroll
    for (int c = 0; c < N; ++c) v[c] = b[c][0] | b[c][1] << 8 | b[c][2] << 16 | b[c][3] << 24;
}

// The groups of slabs of a CTA's tiles, in the order that the MMAs take them.
template <int MODE, int N>
struct Groups {
    static constexpr bool PAIR = MODE != kAlone;
    static constexpr int kQ = MODE == kWide ? 16 : 8, kWords = 4 + kQ;
    const Launch<N>& L;
    Tiles<MODE, N> w;
    const int lane;
    const uint32_t rank;
    int kb, p0, q0;
    __device__ Groups(const Launch<N>& l, uint32_t r) : L(l), w(l, r), lane(threadIdx.x & 31), rank(r) {
        kb = w.lo;
        if (w.lo == w.hi) w.tile = w.count;
        place();
    }
    __device__ void place() {
        if (!w.more()) return;
        const Problem& pr = w.problem(L);
        int tp, tq;
        tile_at(w.tile, pr, tp, tq);
        p0 = (PAIR ? 2 * tp + int(rank) : tp) * kRows + lane;
        q0 = tq * pr.cols + lane;
    }
    // This lane's words of the group at hand, and on to the next.
    __device__ bool take(uint32_t (&v)[kWords]) {
        if (!w.more()) return false;
        const Problem& pr = w.problem(L);
        scale_words<4>(pr.p, p0, kb, pr.slabs, 0, 0, v);
#pragma unroll
        for (int j = 0; j < kQ; j += 8) scale_words<8>(pr.q, q0, kb, pr.slabs, MODE == kWide ? pr.cols / 64 : 0, j, v + 4 + j);
        kb += kGroup;
        if (kb >= w.hi) {
            w.next(L);
            kb = w.lo;
            place();
        }
        return true;
    }
};

// Words are loaded two groups ahead of their use (wide tiles, of longer groups: one).
template <int MODE, int N>
__device__ void write_scales(const Launch<N>& L, Barriers* bars, uint32_t tmem, uint32_t rank) {
    constexpr bool PAIR = MODE != kAlone;
    constexpr int kWords = Groups<MODE, N>::kWords;
    volatile int32_t* abort = &bars->abort;
    const int lane = threadIdx.x & 31;
    const uint32_t lanes = uint32_t((threadIdx.x >> 5) & 3) << 21;   // this warp's quarter, 32 lanes each
    int slot = 0;
    uint32_t phase = 0;
    auto write = [&](const uint32_t (&v)[kWords]) {
        const bool free = wait_phase(&bars->sempty[slot], phase ^ 1u, abort);
        if (!__all_sync(0xffffffffu, free)) {
            give_up(abort, L.flags);
            return false;
        }
        tc_fence_after();
        const uint32_t at = tmem + lanes + kScaleBase + uint32_t(slot) * kSlotCols<MODE>;
        asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                     "r"(v[3])
                     : "memory");
#pragma unroll
        for (int c = 4; c < kWords; c += 8)
            asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at + 4 + c),
                         "r"(v[c]), "r"(v[c + 1]), "r"(v[c + 2]), "r"(v[c + 3]), "r"(v[c + 4]), "r"(v[c + 5]), "r"(v[c + 6]),
                         "r"(v[c + 7])
                         : "memory");
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
            if (PAIR)
                remote_arrive(peer_addr(&bars->sfull[slot], 0));
            else
                mbar_arrive(&bars->sfull[slot]);
        }
        if (++slot == kSlots<MODE>) {
            slot = 0;
            phase ^= 1u;
        }
        return true;
    };
    Groups<MODE, N> g(L, rank);
    uint32_t a[kWords], b[kWords];
    bool na = g.take(a), nb = g.take(b);
    if constexpr (MODE == kWide) {
        while (na) {
            if (!write(a)) return;
            na = g.take(a);
            if (!nb || !write(b)) return;
            nb = g.take(b);
        }
    } else {
        uint32_t c[kWords];
        bool nc = g.take(c);
        while (na) {
            if (!write(a)) return;
            na = g.take(a);
            if (!nb || !write(b)) return;
            nb = g.take(b);
            if (!nc || !write(c)) return;
            nc = g.take(c);
        }
    }
}

__device__ __forceinline__ void store_one(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_one(acrl_bf16* p, float v) { *p = acrl_bf16(pack_bf16x2(v, 0.f) & 0xffffu); }

// Accumulators of a pair's tile: each warp its 32 rows, 32 columns at a time, rounded, staged in shared memory and
// stored by a TMA copy, which leaves out what is beyond the matrix.
// T: the outputs' type, of two problems the larger (Problem::f32 says which each has).
template <typename T, int MODE, int N>
__device__ void pair_epilogue(const Launch<N>& L, Barriers* bars, uint32_t tmem, uint8_t* staging, uint32_t rank) {
    volatile int32_t* abort = &bars->abort;
    const int lane = threadIdx.x & 31, quarter = (threadIdx.x >> 5) & 3;
    constexpr int kBuf = kBlocks<T, MODE>, kStep = 32 * (kDrain<MODE> / 4);   // the warps of a quarter take chunks in turn
    const int first = 32 * (((threadIdx.x >> 5) - 6) >> 2);
    uint8_t* blocks = staging + ((threadIdx.x >> 5) - 6) * kBuf * kOutBlock<T>;
    int buf = 0, acc = 0;
    uint32_t phase = 0;
    // 32 columns of this warp's rows to `out`, rounded to U
    auto store = [&](auto type, const Problem& pr, const CUtensorMap* tmO, const uint32_t (&r)[32], int row0, int col0) {
        using U = decltype(type);
        if (row0 >= pr.p.rows || col0 >= pr.q.rows) return;   // the same for the whole warp
        if (col0 + 32 > pr.q.rows && (pr.q.rows * int(sizeof(U)) & 15) != 0) {
            // a TMA store leaves columns out in 16-byte pieces: here the last ones would write beyond the matrix
            U* out = static_cast<U*>(pr.out) + int64_t(row0 + lane) * pr.ldo + col0;
            if (row0 + lane < pr.p.rows)
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (col0 + j < pr.q.rows) store_one(out + j, __uint_as_float(r[j]));
            return;
        }
        if (lane == 0) bulk_wait_read<kBuf - 1>();              // the store that last read this block is done
        __syncwarp();
        // row `lane` of a block, its 16-byte pieces permuted by the swizzle of the output's map: 64-byte rows in fours
        // (bf16), 128-byte rows in eights (fp32)
        constexpr int kPieces = 32 * int(sizeof(U)) / 16;
        const uint32_t swz = kPieces == 4 ? uint32_t((lane >> 1) & 3) : uint32_t(lane & 7);
        uint8_t* block = blocks + buf * kOutBlock<T>;
        const uint32_t to = smem_u32(block) + uint32_t(lane * 32 * int(sizeof(U)));
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            uint4 v;
            if constexpr (sizeof(U) == 2)
                v = make_uint4(pack_bf16x2(__uint_as_float(r[8 * k]), __uint_as_float(r[8 * k + 1])),
                               pack_bf16x2(__uint_as_float(r[8 * k + 2]), __uint_as_float(r[8 * k + 3])),
                               pack_bf16x2(__uint_as_float(r[8 * k + 4]), __uint_as_float(r[8 * k + 5])),
                               pack_bf16x2(__uint_as_float(r[8 * k + 6]), __uint_as_float(r[8 * k + 7])));
            else
                v = make_uint4(r[4 * k], r[4 * k + 1], r[4 * k + 2], r[4 * k + 3]);
            st_shared16(to + ((uint32_t(k) ^ swz) << 4), v);
        }
        fence_async_shared();
        __syncwarp();
        if (lane == 0) tma_store_2d(tmO, block, col0, row0);
        if (kBuf > 1) buf ^= 1;
    };
    for (Tiles<MODE, N> w(L, rank); w.more(); w.next(L)) {
        const Problem& pr = w.problem(L);
        const CUtensorMap* tmO = &L.o[N == 2 ? w.which : 0];
        int tp, tq;
        tile_at(w.tile, pr, tp, tq);
        const int row0 = (2 * tp + int(rank)) * kRows + quarter * 32;
        bool ready = true;
#pragma unroll 1
        for (int part = 0; part < (MODE == kWide ? 2 : 1); ++part) {
            const int a = MODE == kWide ? part : acc;
            const int c0 = part * kPart + first, end = MODE == kWide && part == 0 ? kPart : pr.cols;
            ready = wait_phase(&bars->tfull[a], phase, abort);
            ready = __all_sync(0xffffffffu, ready);
            if (!ready) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = c0; c < end; c += kStep) {
                uint32_t r[32];
                __syncwarp();
                tmem_ld32(tmem + uint32_t((MODE == kWide ? 0 : acc * L.acc_cols) + c) + (uint32_t(quarter * 32) << 16), r);
                if (c + kStep >= end) {   // read out: the even CTA's MMA warp may fill it again
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) remote_arrive(peer_addr(&bars->tempty[a], 0));
                }
                const int col0 = tq * pr.cols + (MODE == kWide ? 32 * wide_chunk(c / 32, pr.cols / 64) : c);
                if (N == 2 && !pr.f32)
                    store(acrl_bf16{}, pr, tmO, r, row0, col0);
                else
                    store(T{}, pr, tmO, r, row0, col0);
            }
            __syncwarp();
        }
        if (!ready) {
            give_up(abort, L.flags);
            break;
        }
        if (MODE == kWide) {
            phase ^= 1u;
        } else if (++acc == 2) {
            acc = 0;
            phase ^= 1u;
        }
    }
    if (lane == 0) bulk_wait_all();   // the blocks stay valid until every store has completed
    __syncwarp();
}

// A CTA alone: row r of P is column r of `out`, a column of the accumulator a row of it, so a warp stores 32 neighbours.
// With a split sum each rank adds up a share of the columns: every rank's accumulators of it wait in its shared memory (`parts`,
// [rank][column of the share][128]; one rank for all took 5 us more for 16 rows of 4,096 x 4,096, 15 more for 64).
template <typename T>
__device__ bool alone_epilogue(const Launch<1>& L, Barriers* bars, uint32_t tmem, float* parts, uint32_t rank, int nct) {
    const Problem& pr = L.pr[0];
    const int lane = threadIdx.x & 31, quarter = (threadIdx.x >> 5) & 3;
    const uint32_t lanes = uint32_t(quarter * 32) << 16;
    int acc = 0;
    uint32_t phase = 0;
    for (Tiles<kAlone, 1> w(L, rank); w.more(); w.next(L)) {
        int tp, tq;
        tile_at(w.tile, pr, tp, tq);
        const bool ready = wait_phase(&bars->tfull[acc], phase, &bars->abort);
        if (!__all_sync(0xffffffffu, ready)) {
            give_up(&bars->abort, L.flags);
            return false;
        }
        tc_fence_after();
        const int row = tp * kRows + quarter * 32 + lane;
        T* out = static_cast<T*>(pr.out) + row;
#pragma unroll 1
        for (int c = 0; c < pr.cols; c += 16) {
            uint32_t r[16];
            __syncwarp();
            asm volatile(
                "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                  "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                : "r"(tmem + uint32_t(acc * L.acc_cols + c) + lanes));
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            if (w.lo == w.hi)   // no slab left for this rank: nothing was accumulated
#pragma unroll
                for (int j = 0; j < 16; ++j) r[j] = 0u;
            const int m0 = tq * pr.cols + c;
            if (nct == 1) {
                if (row < pr.p.rows)
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (m0 + j < pr.q.rows) store_one(out + int64_t(m0 + j) * pr.ldo, __uint_as_float(r[j]));
            } else {
                const int per = pr.cols / nct;      // of the share: a power of two of ranks divides the columns
                const float* to = parts + int(rank) * per * kRows + quarter * 32 + lane;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int owner = (c + j) / per, at = c + j - owner * per;
                    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(peer_addr(to + at * kRows, uint32_t(owner))), "r"(r[j])
                                 : "memory");
                }
            }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->tempty[acc]);
        if (++acc == 2) {
            acc = 0;
            phase ^= 1u;
        }
    }
    return true;
}

// A rank's share of a split sum: the ranks' accumulators in their order.
template <typename T>
__device__ void join(const float* parts, const Problem& pr, uint32_t rank, int nct) {
    const int at = int(threadIdx.x) & (kRows - 1), per = pr.cols / nct;   // four warps, a row of P a thread
    int tp, tq;
    tile_at(int(blockIdx.x) / nct, pr, tp, tq);
    const int row = tp * kRows + at, m0 = tq * pr.cols + int(rank) * per;
    if (row >= pr.p.rows) return;
    T* out = static_cast<T*>(pr.out) + row;
    for (int j = 0; j < per && m0 + j < pr.q.rows; ++j) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < kMaxSplit; ++k)
            if (k < nct) v += parts[(k * per + j) * kRows + at];
        store_one(out + int64_t(m0 + j) * pr.ldo, v);
    }
}

template <typename T, int MODE, int N>
__global__ void __launch_bounds__(kThreads<MODE>, 1) fp8_matmul_kernel(const __grid_constant__ Launch<N> L) {
    constexpr bool PAIR = MODE != kAlone;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* staging = ring + kRingBytes<T, MODE>;
    Barriers* bars = reinterpret_cast<Barriers*>(staging + kStaging<T, MODE>);
    const int warp = threadIdx.x >> 5;
    const uint32_t rank = cluster_rank();
    const int nct = int(cluster_size());
    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            mbar_init(&bars->full[s], 1);
            mbar_init(&bars->empty[s], 1);
        }
        for (int s = 0; s < kScaleSlots; ++s) {
            mbar_init(&bars->sfull[s], PAIR ? 8 : 4);
            mbar_init(&bars->sempty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&bars->tfull[b], 1);
            mbar_init(&bars->tempty[b], (PAIR ? 2 : 1) * kDrain<MODE>);
        }
        mbar_init(&bars->mma_done, 1);
        bars->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&L.p[0])) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&L.q[0])) : "memory");
    }
    grid_begin();
    if (warp == 2) {
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
    if (PAIR || nct > 1) cluster_sync();   // the others' barriers are initialised, and they run
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;
    // the parts of a split sum, behind the stages
    float* parts = reinterpret_cast<float*>(ring + L.stages * L.stage_bytes);
    bool ok = true;
    if (warp == 0) {
        produce<MODE, N>(L, ring, bars, rank);
    } else if (warp == 1) {
        if (!PAIR || rank == 0) issue_mmas<MODE, N>(L, ring, bars, tmem, rank);
    } else if (warp < 6) {
        write_scales<MODE, N>(L, bars, tmem, rank);
    } else if constexpr (PAIR) {
        pair_epilogue<T, MODE, N>(L, bars, tmem, staging, rank);
    } else {
        ok = alone_epilogue<T>(L, bars, tmem, parts, rank, nct);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (PAIR || nct > 1) cluster_sync();   // no CTA frees its TMEM or leaves while another may still touch it
    if constexpr (!PAIR) {
        if (nct > 1 && warp >= 6 && ok) join<T>(parts, L.pr[0], rank, nct);
    }
    if (warp == 2) {
        tc_fence_after();
        if (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

Operand operand(const Matrix& m) {
    return Operand{m.scale, m.lds, int(m.rows), m.block == ACRL_FP8_TILE ? 7 : 0,
                   (m.lds & 3) == 0 && (reinterpret_cast<uintptr_t>(m.scale) & 3) == 0};
}

// Rows up to kAloneRows become the MMA's columns, where the weight has tiles for more than half of the SMs; with fewer tiles
// the sum is split, at a price that grows with the rows, and the rows are up to kSplitRows, or kSplitRowsASlab for each slab of
// the sum.  us, alone / as pairs, for 16, 64 and 128 rows:
//     16,384 x 4,096  14.4 / 24.0  15.7 / 20.5  18.0 / 20.9        4,096 x 4,096   7.8 / 18.7  10.1 / 17.1  13.2 / 17.3
//    151,936 x 4,096  99.9 / 121   99.1 / 122    102 / 128         1,024 x 2,048   5.4 / 9.3    7.7 / 9.5   10.7 / 9.7
//      9,800 x 1,024   5.6 / 8.9    7.1 / 8.8    9.2 / 8.4         4,096 x 1,024   6.0 / 7.9    9.0 / 7.7   13.2 / 7.4
constexpr int64_t kAloneRows = 128, kSplitRows = 32, kSplitRowsASlab = 6;

// The tensor maps of a problem: P's rows and Q's, and the output's for a pair's stores.
template <int MODE>
bool maps_of(const Matrix& p, const Matrix& q, int64_t K, const Problem& pr, CUtensorMap* tmP, CUtensorMap* tmQ, CUtensorMap* tmO) {
    auto map = [&](CUtensorMap* m, const Matrix& x, int box_rows) {
        return encode_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, x.q, uint64_t(x.rows), uint64_t(K), uint64_t(x.ld), box_rows,
                          kSlab, CU_TENSOR_MAP_SWIZZLE_128B);
    };
    if (!map(tmP, p, kRows) || !map(tmQ, q, MODE == kAlone ? pr.cols : pr.cols / 2)) return false;
    if (MODE == kAlone) {
        *tmO = *tmP;   // not used
        return true;
    }
    return encode_map(tmO, pr.f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, pr.f32 ? 4 : 2, pr.out,
                      uint64_t(p.rows), uint64_t(q.rows), uint64_t(pr.ldo), 32, 32,
                      pr.f32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}

// Allows the kernel its shared memory; the pairs of CTAs that can be resident at once.
template <typename T, int MODE, int N>
int64_t resident_pairs() {
    auto* kernel = fp8_matmul_kernel<T, MODE, N>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    return MODE == kAlone ? kMaxGrid : resident_clusters(reinterpret_cast<const void*>(kernel), kThreads<MODE>, kSmemBytes, 2);
}

// `grid`: of pairs' launches twice the tiles, of which as many run as can be resident at once: they are persistent.
template <typename T, int MODE, int N>
acrl_status launch_kernel(const Launch<N>& L, int64_t grid, int cluster, cudaStream_t s) {
    const int64_t most = resident_pairs<T, MODE, N>();
    if (most < 1) return ACRL_ERR_CUDA;
    if (MODE != kAlone) grid = std::min<int64_t>(grid, 2 * most);
    return launch(fp8_matmul_kernel<T, MODE, N>, grid, kThreads<MODE>, kSmemBytes, cluster, s, L);
}

template <typename T, int MODE>
acrl_status launch_one(const Matrix& p, const Matrix& q, int64_t K, const Problem& pr, int stage_bytes, int stages, int64_t grid,
                       int cluster, int32_t* flags, cudaStream_t s) {
    Launch<1> L = {};
    L.pr[0] = pr;
    L.stages = std::min(kMaxStages, stages);
    L.stage_bytes = stage_bytes;
    L.acc_cols = pr.cols;
    L.flags = flags;
    if (!maps_of<MODE>(p, q, K, pr, &L.p[0], &L.q[0], &L.o[0])) return ACRL_ERR_CUDA;
    return launch_kernel<T, MODE, 1>(L, grid, cluster, s);
}

// out = A B^T, as a problem of pairs or alone.
Problem problem_of(const Matrix& p, const Matrix& q, int64_t K, void* out, int64_t ldo, bool f32) {
    Problem pr = {};
    pr.p = operand(p);
    pr.q = operand(q);
    pr.slabs = int((K + kSlab - 1) / kSlab);
    pr.out = out;
    pr.ldo = ldo;
    pr.f32 = f32;
    pr.idesc = kIdescBase | uint32_t(p.format) << 7 | uint32_t(q.format) << 10;
    return pr;
}

// Whether A's rows become the MMA's columns.
bool rows_alone(int64_t rows, int64_t cols, int64_t K, int sms) {
    const int64_t slabs = (K + kSlab - 1) / kSlab, tiles = (cols + kRows - 1) / kRows;
    return rows <= (2 * tiles > sms ? kAloneRows : std::min(kAloneRows, std::max(kSplitRows, kSplitRowsASlab * slabs)));
}

// The cost of a pair's tile, in loads of one of a slab's rows (1.5 ns): the loads of a slab, 128 rows of P and half the
// columns a CTA, take longest; a wide tile's MMAs also wait for the drain of the one before, and an fp32 output's stores take
// their share of the way to L2 (8,200 x 2,048 x 2,504 in tiles of 224 columns 9.4 us a tile, 7.5 as bf16).
int64_t tile_cost(const Problem& pr) {
    constexpr int64_t kTileCost = 300, kWideCost = 2000;
    return int64_t(pr.slabs) * (128 + pr.cols / 2) + (pr.cols > kPart ? kWideCost : kTileCost) + (pr.f32 ? 5 * pr.cols : 0);
}

// Sets a pair's tiles to `cols` columns.
void cut(Problem& pr, int cols) {
    pr.cols = cols;
    pr.p_tiles = (pr.p.rows + 2 * kRows - 1) / (2 * kRows);
    pr.q_tiles = (pr.q.rows + cols - 1) / cols;
}
void describe(Problem& pr) {
    pr.idesc2 = pr.idesc | uint32_t((pr.cols - kPart) >> 3) << 17 | 2u << 27;
    pr.idesc |= uint32_t(std::min(pr.cols, kPart) >> 3) << 17 | 2u << 27;
}
int64_t tiles_of(const Problem& pr) { return int64_t(pr.p_tiles) * pr.q_tiles; }

// Columns of a pair's tile: all pairs run whole rounds of tiles, so the least rounds x cost.  224 / 320 / 448
// columns: 4,096 x 4,096 x 4,096 (76 pairs: 4, 3 and 3 rounds) 52 / 56 / 63 us, 2,504 x 2,048 x 8,200 (2, 1 and 1) 61 / 44 / 47,
// 8,192 x 8,192 x 1,024 (16, 11 and 8) 65 / 77 / 69, 4,096 x 151,936 x 4,096 (143, 101 and 72) 1,680 / 1,660 / 1,510.
// Narrow ones where the last round would be short: 1,500 x 6,000 x 1,024 of 192 / 224: 18.1 / 18.7 us.
int64_t cut_best(Problem& pr, int pairs) {
    int64_t least = 0;
    int best = 0;
    for (int cols = 2 * kPairCols; cols >= 96; cols -= cols > kPart ? 64 : 32) {
        cut(pr, cols);
        const int64_t cost = (tiles_of(pr) + pairs - 1) / pairs * tile_cost(pr);
        if (least == 0 || cost < least) {
            least = cost;
            best = cols;
        }
        if (cols == kPart + 64) cols = kPairCols + 32;   // two accumulators of 256 do not fit
    }
    cut(pr, best);
    return least;
}

bool sms_of_device(int& sms) {
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess;
}

template <typename T>
acrl_status launch_matmul(const Matrix& a, const Matrix& b, int64_t K, void* out, int64_t ldo, int32_t* flags,
                          cudaStream_t s) {
    int sms = 0;
    if (!sms_of_device(sms)) return launch_status();
    const bool alone = rows_alone(a.rows, b.rows, K, sms);
    const Matrix &p = alone ? b : a, &q = alone ? a : b;
    Problem pr = problem_of(p, q, K, out, ldo, sizeof(T) == 4);
    if (alone) {
        pr.cols = int((q.rows + 15) / 16 * 16);
        pr.p_tiles = int((p.rows + kRows - 1) / kRows);
        pr.q_tiles = 1;
        pr.idesc |= uint32_t(pr.cols >> 3) << 17 | 1u << 27;
        const int bytes = (kRows + pr.cols) * kSlab;
        // as many CTAs a tile as keep all SMs busy, each with four slabs or more
        int split = 1;
        while (split < kMaxSplit && 2 * split * pr.p_tiles <= sms && (pr.slabs + kGroup - 1) / kGroup >= 2 * split) split *= 2;
        const int parts = split > 1 ? pr.cols * kRows * 4 : 0;
        const int64_t grid = split > 1 ? int64_t(pr.p_tiles) * split : std::min(pr.p_tiles, sms);
        return launch_one<T, kAlone>(p, q, K, pr, bytes, (kRingBytes<T, kAlone> - parts) / bytes, grid, split, flags, s);
    }
    cut_best(pr, sms / 2);
    if (tiles_of(pr) > kMaxGrid / 2) return ACRL_ERR_INVALID_ARG;
    describe(pr);
    const int bytes = (kRows + pr.cols / 2) * kSlab;
    return pr.cols > kPart
               ? launch_one<T, kWide>(p, q, K, pr, bytes, kRingBytes<T, kWide> / bytes, 2 * tiles_of(pr), 2, flags, s)
               : launch_one<T, kPair>(p, q, K, pr, bytes, kRingBytes<T, kPair> / bytes, 2 * tiles_of(pr), 2, flags, s);
}

// Checked operands of one row or more each.
acrl_status product(const Matrix& a, const Matrix& b, int64_t K, void* out, acrl_dtype out_dtype, int64_t ldo, int32_t* flags,
                    cudaStream_t s) {
    if (K == 0) {   // an empty sum
        const size_t size = out_dtype == ACRL_BF16 ? 2 : 4;
        return cudaMemset2DAsync(out, size_t(ldo) * size, 0, size_t(b.rows) * size, size_t(a.rows), s) == cudaSuccess
                   ? ACRL_OK
                   : launch_status();
    }
    const acrl_status few = matmul_few(a, nullptr, b, K, out, out_dtype, flags, s);
    if (few != kFewNot) return few;
    return out_dtype == ACRL_BF16 ? launch_matmul<acrl_bf16>(a, b, K, out, ldo, flags, s)
                                  : launch_matmul<float>(a, b, K, out, ldo, flags, s);
}

acrl_status matmul(const Matrix& a, const Matrix& b, int64_t K, void* out, acrl_dtype out_dtype, int64_t ldo,
                   int32_t* flags, cudaStream_t s) {
    if (K < 0 || K > kMaxGrid - 512 || !matrix_ok(a, K) || !matrix_ok(b, K)) return ACRL_ERR_INVALID_ARG;
    if ((out_dtype != ACRL_BF16 && out_dtype != ACRL_F32) || ldo < b.rows || (ldo & 7)) return ACRL_ERR_INVALID_ARG;
    if (a.rows == 0 || b.rows == 0) return ACRL_OK;
    if (!out || !aligned16(out)) return ACRL_ERR_INVALID_ARG;
    if (K > 0) {
        if (!a.q || !b.q || !a.scale || !b.scale || !aligned16(a.q) || !aligned16(b.q)) return ACRL_ERR_INVALID_ARG;
        if (!few_rows(a.rows, b.rows, K) && !operands_on_current_device({a.q, b.q, out})) return ACRL_ERR_INVALID_ARG;
    }
    return product(a, b, K, out, out_dtype, ldo, flags, s);
}

// Two products at once: their tiles share the pairs, so that a part-filled last round of one is filled by the other, and one
// launch's start and end are saved.  Both gradients with their quantisation, together / apart, us, by rows, K and N: 200 x 1,024 x
// 1,024 14 / 20, 1,024 x 1,024 x 4,096 26 / 37, 1,500 x 1,536 x 6,000 48 / 64, 4,096 x 4,096 x 4,096 135 / 146; narrow tiles only, so
// the largest stay apart (4,096 x 4,096 x 16,384 502 / 473).
struct Product {
    const Matrix &a, &b;
    int64_t K;
    void* out;
    acrl_dtype type;
    int64_t ldo;
};

// How the second problem's n1 tiles of cost c1 are shared out among the pairs when n0 of cost c0 were taken in turn; the time
// of the busiest pair.
int64_t share_out(int64_t n0, int64_t c0, int64_t n1, int64_t c1, int64_t pairs, Launch<2>& L) {
    const int64_t full = n0 % pairs, each = n0 / pairs, others = pairs - full;
    const int64_t even = ((n0 * c0 + n1 * c1) / pairs - (each + 1) * c0) / c1;    // for a pair with one more of the first
    int64_t least = 0;
    for (int64_t m = std::max<int64_t>(0, even); m <= std::max<int64_t>(0, even) + 1; ++m) {
        if (full * m > n1) break;
        const int64_t left = n1 - full * m, some = left / others, extra = left % others;
        const int64_t time = std::max(full > 0 ? (each + 1) * c0 + m * c1 : 0, each * c0 + (some + (extra > 0)) * c1);
        if (least > 0 && time >= least) continue;
        least = time;
        L.more_first = int(m);
        L.most_else = int(some);
        L.extra = int(extra);
    }
    return least > 0 ? least : kMaxGrid * kMaxGrid / 4;
}

acrl_status two_products(const Product& x, const Product& y, int32_t* flags, cudaStream_t s) {
    constexpr int64_t kLaunchCost = 3000;   // of a launch's start and end, 4.5 us
    int sms = 0;
    if (!sms_of_device(sms)) return launch_status();
    auto pairs_work = [&](const Product& p) { return !few_rows(p.a.rows, p.b.rows, p.K) && !rows_alone(p.a.rows, p.b.rows, p.K, sms); };
    if (x.K > 0 && y.K > 0 && pairs_work(x) && pairs_work(y)) {
        const int64_t resident = resident_pairs<float, kPair, 2>();
        Launch<2> L = {};
        const Product* of[2] = {&x, &y};
        Problem pr[2];
        int64_t apart = kLaunchCost, cost[2];
        for (int i = 0; i < 2; ++i) {
            const Product& p = *of[i];
            pr[i] = problem_of(p.a, p.b, p.K, p.out, p.ldo, p.type == ACRL_F32);
            apart += cut_best(pr[i], sms / 2);
            int best = 0;
            for (int cols = kPairCols; cols >= 96; cols -= 32) {   // the least work: there are no rounds to fill
                cut(pr[i], cols);
                const int64_t c = tiles_of(pr[i]) * tile_cost(pr[i]);
                if (best == 0 || c < cost[i]) {
                    cost[i] = c;
                    best = cols;
                }
            }
            cut(pr[i], best);
            cost[i] = tile_cost(pr[i]);
            describe(pr[i]);
        }
        const int first = cost[0] >= cost[1] ? 0 : 1;              // the longer tiles
        const int64_t n0 = tiles_of(pr[first]), n1 = tiles_of(pr[1 - first]), pairs = std::min(resident, n0 + n1);
        if (pairs > 0 && n0 + n1 <= kMaxGrid / 2 && share_out(n0, cost[first], n1, cost[1 - first], pairs, L) < apart) {
            for (int i = 0; i < 2; ++i) {
                const int k = i == 0 ? first : 1 - first;
                L.pr[i] = pr[k];
                L.stage_bytes = std::max(L.stage_bytes, (kRows + pr[k].cols / 2) * kSlab);
                if (!maps_of<kPair>(of[k]->a, of[k]->b, of[k]->K, pr[k], &L.p[i], &L.q[i], &L.o[i])) return ACRL_ERR_CUDA;
            }
            L.stages = std::min(kMaxStages, kRingBytes<float, kPair> / L.stage_bytes);
            L.acc_cols = kPairCols;
            L.flags = flags;
            return launch_kernel<float, kPair, 2>(L, 2 * pairs, 2, s);
        }
    }
    const acrl_status st = product(x.a, x.b, x.K, x.out, x.type, x.ldo, flags, s);
    return st != ACRL_OK ? st : product(y.a, y.b, y.K, y.out, y.type, y.ldo, flags, s);
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

// Rows of quantised activations at a stride of 16 bytes, then their scales at one of four; none where the product's
// kernel quantises a row itself.
extern "C" int64_t acrl_fp8_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N < 0 || K < 0) return -1;
    return few_rows(M, N, K) ? 0 : M * ((K + 15) / 16 * 16 + ((K + 127) / 128 + 3) / 4 * 4);
}

extern "C" acrl_status acrl_fp8_linear(const acrl_bf16* x, int64_t M, int64_t K, int64_t ldx, acrl_fp8_format x_format,
                                       const uint8_t* w, int64_t N, int64_t ldw, acrl_fp8_format w_format,
                                       const uint8_t* w_scale, int64_t ldws, acrl_fp8_block w_block, void* out,
                                       acrl_dtype out_dtype, int64_t ldo, void* workspace, int64_t workspace_bytes,
                                       int32_t* dev_flags, acrl_stream stream) {
    if (M < 0 || N < 0 || K < 0 || workspace_bytes < acrl_fp8_linear_workspace_bytes(M, N, K)) return ACRL_ERR_INVALID_ARG;
    const int64_t ldq = (K + 15) / 16 * 16, lds = ((K + 127) / 128 + 3) / 4 * 4;
    if (workspace_bytes < 0 || (M > 0 && N > 0 && K > 0 && !few_rows(M, N, K) && (!workspace || !aligned16(workspace)))) return ACRL_ERR_INVALID_ARG;
    uint8_t* q = static_cast<uint8_t*>(workspace);
    const Matrix a{q, M, ldq, x_format, q + M * ldq, lds, ACRL_FP8_ROW};
    const Matrix b{w, N, ldw, w_format, w_scale, ldws, w_block};
    // the product's arguments are checked before anything is launched
    if (!matrix_ok(a, K) || !matrix_ok(b, K) || (out_dtype != ACRL_BF16 && out_dtype != ACRL_F32) || ldo < N || (ldo & 7) ||
        ldx < K || (ldx & 7))
        return ACRL_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return ACRL_OK;
    if (!out || !aligned16(out) || (K > 0 && (!x || !w || !w_scale || !aligned16(x) || !aligned16(w)))) return ACRL_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (K > 0) {
        const acrl_status few = matmul_few(a, x, b, K, out, out_dtype, dev_flags, s);
        if (few != kFewNot) return few;
        if (!operands_on_current_device({w, q, out})) return ACRL_ERR_INVALID_ARG;
    }
    const acrl_status st = acrl_fp8_quantize(x, ACRL_BF16, M, K, ldx, x_format, ACRL_FP8_ROW, 0, q, ldq, q + M * ldq, lds,
                                             dev_flags, stream);
    if (st != ACRL_OK) return st;
    return product(a, b, K, out, out_dtype, ldo, dev_flags, s);
}

namespace acrl {
namespace {

// The backward's workspace: dy by rows, dy's transpose, x's transpose, each its elements and then its scales.
struct Part {
    int64_t rows, ldq, lds, at;   // at: of the elements; the scales follow
    int64_t end() const { return (at + rows * (ldq + lds) + 15) / 16 * 16; }
};

struct BackwardParts {
    Part dy, dyt, xt;
    BackwardParts(int64_t M, int64_t N, int64_t K) {
        auto part = [](int64_t rows, int64_t cols, int64_t at) {
            return Part{rows, (cols + 15) / 16 * 16, ((cols + 127) / 128 + 3) / 4 * 4, at};
        };
        dy = part(M, N, 0);
        dyt = part(N, M, dy.end());
        xt = part(K, M, dyt.end());
    }
};

Matrix matrix_of(uint8_t* base, const Part& p, acrl_fp8_format format) {
    return Matrix{base + p.at, p.rows, p.ldq, format, base + p.at + p.rows * p.ldq, p.lds, ACRL_FP8_ROW};
}

}  // namespace
}  // namespace acrl

extern "C" int64_t acrl_fp8_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    return M < 0 || N < 0 || K < 0 ? -1 : BackwardParts(M, N, K).xt.end();
}

extern "C" acrl_status acrl_fp8_linear_backward(const acrl_bf16* dy, int64_t M, int64_t N, int64_t lddy,
                                                acrl_fp8_format dy_format, const acrl_bf16* x, int64_t K, int64_t ldx,
                                                acrl_fp8_format x_format, const uint8_t* wt, int64_t ldwt,
                                                acrl_fp8_format w_format, const uint8_t* wt_scale, int64_t ldwts,
                                                acrl_fp8_block w_block, void* dx, acrl_dtype dx_dtype, int64_t lddx, void* dw,
                                                acrl_dtype dw_dtype, int64_t lddw, void* workspace, int64_t workspace_bytes,
                                                int32_t* dev_flags, acrl_stream stream) {
    if (M < 0 || N < 0 || K < 0 || M > kMaxGrid / 2 || N > kMaxGrid / 2 || K > kMaxGrid / 2) return ACRL_ERR_INVALID_ARG;
    const BackwardParts parts(M, N, K);
    const Matrix w{wt, K, ldwt, w_format, wt_scale, ldwts, w_block};
    auto format_ok = [](acrl_fp8_format f) { return f == ACRL_FP8_E4M3 || f == ACRL_FP8_E5M2; };
    auto dtype_ok = [](acrl_dtype d) { return d == ACRL_BF16 || d == ACRL_F32; };
    if (!format_ok(dy_format) || !format_ok(x_format) || !matrix_ok(w, N) || !dtype_ok(dx_dtype) || !dtype_ok(dw_dtype))
        return ACRL_ERR_INVALID_ARG;
    if (lddy < N || (lddy & 7) || ldx < K || (ldx & 7) || lddx < K || (lddx & 7) || lddw < K || (lddw & 7)) return ACRL_ERR_INVALID_ARG;
    if (workspace_bytes < parts.xt.end()) return ACRL_ERR_INVALID_ARG;
    if (K == 0 || (M == 0 && N == 0)) return ACRL_OK;
    if ((M > 0 && (!dx || !aligned16(dx) || !x || !aligned16(x))) || (N > 0 && (!dw || !aligned16(dw) || !wt || !wt_scale || !aligned16(wt))))
        return ACRL_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    uint8_t* base = static_cast<uint8_t*>(workspace);
    const Matrix a = matrix_of(base, parts.dy, dy_format), at = matrix_of(base, parts.dyt, dy_format),
                 xt = matrix_of(base, parts.xt, x_format);
    if (M == 0) return product(at, xt, 0, dw, dw_dtype, lddw, dev_flags, s);     // empty sums
    if (N == 0) return product(a, w, 0, dx, dx_dtype, lddx, dev_flags, s);
    if (!dy || !aligned16(dy) || !workspace || !aligned16(workspace) || !operands_on_current_device({wt, base, dx, dw}))
        return ACRL_ERR_INVALID_ARG;
    auto into = [&](const Part& p, const Matrix& m) { return Quantised{base + p.at, p.ldq, const_cast<uint8_t*>(m.scale), p.lds}; };
    acrl_status st = quantize_backward(dy, M, N, lddy, dy_format, into(parts.dy, a), into(parts.dyt, at), x, K, ldx, x_format,
                                       into(parts.xt, xt), dev_flags, s);
    if (st == ACRL_OK) st = two_products({a, w, N, dx, dx_dtype, lddx}, {at, xt, M, dw, dw_dtype, lddw}, dev_flags, s);
    return st;
}
