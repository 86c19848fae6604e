// acrl_orthogonalize: Newton-Schulz steps on an update.  With X (m x n, m <= n; a tall matrix's transpose) a step is
//
//     A = X X^T,   Q = a I + b A + c A A,   X <- Q X,
//
// so that the polynomial in the Gram matrix is made on its m x m elements, and X is read twice and written once.  A and Q are
// symmetric: tiles above the diagonal are left out and written as mirror images, 3 m^2 n + m^3 multiply-adds a step where the
// plain products have 4 m^2 n + 2 m^3.
//
// All steps are one cooperative launch: CTA pairs, one CTA an SM, go through the tiles of all products of all steps, in one
// order, every pairs-th.  A tile of a product waits until its matrix's product before is written: a counter for each matrix says
// how far it is (each wait is bounded in time).  So the matrices of a batch run into one another, and neither a part-filled round
// nor the last tiles' stores hold up the next product: 24 x 1,024 x 1,024, launched product by product, 1,290 us; with a barrier of
// the grid between them 1,274; as it is 1,150-1,220, by the GPU.
//
// Operands are two bf16 numbers each, x = x0 + x1 with x0 the rounding of x and x1 that of what is left, which together are
// within 2^-16 of it, and a product is three of the tensor cores' (bf16_product.cuh).  One bf16 number would not do: gradients
// have a few strong directions and many weak ones, whose singular values the steps amplify by up to a^steps (485 for five
// steps of the usual quintic), and with them whatever the rounding of the strong ones has put in their place.
#include <algorithm>

#include "acrl_device.cuh"
#include "acrl_host.h"
#include "activation.cuh"
#include "bf16_product.cuh"

namespace acrl {
namespace {

constexpr int kMostSteps = 64;
constexpr int kSumCtas = 608;      // four of an SM's: CTAs that add up squares

struct Update {
    const void* g;
    bool f32, wide;        // wide: every eighth of a row's numbers starts on 16 bytes
    int64_t ld, stride;
    int m, n;              // as given
};

// ---------------------------------------------------------------------------------------------------------------
// the first iterate
// ---------------------------------------------------------------------------------------------------------------

// A sum of squares of numbers of any size, in three sums whose terms stay within fp32: of numbers from 2^50 on scaled by
// 2^-80, of those below 2^-50 by 2^80, and of the others.
struct Squares {
    float low = 0.f, mid = 0.f, high = 0.f;
    __device__ __forceinline__ void add(float x) {
        const float a = fabsf(x);
        if (a > 0x1p50f) {
            x *= 0x1p-80f;
            high = fmaf(x, x, high);
        } else if (a < 0x1p-50f) {
            x *= 0x1p80f;
            low = fmaf(x, x, low);
        } else {
            mid = fmaf(x, x, mid);   // a NaN as well
        }
    }
    __device__ __forceinline__ double total() const { return double(low) * 0x1p-160 + double(mid) + double(high) * 0x1p160; }
};

// A matrix's rows are gone through in pieces of kPiece columns, a warp a piece; `ctas` CTAs a matrix take them in turn.
constexpr int kPiece = 1024, kVec = 8, kTurns = kPiece / (32 * kVec);

struct Pieces {
    int per_row, all, at, step;
    __device__ Pieces(const Update& u, int cta, int ctas) {
        per_row = (u.n + kPiece - 1) / kPiece;
        all = u.m * per_row;
        at = cta * 8 + int(threadIdx.x >> 5);
        step = ctas * 8;
    }
};

// Eight of a row's numbers from column c on, zeros beyond its end.
__device__ __forceinline__ void load8(const Update& u, int64_t row, int c, float (&v)[8]) {
    if (c + 8 > u.n || !u.wide) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < u.n ? load_float(u.g, u.f32, row + c + j) : 0.f;
    } else if (u.f32) {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(u.g) + row + c);
        const float4 a = p[0], b = p[1];
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
        const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const acrl_bf16*>(u.g) + row + c);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bf16_lo(w[j]);
            v[2 * j + 1] = bf16_hi(w[j]);
        }
    }
}

// Partial sums of a matrix's squares, `ctas` of them.  HBM bounds it.  It also clears the matrix's counter.
__global__ void __launch_bounds__(256) squares_kernel(Update u, int ctas, double* sums, unsigned* done) {
    __shared__ double part[8];
    grid_begin();
    const int b = int(blockIdx.x) / ctas, lane = threadIdx.x & 31;
    if (int(blockIdx.x) == b * ctas && threadIdx.x == 0) done[b] = 0;
    Squares s;
    Pieces p(u, int(blockIdx.x) - b * ctas, ctas);
    for (; p.at < p.all; p.at += p.step) {
        const int r = p.at / p.per_row, c = (p.at - r * p.per_row) * kPiece + lane * kVec;
        const int64_t row = b * u.stride + r * u.ld;
        float v[kTurns][8];
#pragma unroll
        for (int i = 0; i < kTurns; ++i) load8(u, row, min(c + i * 32 * kVec, u.n), v[i]);
#pragma unroll
        for (int i = 0; i < kTurns; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s.add(v[i][j]);
    }
    const double sum = warp_sum(s.total());
    if (lane == 0) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int i = 0; i < 8; ++i) t += part[i];
        sums[blockIdx.x] = t;
    }
}

// Two bf16 numbers for each of eight, from a column that is a multiple of eight.
__device__ __forceinline__ void halves8(const float (&v)[8], acrl_bf16* hi, acrl_bf16* lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        h[j] = pack_bf16x2(v[2 * j], v[2 * j + 1]);
        l[j] = pack_bf16x2(v[2 * j] - bf16_lo(h[j]), v[2 * j + 1] - bf16_hi(h[j]));
    }
    *reinterpret_cast<uint4*>(hi) = make_uint4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<uint4*>(lo) = make_uint4(l[0], l[1], l[2], l[3]);
}

// X_0 = G / (|G| + eps) in two bf16 matrices, turned where G is tall, in blocks of 64 x 64 through shared memory.  The factor is
// a power of two times a number in [1, 2): an update of any size is brought near 1 before it is divided.  `ctas` CTAs a matrix
// (each adds up the squares for itself; a CTA for each block of 32 x 32 took 95 us for 24 x 1,024 x 1,024, these 24).
__global__ void __launch_bounds__(256) first_kernel(Update u, int ctas, const double* sums, float eps, acrl_bf16* hi, acrl_bf16* lo,
                                                    int64_t ldx, int64_t size, int32_t* flags) {
    __shared__ float block[64][65];
    __shared__ float by[3];
    grid_begin();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = int(blockIdx.x) / ctas, cta = int(blockIdx.x) - b * ctas;
    if (warp == 0) {
        double sum = 0.0;
        for (int i = lane; i < ctas; i += 32) sum += sums[int64_t(b) * ctas + i];
        sum = warp_sum(sum);
        if (lane == 0) {
            const bool bad = !(sum <= 1.7e308);   // an infinity or a NaN: no finite matrix comes near
            if (bad && cta == 0) raise_flag(flags, ACRL_FLAG_NONFINITE);
            int e = 0;
            const double f = frexp(sqrt(sum) + double(eps), &e);   // f 2^e
            by[0] = exp2f(float(-e / 2));
            by[1] = exp2f(float(-e - -e / 2));
            by[2] = bad ? __int_as_float(0x7fc00000) : f > 0.0 ? float(1.0 / f) : 0.f;
        }
    }
    __syncthreads();
    const float one = by[0], two = by[1], rest = by[2];
    acrl_bf16 *h = hi + b * size, *l = lo + b * size;
    if (u.m <= u.n) {
        Pieces p(u, cta, ctas);
        for (; p.at < p.all; p.at += p.step) {
            const int r = p.at / p.per_row, c = (p.at - r * p.per_row) * kPiece + lane * kVec;
            float v[kTurns][8];
#pragma unroll
            for (int i = 0; i < kTurns; ++i) load8(u, b * u.stride + r * u.ld, min(c + i * 32 * kVec, u.n), v[i]);
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                const int at = c + i * 32 * kVec;
                if (at >= u.n) break;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = v[i][j] * one * two * rest;
                halves8(v[i], h + r * ldx + at, l + r * ldx + at);   // the last ones' zeros are within ldx
            }
        }
        return;
    }
    const int cols = (u.n + 63) / 64, blocks = (u.m + 63) / 64 * cols, k = int(threadIdx.x & 7) * 8, row = int(threadIdx.x >> 3);
    for (int at = cta; at < blocks; at += ctas) {
        const int r0 = at / cols * 64, c0 = at % cols * 64;
#pragma unroll
        for (int i = 0; i < 64; i += 32) {
            float v[8] = {};
            const int r = r0 + row + i;
            if (r < u.m && c0 + k < u.n) load8(u, b * u.stride + r * u.ld, c0 + k, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) block[row + i][k + j] = v[j] * one * two * rest;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 64; i += 32) {
            const int r = c0 + row + i, c = r0 + k;   // of X
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = block[k + j][row + i];
            if (r < u.n && c < u.m) halves8(v, h + r * ldx + c, l + r * ldx + c);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------------
// the steps' products
// ---------------------------------------------------------------------------------------------------------------

// What is made of the sums: A itself; Q = a I + b A + c sum; X; and the last X as the result.
enum Kind { kGram, kPolynomial, kIterate, kResult };

struct Finish {
    int kind;
    float a, b, c, scale;
    const acrl_bf16 *hi_in, *lo_in;    // A, for the polynomial
    acrl_bf16 *hi, *lo;                // A, Q or X
    int64_t ld, size;                  // of all of these, and from one matrix to the next
    acrl_bf16* out;                    // the result
    int64_t ldo, out_stride;
    bool tall, wide;                   // the result is turned back; every eighth of its numbers starts on 16 bytes
};

// a I + b A + c v at row i, columns j .. j + 31; what is beyond the matrix is left out of the result.  A row's 64 bytes of each
// half come in 16-byte loads, all of them in flight together: no test is around a load, and those beyond the matrix are of its
// first row or column (one after the other they took 1.1 us of a tile's 2.6).
__device__ __forceinline__ void polynomial(const Finish& f, int z, int i, int j, int m, float (&v)[32]) {
    if (m == 0) return;
    const int64_t row = z * f.size + min(i, m - 1) * f.ld;
    uint4 h[4], l[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t at = row + (j + 8 * k < f.ld ? j + 8 * k : 0);   // ld is a multiple of eight
        h[k] = __ldcg(reinterpret_cast<const uint4*>(f.hi_in + at));
        l[k] = __ldcg(reinterpret_cast<const uint4*>(f.lo_in + at));
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t hw[4] = {h[k].x, h[k].y, h[k].z, h[k].w}, lw[4] = {l[k].x, l[k].y, l[k].z, l[k].w};
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const float A = n & 1 ? bf16_hi(hw[n >> 1]) + bf16_hi(lw[n >> 1]) : bf16_lo(hw[n >> 1]) + bf16_lo(lw[n >> 1]);
            v[8 * k + n] = fmaf(f.c, v[8 * k + n], fmaf(f.b, A, i == j + 8 * k + n ? f.a : 0.f));
        }
    }
}

struct StepEpilogue {
    Finish f;
    float* parts;   // of the tiles

    // Whole sums of 32 x 32: a lane has a row, or with `turned` a column.
    __device__ __forceinline__ void finish(const Problem& pr, const Unit& t, float (&v)[32], int row0, int col0, int rows, int cols,
                                           bool turned, const WarpOut& out) const {
        if (f.kind == kResult) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] *= f.scale;
            acrl_bf16* to = f.out + t.z * f.out_stride;
            // of the matrix, or of its transpose
            const int R = f.tall ? cols : rows, C = f.tall ? rows : cols, r = f.tall ? col0 : row0, c = f.tall ? row0 : col0;
            if (turned != f.tall) out.store_turned(to, f.ldo, R, C, v, r, c, f.wide);
            else out.store(to, f.ldo, R, C, v, r, c, f.wide);
            return;
        }
        if (f.kind == kPolynomial)   // A is symmetric: its column is its row
            polynomial(f, t.z, (turned ? col0 : row0) + out.lane, turned ? row0 : col0, rows, v);
        uint32_t h[16], l[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            h[j] = pack_bf16x2(v[2 * j], v[2 * j + 1]);
            l[j] = pack_bf16x2(v[2 * j] - bf16_lo(h[j]), v[2 * j + 1] - bf16_hi(h[j]));
        }
        acrl_bf16 *hi = f.hi + t.z * f.size, *lo = f.lo + t.z * f.size;
        const bool twice = pr.lower && col0 < t.tp * 2 * kRows;   // a tile above the diagonal has no other way to be written
        if (!turned || twice) {
            const bool other = turned;   // the lane's values, as a row of the transpose
            out.store_halves(hi, lo, f.ld, other ? cols : rows, other ? rows : cols, h, l, other ? col0 : row0, other ? row0 : col0);
        }
        if (turned || twice) {
            const bool other = !turned;
            out.store_halves_turned(hi, lo, f.ld, other ? cols : rows, other ? rows : cols, h, l, other ? col0 : row0, other ? row0 : col0);
        }
    }

    __device__ __forceinline__ void chunk(const Problem& pr, const Unit& t, const uint32_t (&r)[32], int row0, int col0, int rows,
                                          int cols, const WarpOut& out) const {
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
        if (pr.parts > 1) {
            const int high = 2 * kRows, wide = pr.cols;
            out.store(parts + (int64_t(t.all) * pr.parts + t.part) * high * wide, wide, rows > 0 ? high : 0, wide, v, row0 - t.tp * high,
                      col0 - t.tq * wide);
            return;
        }
        finish(pr, t, v, row0, col0, rows, cols, false, out);
    }

    // The parts of the tiles in their order, and what is made of them: block after block of 32 x 32, a warp each.  A lane has a
    // column of the block, so that a row of it is one load.
    __device__ void join(const Problem& pr, int warp, int warps, const WarpOut& out) const {
        const int across = pr.cols / 32, each = 2 * kRows / 32 * across, tiles = pr.tiles * pr.batch;
        const int64_t size = int64_t(2 * kRows) * pr.cols;
        for (int64_t k = warp; k < int64_t(tiles) * each; k += warps) {
            const Unit t = tile_at(pr, int(k / each));
            const int in = int(k - int64_t(t.all) * each), r = in / across * 32, c = in % across * 32;   // in the tile
            const int row0 = t.tp * 2 * kRows + r, col0 = t.tq * pr.cols + c;
            if (row0 >= pr.rows || col0 >= pr.cols_all) continue;
            float v[32] = {};
            const float* p = parts + t.all * pr.parts * size + int64_t(r) * pr.cols + c + out.lane;
            for (int j = 0; j < pr.parts; ++j)
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] += __ldcg(p + j * size + i * pr.cols);
            finish(pr, t, v, row0, col0, pr.rows, pr.cols_all, true, out);
        }
    }
};

// The products of a step: A = X X^T, Q from A A, Q X.
enum { kProducts = 3 };

struct StepsLaunch {
    // of X (each of two buffers), A and Q: 128 rows as p, half a tile's columns as q, blocks turned
    CUtensorMap x_p[2], x_q[2], x_turned[2], a_p, a_q, q_p;
    Problem pr[kProducts];
    Finish f[kProducts + 1];          // of A, Q, X in the first buffer, X in the second
    float coeffs[3 * kMostSteps];
    int steps;
    float* parts;
    unsigned* done;                   // warps' shares of units written so far, of each matrix; with parts, of all
    int each;                         // a counter for each matrix
    int stages, stage_bytes;
    int32_t* flags;
};

// Where a role is among the products: their units in order, every pairs-th.
struct Place {
    const StepsLaunch& l;
    int k = 0, pair, pairs, last;
    int offset = 0;          // units of the products before, modulo the pairs
    unsigned before = 0;     // of a counter: what the products before add up to
    __device__ explicit Place(const StepsLaunch& launch) : l(launch) {
        pair = int(blockIdx.x >> 1);
        pairs = int(gridDim.x >> 1);
        last = kProducts * l.steps - 1;
    }
    __device__ __forceinline__ bool more() const { return k <= last; }
    __device__ __forceinline__ int kind() const { return k % kProducts; }
    __device__ __forceinline__ int step() const { return k / kProducts; }
    __device__ __forceinline__ int first() const { return pair >= offset ? pair - offset : pair - offset + pairs; }
    // This product's units add up to this much: the epilogue warps of two CTAs each.
    __device__ __forceinline__ unsigned units(const Problem& pr) const {
        return 2u * unsigned(kDrain) * unsigned(l.each ? pr.tiles : pr.units);
    }
    __device__ __forceinline__ void next(const Problem& pr) {
        before += units(pr) + (pr.parts > 1 ? gridDim.x * unsigned(kDrain) : 0u);
        offset = (offset + pr.units) % pairs;
        ++k;
    }
};

// Until `counter` has come to `want`: what was written before it did is visible then.  False after the time limit, or once the
// CTA has given up.
__device__ __forceinline__ bool wait_done(const unsigned* counter, unsigned want, volatile int32_t* abort) {
    uint64_t t0 = 0;
    for (uint32_t i = 0;; ++i) {
        unsigned n;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(n) : "l"(counter) : "memory");
        if (int(n - want) >= 0) return true;
        if ((i & 63u) == 63u) {
            if (t0 == 0) t0 = global_ns();
            if (*abort || global_ns() - t0 > kWaitNs) return false;
        }
    }
}

// Whether all of the CTA's epilogue threads say so.  All of them come, whatever they say, and what they have written before is
// visible to all of them.
__device__ __forceinline__ bool epilogue_vote(bool ok) {
    int all;
    __syncwarp();
    asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n bar.red.and.pred q, 1, %2, p;\n selp.b32 %0, 1, 0, q;\n}"
                 : "=r"(all)
                 : "r"(int(ok)), "n"(32 * kDrain)
                 : "memory");
    return all != 0;
}

__global__ void __launch_bounds__(kProductThreads, 1) steps_kernel(const __grid_constant__ StepsLaunch l) {
    extern __shared__ uint8_t smem_raw[];
    const Begun b = begin_products<true>(smem_raw, l.stages, l.stage_bytes, &l.x_p[0], &l.x_q[0], l.flags);
    const int warp = threadIdx.x >> 5;
    ProductBarriers* bars = b.ring.bars;
    volatile int32_t* abort = &bars->abort;
    bool ok = true;
    if (warp == 0) {
        Producer<true, 3> role{b.ring};
        for (Place at(l); at.more() && ok;) {
            const Problem pr = l.pr[at.kind()];
            const int kind = at.kind(), x = at.step() & 1;
            const CUtensorMap* p = kind == 0 ? &l.x_p[x] : kind == 1 ? &l.a_p : &l.q_p;
            const CUtensorMap* q = kind == 0 ? &l.x_q[x] : kind == 1 ? &l.a_q : &l.x_turned[x];
            int known = -1;   // the matrix whose product before is written
            for (int u = at.first(); u < pr.units && ok; u += at.pairs) {
                const Unit t = unit_at(pr, u);
                const int z = l.each ? t.z : 0;
                if (z != known) {
                    known = z;
                    // Every lane, whichever is elected for the copies: a vote would order no memory between one that has waited and
                    // the others.  (256 x 256 97.7 us; one lane and a __syncwarp 103.)
                    ok = __all_sync(0xffffffffu, wait_done(l.done + z, at.before, abort));
                    if (!ok) {
                        give_up(abort, l.flags);
                        role.land();
                        break;
                    }
                    asm volatile("fence.proxy.async;" ::: "memory");   // copies read what others' stores have written
                }
                ok = role.unit(pr, t, p, q);
            }
            at.next(pr);
        }
    } else if (warp == 1 && b.ring.rank == 0) {
        Multiplier<true, 3> role{b.ring, b.tmem};
        for (Place at(l); at.more() && ok;) {
            const Problem pr = l.pr[at.kind()];
            for (int u = at.first(); u < pr.units && ok; u += at.pairs) ok = role.unit(pr, unit_at(pr, u));
            at.next(pr);
        }
        role.finish();
    } else if (warp >= 4) {
        Drain<true, false> role(b.ring, b.tmem, b.staging);
        // What the warp, or after a vote the CTA's epilogue, has written is visible to those who find it counted.  Every warp for
        // itself, 256 x 256 took 100 us, through a warp of the CTA that has waited for all 104; on the one counter that split sums
        // have, 2,051 x 1,000 took 258 so, and 242 with a vote.
        auto tell = [&](unsigned* counter, unsigned shares) {
            __syncwarp();
            if (role.lane == 0) {
                __threadfence();
                asm volatile("red.relaxed.gpu.global.add.u32 [%0], %1;" ::"l"(counter), "r"(shares) : "memory");
            }
        };
        const bool first = warp == 4;
#pragma unroll 1
        for (Place at(l); at.more() && ok;) {
            const Problem pr = l.pr[at.kind()];
            StepEpilogue e{l.f[at.kind() < 2 ? at.kind() : 2 + (1 - (at.step() & 1))], l.parts};
            if (at.kind() == 1) {
                e.f.a = l.coeffs[3 * at.step()];
                e.f.b = l.coeffs[3 * at.step() + 1];
                e.f.c = l.coeffs[3 * at.step() + 2];
            }
            if (at.k == at.last) e.f.kind = kResult;
#pragma unroll 1
            for (int u = at.first(); u < pr.units && ok; u += at.pairs) {
                ok = role.unit(pr, u, e);
                if (l.each) {
                    if (ok) tell(l.done + u / pr.tiles, 1);
                } else {
                    ok = epilogue_vote(ok);
                    if (ok && first) tell(l.done, kDrain);
                }
            }
            if (pr.parts > 1 && ok) {
                ok = epilogue_vote(!first || role.lane != 0 || wait_done(l.done, at.before + at.units(pr), abort));
                if (!ok) give_up(abort, l.flags);
                else {
                    e.join(pr, int(blockIdx.x) * kDrain + warp - 4, int(gridDim.x) * kDrain, role.out);
                    epilogue_vote(true);
                    if (first) tell(l.done, kDrain);
                }
            }
            at.next(pr);
        }
    }
    end_products<true>(b.tmem);
}

// ---------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------

struct Plan {
    Shape shape;
    Cut cut;
    int64_t workspace;
};

Plan plan_of(int64_t batch, int64_t rows, int64_t cols, int64_t K, bool lower, bool q_turned) {
    const Shape s{true, rows, cols, K, batch, lower, 3, 256, q_turned ? 128 : 64, 0, 2 * kRows};
    const Cut cut = best_cut(s);
    return Plan{s, cut, parts_bytes(s, cut)};
}

// The workspace, in bytes: sums of squares; X twice, A and Q, each in two matrices; the parts of a split sum.
struct Layout {
    int64_t m, n, ldx, lda, ctas;
    int64_t done, x[2], gram, q, parts, end;
    Plan plan_gram, plan_q, plan_x;
    Layout(int64_t batch, int64_t rows, int64_t cols) {
        m = std::min(rows, cols);
        n = std::max(rows, cols);
        ldx = (n + 7) / 8 * 8;
        lda = (m + 7) / 8 * 8;
        ctas = std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(1, kSumCtas / batch), m * n / 4096));
        int64_t at = (batch * ctas * 8 + 127) / 128 * 128;
        auto take = [&](int64_t bytes) {
            const int64_t here = at;
            at += (bytes + 127) / 128 * 128;
            return here;
        };
        done = take(batch * 4);
        for (int64_t& one : x) one = take(batch * m * ldx * 4);   // a half after the other
        gram = take(batch * m * lda * 4);
        q = take(batch * m * lda * 4);
        plan_gram = plan_of(batch, m, m, n, true, false);
        plan_q = plan_of(batch, m, m, m, true, false);
        plan_x = plan_of(batch, m, n, m, false, true);
        parts = take(std::max(plan_gram.workspace, std::max(plan_q.workspace, plan_x.workspace)));
        end = at;
    }
};

struct Halves {
    acrl_bf16 *hi, *lo;
    int64_t ld, size;   // from one matrix to the next
};

// All pairs are resident at once, or the launch is refused: cooperative.  The most that are, of the calling thread's last device.
int64_t resident_pairs() {
    static thread_local int known = -1;
    static thread_local int64_t most = 0;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    if (dev == known) return most;
    if (cudaFuncSetAttribute(steps_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kProductSmem) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    most = resident_clusters(reinterpret_cast<const void*>(steps_kernel), kProductThreads, kProductSmem, 2);
    if (most > 0) known = dev;
    return most;
}

acrl_status launch_steps(const StepsLaunch& l, int64_t pairs, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(2 * pairs), 1, 1);
    cfg.blockDim = dim3(kProductThreads, 1, 1);
    cfg.dynamicSmemBytes = kProductSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    (void)cudaLaunchKernelEx(&cfg, steps_kernel, l);
    return launch_status();
}

}  // namespace
}  // namespace acrl

using namespace acrl;

namespace {
bool sizes_ok(int64_t batch, int64_t m, int64_t n) {
    return batch >= 0 && m >= 0 && n >= 0 && batch <= kMostSize && m <= kMostSize && n <= kMostSize;
}
// Tiles, pieces and blocks of a launch are counted in 32 bits.
bool blocks_ok(int64_t batch, int64_t m, int64_t n) {
    return double(batch) * double((m + 31) / 32) * double((n + 31) / 32) < double(1 << 30);
}
}  // namespace

extern "C" int64_t acrl_orthogonalize_workspace_bytes(int64_t batch, int64_t m, int64_t n) {
    if (batch < 0 || m < 0 || n < 0) return -1;
    return batch == 0 || m == 0 || n == 0 || !sizes_ok(batch, m, n) || !blocks_ok(batch, m, n) ? 0 : Layout(batch, m, n).end;
}

extern "C" acrl_status acrl_orthogonalize(const void* g, acrl_dtype g_dtype, int64_t batch, int64_t m, int64_t n, int64_t ldg,
                                          int64_t g_stride, const float* coeffs, int32_t steps, float eps, float scale,
                                          acrl_bf16* out, int64_t ldo, int64_t out_stride, void* workspace, int64_t workspace_bytes,
                                          int32_t* dev_flags, acrl_stream stream) {
    if (!sizes_ok(batch, m, n)) return ACRL_ERR_INVALID_ARG;
    if ((g_dtype != ACRL_BF16 && g_dtype != ACRL_F32) || steps < 1 || steps > kMostSteps || !coeffs) return ACRL_ERR_INVALID_ARG;
    if (!(eps >= 0.f && eps < INFINITY) || !(scale > -INFINITY && scale < INFINITY)) return ACRL_ERR_INVALID_ARG;
    for (int i = 0; i < 3 * steps; ++i)
        if (!(coeffs[i] > -INFINITY && coeffs[i] < INFINITY)) return ACRL_ERR_INVALID_ARG;
    if (workspace_bytes < acrl_orthogonalize_workspace_bytes(batch, m, n)) return ACRL_ERR_INVALID_ARG;
    if (batch == 0 || m == 0 || n == 0) return ACRL_OK;
    if (!blocks_ok(batch, m, n)) return ACRL_ERR_INVALID_ARG;
    if (!g || (reinterpret_cast<uintptr_t>(g) & (g_dtype == ACRL_BF16 ? 1 : 3)) || ldg < n || !out ||
        (reinterpret_cast<uintptr_t>(out) & 1) || ldo < n || !workspace || !aligned16(workspace))
        return ACRL_ERR_INVALID_ARG;
    if (batch > 1 && (g_stride < (m - 1) * ldg + n || out_stride < (m - 1) * ldo + n)) return ACRL_ERR_INVALID_ARG;
    if (!operands_on_current_device({g, out, workspace})) return ACRL_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const Layout l(batch, m, n);
    uint8_t* base = static_cast<uint8_t*>(workspace);
    auto halves_at = [&](int64_t at, int64_t ld) {
        acrl_bf16* hi = reinterpret_cast<acrl_bf16*>(base + at);
        return Halves{hi, hi + batch * l.m * ld, ld, l.m * ld};
    };
    const Halves x[2] = {halves_at(l.x[0], l.ldx), halves_at(l.x[1], l.ldx)}, gram = halves_at(l.gram, l.lda), q = halves_at(l.q, l.lda);
    double* sums = reinterpret_cast<double*>(base);
    StepsLaunch t = {};
    t.steps = steps;
    t.parts = reinterpret_cast<float*>(base + l.parts);
    t.done = reinterpret_cast<unsigned*>(base + l.done);
    t.each = 1;
    t.flags = dev_flags;
    std::copy(coeffs, coeffs + 3 * steps, t.coeffs);
    const Plan* plans[kProducts] = {&l.plan_gram, &l.plan_q, &l.plan_x};
    int64_t units = 0;
    for (int k = 0; k < kProducts; ++k) {
        const Plan& p = *plans[k];
        t.pr[k] = problem_of(p.shape, p.cut, false, k == 2, false);
        t.stage_bytes = std::max(t.stage_bytes, 2 * (kRows + p.cut.cols / 2) * kRowBytes);
        units = std::max(units, p.cut.units());
        if (p.cut.parts > 1) t.each = 0;   // parts are of all matrices at once
    }
    t.stages = std::min(kMaxStages, kRingBytes / t.stage_bytes);
    bool ok = true;
    auto map = [&](CUtensorMap& to, const Halves& h, int64_t rows, bool turned, int64_t K, int box) {
        ok = ok && operand_map(&to, Matrix{h.hi, rows, h.ld, turned, batch, h.size, batch * h.size}, K, box);
    };
    for (int b = 0; b < 2; ++b) {
        map(t.x_p[b], x[b], l.m, false, l.n, kRows);
        map(t.x_q[b], x[b], l.m, false, l.n, l.plan_gram.cut.cols / 2);
        map(t.x_turned[b], x[b], l.n, true, l.m, kSlab);
    }
    map(t.a_p, gram, l.m, false, l.m, kRows);
    map(t.a_q, gram, l.m, false, l.m, l.plan_q.cut.cols / 2);
    map(t.q_p, q, l.m, false, l.m, kRows);
    if (!ok) return ACRL_ERR_CUDA;
    auto finish = [&](Finish& f, Kind kind, const Halves& to) {
        f.kind = kind;
        f.hi = to.hi;
        f.lo = to.lo;
        f.ld = to.ld;
        f.size = to.size;
        f.hi_in = gram.hi;
        f.lo_in = gram.lo;
        f.scale = scale;
        f.out = out;
        f.ldo = ldo;
        f.out_stride = out_stride;
        f.tall = m > n;
        f.wide = aligned16(out) && (ldo & 7) == 0 && (batch == 1 || (out_stride & 7) == 0);
    };
    finish(t.f[0], kGram, gram);
    finish(t.f[1], kPolynomial, q);
    finish(t.f[2], kIterate, x[0]);
    finish(t.f[3], kIterate, x[1]);
    const int64_t most = resident_pairs();
    if (most < 1) return ACRL_ERR_CUDA;
    const int64_t to = g_dtype == ACRL_BF16 ? 7 : 3;
    const bool wide = aligned16(g) && (ldg & to) == 0 && (batch == 1 || (g_stride & to) == 0);
    const Update u{g, g_dtype == ACRL_F32, wide, ldg, g_stride, int(m), int(n)};
    acrl_status st = launch(squares_kernel, batch * l.ctas, 256, 0, 0, s, u, int(l.ctas), sums, t.done);
    if (st == ACRL_OK)
        st = launch(first_kernel, batch * l.ctas, 256, 0, 0, s, u, int(l.ctas), static_cast<const double*>(sums), eps, x[0].hi, x[0].lo, l.ldx,
                    x[0].size, dev_flags);
    return st != ACRL_OK ? st : launch_steps(t, std::min(units, most), s);
}
