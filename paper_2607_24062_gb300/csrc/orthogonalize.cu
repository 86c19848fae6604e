// acrl_orthogonalize: Newton-Schulz steps on an update.  With X (m x n, m <= n; a tall matrix's transpose) a step is
//
//     A = X X^T,   Q = a I + b A + c A A,   X <- Q X,
//
// so that the polynomial in the Gram matrix is made on its m x m elements, and X is read twice and written once.  A and Q are
// symmetric: tiles above the diagonal are left out and written as mirror images, 3 m^2 n + m^3 multiply-adds a step where the
// plain products have 4 m^2 n + 2 m^3.
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
constexpr int kPairs = 76;
constexpr int kSumCtas = 608;      // four of an SM's: CTAs that add up squares

struct Update {
    const void* g;
    bool f32;
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

// Partial sums of a matrix's squares, `ctas` of them: rows in turn, 16 bytes a thread.  HBM bounds it.
__global__ void __launch_bounds__(256) squares_kernel(Update u, int ctas, double* sums) {
    __shared__ double part[8];
    grid_begin();
    const int b = int(blockIdx.x) / ctas, c = int(blockIdx.x) - b * ctas;
    const int V = u.f32 ? 4 : 8, vectors = (u.n + V - 1) / V;
    Squares s;
    const int64_t all = int64_t(u.m) * vectors;
    for (int64_t i = int64_t(c) * 256 + threadIdx.x; i < all; i += int64_t(ctas) * 256) {
        const int64_t r = i / vectors;
        const int at = int(i - r * vectors) * V;
        const int64_t row = b * u.stride + r * u.ld + at;
        if (at + V > u.n) {
            for (int j = at; j < u.n; ++j) s.add(load_float(u.g, u.f32, row + j - at));
        } else if (u.f32) {
            const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(u.g) + row);
            s.add(x.x);
            s.add(x.y);
            s.add(x.z);
            s.add(x.w);
        } else {
            const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const acrl_bf16*>(u.g) + row);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s.add(bf16_lo(w[j]));
                s.add(bf16_hi(w[j]));
            }
        }
    }
    const double sum = warp_sum(s.total());
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int i = 0; i < 8; ++i) t += part[i];
        sums[blockIdx.x] = t;
    }
}

// Two bf16 numbers for one.
__device__ __forceinline__ void halves(float x, acrl_bf16& hi, acrl_bf16& lo) {
    hi = to_bf16(x);
    lo = to_bf16(x - bf16_to_float(hi));
}

// X_0 = G / (|G| + eps) in two bf16 matrices, 32 x 32 blocks, turned where G is tall.  The factor is a power of two times a
// number in [1, 2): an update of any size is brought near 1 before it is divided.
__global__ void __launch_bounds__(256) first_kernel(Update u, int ctas, const double* sums, float eps, acrl_bf16* hi, acrl_bf16* lo,
                                                    int64_t ldx, int64_t size, int32_t* flags) {
    __shared__ float block[32][33];
    __shared__ float by[3];
    grid_begin();
    const int64_t rows = (u.m + 31) / 32, cols = (u.n + 31) / 32, blocks = rows * cols;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int b = int(int64_t(blockIdx.x) / blocks);
    const int64_t k = int64_t(blockIdx.x) - b * blocks;
    const int r0 = int(k / cols) * 32, c0 = int(k % cols) * 32;
    if (warp == 0) {
        double sum = 0.0;
        for (int i = lane; i < ctas; i += 32) sum += sums[int64_t(b) * ctas + i];
        sum = warp_sum(sum);
        if (lane == 0) {
            const bool bad = !(sum <= 1.7e308);   // an infinity or a NaN: no finite matrix comes near
            if (bad && k == 0) raise_flag(flags, ACRL_FLAG_NONFINITE);
            int e = 0;
            const double f = frexp(sqrt(sum) + double(eps), &e);   // f 2^e
            by[0] = exp2f(float(-e / 2));
            by[1] = exp2f(float(-e - -e / 2));
            by[2] = bad ? __int_as_float(0x7fc00000) : f > 0.0 ? float(1.0 / f) : 0.f;
        }
    }
    __syncthreads();
    const float one = by[0], two = by[1], rest = by[2];
    const bool tall = u.m > u.n;
    acrl_bf16 *h = hi + b * size, *l = lo + b * size;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + warp + 8 * i, c = c0 + lane;
        float x = 0.f;
        if (r < u.m && c < u.n) x = load_float(u.g, u.f32, b * u.stride + r * u.ld + c) * one * two * rest;
        if (tall)
            block[warp + 8 * i][lane] = x;
        else if (r < u.m && c < u.n)
            halves(x, h[r * ldx + c], l[r * ldx + c]);
    }
    if (!tall) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = c0 + warp + 8 * i, c = r0 + lane;   // of X
        if (r < u.n && c < u.m) halves(block[lane][warp + 8 * i], h[r * ldx + c], l[r * ldx + c]);
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
    bool tall;                         // the result is turned back
};

// Four of A's numbers from their halves.
__device__ __forceinline__ void add_halves(uint2 h, uint2 l, float (&A)[4]) {
    A[0] = bf16_lo(h.x) + bf16_lo(l.x);
    A[1] = bf16_hi(h.x) + bf16_hi(l.x);
    A[2] = bf16_lo(h.y) + bf16_lo(l.y);
    A[3] = bf16_hi(h.y) + bf16_hi(l.y);
}

// a I + b A + c v at row i, columns j .. j + 31; what is beyond the matrix is left out of the result.  A row's 64 bytes of each half come in 16-byte loads: one by one they took three times as long as the product (24 x 1,024 x
// 1,024: 220 us a step against 66 for A itself).
__device__ __forceinline__ void polynomial(const Finish& f, int64_t at, int i, int j, int m, float (&v)[32]) {
#pragma unroll
    for (int k = 0; k < 32; k += 8) {
        uint4 h = make_uint4(0u, 0u, 0u, 0u), l = h;
        if (i < m && j + k < f.ld) {   // ld is a multiple of eight
            h = *reinterpret_cast<const uint4*>(f.hi_in + at + k);
            l = *reinterpret_cast<const uint4*>(f.lo_in + at + k);
        }
        float A[8];
        add_halves(make_uint2(h.x, h.y), make_uint2(l.x, l.y), *reinterpret_cast<float (*)[4]>(A));
        add_halves(make_uint2(h.z, h.w), make_uint2(l.z, l.w), *reinterpret_cast<float (*)[4]>(A + 4));
#pragma unroll
        for (int n = 0; n < 8; ++n) v[k + n] = fmaf(f.c, v[k + n], fmaf(f.b, A[n], i < m && i == j + k + n ? f.a : 0.f));
    }
}

struct StepEpilogue {
    Finish f;
    float* parts;                  // where the sum is split: [matrix][part][row][ldparts]
    int64_t ldparts, part_size;

    __device__ __forceinline__ void chunk(const Problem& pr, const Unit& t, const uint32_t (&r)[32], int row0, int col0, int rows,
                                          int cols, const WarpOut& out) const {
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
        if (parts) {
            out.store(parts + (int64_t(t.z) * pr.parts + t.part) * part_size, ldparts, rows, cols, v, row0, col0);
            return;
        }
        if (f.kind == kResult) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] *= f.scale;
            acrl_bf16* to = f.out + t.z * f.out_stride;
            if (f.tall) out.store_turned(to, f.ldo, cols, rows, v, col0, row0);
            else out.store(to, f.ldo, rows, cols, v, row0, col0);
            return;
        }
        const int row = row0 + out.lane;
        if (f.kind == kPolynomial) polynomial(f, t.z * f.size + row * f.ld + col0, row, col0, rows, v);
        const bool twice = pr.lower && col0 < t.tp * 2 * kRows;   // a tile above the diagonal has no other way to be written
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            acrl_bf16* to = (half ? f.lo : f.hi) + t.z * f.size;
            out.store(to, f.ld, rows, cols, v, row0, col0);
            if (twice) out.store_turned(to, f.ld, cols, rows, v, col0, row0);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] -= bf16_to_float(to_bf16(v[j]));   // what is left for the other
        }
    }
};

// The parts of a split sum in their order, and what is made of them, a block of 32 x 32 a CTA; of a symmetric matrix those
// that were computed, and their mirror images.
__global__ void __launch_bounds__(256) join_kernel(Finish f, const float* parts, int count, int64_t ldparts, int64_t part_size, int lower,
                                                   int rows, int cols) {
    __shared__ float block[32][33];
    grid_begin();
    const int64_t across = (cols + 31) / 32, blocks = (rows + 31) / 32 * across, z = int64_t(blockIdx.x) / blocks;
    const int64_t k = int64_t(blockIdx.x) - z * blocks;
    const int r0 = int(k / across) * 32, c0 = int(k % across) * 32, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tile = r0 / (2 * kRows) * 2 * kRows;   // the first row, and column, of the diagonal's tile
    if (lower && c0 >= tile + 2 * kRows) return;
    const bool turn = f.kind == kResult && f.tall, twice = lower && c0 < tile;
    float v[4] = {};
    const int c = c0 + lane;
    for (int j = 0; j < count; ++j) {
        const float* p = parts + (z * count + j) * part_size + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + warp + 8 * i;
            if (r < rows && c < cols) v[i] += p[r * ldparts];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + warp + 8 * i;
        const bool in = r < rows && c < cols;
        const int64_t at = z * f.size + r * f.ld + c;
        if (f.kind == kResult) {
            v[i] *= f.scale;
            if (in && !turn) f.out[z * f.out_stride + r * f.ldo + c] = to_bf16(v[i]);
        } else {
            if (f.kind == kPolynomial && in)
                v[i] = fmaf(f.c, v[i], fmaf(f.b, bf16_to_float(f.hi_in[at]) + bf16_to_float(f.lo_in[at]), r == c ? f.a : 0.f));
            if (in) halves(v[i], f.hi[at], f.lo[at]);
        }
        block[warp + 8 * i][lane] = v[i];
    }
    if (!turn && !twice) return;   // the same for the CTA
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = c0 + warp + 8 * i, d = r0 + lane;   // of the turned block
        if (r >= cols || d >= rows) continue;
        const float x = block[lane][warp + 8 * i];
        if (turn)
            f.out[z * f.out_stride + r * f.ldo + d] = to_bf16(x);
        else
            halves(x, f.hi[z * f.size + r * f.ld + d], f.lo[z * f.size + r * f.ld + d]);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------

struct Plan {
    Cut cut;
    int64_t cost, workspace, ldparts, part_size;
};

// The cut of a product rows x cols over K with the least estimated time, as for a layer's.
Plan plan_of(int64_t batch, int64_t rows, int64_t cols_all, int64_t K, bool lower, bool q_turned) {
    constexpr int64_t kTile = 4000, kJoin = 6000, kJoinBytes = 3000;
    const int64_t slabs = (K + kSlab - 1) / kSlab, p_tiles = (rows + 2 * kRows - 1) / (2 * kRows);
    Plan best = {};
    best.ldparts = (cols_all + 7) / 8 * 8;
    best.part_size = rows * best.ldparts;
    for (int cols = 256; cols >= (q_turned ? 128 : 64); cols /= 2) {
        const int64_t q_tiles = (cols_all + cols - 1) / cols, r = 2 * kRows / cols;
        const int64_t tiles = batch * (lower ? r * (p_tiles - 1) * p_tiles / 2 + q_tiles : p_tiles * q_tiles);
        const int64_t slab = std::max(6 * cols, 4 * (kRows + cols / 2));
        for (int64_t parts = 1; parts <= 16 && parts <= slabs; ++parts) {
            const int64_t per = (slabs + parts - 1) / parts;
            if ((slabs + per - 1) / per != parts) continue;
            const int64_t rounds = (tiles * parts + kPairs - 1) / kPairs;
            const int64_t cost = rounds * (per * slab + kTile) +
                                 (parts > 1 ? kJoin + (parts + 1) * batch * best.part_size * 4 / kJoinBytes : 0);
            if (best.cost == 0 || cost < best.cost) {
                best.cost = cost;
                best.cut = Cut{cols, int(parts), int(per)};
            }
        }
    }
    best.workspace = best.cut.parts > 1 ? best.cut.parts * batch * best.part_size * 4 : 0;
    return best;
}

// The workspace, in bytes: sums of squares; X twice, A and Q, each in two matrices; the parts of a split sum.
struct Layout {
    int64_t m, n, ldx, lda, ctas;
    int64_t x[2][2], gram[2], q[2], parts, end;
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
        for (auto& pair : x)
            for (int64_t& half : pair) half = take(batch * m * ldx * 2);
        for (int64_t& half : gram) half = take(batch * m * lda * 2);
        for (int64_t& half : q) half = take(batch * m * lda * 2);
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

// One product of the steps: rows x cols over K.
acrl_status step_product(const Plan& plan, int64_t batch, int64_t rows, int64_t cols, int64_t K, const Halves& p, const Halves& q,
                         bool q_turned, bool lower, const Finish& f, float* parts, int32_t* flags, cudaStream_t s) {
    ProductLaunch<1, 3, StepEpilogue> l = {};
    l.pr[0] = problem_of(true, rows, cols, K, batch, false, q_turned, lower, false, plan.cut);
    StepEpilogue& e = l.epi[0];
    e.f = f;
    e.parts = plan.cut.parts > 1 ? parts : nullptr;
    e.ldparts = plan.ldparts;
    e.part_size = plan.part_size;
    for (int i = 0; i < 2; ++i) {
        if (!operand_map(&l.p[0][i], Matrix{i ? p.lo : p.hi, rows, p.ld, false, batch, p.size}, K, kRows) ||
            !operand_map(&l.q[0][i], Matrix{i ? q.lo : q.hi, cols, q.ld, q_turned, batch, q.size}, K, plan.cut.cols / 2))
            return ACRL_ERR_CUDA;
    }
    const acrl_status st = launch_product<true, false>(l, flags, s);
    if (st != ACRL_OK || !e.parts) return st;
    return launch(join_kernel, batch * ((rows + 31) / 32) * ((cols + 31) / 32), 256, 0, 0, s, f, static_cast<const float*>(parts),
                  plan.cut.parts, plan.ldparts, plan.part_size, int(lower), int(rows), int(cols));
}

}  // namespace
}  // namespace acrl

using namespace acrl;

namespace {
bool sizes_ok(int64_t batch, int64_t m, int64_t n) {
    constexpr int64_t kMost = kMaxGrid - 512;
    return batch >= 0 && m >= 0 && n >= 0 && batch <= kMost && m <= kMost && n <= kMost;
}
// One launch's blocks, and the parts' too, stay within a grid.
bool blocks_ok(int64_t batch, int64_t m, int64_t n) {
    return double(batch) * double((m + 31) / 32) * double((n + 31) / 32) < double(kMaxGrid);
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
    const int64_t to = g_dtype == ACRL_BF16 ? 7 : 3;
    if (!g || !aligned16(g) || ldg < n || (ldg & to) || (g_stride & to) || !out || !aligned16(out) || ldo < n || (ldo & 7) ||
        (out_stride & 7) || !workspace || !aligned16(workspace))
        return ACRL_ERR_INVALID_ARG;
    if (batch > 1 && (g_stride < (m - 1) * ldg + n || out_stride < (m - 1) * ldo + n)) return ACRL_ERR_INVALID_ARG;
    if (!operands_on_current_device({g, out, workspace})) return ACRL_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const Layout l(batch, m, n);
    uint8_t* base = static_cast<uint8_t*>(workspace);
    auto halves_at = [&](const int64_t (&at)[2], int64_t ld) {
        return Halves{reinterpret_cast<acrl_bf16*>(base + at[0]), reinterpret_cast<acrl_bf16*>(base + at[1]), ld, l.m * ld};
    };
    const Halves x[2] = {halves_at(l.x[0], l.ldx), halves_at(l.x[1], l.ldx)}, gram = halves_at(l.gram, l.lda), q = halves_at(l.q, l.lda);
    float* parts = reinterpret_cast<float*>(base + l.parts);
    double* sums = reinterpret_cast<double*>(base);
    const Update u{g, g_dtype == ACRL_F32, ldg, g_stride, int(m), int(n)};
    acrl_status st = launch(squares_kernel, batch * l.ctas, 256, 0, 0, s, u, int(l.ctas), sums);
    if (st != ACRL_OK) return st;
    st = launch(first_kernel, batch * ((m + 31) / 32) * ((n + 31) / 32), 256, 0, 0, s, u, int(l.ctas), static_cast<const double*>(sums), eps, x[0].hi,
                x[0].lo, l.ldx, x[0].size, dev_flags);
    for (int i = 0; i < steps && st == ACRL_OK; ++i) {
        const Halves &from = x[i & 1], &into = x[1 - (i & 1)];
        Finish f = {};
        f.kind = kGram;
        f.hi = gram.hi;
        f.lo = gram.lo;
        f.ld = gram.ld;
        f.size = gram.size;
        st = step_product(l.plan_gram, batch, l.m, l.m, l.n, from, from, false, true, f, parts, dev_flags, s);
        if (st != ACRL_OK) break;
        f.kind = kPolynomial;
        f.a = coeffs[3 * i];
        f.b = coeffs[3 * i + 1];
        f.c = coeffs[3 * i + 2];
        f.hi_in = gram.hi;
        f.lo_in = gram.lo;
        f.hi = q.hi;
        f.lo = q.lo;
        st = step_product(l.plan_q, batch, l.m, l.m, l.m, gram, gram, false, true, f, parts, dev_flags, s);
        if (st != ACRL_OK) break;
        f.kind = i + 1 < steps ? kIterate : kResult;
        f.hi = into.hi;
        f.lo = into.lo;
        f.ld = into.ld;
        f.size = into.size;
        f.scale = scale;
        f.out = out;
        f.ldo = ldo;
        f.out_stride = out_stride;
        f.tall = m > n;
        st = step_product(l.plan_x, batch, l.m, l.n, l.m, q, from, true, false, f, parts, dev_flags, s);
    }
    return st;
}
