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
    if (c + 8 > u.n) {
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

// Partial sums of a matrix's squares, `ctas` of them.  HBM bounds it.
__global__ void __launch_bounds__(256) squares_kernel(Update u, int ctas, double* sums) {
    __shared__ double part[8];
    grid_begin();
    const int b = int(blockIdx.x) / ctas, lane = threadIdx.x & 31;
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

// Two bf16 numbers for one.
__device__ __forceinline__ void halves(float x, acrl_bf16& hi, acrl_bf16& lo) {
    hi = to_bf16(x);
    lo = to_bf16(x - bf16_to_float(hi));
}

// Eight of them, from a column that is a multiple of eight.
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
    float* parts;                  // of the tiles

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

// The parts of the tiles in their order, and what is made of them, a block of 32 x 32 a CTA; of a symmetric matrix the
// mirror image as well.
__global__ void __launch_bounds__(256) join_kernel(Finish f, const float* parts, Problem pr) {
    __shared__ float block[32][33];
    grid_begin();
    const int across = pr.cols / 32, blocks = 2 * kRows / 32 * across, tile = int(blockIdx.x) / blocks, k = int(blockIdx.x) - tile * blocks;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rows = pr.rows, cols = pr.cols_all;
    const Unit t = tile_at(pr, tile);
    const int64_t z = t.z;
    const int rt = k / across * 32, ct = k % across * 32, r0 = t.tp * 2 * kRows + rt, c0 = t.tq * pr.cols + ct;   // in the tile, in all
    if (r0 >= rows || c0 >= cols) return;
    const bool turn = f.kind == kResult && f.tall, twice = pr.lower && c0 < t.tp * 2 * kRows;
    float v[4] = {};
    const int c = c0 + lane;
    const int64_t size = int64_t(2 * kRows) * pr.cols;
    const float* p = parts + tile * pr.parts * size + (rt + warp) * pr.cols + ct + lane;
    for (int j = 0; j < pr.parts; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += p[j * size + 8 * i * pr.cols];
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
    Shape shape;
    Cut cut;
    int64_t workspace;
};

Plan plan_of(int64_t batch, int64_t rows, int64_t cols, int64_t K, bool lower, bool q_turned) {
    const Shape s{true, rows, cols, K, batch, lower, 3, 256, q_turned ? 128 : 64, 0};
    const Cut cut = best_cut(s);
    return Plan{s, cut, parts_bytes(s, cut)};
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

// One product of the steps.
acrl_status step_product(const Plan& plan, const Halves& p, const Halves& q, bool q_turned, const Finish& f, float* parts, int32_t* flags,
                         cudaStream_t s) {
    const Shape& sh = plan.shape;
    ProductLaunch<1, 3, StepEpilogue> l = {};
    l.pr[0] = problem_of(sh, plan.cut, false, q_turned, false);
    l.epi[0].f = f;
    l.epi[0].parts = parts;
    for (int i = 0; i < 2; ++i) {
        if (!operand_map(&l.p[0][i], Matrix{i ? p.lo : p.hi, sh.rows, p.ld, false, sh.batch, p.size}, sh.K, kRows) ||
            !operand_map(&l.q[0][i], Matrix{i ? q.lo : q.hi, sh.cols_all, q.ld, q_turned, sh.batch, q.size}, sh.K, plan.cut.cols / 2))
            return ACRL_ERR_CUDA;
    }
    const acrl_status st = launch_product<true, false>(l, flags, s);
    if (st != ACRL_OK || plan.cut.parts == 1) return st;
    return launch(join_kernel, plan.cut.tiles * (2 * kRows / 32) * (plan.cut.cols / 32), 256, 0, 0, s, f, static_cast<const float*>(parts), l.pr[0]);
}

}  // namespace
}  // namespace acrl

using namespace acrl;

namespace {
bool sizes_ok(int64_t batch, int64_t m, int64_t n) {
    constexpr int64_t kMost = kMaxGrid - 512;
    return batch >= 0 && m >= 0 && n >= 0 && batch <= kMost && m <= kMost && n <= kMost;
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
    st = launch(first_kernel, batch * l.ctas, 256, 0, 0, s, u, int(l.ctas), static_cast<const double*>(sums), eps, x[0].hi,
                x[0].lo, l.ldx, x[0].size, dev_flags);
    for (int i = 0; i < steps && st == ACRL_OK; ++i) {
        const Halves &from = x[i & 1], &into = x[1 - (i & 1)];
        Finish f = {};
        f.kind = kGram;
        f.hi = gram.hi;
        f.lo = gram.lo;
        f.ld = gram.ld;
        f.size = gram.size;
        st = step_product(l.plan_gram, from, from, false, f, parts, dev_flags, s);
        if (st != ACRL_OK) break;
        f.kind = kPolynomial;
        f.a = coeffs[3 * i];
        f.b = coeffs[3 * i + 1];
        f.c = coeffs[3 * i + 2];
        f.hi_in = gram.hi;
        f.lo_in = gram.lo;
        f.hi = q.hi;
        f.lo = q.lo;
        st = step_product(l.plan_q, gram, gram, false, f, parts, dev_flags, s);
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
        st = step_product(l.plan_x, q, from, true, f, parts, dev_flags, s);
    }
    return st;
}
