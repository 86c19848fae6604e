// A layer of up to 16 rows, single tokens first of all, and a small layer of up to 256.  Up to 32 rows every byte of the weight is
// read once, and HBM bounds it; each further block of 32 reads the weight again, from L2.  Neither tensor memory nor a ring of copies: their start and end, and the join of a split sum, take longer
// than the weight of a layer.
// A CTA has 16 rows of the weight; its eight warps take turns along the sum, 128 columns each, and their sums meet in shared
// memory.  The products are mma.sync m16n8k16, the weight's rows the 16 and those of x the eight: the pipes of tcgen05 would
// wait for the same bytes.  A lane loads 16 bytes of a weight's row, eight neighbours of the sum, where the instruction's
// layout has four pairs: which eight of a slab's 32 columns a lane holds does not matter as long as both operands agree.
#include <algorithm>

#include "linear.cuh"

namespace acrl {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kW = 16;          // rows of the weight, of a CTA
constexpr int kAhead = 4;       // slabs of 32 columns in flight
constexpr int kTurn = 32 * kAhead;

struct FewArgs {
    const acrl_bf16 *x, *w;
    int64_t ldx, ldw;
    int M, N, K;
    int ctas;   // of a block
    Finish f;
};

// Eight numbers of a row from column k on, zeros beyond its end.
__device__ __forceinline__ uint4 load8(const acrl_bf16* row, int k, int K) {
    uint32_t v[4] = {};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (k + j < K) v[j >> 1] |= uint32_t(row[k + j]) << (j & 1) * 16;
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// Eight numbers, or zeros, without a branch around the load; of the weight, which a CTA reads once, past L1.
template <bool ONCE>
__device__ __forceinline__ uint4 eight(const acrl_bf16* p, bool there) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (ONCE)
        asm volatile(
            "{\n .reg .pred q;\n setp.ne.b32 q, %5, 0;\n @q ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
            : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w)
            : "l"(p), "r"(uint32_t(there)));
    else
        asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %5, 0;\n @q ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
                     : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w)
                     : "l"(p), "r"(uint32_t(there)));
    return v;
}

__device__ __forceinline__ void mma_16x8(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// T: eights of x's rows, of all or of each of the BLOCKS that they are cut into.
template <int T, bool BLOCKS>
__global__ void __launch_bounds__(kThreads, T == 1 ? 3 : 2) few_kernel(const __grid_constant__ FewArgs A) {
    __shared__ float red[kWarps][8 * T][kW + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int block = BLOCKS ? int(blockIdx.x) / A.ctas : 0;
    const int n0 = (int(blockIdx.x) - block * A.ctas) * kW, m0 = block * 8 * T, M = BLOCKS ? min(A.M - m0, 8 * T) : A.M, K = A.K;
    const acrl_bf16* X = A.x + m0 * A.ldx;
    const acrl_bf16* w0 = A.w + int64_t(min(n0 + g, A.N - 1)) * A.ldw;
    const acrl_bf16* w1 = A.w + int64_t(min(n0 + g + 8, A.N - 1)) * A.ldw;
    // The weight's first columns on their way to L2 before the launch before this one has ended.  (L2 is where all writes go: what
    // that launch still writes of them is what the loads will find.)
    if (warp * kTurn < K) {
        asm volatile("prefetch.global.L2 [%0];" ::"l"(w0 + min(warp * kTurn + 32 * t, K - 1)));
        asm volatile("prefetch.global.L2 [%0];" ::"l"(w1 + min(warp * kTurn + 32 * t, K - 1)));
    }
    grid_begin();
    float c[T][4] = {};
    const int whole = K & ~7;
    for (int k0 = warp * kTurn; k0 < whole; k0 += kWarps * kTurn) {
        uint4 a[kAhead], b[kAhead], x[T][kAhead];
        // With eight rows of x three CTAs are resident and a thread has 80 registers: predicates for the loads would not fit (1 x
        // 16,384 x 4,096 26.4 us against 22.5), and the sum's end is gone through slab by slab instead.
        if (T == 1 && k0 + kTurn > whole) {
#pragma unroll 1
            for (int k = k0 + 8 * t; k < k0 + 8 * t + kTurn && k - 8 * t < whole; k += 32) {
                const uint4 a = eight<true>(w0 + k, k < whole), b = eight<true>(w1 + k, k < whole);
                const uint4 x = eight<false>(X + g * A.ldx + k, g < M && k < whole);
                mma_16x8(c[0], a.x, b.x, a.y, b.y, x.x, x.y);
                mma_16x8(c[0], a.z, b.z, a.w, b.w, x.z, x.w);
            }
            break;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = k0 + 32 * i + 8 * t;
            a[i] = T == 1 ? ld_stream(reinterpret_cast<const uint4*>(w0 + k)) : eight<true>(w0 + k, k < whole);
            b[i] = T == 1 ? ld_stream(reinterpret_cast<const uint4*>(w1 + k)) : eight<true>(w1 + k, k < whole);
        }
#pragma unroll
        for (int r = 0; r < T; ++r)
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int k = k0 + 32 * i + 8 * t;
                const acrl_bf16* p = X + (8 * r + g) * A.ldx + k;
                if (T == 1) x[r][i] = g < M ? __ldg(reinterpret_cast<const uint4*>(p)) : make_uint4(0u, 0u, 0u, 0u);
                else x[r][i] = eight<false>(p, 8 * r + g < M && k < whole);
            }
        // each turn's products in a sum of their own: the tensor cores cut partial sums off, an error that grows with their number
#pragma unroll
        for (int r = 0; r < T; ++r) {
            float d[4] = {};
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                mma_16x8(d, a[i].x, b[i].x, a[i].y, b[i].y, x[r][i].x, x[r][i].y);
                mma_16x8(d, a[i].z, b[i].z, a[i].w, b[i].w, x[r][i].z, x[r][i].w);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) c[r][j] += d[j];
        }
    }
    if (warp == kWarps - 1 && whole < K) {   // fewer than eight columns: the first of a row's lanes has them
        const uint4 a = load8(w0, whole, t == 0 ? K : 0), b = load8(w1, whole, t == 0 ? K : 0);
#pragma unroll
        for (int r = 0; r < T; ++r) {
            const uint4 x = load8(X + (8 * r + g) * A.ldx, whole, t == 0 && 8 * r + g < M ? K : 0);
            mma_16x8(c[r], a.x, b.x, a.y, b.y, x.x, x.y);
            mma_16x8(c[r], a.z, b.z, a.w, b.w, x.z, x.w);
        }
    }
#pragma unroll
    for (int r = 0; r < T; ++r) {
        red[warp][8 * r + 2 * t][g] = c[r][0];
        red[warp][8 * r + 2 * t + 1][g] = c[r][1];
        red[warp][8 * r + 2 * t][g + 8] = c[r][2];
        red[warp][8 * r + 2 * t + 1][g + 8] = c[r][3];
    }
    __syncthreads();
    const int64_t n = n0 + (threadIdx.x & (kW - 1));
    const Finish& f = A.f;
#pragma unroll 1
    for (int i = threadIdx.x / kW; i < M && n < A.N; i += kThreads / kW) {
        const int64_t m = m0 + i;
        float v[1] = {};
#pragma unroll
        for (int j = 0; j < kWarps; ++j) v[0] += red[j][i][n - n0];
        if (f.bias) v[0] += load_float(f.bias, f.bias_f32, n);
        if (f.pre) f.pre[m * f.ldp + n] = to_bf16(v[0]);
        apply(f.act, v);
        if (f.residual) v[0] += load_float(f.residual, f.residual_f32, m * f.ldr + n);
        store_float(f.out, f.out_f32, m * f.ldo + n, v[0]);
        if (T <= 2) break;
    }
}

constexpr int kMostFew = 256, kBlock = 32;   // rows of x, and of a block of them

}  // namespace

// Above 16 rows the CTAs' loads of x count: with those of their 16 rows of the weight they come from L2 at some 80 bytes a
// nanosecond of an SM, and a CTA has 0.4 us more.  Tensor memory's way reads x for 128 rows of the weight at once and HBM bounds
// it, 5.9 TB/s, but it takes 3.5 us more to begin and to end, and of up to 128 rows 2 more where its tiles are so few that their
// sums are split.  Measured, us here and there: 32 x 2,048 x 2,048 4.7 and 8.8, 64 x 2,048 x 2,048 6.3 and 9.7, 100 x 1,000 x 1,000
// 4.5 and 8.2, 256 x 768 x 768 5.8 and 6.6, 128 x 4,096 x 512 6.9 and 10.1, 32 x 4,096 x 4,096 11.1 and 12.3; 48 x 4,096 x 4,096 18 and
// 13, 64 x 1,024 x 5,120 9.8 and 8.4, 256 x 1,000 x 1,000 8.2 and 7.7.
bool linear_few_rows(int64_t M, int64_t N, int64_t K) {
    if (M <= 0 || M > kMostFew || N <= 0 || K <= 0) return false;
    if (M <= 16) return true;
    const int64_t blocks = (M + kBlock - 1) / kBlock, T = blocks > 1 ? kBlock / 8 : (M + 7) / 8;
    const double cta = double(kW + 8 * T) * 2.0 * double(K) / 80.0 + 400.0;
    const double split = M <= 128 && (N + 127) / 128 * 4 <= 152 ? 2000.0 : 0.0;
    return std::max(1.0, double(blocks * ((N + kW - 1) / kW)) / 152.0) * cta < 3500.0 + split + 2.0 * double(N) * double(K) / 5900.0;
}

acrl_status linear_few(const acrl_bf16* x, int64_t M, int64_t K, int64_t ldx, const acrl_bf16* w, int64_t N, int64_t ldw, const Finish& f,
                       cudaStream_t s) {
    const int64_t blocks = (M + kBlock - 1) / kBlock, ctas = (N + kW - 1) / kW, T = blocks > 1 ? kBlock / 8 : (M + 7) / 8;
    const FewArgs A{x, w, ldx, ldw, int(M), int(N), int(K), int(ctas), f};
    return launch(blocks > 1 ? few_kernel<4, true> : T == 1 ? few_kernel<1, false> : T == 2 ? few_kernel<2, false> :
                  T == 3 ? few_kernel<3, false> : few_kernel<4, false>, blocks * ctas, kThreads, 0, 0, s, A);
}

}  // namespace acrl
