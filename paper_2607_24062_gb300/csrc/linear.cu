// acrl_linear and acrl_linear_backward: a bf16 layer with bias, activation and residual, and its gradients.
#include <algorithm>

#include "acrl_host.h"
#include "bf16_product.cuh"
#include "linear.cuh"

namespace acrl {
namespace {

constexpr int64_t kAloneRows = 128;  // rows that become a CTA's columns

// A tile's accumulators on their way out.  Pair: a lane has a row of the result and 32 of its columns.  Alone: p is the
// weight, a lane has a column of the result and 32 rows, and a warp's stores are of neighbours.
template <bool PAIR>
struct LinearEpilogue {
    Finish f;
    float* parts;                   // of the tiles

    __device__ __forceinline__ void chunk(const Problem& pr, const Unit& t, const uint32_t (&r)[32], int row0, int col0, int rows,
                                          int cols, const WarpOut& out) const {
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
        if constexpr (PAIR) {
            if (pr.parts > 1) {
                const int high = pr.tile_rows(), wide = pr.tile_cols();
                out.store(parts + (int64_t(t.all) * pr.parts + t.part) * high * wide, wide, rows > 0 ? high : 0, wide, v,
                          row0 - t.tp * high, col0 - t.tq * wide);
                return;
            }
            const int row = row0 + out.lane;
            if (f.bias) {
                const float b = col0 + out.lane < cols ? load_float(f.bias, f.bias_f32, col0 + out.lane) : 0.f;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(0xffffffffu, b, j);
            }
            if (f.pre) out.store(f.pre, f.ldp, rows, cols, v, row0, col0);
            apply(f.act, v);
            if (f.residual && row < rows) {
                float add[32];
                load_row(f.residual, f.residual_f32, row * f.ldr, col0, cols, add);
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] += add[j];
            }
            if (f.out_f32)
                out.store(static_cast<float*>(f.out), f.ldo, rows, cols, v, row0, col0);
            else
                out.store(static_cast<acrl_bf16*>(f.out), f.ldo, rows, cols, v, row0, col0);
        } else {
            const int64_t n = row0 + out.lane;
            if (n >= rows) return;
            const int count = cols - col0;   // of the result's rows that this chunk has, of 32
            if (pr.parts > 1) {
                float* to = parts + ((int64_t(t.all) * pr.parts + t.part) * pr.cols + col0 - t.tq * pr.cols) * pr.high + n - t.tp * pr.high;
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (j < count) to[j * pr.high] = v[j];
                return;
            }
            const float b = f.bias ? load_float(f.bias, f.bias_f32, n) : 0.f;
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += b;
            if (f.pre)
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (j < count) f.pre[(col0 + j) * f.ldp + n] = to_bf16(v[j]);
            apply(f.act, v);
            if (f.residual) {
                float add[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) add[j] = j < count ? load_float(f.residual, f.residual_f32, (col0 + j) * f.ldr + n) : 0.f;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] += add[j];
            }
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < count) store_float(f.out, f.out_f32, (col0 + j) * f.ldo + n, v[j]);
        }
    }
};

// The parts of the tiles in their order, and what follows; without parts the sum is empty.  A CTA has kJoinRows rows of a
// tile, a thread four columns of some.
constexpr int kJoinRows = 16;

__global__ void __launch_bounds__(256) join_kernel(Finish f, const float* parts, Problem pr, int M, int N) {
    grid_begin();
    const int high = pr.tile_rows(), wide = pr.tile_cols(), strips = (high + kJoinRows - 1) / kJoinRows;
    const int tile = int(blockIdx.x) / strips, strip = int(blockIdx.x) - tile * strips;
    const Unit t = tile_at(pr, tile);
    const int r0 = (pr.pair ? t.tp : t.tq) * high, c0 = (pr.pair ? t.tq : t.tp) * wide, quads = wide / 4;
    for (int i = threadIdx.x; i < kJoinRows * quads; i += 256) {
        const int r = strip * kJoinRows + i / quads, at = i % quads * 4, c = c0 + at;
        const int64_t row = r0 + r;
        if (r >= high || row >= M || c >= N) continue;
        float v[4] = {};
        const float* p = parts + (int64_t(tile) * pr.parts * high + r) * wide + at;
        for (int k = 0; k < pr.parts; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(p + int64_t(k) * high * wide);
            v[0] += x.x;
            v[1] += x.y;
            v[2] += x.z;
            v[3] += x.w;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (f.bias && c + j < N) v[j] += load_float(f.bias, f.bias_f32, c + j);
        auto store = [&](void* to, bool f32, int64_t ld) {
            if (c + 4 > N) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + j < N) store_float(to, f32, row * ld + c + j, v[j]);
            } else if (f32) {
                *reinterpret_cast<float4*>(static_cast<float*>(to) + row * ld + c) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
                *reinterpret_cast<uint2*>(static_cast<acrl_bf16*>(to) + row * ld + c) =
                    make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            }
        };
        if (f.pre) store(f.pre, false, f.ldp);
        apply(f.act, v);
        if (f.residual) {
            float add[4];
            load_row(f.residual, f.residual_f32, row * f.ldr, c, N, add);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += add[j];
        }
        store(f.out, f.out_f32, f.ldo);
    }
}

// How a product of M x N results over K is made: x has the rows, w the columns, either turned.
struct Plan {
    Shape shape;
    Cut cut;
    int64_t workspace;
};

Shape shape_of(int64_t M, int64_t N, int64_t K, bool x_turned, bool w_turned) {
    if (M > kAloneRows)   // blocks of 64 a CTA
        return Shape{true, M, N, K, 1, false, 1, 256, w_turned ? 128 : 64, w_turned ? 128 : 32, 2 * kRows};
    const int64_t to = x_turned ? 64 : 16;
    const int cols = int(std::max<int64_t>(1, (M + to - 1) / to) * to);
    return Shape{false, N, M, K, 1, false, 1, cols, cols, cols, kRows};
}

Plan plan_of(const Shape& s, const Cut& cut) { return Plan{s, cut, parts_bytes(s, cut)}; }

// Alone, the tiles of whole sums have fewer than 128 rows of p where the last round is fuller then, which HBM bounds like the
// others (the MMAs are of 128 all the same).  Measured, us with 128 and with these: 48 x 40,960 x 4,096 67.5 and 59.6, 100 x
// 28,672 x 4,096 55.6 and 47.6, 48 x 20,000 x 1,024 14.4 and 13.4; where nothing is gained, as with 16,384 columns, 128 stay.
Plan plan_of(Shape s, bool any_high) {
    Plan best = plan_of(s, best_cut(s));
    if (s.pair || !any_high || best.cut.parts > 1) return best;
    int64_t least = cut_cycles(s, best.cut);
    for (s.high = kRows - 8; s.high >= kRows / 2; s.high -= 8) {
        Cut c = best.cut;
        c.tiles = s.tiles(c.cols);
        const int64_t cost = cut_cycles(s, c);
        if (cost >= least) continue;
        least = cost;
        best = plan_of(s, c);
    }
    return best;
}

Plan plan_of(int64_t M, int64_t N, int64_t K, bool x_turned, bool w_turned) {
    return plan_of(shape_of(M, N, K, x_turned, w_turned), !w_turned);
}

// Both products of a backward pass, in one launch where both are made by pairs.
struct BackwardPlan {
    Plan dx, dw;
    bool together;
};

BackwardPlan plan_backward(int64_t M, int64_t N, int64_t K) {
    const Shape sx = shape_of(M, K, N, false, true), sw = shape_of(N, K, M, true, true);
    if (!sx.pair || !sw.pair || K == 0) return BackwardPlan{plan_of(sx, false), plan_of(sw, false), false};
    Cut cx = {}, cw = {};
    best_cuts(sx, sw, cx, cw);
    return BackwardPlan{plan_of(sx, cx), plan_of(sw, cw), true};
}

// Plans of the sizes that the calling thread asked for last: a call asks twice, for its workspace and for its launches.
template <typename P, typename F>
P planned(int64_t M, int64_t N, int64_t K, F make) {
    struct Known {
        int64_t M, N, K;
        P plan;
    };
    static thread_local Known known[4] = {{-1, -1, -1, P{}}, {-1, -1, -1, P{}}, {-1, -1, -1, P{}}, {-1, -1, -1, P{}}};
    static thread_local int turn = 0;
    for (const Known& k : known)
        if (k.M == M && k.N == N && k.K == K) return k.plan;
    turn = (turn + 1) % 4;
    known[turn] = Known{M, N, K, make()};
    return known[turn].plan;
}

Plan plan_linear(int64_t M, int64_t N, int64_t K) {
    return planned<Plan>(M, N, K, [&] { return plan_of(M, N, K, false, false); });
}

// One product: x has the result's rows, w its columns.
struct Product {
    const Plan& plan;
    Matrix x, w;
    int64_t K;
    const Finish& f;
    float* parts;
};

// An fp32 result of more than one run, and any of a very long sum.
bool has_runs(const Product& p) { return p.plan.shape.slabs() > (p.f.out_f32 ? kRun : kLongest); }

template <bool PAIR, int NP>
bool describe(ProductLaunch<NP, 1, LinearEpilogue<PAIR>>& l, int at, const Product& d) {
    const Matrix &p = PAIR ? d.x : d.w, &q = PAIR ? d.w : d.x;
    const Cut& cut = d.plan.cut;
    l.pr[at] = problem_of(d.plan.shape, cut, p.turned, q.turned, has_runs(d));
    l.epi[at].f = d.f;
    l.epi[at].parts = d.parts;
    return operand_map(&l.p[at], p, d.K, PAIR ? kRows : d.plan.shape.high) && operand_map(&l.q[at], q, d.K, PAIR ? cut.cols / 2 : cut.cols);
}

acrl_status join(const Problem& pr, const Product& d, cudaStream_t s) {
    const int64_t ctas = d.plan.cut.tiles * ((pr.tile_rows() + kJoinRows - 1) / kJoinRows);
    if (ctas > kMaxGrid) return ACRL_ERR_INVALID_ARG;
    return launch(join_kernel, ctas, 256, 0, 0, s, d.f, static_cast<const float*>(d.parts), pr, int(d.x.rows), int(d.w.rows));
}

template <bool PAIR, int NP>
acrl_status run_products(const Product (&d)[NP], const ColumnSums& sums, int32_t* flags, cudaStream_t s) {
    ProductLaunch<NP, 1, LinearEpilogue<PAIR>> l = {};
    l.sums = sums;
    bool runs = false;
    for (int i = 0; i < NP; ++i) {
        if (!units_fit(d[i].plan.cut)) return ACRL_ERR_INVALID_ARG;
        if (!describe<PAIR, NP>(l, i, d[i])) return ACRL_ERR_CUDA;
        runs = runs || has_runs(d[i]);
    }
    acrl_status st = runs ? launch_product<PAIR, true>(l, flags, s) : launch_product<PAIR, false>(l, flags, s);
    for (int i = 0; i < NP && st == ACRL_OK; ++i)
        if (d[i].plan.cut.parts > 1) st = join(l.pr[i], d[i], s);
    return st;
}

// f(x w^T + ...): K > 0 columns, or an empty sum.
acrl_status product(const Product& d, const ColumnSums& sums, int32_t* flags, cudaStream_t s) {
    if (d.K == 0) {   // of no rows, or of no columns: there are no columns' sums to join beside it
        const Cut& c = d.plan.cut;
        if (!units_fit(c)) return ACRL_ERR_INVALID_ARG;
        Problem pr = problem_of(d.plan.shape, c, d.x.turned, d.w.turned, false);
        pr.parts = 0;
        return join(pr, d, s);
    }
    const Product one[1] = {d};
    return d.plan.shape.pair ? run_products<true, 1>(one, sums, flags, s) : run_products<false, 1>(one, sums, flags, s);
}

// g = dy f'(u), rounded, and the columns' sums of the unrounded.  A lane has eight columns, a warp 256, and the eight warps of a
// CTA take its rows in turn, four at a time in flight; their sums meet in shared memory.  6 bytes an element
// (2 without an activation), but its arithmetic is in the way of HBM's rate: 4,096 x 16,384 with GELU 76-78 us, 5.2 TB/s, and 89 before
// the activations took packed instructions.
constexpr int kSlopeCols = 256, kSlopeAhead = 4;

// Rows of a CTA: as many as still make a few CTAs for each SM.
int64_t slope_rows(int64_t M, int64_t N) { return (M + 127) / 128 * ((N + kSlopeCols - 1) / kSlopeCols) >= 1024 ? 128 : 32; }

template <int ACT>
__global__ void __launch_bounds__(256) slope_kernel(const acrl_bf16* dy, int64_t lddy, const acrl_bf16* pre, int64_t ldp, int M,
                                                    int N, int rows, acrl_bf16* g, int64_t ldg, float* sums, int64_t ldsums) {
    __shared__ float part[8][kSlopeCols];
    grid_begin();
    const int tiles = (N + kSlopeCols - 1) / kSlopeCols, at = int(blockIdx.x) / tiles;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = int(int64_t(blockIdx.x) - int64_t(at) * tiles) * kSlopeCols + lane * 8;
    const int64_t m0 = int64_t(at) * rows, end = min(int64_t(M), m0 + rows);
    const bool whole = c + 8 <= N;
    float sum[8] = {};
    // g's eight values of a row; beyond the matrix there are zeros in dy, and nothing is stored
    auto row = [&](int64_t m, const uint4& d, const uint4& u) {
        const uint32_t dw[4] = {d.x, d.y, d.z, d.w}, uw[4] = {u.x, u.y, u.z, u.w};
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bf16_lo(dw[j]);
            v[2 * j + 1] = bf16_hi(dw[j]);
            if (ACT != ACRL_ACT_NONE) {   // the same with and without g: no fma into the sum
                float u[2] = {bf16_lo(uw[j]), bf16_hi(uw[j])};
                act_slope2<ACT>(u);
                v[2 * j] = __fmul_rn(v[2 * j], u[0]);
                v[2 * j + 1] = __fmul_rn(v[2 * j + 1], u[1]);
            }
        }
        if (ACT != ACRL_ACT_NONE && g) {
            acrl_bf16* to = g + m * ldg + c;
            if (whole) {
                *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                                           pack_bf16x2(v[6], v[7]));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < N) to[j] = to_bf16(v[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[j];
    };
    auto load = [&](const acrl_bf16* p) {
        if (whole) return *reinterpret_cast<const uint4*>(p);
        uint32_t w[4] = {};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < N) w[j >> 1] |= uint32_t(p[j]) << (j & 1) * 16;
        return make_uint4(w[0], w[1], w[2], w[3]);
    };
    if (c < N) {
        for (int64_t m = m0 + warp; m < end; m += 8 * kSlopeAhead) {
            uint4 d[kSlopeAhead], u[kSlopeAhead] = {};
#pragma unroll
            for (int i = 0; i < kSlopeAhead; ++i)
                if (m + 8 * i < end) {
                    d[i] = load(dy + (m + 8 * i) * lddy + c);
                    if (ACT != ACRL_ACT_NONE) u[i] = load(pre + (m + 8 * i) * ldp + c);
                }
#pragma unroll
            for (int i = 0; i < kSlopeAhead; ++i)
                if (m + 8 * i < end) row(m + 8 * i, d[i], u[i]);
        }
    }
    if (!sums) return;   // the same for the CTA
#pragma unroll
    for (int j = 0; j < 8; ++j) part[warp][lane * 8 + j] = sum[j];
    __syncthreads();
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) total += part[w][threadIdx.x];
    sums[at * ldsums + (int64_t(blockIdx.x) - int64_t(at) * tiles) * kSlopeCols + threadIdx.x] = total;
}

// The columns' sums where no product is made beside.
__global__ void __launch_bounds__(32) sums_kernel(ColumnSums sums) {
    grid_begin();
    sums.run(int(blockIdx.x), int(gridDim.x));
}

bool dtype_ok(acrl_dtype d) { return d == ACRL_BF16 || d == ACRL_F32; }
bool on_its_type(const void* p, bool f32) { return (reinterpret_cast<uintptr_t>(p) & (f32 ? 3 : 1)) == 0; }
bool matrix_ok(const void* p, int64_t cols, int64_t ld) { return p && aligned16(p) && ld >= cols && (ld & 7) == 0; }

// A call's sizes; of a matrix of more than 2^48 numbers, which no GPU holds, the bytes of the workspace could leave 64 bits.
bool sizes_ok(int64_t M, int64_t N, int64_t K) {
    auto fits = [](int64_t a, int64_t b) { return double(a) * double(b) < 281474976710656.0; };
    return M >= 0 && N >= 0 && K >= 0 && M <= kMostSize && N <= kMostSize && K <= kMostSize && fits(M, N) && fits(M, K) && fits(N, K);
}

// The backward's workspace: g, the columns' sums of its parts, the parts of the products' split sums.
struct BackwardParts {
    BackwardPlan plan;
    int64_t ldg, rows, count, ldsums;   // of a part of the columns' sums, and how many there are
    int64_t sums, dx, dw, end;          // bytes
    BackwardParts(int64_t M, int64_t N, int64_t K)
        : plan(planned<BackwardPlan>(M, N, K, [&] { return plan_backward(M, N, K); })) {
        ldg = (N + 7) / 8 * 8;
        sums = M * ldg * 2;
        rows = slope_rows(M, N);
        count = (M + rows - 1) / rows;
        ldsums = (N + kSlopeCols - 1) / kSlopeCols * kSlopeCols;
        dx = sums + count * ldsums * 4;
        dw = dx + plan.dx.workspace;
        end = dw + plan.dw.workspace;
    }
};

}  // namespace
}  // namespace acrl

using namespace acrl;

extern "C" int64_t acrl_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N < 0 || K < 0) return -1;
    return M == 0 || N == 0 || K == 0 || !sizes_ok(M, N, K) || linear_few_rows(M, N, K) ? 0 : plan_linear(M, N, K).workspace;
}

extern "C" acrl_status acrl_linear(const acrl_bf16* x, int64_t M, int64_t K, int64_t ldx, const acrl_bf16* w, int64_t N, int64_t ldw,
                                   const void* bias, acrl_dtype bias_dtype, acrl_activation act, const void* residual,
                                   acrl_dtype residual_dtype, int64_t ldr, acrl_bf16* pre, int64_t ldp, void* out,
                                   acrl_dtype out_dtype, int64_t ldo, void* workspace, int64_t workspace_bytes, int32_t* dev_flags,
                                   acrl_stream stream) {
    if (!sizes_ok(M, N, K)) return ACRL_ERR_INVALID_ARG;
    if (act < ACRL_ACT_NONE || act > ACRL_ACT_SILU || !dtype_ok(out_dtype) || (bias && !dtype_ok(bias_dtype)) ||
        (residual && !dtype_ok(residual_dtype)))
        return ACRL_ERR_INVALID_ARG;
    if (workspace_bytes < acrl_linear_workspace_bytes(M, N, K)) return ACRL_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return ACRL_OK;
    if (!matrix_ok(out, N, ldo) || (residual && !matrix_ok(residual, N, ldr)) || (pre && !matrix_ok(pre, N, ldp)))
        return ACRL_ERR_INVALID_ARG;
    if (K > 0 && (!matrix_ok(x, K, ldx) || !matrix_ok(w, K, ldw))) return ACRL_ERR_INVALID_ARG;
    // each lane adds what it has read before it stores, if the two are the same matrix
    if (residual == out && (residual_dtype != out_dtype || (M > 1 && ldr != ldo))) return ACRL_ERR_INVALID_ARG;
    if (bias && !on_its_type(bias, bias_dtype == ACRL_F32)) return ACRL_ERR_INVALID_ARG;
    const int64_t need = acrl_linear_workspace_bytes(M, N, K);
    if (need > 0 && (!workspace || !aligned16(workspace))) return ACRL_ERR_INVALID_ARG;
    auto used = [](bool is, const void* p) { return is ? p : nullptr; };
    if (!operands_on_current_device({out, used(K > 0, x), used(K > 0, w), used(need > 0, workspace), bias, residual, pre}, true))
        return ACRL_ERR_INVALID_ARG;
    const Finish f{bias, residual, out, pre, ldr, ldp, ldo, int(act), bias_dtype == ACRL_F32, residual_dtype == ACRL_F32,
                   out_dtype == ACRL_F32};
    if (linear_few_rows(M, N, K)) return linear_few(x, M, K, ldx, w, N, ldw, f, reinterpret_cast<cudaStream_t>(stream));
    const Plan plan = plan_linear(M, N, K);
    return product({plan, Matrix{x, M, ldx, false, 1, M * ldx, 0}, Matrix{w, N, ldw, false, 1, N * ldw, 0}, K, f, static_cast<float*>(workspace)},
                   ColumnSums{}, dev_flags, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" int64_t acrl_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    return M < 0 || N < 0 || K < 0 ? -1 : sizes_ok(M, N, K) ? BackwardParts(M, N, K).end : 0;
}

extern "C" acrl_status acrl_linear_backward(const acrl_bf16* dy, int64_t M, int64_t N, int64_t lddy, const acrl_bf16* x, int64_t K,
                                            int64_t ldx, const acrl_bf16* w, int64_t ldw, acrl_activation act,
                                            const acrl_bf16* pre, int64_t ldp, void* dx, acrl_dtype dx_dtype, int64_t lddx, void* dw,
                                            acrl_dtype dw_dtype, int64_t lddw, float* dbias, void* workspace,
                                            int64_t workspace_bytes, int32_t* dev_flags, acrl_stream stream) {
    if (!sizes_ok(M, N, K)) return ACRL_ERR_INVALID_ARG;
    if (act < ACRL_ACT_NONE || act > ACRL_ACT_SILU || (dx && !dtype_ok(dx_dtype)) || (dw && !dtype_ok(dw_dtype)))
        return ACRL_ERR_INVALID_ARG;
    const BackwardParts parts(M, N, K);
    if (workspace_bytes < parts.end) return ACRL_ERR_INVALID_ARG;
    const bool has_dx = dx && M > 0 && K > 0, has_dw = dw && N > 0 && K > 0, has_g = M > 0 && N > 0;
    if ((has_dx && !matrix_ok(dx, K, lddx)) || (has_dw && !matrix_ok(dw, K, lddw))) return ACRL_ERR_INVALID_ARG;
    if (has_g && (!matrix_ok(dy, N, lddy) || (act != ACRL_ACT_NONE && !matrix_ok(pre, N, ldp)))) return ACRL_ERR_INVALID_ARG;
    if (act == ACRL_ACT_NONE && pre) return ACRL_ERR_INVALID_ARG;
    if (has_g && ((has_dx && !matrix_ok(w, K, ldw)) || (has_dw && !matrix_ok(x, K, ldx)))) return ACRL_ERR_INVALID_ARG;
    if (!has_dx && !has_dw && !(dbias && N > 0)) return ACRL_OK;
    if (has_g && (!workspace || !aligned16(workspace))) return ACRL_ERR_INVALID_ARG;
    if (dbias && !on_its_type(dbias, true)) return ACRL_ERR_INVALID_ARG;
    auto used = [](bool is, const void* p) { return is ? p : nullptr; };
    if (!operands_on_current_device({used(has_g, dy), used(has_g, workspace), used(has_g, pre), used(has_dx, dx), used(has_dw, dw),
                                     used(has_g && has_dx, w), used(has_g && has_dw, x), used(N > 0, dbias)}, true))
        return ACRL_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    uint8_t* base = static_cast<uint8_t*>(workspace);
    const acrl_bf16* g = dy;
    int64_t ldg = lddy;
    acrl_status st = ACRL_OK;
    ColumnSums columns = {};
    if (has_g && (act != ACRL_ACT_NONE || dbias)) {
        acrl_bf16* to = act == ACRL_ACT_NONE || !(has_dx || has_dw) ? nullptr : reinterpret_cast<acrl_bf16*>(base);
        float* sums = dbias ? reinterpret_cast<float*>(base + parts.sums) : nullptr;
        const int64_t tiles = (N + kSlopeCols - 1) / kSlopeCols;
        if (parts.count * tiles > kMaxGrid) return ACRL_ERR_INVALID_ARG;
        st = by_act(act, [&](auto a) {
            return launch(slope_kernel<a>, parts.count * tiles, 256, 0, 0, s, dy, lddy, pre, ldp, int(M), int(N), int(parts.rows), to,
                          parts.ldg, sums, parts.ldsums);
        });
        if (st != ACRL_OK) return st;
        if (to) {
            g = to;
            ldg = parts.ldg;
        }
        if (dbias) columns = ColumnSums{sums, parts.ldsums, int(parts.count), int(N), dbias};
        if (dbias && !has_dx && !has_dw) return launch(sums_kernel, std::min<int64_t>((N + 31) / 32, 4096), 32, 0, 0, s, columns);
    } else if (dbias && N > 0) {
        if (cudaMemsetAsync(dbias, 0, size_t(N) * 4, s) != cudaSuccess) return launch_status();
    }
    // without rows, or without columns of dy, the sums are empty
    Finish fx = {}, fw = {};
    fx.out = dx;
    fx.ldo = lddx;
    fx.out_f32 = dx_dtype == ACRL_F32;
    fw.out = dw;
    fw.ldo = lddw;
    fw.out_f32 = dw_dtype == ACRL_F32;
    const Product both[2] = {{parts.plan.dx, Matrix{g, M, ldg, false, 1, M * ldg, 0}, Matrix{w, K, ldw, true, 1, N * ldw, 0}, has_g ? N : 0, fx,
                              reinterpret_cast<float*>(base + parts.dx)},
                             {parts.plan.dw, Matrix{g, N, ldg, true, 1, M * ldg, 0}, Matrix{x, K, ldx, true, 1, M * ldx, 0}, has_g ? M : 0, fw,
                              reinterpret_cast<float*>(base + parts.dw)}};
    if (has_dx && has_dw && has_g && parts.plan.together) return run_products<true, 2>(both, columns, dev_flags, s);
    if (has_dx) st = product(both[0], columns, dev_flags, s);
    if (has_dw && st == ACRL_OK) st = product(both[1], has_dx ? ColumnSums{} : columns, dev_flags, s);
    return st;
}
