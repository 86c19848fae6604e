// acrl_policy_loss_grad_logits: a row's log-prob, the clipped policy loss with a KL
// term towards a reference policy, and its gradient with respect to the logits,
// in one pass over the logits.
//
//     lse = log sum_j e^(z_j),  logp = z_a - lse,  ratio = e^(logp - old_logp)
//     token_loss = clipped(ratio; coef) + kl_coef KL
//     grad_j = c (p_j - 1[j = a]) + kl_coef dKL/dz_j,   c = -d clipped / d logp
//
// KL over the vocabulary, against the reference's logits x (q = softmax(x)):
//     exact    sum p (log p - log q)     dKL/dz_j = p_j (log p_j - log q_j - KL)
//     reverse  sum q (log q - log p)     dKL/dz_j = p_j - q_j
// or from the reference's log-prob of the sampled token, d = logp - ref_logp:
//     k1 d,  k2 d^2 / 2,  k3 e^-d - 1 + d, whose slope in logp joins c.
//
// The gradient needs the sums of the whole row, so a row is swept twice; HBM sees it
// once.  A CTA takes one row and keeps what fits of it in shared memory between the sweeps
// (a bulk copy that runs while the threads load the rest); the rest of long rows comes from L2 the second
// time.  CTAs are as small as the row allows, so that several rows share an SM and one is read while another is
// written: HBM takes loads alone at 7.1 TB/s, stores alone at 4.0 and both together at 6.8.  Where rows are few, a
// cluster of CTAs shares each (one state per CTA goes through distributed shared memory).  HBM bounds it: 2 bytes of z,
// 2 of x and 2 of the gradient an element.
//
// Tried and slower, us for 2,632 rows of 151,936 columns with KL over the vocabulary (this: 480): persistent CTAs with a
// ring of chunks and one role per warp 580-620 (the roles' warps are too few to hide their latencies); persistent CTAs
// whose one pass writes a row's gradient and folds the next row 680; persistent CTAs that copy the next
// row's part early 494, and 192 KB more of a row in tensor memory 514: CTAs that stay begin and end their rows together
// and HBM reads and writes in turn; a cluster of two, four or eight CTAs a row 530-790.
#include <algorithm>
#include <cmath>

#include "acrl_device.cuh"
#include "acrl_host.h"
#include "mbarrier.cuh"
#include "row_lse.cuh"

namespace acrl {
namespace {

constexpr int kMaxCluster = 8;

enum Kind { kSampled, kExact, kReverse, kMean };   // which sums a row needs; kMean: the log-probs by themselves
template <Kind KIND>
constexpr bool kTwo = KIND == kExact || KIND == kReverse;   // two operands

struct PolicyArgs {
    const acrl_bf16 *z, *x;
    int64_t ldz, ldx;
    int V;
    int64_t T;
    int keep;      // vectors of each operand that a CTA keeps of a row in shared memory
    uint32_t first_wave;   // CTAs that begin one after another, and by how much
    int phase_ns;
    const int32_t* ids;
    const uint8_t* mask;
    const float *coef, *kl_coef, *old_logp, *ref_logp;
    int kl;        // acrl_kl
    float low, high, dual;
    acrl_bf16* grad;
    int64_t ldg;
    float *logp, *kl_out, *token_loss;
    int32_t* flags;
};

// A row's (or part's) running state in base 2: maxima, exponents U = max log2 e as whole numbers, sums
// against them, and the cross sum: exact  sum 2^(u - U) (z - x),  reverse  sum 2^(w - W) (x - z),  mean  sum 2^(u - U) z.
// `off` = sx - sz where U = W: KL of two close distributions needs the logarithm of the sums' ratio to better than the
// sums' own roundings, and the difference, summed by itself from the lanes on, is rounded at its own size.
struct State {
    float mz, U, sz, mx, W, sx, cross, off;   // mz, mx: of some columns, near the maxima
};

__device__ __forceinline__ State empty_state() { return State{-INFINITY, kLowestU, 0.f, -INFINITY, kLowestU, 0.f, 0.f, 0.f}; }

// log2 e less its nearest fp32 number: left out of the exponents, as here, it tilts lse by 1.3e-8 of the distribution's mean logit,
// and every log-prob with it, which a sum over a response's tokens carries; so lse takes it afterwards.  (In the exponents it
// would be lost to their rounding where a column lies far above those of U.)  The log-probs by themselves, bound by HBM, sum the
// mean too.  A loss's sums leave no room for another product a column (2-8 % of the time): halfway between lse, which is the
// mean and the entropy, and the sampled logit, which is the mean over tokens sampled from the row, is near enough, and for an
// unlikely token the difference is below the rounding of its log-prob.  p's and q's tilts cancel in the KL.  (Mean error over rows
// of 4,096 columns around 0 / 20, KL over the vocabulary: 9.4e-8 / 3.6e-7 before, 2e-8 / 3e-8 so.)
constexpr float kLog2eLow = 1.92596303e-8f;

// Whole numbers: sums are brought from one to another without a rounding.
__device__ __forceinline__ float exponent_of(float m) { return rintf(max_exponent<true>(m)); }
// That of the reference's columns: the policy's where they are near.
__device__ __forceinline__ float exponent_beside(float mx, float U) {
    const float W = exponent_of(mx);
    return fabsf(W - U) <= 16.f ? U : W;
}

// z - log(2^U s) in two parts.  U log 2 in two as well, the first of 15 bits, so that z less it is exact for every bf16 z of
// ordinary size and one rounding, at the size of what is computed from the parts, is left: a log-prob's difference from another
// is far smaller than either.  Beyond, by differences of the logits, which are as coarse as units there.
struct LogShare {
    float whole, rest;     // whole - rest
    __device__ __forceinline__ float value() const { return whole - rest; }
    __device__ __forceinline__ float less(float other) const { return (whole - other) - rest; }
};
__device__ __forceinline__ LogShare less_log(float z, float m, float U, float s) {
    constexpr float kHi = 22713.f / 32768.f, kLo = 1.42860682e-6f;   // log 2 = kHi + kLo
    const int bits = __float_as_int(s), e = (bits - 0x3f400000) >> 23;   // s = 2^e f, 3/4 <= f < 3/2
    const bool normal = s > 1e-37f && s < 3e38f;                         // else (0, infinite, NaN): its own logarithm
    const float f = normal ? __int_as_float(bits - e * (1 << 23)) : s, n = normal ? U + float(e) : U;
    const float l = kLn2 * log2f(f);
    if (fabsf(U) < 1e6f) return LogShare{fmaf(-n, kHi, z), fmaf(n, kLo, l)};
    return LogShare{z - m, l + kLn2 * (n - U - fmaf(m, kLog2e, -U))};
}

// That of a row's own logits, with what the exponents lack; z: the sampled one's (0 with kMean: -lse).
template <Kind KIND>
__device__ __forceinline__ LogShare log_share(float z, const State& row) {
    LogShare r = less_log(z, row.mz, row.U, row.sz);
    const float lse = kLn2 * (row.U + log2f(row.sz)), mean = row.cross / row.sz;
    r.rest = fmaf(kLog2eLow * kLn2, KIND != kMean ? 0.5f * (z + lse) : isfinite(mean) ? mean : lse, r.rest);
    return r;
}

// Two fp32 numbers in a register pair: sums, products and fused products of both in one instruction (issue bounds these
// sweeps next to HBM; one number at a time took 36 instructions a column pair where this takes some 16).
using Two = unsigned long long;

__device__ __forceinline__ Two two(float lo, float hi) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split(Two a, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a)); }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Two ex2_2(Two a) {
    float lo, hi;
    split(a, lo, hi);
    return two(ex2(lo), ex2(hi));
}
// d where the weight is not 0, 0 elsewhere.
__device__ __forceinline__ Two where_weighted(Two w, Two d) {
    float w0, w1, d0, d1;
    split(w, w0, w1);
    split(d, d0, d1);
    return two(w0 > 0.f ? d0 : 0.f, w1 > 0.f ? d1 : 0.f);
}
__device__ __forceinline__ Two widen(uint32_t pair) { return two(bf16_lo(pair), bf16_hi(pair)); }
__device__ __forceinline__ float sum_of(Two a) {
    float lo, hi;
    split(a, lo, hi);
    return lo + hi;
}

__device__ __forceinline__ uint32_t max_pairs(const uint4& v) {
    return max_bf16x2(max_bf16x2(v.x, v.y), max_bf16x2(v.z, v.w));
}

// A new running maximum m of one operand: its exponent, and the factor that brings sums to it.
__device__ __forceinline__ float raise_max(float m, float& mx, float& U) {
    const float Un = exponent_of(m), f = ex2(U - Un);
    U = Un;
    mx = m;
    return f;
}

// Fold N vectors of each operand: the careful way, with a running maximum, and where a column of probability 0 adds
// nothing to the cross sum, whatever the other side holds there (an infinite difference times 0 would be NaN).
template <Kind KIND, int N>
__device__ __forceinline__ void fold(State& st, const uint4 (&z)[N], const uint4 (&x)[N]) {
    uint32_t pm = max_pairs(z[0]);
#pragma unroll
    for (int k = 1; k < N; ++k) pm = max_bf16x2(pm, max_pairs(z[k]));
    const float vm = fmaxf(bf16_lo(pm), bf16_hi(pm));
    if (vm > st.mz) {
        const float f = raise_max(vm, st.mz, st.U);
        st.sz *= f;
        if (KIND != kReverse) st.cross *= f;
    }
    if constexpr (kTwo<KIND>) {
        uint32_t qm = max_pairs(x[0]);
#pragma unroll
        for (int k = 1; k < N; ++k) qm = max_bf16x2(qm, max_pairs(x[k]));
        const float wm = fmaxf(bf16_lo(qm), bf16_hi(qm));
        if (wm > st.mx) {
            const float f = raise_max(wm, st.mx, st.W);
            st.sx *= f;
            if (KIND == kReverse) st.cross *= f;
        }
    }
    const Two l2e = two(kLog2e, kLog2e), nU = two(-st.U, -st.U), nW = two(-st.W, -st.W), minus = two(-1.f, -1.f);
    Two sz = two(0.f, 0.f), sx = sz, cr = sz;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t zw[4] = {z[k].x, z[k].y, z[k].z, z[k].w}, xw[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const Two a = widen(zw[j]), e = ex2_2(fma2(a, l2e, nU));
            sz = add2(sz, e);
            if constexpr (KIND == kMean) cr = fma2(e, where_weighted(e, a), cr);
            if constexpr (kTwo<KIND>) {
                const Two b = widen(xw[j]), h = ex2_2(fma2(b, l2e, nW));
                sx = add2(sx, h);
                const Two w = KIND == kExact ? e : h, d = KIND == kExact ? fma2(b, minus, a) : fma2(a, minus, b);
                cr = fma2(w, where_weighted(w, d), cr);
            }
        }
    }
    st.sz += sum_of(sz);
    st.cross += sum_of(cr);
    if (kTwo<KIND>) st.sx += sum_of(sx);
}

// The quick way: sums against exponents that are fixed for a warp's share of the row, those of some of its columns.  Sums are as
// exact against any exponent from which they neither overflow nor vanish.  A warp that holds a lane's sum of kQuickMost or more
// (columns 44 above those of the exponents, an infinity, a column taken out on one side) folds its share again the careful way.
// The bound is for what comes after: 2^13 lanes of a cluster and factors of up to 2^32 between their exponents leave the row's
// sum below 2^109; and a factor that is flushed to 0, below 2^-126, has taken less than 2^-49 from a sum that is 2^-16 or more.
// Where the careful way is not needed both give the same cross sum's terms; the careful way costs nearly half as much again.
constexpr float kQuickMost = 0x1p64f;
// BY_VECTORS: a vector's columns are added up by themselves before they meet the lane's sum.  One by one beside a sum that holds a
// column far above them, small ones are lost, all in one direction: rows of 151,936 whose likeliest token has 0.9 had log-probs
// 5.7e-7 (256 threads) or 2.1e-7 (512) too high on average, 3e-8 and 6e-8 too low so.  In the statistics at no cost; from
// log-probs with 256 threads or more (2,632 x 151,936 319 us against 324, but 146,000 x 2,048 in CTAs of 32 216 against 207, where
// a lane adds up few columns); with KL over the vocabulary registers are short (2,632 x 151,936 485 against 475).
template <Kind KIND, bool BY_VECTORS>
struct Quick {
    float mz, mx;
    Two nU, nW, sz, sx, cr;

    // `z`, `x`: vectors of every lane of a warp.
    __device__ __forceinline__ void start(const uint4& z, const uint4& x) {
        mz = warp_max_of(max_pairs(z));
        const float U = exponent_of(mz);
        nU = two(-U, -U);
        sz = sx = cr = two(0.f, 0.f);
        if constexpr (kTwo<KIND>) {
            mx = warp_max_of(max_pairs(x));
            const float W = exponent_beside(mx, U);
            nW = two(-W, -W);
        }
    }
    static __device__ __forceinline__ float warp_max_of(uint32_t pair) {
        const int a = __float_as_int(fmaxf(bf16_lo(pair), bf16_hi(pair)));
        const int m = __reduce_max_sync(0xffffffffu, a ^ ((a >> 31) & 0x7fffffff));   // ordered as the numbers are
        return __int_as_float(m ^ ((m >> 31) & 0x7fffffff));
    }
    template <int N>
    __device__ __forceinline__ void fold(const uint4 (&z)[N], const uint4 (&x)[N]) {
        const Two l2e = two(kLog2e, kLog2e), minus = two(-1.f, -1.f);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t zw[4] = {z[k].x, z[k].y, z[k].z, z[k].w}, xw[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
            Two e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Two a = widen(zw[j]);
                e[j] = ex2_2(fma2(a, l2e, nU));
                if constexpr (!BY_VECTORS) sz = add2(sz, e[j]);
                if constexpr (KIND == kMean) cr = fma2(e[j], a, cr);     // NaN beside a column at -infinity: log_share() looks
                if constexpr (kTwo<KIND>) {
                    const Two b = widen(xw[j]), h = ex2_2(fma2(b, l2e, nW));
                    sx = add2(sx, h);
                    cr = KIND == kExact ? fma2(e[j], fma2(b, minus, a), cr) : fma2(h, fma2(a, minus, b), cr);
                }
            }
            if constexpr (BY_VECTORS) sz = add2(sz, add2(add2(e[0], e[1]), add2(e[2], e[3])));
        }
    }
    __device__ __forceinline__ State state() const {
        State s = empty_state();
        s.mz = mz;
        s.U = exponent_of(mz);
        s.sz = sum_of(sz);
        s.cross = sum_of(cr);
        if constexpr (kTwo<KIND>) {
            s.mx = mx;
            s.W = exponent_beside(mx, s.U);
            s.sx = sum_of(sx);
            s.off = s.sx - s.sz;
        }
        return s;
    }
};

// The state against common maxima: one exponential for each.
template <Kind KIND>
__device__ __forceinline__ State bring(const State& s, float mz, float mx) {
    State r;
    r.mz = mz;
    r.U = exponent_of(mz);
    const float f = ex2(s.U - r.U);
    r.sz = s.sz * f;
    if constexpr (!kTwo<KIND>) {
        r.mx = mx;
        r.W = r.sx = r.off = 0.f;
        r.cross = KIND == kMean ? s.cross * f : 0.f;
    } else {
        r.mx = mx;
        r.W = exponent_beside(mx, r.U);
        const float g = ex2(s.W - r.W);
        r.sx = s.sx * g;
        r.cross = s.cross * (KIND == kExact ? f : g);
        r.off = s.U == s.W && f == g ? s.off * f : r.sx - r.sz;
    }
    return r;
}

// All of a group of lanes' states, in every lane (fixed order).
template <Kind KIND, int LANES>
__device__ __forceinline__ State meet(State s) {
    float mz = s.mz, mx = s.mx;
#pragma unroll
    for (int m = LANES / 2; m >= 1; m >>= 1) {
        mz = fmaxf(mz, __shfl_xor_sync(0xffffffffu, mz, m));
        if (kTwo<KIND>) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, m));
    }
    s = bring<KIND>(s, mz, mx);
#pragma unroll
    for (int m = LANES / 2; m >= 1; m >>= 1) {
        s.sz += __shfl_xor_sync(0xffffffffu, s.sz, m);
        if (KIND != kSampled) s.cross += __shfl_xor_sync(0xffffffffu, s.cross, m);
        if (kTwo<KIND>) {
            s.sx += __shfl_xor_sync(0xffffffffu, s.sx, m);
            s.off += __shfl_xor_sync(0xffffffffu, s.off, m);
        }
    }
    return s;
}

__device__ __forceinline__ void bulk_in(void* dst, const void* src, uint32_t bytes, uint64_t* bar, uint64_t pol) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::
            "r"(smem_u32(dst)),
        "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(pol)
        : "memory");
}

__device__ __forceinline__ void st_peer4(const float4* p, uint32_t rank, const float4& v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(peer_addr(p, rank)), "f"(v.x), "f"(v.y), "f"(v.z),
                 "f"(v.w)
                 : "memory");
}

// What the gradient of a row's elements needs.
struct RowGrad {
    float U, W;        // lse log2 e of z, of x
    float c;           // of the one-hot term
    float k;           // kl_coef
    float c2;          // exact: c - k (lse_z - lse_x + KL); reverse: c + k
    float target;
    int a;
};

// SAFE: as in fold.
template <Kind KIND, bool SAFE>
__device__ __forceinline__ Two grad_two(Two z, Two x, const RowGrad& g) {
    const Two l2e = two(kLog2e, kLog2e), p = ex2_2(fma2(z, l2e, two(-g.U, -g.U)));
    if constexpr (!kTwo<KIND>) return mul2(p, two(g.c, g.c));
    if constexpr (KIND == kReverse) {
        const Two q = ex2_2(fma2(x, l2e, two(-g.W, -g.W)));
        return fma2(p, two(g.c2, g.c2), mul2(q, two(-g.k, -g.k)));
    }
    Two d = fma2(x, two(-1.f, -1.f), z);
    if constexpr (SAFE) d = where_weighted(p, d);
    return mul2(p, fma2(two(g.k, g.k), d, two(g.c2, g.c2)));
}

template <Kind KIND, bool SAFE>
__device__ __forceinline__ uint4 grad_vec8(const uint4& zv, const uint4& xv, const RowGrad& g, int rel) {
    const uint32_t zw[4] = {zv.x, zv.y, zv.z, zv.w}, xw[4] = {xv.x, xv.y, xv.z, xv.w};
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float lo, hi;
        split(grad_two<KIND, SAFE>(widen(zw[j]), widen(xw[j]), g), lo, hi);
        o[j] = pack_bf16x2(lo, hi);
    }
    if (unsigned(rel) < 8u) {
        const uint32_t target = pack_bf16x2(g.target, g.target), half = rel & 1 ? 0xffff0000u : 0xffffu;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j == rel >> 1) o[j] = (o[j] & ~half) | (target & half);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// A slice of a row: vectors [begin, end) of it, the first `kept` of them in shared memory; the last slice also has
// the columns beyond the whole vectors.
struct Slice {
    int begin, end, kept;
    bool last;
};

// What comes after a row's sums.
enum { kWrite, kWriteSafe, kFillZero, kFillNaN };

// The row's scalars from its merged state, in every lane of a warp; `writes`: this thread stores the row's outputs.
template <Kind KIND>
__device__ __forceinline__ int row_scalars(const PolicyArgs& A, int64_t t, const State& row, int a, float za, float xa,
                                           float c0, float kc, float old, float ref, bool writes, RowGrad& g) {
    const bool sums = row.sz > 0.f && isfinite(row.sz) && isfinite(row.mz);
    const LogShare share = log_share<KIND>(za, row);
    const float logp = share.value();
    float KL = 0.f, apart = 0.f, logq = 0.f;                                      // apart = lse_z - lse_x
    g.a = a;
    g.k = kc;
    g.U = row.U + log2f(row.sz);
    g.W = 0.f;
    float slope = 0.f;                                                            // of the sampled estimators, in logp
    if constexpr (kTwo<KIND>) {
        const float off = isfinite(row.off) ? row.off : row.sx - row.sz;
        const float ratio = row.U == row.W && fabsf(off) < 0.5f * row.sx ? log1pf(-off / row.sx) : kLn2 * log2f(row.sz / row.sx);
        apart = fabsf(row.U) < 1e6f && fabsf(row.W) < 1e6f
                    ? fmaf(row.U - row.W, kLn2, ratio)
                    : (row.mz - row.mx) + (ratio - kLn2 * (fmaf(row.mz, kLog2e, -row.U) - fmaf(row.mx, kLog2e, -row.W)));
        logq = less_log(xa, row.mx, row.W, row.sx).value();
        KL = KIND == kExact ? row.cross / row.sz - apart : row.cross / row.sx + apart;
        g.W = row.W + log2f(row.sx);
    } else {
        const float d = share.less(ref);
        if (A.kl == ACRL_KL_K1) {
            KL = d;
            slope = 1.f;
        } else if (A.kl == ACRL_KL_K2) {
            KL = 0.5f * d * d;
            slope = d;
        } else if (A.kl == ACRL_KL_K3) {
            const float e = expm1f(-d);
            KL = e + d;
            slope = -e;
        }
    }
    const float ratio = A.old_logp ? expf(share.less(old)) : 1.f;
    float surrogate = 0.f;
    g.c = 0.f;
    if (c0 != 0.f) {
        const bool up = c0 >= 0.f;
        const float capped = up ? fminf(ratio, 1.f + A.high) : fminf(fmaxf(ratio, 1.f - A.low), A.dual);
        const bool live = up ? ratio <= 1.f + A.high : (ratio >= 1.f - A.low && ratio <= A.dual);
        surrogate = -c0 * capped;
        if (live) g.c = c0 * ratio;
    }
    if (kc != 0.f && !kTwo<KIND>) g.c -= kc * slope;
    const float loss = kc != 0.f ? fmaf(kc, KL, surrogate) : surrogate;
    const bool defined = isfinite(logp) && sums, estimated = defined && isfinite(KL);   // the log-prob; the KL (0 if there is none)
    const bool carries = c0 != 0.f || kc != 0.f;
    // a NaN ratio is lost in the clip; one that is infinite, or a coefficient that is no number, shows in what it makes
    const bool undefined = carries && (!(!kTwo<KIND> ? defined : estimated) || (c0 != 0.f && isnan(ratio)) || !isfinite(loss) ||
                                       !isfinite(g.c));
    if (writes) {
        const float nan = __int_as_float(0x7fc00000);
        A.logp[t] = defined ? logp : nan;
        if (A.kl_out) A.kl_out[t] = estimated ? KL : nan;
        A.token_loss[t] = undefined ? nan : loss;
        if (!estimated || undefined) raise_flag(A.flags, ACRL_FLAG_NONFINITE);
    }
    if (!carries || undefined) return undefined ? kFillNaN : kFillZero;
    g.target = g.c * expm1f(logp);
    g.c2 = g.c;
    if (KIND == kExact) {
        g.c2 = fmaf(-kc, apart + KL, g.c);
        g.target = fmaf(kc * expf(logp), logp - logq - KL, g.target);
    }
    if (KIND == kReverse) {
        g.c2 = g.c + kc;
        g.target = fmaf(kc, expf(logp) - expf(logq), g.target);
    }
    return kWrite;
}

// A row's sampled column, or -1 for a row that is left out (masked, or an id outside the vocabulary).
__device__ __forceinline__ int column_of(const PolicyArgs& A, int64_t t) {
    const int a = A.ids[t];
    return (A.mask && A.mask[t] == 0) || a < 0 || a >= A.V ? -1 : a;
}

__device__ __forceinline__ bool was_careful(const float4* from) { return !isfinite(from[1].w); }
__device__ __forceinline__ void put(float4* to, const State& s, bool careful) {
    to[0] = make_float4(s.mz, s.U, s.sz, s.mx);
    to[1] = make_float4(s.W, s.sx, s.cross, careful ? INFINITY : s.off);   // finite where not careful
}
__device__ __forceinline__ State get(const float4* from) {
    const float4 a = from[0], b = from[1];
    return State{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}

template <int THREADS>
struct Shared {
    uint64_t landed;
    float4 warps[THREADS / 32][2];
    float4 parts[kMaxCluster][2];      // the CTAs' states
    RowGrad grad;
    int what;
};

template <Kind KIND, int THREADS>
struct Cta {
    static constexpr int kOps = !kTwo<KIND> ? 1 : 2;
    static constexpr int kWide = 4 / kOps;             // vectors of each operand that a thread has in flight
    static constexpr int kStep = kWide * THREADS;      // vectors of a step of the CTA
    const PolicyArgs& A;
    Shared<THREADS>& sh;
    const uint4 *sz, *sx;      // the part in shared memory
    int begin, n, kept;        // this CTA's vectors of a row: the first, how many, of them in shared memory
    bool last;                 // the columns beyond the whole vectors are this CTA's

    // one thread: the copies of the part in shared memory
    __device__ void load(int64_t t) const {
        if (kept == 0) return;
        const uint64_t once = policy_evict_first();
        const uint32_t bytes = uint32_t(kept) * 16u;
        mbar_expect_tx(&sh.landed, kOps * bytes);
        bulk_in(const_cast<uint4*>(sz), reinterpret_cast<const uint4*>(A.z + t * A.ldz) + begin, bytes, &sh.landed, once);
        if (kTwo<KIND>)
            bulk_in(const_cast<uint4*>(sx), reinterpret_cast<const uint4*>(A.x + t * A.ldx) + begin, bytes, &sh.landed, once);
    }

    // f(z, x) on the vectors that are not in shared memory: from global memory, kWide of each operand at a time, with an
    // L2 policy.
    template <typename Fn>
    __device__ __forceinline__ void rest(const uint4* gz, const uint4* gx, uint64_t pol, Fn f) const {
        int v = kept + threadIdx.x;
        for (; v + (kWide - 1) * THREADS < n; v += kStep) {
            uint4 z[kWide], x[kWide];
#pragma unroll
            for (int k = 0; k < kWide; ++k) {
                z[k] = ld_policy(gz + v + k * THREADS, pol);
                if constexpr (kTwo<KIND>) x[k] = ld_policy(gx + v + k * THREADS, pol);
                else x[k] = z[k];
            }
#pragma unroll
            for (int k = 0; k < kWide; ++k) f(z[k], x[k], v + k * THREADS);
        }
        for (; v < n; v += THREADS) {
            const uint4 z = ld_policy(gz + v, pol);
            uint4 x = z;
            if constexpr (kTwo<KIND>) x = ld_policy(gx + v, pol);
            f(z, x, v);
        }
    }
    __device__ __forceinline__ State fold_row(int64_t t, bool& careful) {
        const int tid = threadIdx.x;
        const acrl_bf16 *zr = A.z + t * A.ldz, *xr = !kTwo<KIND> ? zr : A.x + t * A.ldx;
        const uint4 *gz = reinterpret_cast<const uint4*>(zr) + begin, *gx = reinterpret_cast<const uint4*>(xr) + begin;
        // the columns beyond the whole vectors, one a thread: a vector whose other columns are both operands' lowest
        // number, which add nothing
        const bool odd = last && tid < (A.V & 7);
        const uint32_t low = 0xff7fff7fu;
        uint4 oz = make_uint4(low, low, low, low), ox = oz;
        if (odd) {
            oz.x = 0xff7f0000u | zr[(A.V & ~7) + tid];
            ox.x = !kTwo<KIND> ? oz.x : 0xff7f0000u | xr[(A.V & ~7) + tid];
        }
        const uint64_t again = policy_evict_last();
        Quick<KIND, KIND == kMean || (KIND == kSampled && THREADS >= 256)> q;
        bool started = false;
        auto first_of = [&](const uint4& z, const uint4& x) {
            if (!started) q.start(z, x);
            started = true;
        };
        // exponents from the first columns that the warp comes to: those of the rest, or of the part in shared memory
        if (kept + (tid & ~31) < n) {
            const int at = min(kept + tid, n - 1);
            const uint4 z = __ldg(gz + at);
            first_of(z, !kTwo<KIND> ? z : __ldg(gx + at));
            rest(gz, gx, again, [&](const uint4& z, const uint4& x, int) {
                const uint4 a[1] = {z}, b[1] = {x};
                q.fold(a, b);
            });
        }
        __syncwarp();
        if (kept > 0) {
            if (!mbar_try_wait(&sh.landed, 0) && !wait_phase_inline(&sh.landed, 0, nullptr)) raise_flag(A.flags, ACRL_FLAG_TIMEOUT);
            __syncwarp();
            if (!started) first_of(sz[min(tid, kept - 1)], sx[min(tid, kept - 1)]);
            int v = tid;
            for (; v + THREADS < kept; v += 2 * THREADS) {
                const uint4 z[2] = {sz[v], sz[v + THREADS]}, x[2] = {sx[v], sx[v + THREADS]};
                q.fold(z, x);
            }
            if (v < kept) {
                const uint4 z[1] = {sz[v]}, x[1] = {sx[v]};
                q.fold(z, x);
            }
        }
        __syncwarp();
        first_of(oz, ox);       // a row of fewer than eight columns
        if (odd) {
            const uint4 a[1] = {oz}, b[1] = {ox};
            q.fold(a, b);
        }
        __syncwarp();
        State st = q.state();
        const bool small = st.sz < kQuickMost && (!kTwo<KIND> || (st.sx < kQuickMost && fabsf(st.cross) < kQuickMost));
        careful = __any_sync(0xffffffffu, !small);     // (a NaN is not below the bound)
        if (careful) {          // once more, from where the vectors are now
            st = empty_state();
            auto f = [&](const uint4& z, const uint4& x, int) {
                const uint4 a[1] = {z}, b[1] = {x};
                fold<KIND, 1>(st, a, b);
            };
            for (int v = tid; v < kept; v += THREADS) f(sz[v], sx[v], v);
            rest(gz, gx, again, f);
            if (odd) f(oz, ox, 0);
        }
        __syncwarp();
        if (careful) st.off = st.sx - st.sz;
        return meet<KIND, 32>(st);
    }

    template <bool SAFE>
    __device__ __forceinline__ void write_part(uint4* out, const RowGrad& g, int rel0) const {
        int v = threadIdx.x;
        for (; v + THREADS < kept; v += 2 * THREADS) {
            const uint4 z[2] = {sz[v], sz[v + THREADS]}, x[2] = {sx[v], sx[v + THREADS]};
#pragma unroll
            for (int k = 0; k < 2; ++k)
                st_stream(out + v + k * THREADS, grad_vec8<KIND, SAFE>(z[k], x[k], g, rel0 - ((v + k * THREADS) << 3)));
        }
        if (v < kept) st_stream(out + v, grad_vec8<KIND, SAFE>(sz[v], sx[v], g, rel0 - (v << 3)));
    }
    template <bool SAFE>
    __device__ __forceinline__ void write_rest(int64_t t, uint4* out, acrl_bf16* gr, const RowGrad& g, int rel0) const {
        const acrl_bf16 *zr = A.z + t * A.ldz, *xr = !kTwo<KIND> ? zr : A.x + t * A.ldx;
        const uint4 *gz = reinterpret_cast<const uint4*>(zr) + begin, *gx = reinterpret_cast<const uint4*>(xr) + begin;
        auto f = [&](const uint4& z, const uint4& x, int v) {
            st_stream(out + v, grad_vec8<KIND, SAFE>(z, x, g, rel0 - (v << 3)));
        };
        rest(gz, gx, policy_evict_first(), f);
        if (last && threadIdx.x < (A.V & 7)) {
            const int j = (A.V & ~7) + int(threadIdx.x);
            const float z = bf16_to_float(zr[j]), x = !kTwo<KIND> ? 0.f : bf16_to_float(xr[j]);
            float v, none;
            split(grad_two<KIND, SAFE>(two(z, z), two(x, x), g), v, none);
            gr[j] = acrl_bf16(pack_bf16x2(j == g.a ? g.target : v, 0.f) & 0xffffu);
        }
    }
    __device__ __forceinline__ void fill(int64_t t, uint32_t pair) const {
        acrl_bf16* gr = A.grad + t * A.ldg;
        uint4* out = reinterpret_cast<uint4*>(gr) + begin;
        for (int v = threadIdx.x; v < n; v += THREADS) st_stream(out + v, make_uint4(pair, pair, pair, pair));
        if (last && threadIdx.x < (A.V & 7)) gr[(A.V & ~7) + threadIdx.x] = acrl_bf16(pair & 0xffffu);
    }
};

// Small CTAs work a row's scalars out in every warp, with one barrier; from 256 threads the first warp does, for a second
// barrier.
template <Kind KIND, int THREADS, int PER_SM>
__global__ void __launch_bounds__(THREADS, PER_SM) policy_kernel(const __grid_constant__ PolicyArgs A) {
    constexpr int kWarps = THREADS / 32;
    constexpr bool kEvery = THREADS < 256;
    extern __shared__ __align__(16) uint4 kept_rows[];
    __shared__ __align__(16) Shared<THREADS> sh;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int nct = int(cluster_size()), rank = int(cluster_rank());
    const int64_t t = int64_t(blockIdx.x) / nct;
    using C = Cta<KIND, THREADS>;
    const int nvec = A.V >> 3, per = (nvec + nct - 1) / nct;
    const int begin = min(nvec, rank * per), n = min(per, nvec - begin), kept = min(n, A.keep);
    C cta{A, sh, kept_rows, kept_rows + (C::kOps - 1) * A.keep, begin, n, kept, rank == nct - 1};
    grid_begin();
    if (blockIdx.x < A.first_wave) {          // see stagger()
        const uint64_t t0 = global_ns(), wait = uint64_t(A.phase_ns) * (PER_SM == 1 ? blockIdx.x & 3u : blockIdx.x / (A.first_wave / PER_SM));
        while (global_ns() - t0 < wait) __nanosleep(200);
    }
    const int a = column_of(A, t);
    if (a < 0) {     // left out: zeros (the same for the whole cluster)
        cta.fill(t, 0u);
        if (rank == 0 && tid == 0) {
            A.logp[t] = A.token_loss[t] = 0.f;
            if (A.kl_out) A.kl_out[t] = 0.f;
            if (!A.mask || A.mask[t]) raise_flag(A.flags, ACRL_FLAG_BAD_ID);
        }
        return;
    }
    if (tid == 0) {
        mbar_init(&sh.landed, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        cta.load(t);
    }
    // what there is one of per row, one number a lane: the sampled column of z and x, and the token's numbers
    float mine = 0.f;
    if ((kEvery || wid == 0) && lane < 6) {
        if (lane >= 2) {
            const float* p = lane == 2 ? A.coef : lane == 3 ? A.kl_coef : lane == 4 ? A.old_logp : A.ref_logp;
            if (p) mine = p[t];
        } else if (lane == 0 || kTwo<KIND>) {
            mine = bf16_to_float(lane == 0 ? A.z[t * A.ldz + a] : A.x[t * A.ldx + a]);
        }
    }
    __syncthreads();                         // the barrier is initialised
    if (nct > 1) cluster_sync();             // every CTA runs before its shared memory is written
    bool careful;
    State st = cta.fold_row(t, careful);
    RowGrad g;
    int what = kWrite;
    auto scalars = [&] {
        auto one = [&](int k) { return __shfl_sync(0xffffffffu, mine, k); };
        what = row_scalars<KIND>(A, t, st, a, one(0), one(1), one(2), one(3), one(4), one(5), rank == 0 && tid == 0, g);
        if (what == kWrite && careful) what = kWriteSafe;
    };
    const State none = empty_state();
    if (kWarps > 1) {
        if (lane == 0) put(sh.warps[wid], st, careful);
        __syncthreads();
        if (kEvery || wid == 0) {
            careful = __any_sync(0xffffffffu, lane < kWarps && was_careful(sh.warps[lane]));
            st = meet<KIND, 32>(lane < kWarps ? get(sh.warps[lane]) : none);
        }
    }
    if (nct > 1) {
        if (wid == 0 && lane < nct) {        // lane r hands this CTA's state to CTA r
            st_peer4(&sh.parts[rank][0], lane, make_float4(st.mz, st.U, st.sz, st.mx));
            st_peer4(&sh.parts[rank][1], lane, make_float4(st.W, st.sx, st.cross, careful ? INFINITY : st.off));
        }
        cluster_sync();
        const int k = lane & (kMaxCluster - 1);
        careful = __any_sync(0xffffffffu, k < nct && was_careful(sh.parts[k]));
        st = meet<KIND, kMaxCluster>(k < nct ? get(sh.parts[k]) : none);
    }
    if constexpr (kEvery) {
        scalars();
    } else {
        if (wid == 0) {
            scalars();
            if (lane == 0) {
                sh.grad = g;
                sh.what = what;
            }
        }
        __syncthreads();
        g = sh.grad;
        what = sh.what;
    }
    acrl_bf16* gr = A.grad + t * A.ldg;
    uint4* out = reinterpret_cast<uint4*>(gr) + begin;
    const int rel0 = a - (begin << 3);
    if (what == kWrite) {
        cta.template write_rest<false>(t, out, gr, g, rel0);
        cta.template write_part<false>(out, g, rel0);
    } else if (what == kWriteSafe) {
        cta.template write_rest<true>(t, out, gr, g, rel0);
        cta.template write_part<true>(out, g, rel0);
    } else {
        cta.fill(t, what == kFillNaN ? 0x7fc07fc0u : 0u);
    }
}

// The statistics alone: lse and the sampled token's log-prob, one row a CTA, nothing kept.  What the errors of a response's
// log-probs have in common adds up in its log ratio: sums against fixed exponents, added up by vectors, with the mean logit's share of
// log2 e, leave 2e-8 at 32,000 columns and 5e-8 at 151,936 (3e-7 rms, fp32's spacing at 8 to 16 being 9.5e-7), where an online
// log-softmax whose sums are rescaled at every new maximum leaves 1.5e-7.  4,096 rows of 151,936 in 176 us, 1.04 of the copy rate.
template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) logp_kernel(const __grid_constant__ PolicyArgs A, float* __restrict__ lse) {
    constexpr int kWarps = THREADS / 32;
    __shared__ __align__(16) Shared<THREADS> sh;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int64_t t = blockIdx.x;
    Cta<kMean, THREADS> cta{A, sh, nullptr, nullptr, 0, A.V >> 3, 0, true};
    grid_begin();
    const bool masked = A.mask && A.mask[t] == 0;
    if (masked) {
        if (tid == 0) lse[t] = A.logp[t] = 0.f;
        return;
    }
    const int a = A.ids[t];
    const bool in = a >= 0 && a < A.V;
    const float za = in && tid == 0 ? bf16_to_float(A.z[t * A.ldz + a]) : 0.f;
    bool careful;
    State st = cta.fold_row(t, careful);
    if (kWarps > 1) {
        if (lane == 0) put(sh.warps[wid], st, careful);
        __syncthreads();
        if (wid != 0) return;
        const State none = empty_state();
        st = meet<kMean, 32>(lane < kWarps ? get(sh.warps[lane]) : none);
    }
    if (tid != 0) return;
    const float l = -log_share<kMean>(0.f, st).value(), lp = in ? log_share<kMean>(za, st).value() : 0.f;
    if (!in) raise_flag(A.flags, ACRL_FLAG_BAD_ID);
    const bool fine = isfinite(l) && isfinite(lp);
    if (!fine) raise_flag(A.flags, ACRL_FLAG_NONFINITE);
    lse[t] = fine ? l : __int_as_float(0x7fc00000);
    A.logp[t] = fine ? lp : __int_as_float(0x7fc00000);
}

constexpr int kSmBytes = 227 * 1024;

// CTAs of long rows all begin together, and as their rows take equally long, HBM then reads and writes in turn.  So the first
// wave begins in phases: with one CTA an SM, quarters of a row's time apart; with more, the CTAs of an SM spread over it.
// 2,632 x 151,936 over the vocabulary 512 / 479 us, sampled 357 / 314; 6,102 x 65,544 316 / 296.  A call of fewer than
// kPhasedWaves waves would lose more than it gains.
constexpr int kPhasedWaves = 6;
constexpr int kSms = 152;
constexpr double kSmBytesPerNs = 44.6;    // an SM's share of HBM's rate

void stagger(PolicyArgs& A, int64_t bytes_moved, int per_sm) {
    if (A.T < int64_t(kPhasedWaves) * kSms * per_sm) return;
    A.first_wave = uint32_t(kSms * per_sm);
    A.phase_ns = int(double(bytes_moved) / kSmBytesPerNs * per_sm / (per_sm == 1 ? 4 : per_sm));
}

template <Kind KIND, int THREADS, int PER_SM>
acrl_status launch_rows(PolicyArgs A, int ctas, cudaStream_t s) {
    constexpr int kVec = !kTwo<KIND> ? 16 : 32;       // bytes of a vector of all operands
    const int nvec = A.V >> 3, slice = (nvec + ctas - 1) / ctas;
    constexpr int room = kSmBytes / PER_SM - 1024 - int(sizeof(Shared<THREADS>));   // the system takes 1 KB of each CTA's
    // whole steps of the CTA, where not all of it
    A.keep = slice <= room / kVec ? slice : room / kVec / (2 * THREADS) * (2 * THREADS);
    if (A.keep < slice && ctas == 1) stagger(A, int64_t(nvec) * (!kTwo<KIND> ? 32 : 48), PER_SM);
    auto* kernel = policy_kernel<KIND, THREADS, PER_SM>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, room) != cudaSuccess) return launch_status();
    const int64_t T = A.T, most = kMaxGrid / ctas;
    for (int64_t t = 0; t < T; t += most) {      // a grid's limit
        PolicyArgs B = A;
        auto at = [t](auto* p, int64_t ld = 1) { return p ? p + t * ld : p; };
        B.T = std::min(most, T - t);
        if (t > 0) B.first_wave = 0;
        B.z = at(A.z, A.ldz);
        B.x = at(A.x, A.ldx);
        B.grad = at(A.grad, A.ldg);
        B.ids = at(A.ids);
        B.mask = at(A.mask);
        B.coef = at(A.coef);
        B.kl_coef = at(A.kl_coef);
        B.old_logp = at(A.old_logp);
        B.ref_logp = at(A.ref_logp);
        B.logp = at(A.logp);
        B.kl_out = at(A.kl_out);
        B.token_loss = at(A.token_loss);
        const acrl_status st = launch(kernel, B.T * ctas, THREADS, size_t(A.keep) * kVec, ctas, s, B);
        if (st != ACRL_OK) return st;
    }
    return ACRL_OK;
}

template <Kind KIND>
acrl_status launch_policy(const PolicyArgs& A, cudaStream_t s) {
    const int64_t bytes = int64_t(A.V >> 3) * (!kTwo<KIND> ? 16 : 32);    // of a row
    // Few rows: several CTAs each, of 16 KB or more.  V = 151,936 over the vocabulary, 1 / 2 / 4 / 8 CTAs a row: 19 rows
    // 27.3 / 19.1 / 15.1 / 15.4 us, 76 rows 27.9 / 21.2 / 29.0 / 31.0, 152 rows 33.5 / 35.7 / 50.9 / 55.9.
    int ctas = 1;
    while (ctas < kMaxCluster && 2 * ctas * A.T <= kSms && bytes / ctas > 16 * 1024) ctas *= 2;
    // Threads by the row's bytes: few enough that rows share an SM, enough that a row's latency shows little.  600 MB of each
    // operand over the vocabulary (from log-probs), us:
    //     row      32         64         128        256        512        1,024
    //      9 KB    185 (210)  226 (213)
    //     11 KB    202 (225)  200 (203)  330 (282)
    //     18 KB    190 (286)  178 (206)  232 (220)
    //     24 KB               182 (247)  193 (203)  276 (278)
    //     44 KB               189 (301)  169 (213)  197 (222)
    //     52 KB                          197 (244)  185 (213)  244 (260)
    //     72 KB                          180 (254)  168 (207)  210 (232)
    //     90 KB                                     192 (236)  190 (217)
    //    310 KB                                     277 (380)  181 (256)  222 (302)
    //    350 KB                                     256 (386)  215 (284)  211 (313)
    //    600 KB                                     310 (497)  250 (349)  191 (343)
    const int64_t slice = bytes / ctas;
    if (slice <= 10 * 1024) return launch_rows<KIND, 32, 24>(A, ctas, s);
    if (slice <= 20 * 1024) return launch_rows<KIND, 64, 13>(A, ctas, s);
    if (slice <= 48 * 1024) return launch_rows<KIND, 128, 5>(A, ctas, s);
    if (slice <= 84 * 1024) return launch_rows<KIND, 256, 3>(A, ctas, s);
    if (!kTwo<KIND> || slice <= 340 * 1024) return launch_rows<KIND, 512, 2>(A, ctas, s);
    return launch_rows<KIND, 1024, 1>(A, ctas, s);
}

}  // namespace

}  // namespace acrl

using namespace acrl;

extern "C" acrl_status acrl_token_logp(const acrl_bf16* logits, int64_t T, int64_t V, int64_t ld, const int32_t* ids,
                                       const uint8_t* mask, float* lse, float* logp, int32_t* dev_flags, acrl_stream stream) {
    if (T < 0 || V < 1 || V > kMaxVocab || ld < V || (ld & 7) != 0) return ACRL_ERR_INVALID_ARG;
    if (T > 0 && (!logits || !ids || !lse || !logp || !aligned16(logits))) return ACRL_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    PolicyArgs A = {};
    A.V = int(V);
    A.ldz = ld;
    A.flags = dev_flags;
    for (int64_t t = 0; t < T; t += kMaxGrid) {
        A.z = logits + t * ld;
        A.ids = ids + t;
        A.mask = mask ? mask + t : nullptr;
        A.logp = logp + t;
        A.T = std::min(kMaxGrid, T - t);
        auto run = [&](auto* kernel, int threads) { return launch(kernel, A.T, threads, 0, 0, s, A, lse + t); };
        // with the pairs and the gradient, 32 / 128 / 256 threads a row: 48,828 x 4,096 218 / 271 / 375 us, 12,207 x 16,384
        // 208 / 204 / 214, 1,316 x 151,936 212 / 212 / 204
        const acrl_status st = V <= 8192 ? run(logp_kernel<32>, 32) : V <= 65536 ? run(logp_kernel<128>, 128) : run(logp_kernel<256>, 256);
        if (st != ACRL_OK) return st;
    }
    return ACRL_OK;
}

extern "C" acrl_status acrl_policy_loss_grad_logits(const acrl_bf16* logits, int64_t T, int64_t V, int64_t ld,
                                                    const int32_t* ids, const uint8_t* mask, const float* old_logp,
                                                    const float* coef, float clip_low, float clip_high, float dual_clip,
                                                    acrl_kl kl, const float* kl_coef, const acrl_bf16* ref_logits,
                                                    int64_t ld_ref, const float* ref_logp, acrl_bf16* grad, float* logp,
                                                    float* kl_out, float* token_loss, float* loss, int32_t* dev_flags,
                                                    acrl_stream stream) {
    if (T < 0 || V < 1 || V > kMaxVocab || ld < V || (ld & 7) != 0 || !loss) return ACRL_ERR_INVALID_ARG;
    if (!(clip_low >= 0.f && clip_low < 1.f) || !(clip_high >= 0.f) || !(dual_clip == 0.f || dual_clip > 1.f))
        return ACRL_ERR_INVALID_ARG;
    if (kl < ACRL_KL_NONE || kl > ACRL_KL_REVERSE) return ACRL_ERR_INVALID_ARG;
    const bool full = kl >= ACRL_KL_EXACT, sampled = kl >= ACRL_KL_K1 && !full;
    if (full && (ld_ref < V || (ld_ref & 7) != 0)) return ACRL_ERR_INVALID_ARG;
    if (kl == ACRL_KL_NONE && (kl_coef || kl_out)) return ACRL_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (T > 0) {
        if (!logits || !ids || !grad || !logp || !token_loss || !aligned16(logits) || !aligned16(grad))
            return ACRL_ERR_INVALID_ARG;
        if ((full && (!ref_logits || !aligned16(ref_logits))) || (sampled && !ref_logp)) return ACRL_ERR_INVALID_ARG;
        PolicyArgs A = {};
        A.z = logits;
        A.ldz = A.ldg = ld;
        A.x = full ? ref_logits : nullptr;
        A.ldx = ld_ref;
        A.V = int(V);
        A.ids = ids;
        A.mask = mask;
        A.coef = coef;
        A.kl_coef = kl_coef;
        A.old_logp = old_logp;
        A.ref_logp = sampled ? ref_logp : nullptr;
        A.kl = kl;
        A.low = clip_low;
        A.high = clip_high;
        A.dual = dual_clip == 0.f ? INFINITY : dual_clip;
        A.grad = grad;
        A.logp = logp;
        A.kl_out = kl_out;
        A.token_loss = token_loss;
        A.flags = dev_flags;
        A.T = T;
        const acrl_status st = kl == ACRL_KL_EXACT     ? launch_policy<kExact>(A, s)
                               : kl == ACRL_KL_REVERSE ? launch_policy<kReverse>(A, s)
                                                       : launch_policy<kSampled>(A, s);
        if (st != ACRL_OK) return st;
    }
    return acrl_reduce_loss(token_loss, T, loss, stream);
}
