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
// The gradient needs the sums of the whole row, so a row is swept twice; it is read
// from memory once.  Persistent CTAs, alone or as a cluster that shares each of its
// rows, run four roles that work on different rows at the same time:
//   warp 0       copies the CTA's slices of row after row into a ring of chunks in
//                shared memory (bulk copies);
//   warp 1       merges the states of a row's slices, works out its scalars and outputs;
//   F warps      fold the running maxima and sums of a slice as its chunks land, and
//                push the slice's state to every CTA of the cluster (distributed
//                shared memory, counted on a barrier there);
//   F warps      write the gradient of a slice from its chunks, and free them.
// So loads, arithmetic, the exchange between CTAs and stores of neighbouring rows
// overlap, and HBM sees every operand once: 2 bytes of z, 2 of x and 2 of the gradient an
// element, which bounds it.
#include <algorithm>
#include <cmath>

#include "acrl_device.cuh"
#include "acrl_host.h"
#include "mbarrier.cuh"
#include "row_lse.cuh"

namespace acrl {
namespace {

constexpr int kMaxCluster = 8;
constexpr int kMaxSlots = 32;      // chunks of a ring
constexpr int kMaxAhead = 7;       // rows that may lie in a ring
constexpr int kStates = 16;        // states of rows under way: a CTA's fold may be 2 kMaxAhead rows ahead of another's merge
constexpr int kGrads = 4;          // rows between the merge and the writing warps

enum Kind { kSampled, kExact, kReverse };   // which sums a row needs

struct PolicyArgs {
    const acrl_bf16 *z, *x;
    int64_t ldz, ldx;
    int V;
    int64_t T;
    int keep;      // vectors of each operand that a CTA keeps of a row
    int slots;     // chunks of the ring
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

// A row's (or part's) running state in base 2: maxima, exponents U = max log2 e, sums
// against them, and the cross sum: exact  sum 2^(u - U) (z - x),  reverse  sum 2^(w - W) (x - z).
struct State {
    float mz, U, sz, mx, W, sx, cross;
};

__device__ __forceinline__ State empty_state() { return State{-INFINITY, kLowestU, 0.f, -INFINITY, kLowestU, 0.f, 0.f}; }

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
    const float Un = max_exponent<true>(m), f = ex2(U - Un);
    U = Un;
    mx = m;
    return f;
}

// Fold N vectors of each operand.  A column of probability 0 adds nothing to the cross sum, whatever the other side
// holds there (an infinite difference times 0 would be NaN).
template <Kind KIND, int N>
__device__ __forceinline__ void fold(State& st, const uint4 (&z)[N], const uint4 (&x)[N]) {
    uint32_t pm = max_pairs(z[0]);
#pragma unroll
    for (int k = 1; k < N; ++k) pm = max_bf16x2(pm, max_pairs(z[k]));
    const float vm = fmaxf(bf16_lo(pm), bf16_hi(pm));
    if (vm > st.mz) {
        const float f = raise_max(vm, st.mz, st.U);
        st.sz *= f;
        if (KIND == kExact) st.cross *= f;
    }
    if constexpr (KIND != kSampled) {
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
            if constexpr (KIND != kSampled) {
                const Two b = widen(xw[j]), h = ex2_2(fma2(b, l2e, nW));
                sx = add2(sx, h);
                const Two w = KIND == kExact ? e : h, d = KIND == kExact ? fma2(b, minus, a) : fma2(a, minus, b);
                cr = fma2(w, where_weighted(w, d), cr);
            }
        }
    }
    st.sz += sum_of(sz);
    if (KIND != kSampled) {
        st.sx += sum_of(sx);
        st.cross += sum_of(cr);
    }
}

// The state against common maxima: one exponential for each.
template <Kind KIND>
__device__ __forceinline__ State bring(const State& s, float mz, float mx) {
    State r;
    r.mz = mz;
    r.U = max_exponent<true>(mz);
    const float f = ex2(s.U - r.U);
    r.sz = s.sz * f;
    if constexpr (KIND == kSampled) {
        r.mx = mx;
        r.W = r.sx = r.cross = 0.f;
    } else {
        r.mx = mx;
        r.W = max_exponent<true>(mx);
        const float g = ex2(s.W - r.W);
        r.sx = s.sx * g;
        r.cross = s.cross * (KIND == kExact ? f : g);
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
        if (KIND != kSampled) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, m));
    }
    s = bring<KIND>(s, mz, mx);
#pragma unroll
    for (int m = LANES / 2; m >= 1; m >>= 1) {
        s.sz += __shfl_xor_sync(0xffffffffu, s.sz, m);
        if (KIND != kSampled) {
            s.sx += __shfl_xor_sync(0xffffffffu, s.sx, m);
            s.cross += __shfl_xor_sync(0xffffffffu, s.cross, m);
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

// A state to CTA `rank` of the cluster, and an arrival on its barrier.
__device__ __forceinline__ void push_state(const float4* slot, uint64_t* bar, uint32_t rank, const float4& a, const float4& b) {
    const uint32_t to = peer_addr(slot, rank);
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to), "f"(a.x), "f"(a.y), "f"(a.z), "f"(a.w)
                 : "memory");
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + 16), "f"(b.x), "f"(b.y), "f"(b.z), "f"(b.w)
                 : "memory");
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(peer_addr(bar, rank)) : "memory");
}

// A phase that other CTAs of the cluster complete: what they wrote before they arrived is visible after it.
__device__ __forceinline__ bool try_wait_cluster(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
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

template <Kind KIND>
__device__ __forceinline__ Two grad_two(Two z, Two x, const RowGrad& g) {
    const Two l2e = two(kLog2e, kLog2e), p = ex2_2(fma2(z, l2e, two(-g.U, -g.U)));
    if constexpr (KIND == kSampled) return mul2(p, two(g.c, g.c));
    if constexpr (KIND == kReverse) {
        const Two q = ex2_2(fma2(x, l2e, two(-g.W, -g.W)));
        return fma2(p, two(g.c2, g.c2), mul2(q, two(-g.k, -g.k)));
    }
    const Two d = where_weighted(p, fma2(x, two(-1.f, -1.f), z));
    return mul2(p, fma2(two(g.k, g.k), d, two(g.c2, g.c2)));
}

template <Kind KIND>
__device__ __forceinline__ uint4 grad_vec8(const uint4& zv, const uint4& xv, const RowGrad& g, int rel) {
    const uint32_t zw[4] = {zv.x, zv.y, zv.z, zv.w}, xw[4] = {xv.x, xv.y, xv.z, xv.w};
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float lo, hi;
        split(grad_two<KIND>(widen(zw[j]), widen(xw[j]), g), lo, hi);
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
enum { kWrite, kFillZero, kFillNaN };

// The row's scalars from its merged state, in every lane of a warp; `writes`: this thread stores the row's outputs.
template <Kind KIND>
__device__ __forceinline__ int row_scalars(const PolicyArgs& A, int64_t t, const State& row, int a, float za, float xa,
                                           float c0, float kc, float old, float ref, bool writes, RowGrad& g) {
    const float lz = kLn2 * (log2f(row.sz) - fmaf(row.mz, kLog2e, -row.U));      // lse_z - max z
    const float logp = (za - row.mz) - lz;
    float KL = 0.f, apart = 0.f, logq = 0.f;                                      // apart = lse_z - lse_x
    g.a = a;
    g.k = kc;
    g.U = row.U + log2f(row.sz);
    g.W = 0.f;
    float slope = 0.f;                                                            // of the sampled estimators, in logp
    if constexpr (KIND != kSampled) {
        const float lx = kLn2 * (log2f(row.sx) - fmaf(row.mx, kLog2e, -row.W));
        apart = (row.mz - row.mx) + (lz - lx);
        logq = (xa - row.mx) - lx;
        KL = KIND == kExact ? row.cross / row.sz - apart : row.cross / row.sx + apart;
        g.W = row.W + log2f(row.sx);
    } else {
        const float d = logp - ref;
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
    const float ratio = A.old_logp ? expf(logp - old) : 1.f;
    float surrogate = 0.f;
    g.c = 0.f;
    if (c0 != 0.f) {
        const bool up = c0 >= 0.f;
        const float capped = up ? fminf(ratio, 1.f + A.high) : fminf(fmaxf(ratio, 1.f - A.low), A.dual);
        const bool live = up ? ratio <= 1.f + A.high : (ratio >= 1.f - A.low && ratio <= A.dual);
        surrogate = -c0 * capped;
        if (live) g.c = c0 * ratio;
    }
    if (kc != 0.f && KIND == kSampled) g.c -= kc * slope;
    const float loss = kc != 0.f ? fmaf(kc, KL, surrogate) : surrogate;
    const bool defined = isfinite(logp) && isfinite(lz) && (KIND == kSampled || isfinite(KL));
    const bool carries = c0 != 0.f || kc != 0.f;
    const bool undefined = carries && (!defined || (c0 != 0.f && isnan(ratio)) || (kc != 0.f && !isfinite(KL)));
    if (writes) {
        const float nan = __int_as_float(0x7fc00000);
        A.logp[t] = defined ? logp : nan;
        if (A.kl_out) A.kl_out[t] = defined ? KL : nan;
        A.token_loss[t] = undefined ? nan : loss;
        if (!defined || undefined) raise_flag(A.flags, ACRL_FLAG_NONFINITE);
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

template <int F>
struct Shared {
    uint64_t full[kMaxSlots];     // a chunk has landed
    uint64_t empty[kMaxSlots];    // the F writing warps are done with it
    uint64_t state[kStates];      // every CTA's state of a row is here
    uint64_t ready[kGrads];       // a row's scalars are here
    uint64_t taken[kGrads];       // the F writing warps have them
    float4 states[kStates][kMaxCluster][2];
    float4 parts[2][F][2];        // the folding warps' states, rows in turn
    RowGrad grads[kGrads];
    int what[kGrads];
    int32_t abort;
};

__device__ __forceinline__ void put(float4* to, const State& s) {
    to[0] = make_float4(s.mz, s.U, s.sz, s.mx);
    to[1] = make_float4(s.W, s.sx, s.cross, 0.f);
}
__device__ __forceinline__ State get(const float4* from) {
    const float4 a = from[0], b = from[1];
    return State{a.x, a.y, a.z, a.w, b.x, b.y, b.z};
}

// Position in a ring.
struct Ring {
    int n, at = 0;
    uint32_t phase = 0;
    __device__ explicit Ring(int size) : n(size) {}
    __device__ void next() {
        if (++at == n) {
            at = 0;
            phase ^= 1u;
        }
    }
};

// A row's sampled column, or -1 for a row that is left out (masked, or an id outside the vocabulary).
__device__ __forceinline__ int column_of(const PolicyArgs& A, int64_t t) {
    if (t >= A.T) return -1;
    const int a = A.ids[t];
    return (A.mask && A.mask[t] == 0) || a < 0 || a >= A.V ? -1 : a;
}

template <Kind KIND, int F>
struct Cta {
    static constexpr int kLanes = 32 * F;          // of a role of F warps
    static constexpr int kChunk = 2 * kLanes;      // vectors of a chunk
    static constexpr int kOps = KIND == kSampled ? 1 : 2;
    const PolicyArgs& A;
    Shared<F>& sh;
    uint4* ring;
    Slice sl;
    int chunks;            // of a row
    int64_t first, step;   // rows
    int rank, nct;

    __device__ const uint4* z_of(int slot) const { return ring + slot * (kOps * kChunk); }
    __device__ const uint4* x_of(int slot) const { return z_of(slot) + (kOps - 1) * kChunk; }
    __device__ void fail() {
        *static_cast<volatile int32_t*>(&sh.abort) = 1;
        raise_flag(A.flags, ACRL_FLAG_TIMEOUT);
    }
    __device__ bool wait(uint64_t* bar, uint32_t parity) {
        const bool ok = mbar_try_wait(bar, parity) || wait_phase_inline(bar, parity, &sh.abort);
        if (__all_sync(0xffffffffu, ok)) return true;
        fail();
        return false;
    }

    __device__ void load() {   // one thread
        const uint64_t once = policy_evict_first();
        Ring r(A.slots);
        int next = column_of(A, first);
        for (int64_t t = first; t < A.T; t += step) {
            const int a = next;
            next = column_of(A, t + step);
            if (a < 0) continue;
            const uint4* zr = reinterpret_cast<const uint4*>(A.z + t * A.ldz) + sl.begin;
            const uint4* xr = KIND == kSampled ? zr : reinterpret_cast<const uint4*>(A.x + t * A.ldx) + sl.begin;
            for (int c = 0; c < chunks; ++c, r.next()) {
                if (!mbar_try_wait(&sh.empty[r.at], r.phase ^ 1u) && !wait_phase_inline(&sh.empty[r.at], r.phase ^ 1u, &sh.abort)) {
                    fail();
                    const uint64_t t0 = global_ns();     // the copies that were started land before the CTA can leave
                    while (global_ns() - t0 < 100000ull) {
                    }
                    return;
                }
                const uint32_t bytes = uint32_t(min(kChunk, sl.kept - c * kChunk)) * 16u;
                mbar_expect_tx(&sh.full[r.at], kOps * bytes);
                bulk_in(const_cast<uint4*>(z_of(r.at)), zr + c * kChunk, bytes, &sh.full[r.at], once);
                if (KIND != kSampled) bulk_in(const_cast<uint4*>(x_of(r.at)), xr + c * kChunk, bytes, &sh.full[r.at], once);
            }
        }
    }

    __device__ void fold_rows(int warp) {
        const int lane = threadIdx.x & 31, tid = warp * 32 + lane;
        Ring r(A.slots), s(kStates);
        int parity = 0, next = column_of(A, first);
        for (int64_t t = first; t < A.T; t += step) {
            const int a = next;
            next = column_of(A, t + step);
            if (a < 0) continue;
            const acrl_bf16 *zr = A.z + t * A.ldz, *xr = KIND == kSampled ? zr : A.x + t * A.ldx;
            // the columns beyond the whole vectors, one a lane, loaded first and folded last
            const int j = (A.V & ~7) + tid;
            const bool odd = sl.last && tid < (A.V & 7);
            uint32_t zj = 0xff7fu, xj = 0xff7fu;
            if (odd) {
                zj = zr[j];
                xj = KIND == kSampled ? zj : xr[j];
            }
            State st = empty_state();
            for (int c = 0; c < chunks; ++c, r.next()) {
                if (!wait(&sh.full[r.at], r.phase)) return;
                const int n = min(kChunk, sl.kept - c * kChunk);
                const uint4 *sz = z_of(r.at), *sx = x_of(r.at);
                if (tid + kLanes < n) {
                    const uint4 z[2] = {sz[tid], sz[tid + kLanes]}, x[2] = {sx[tid], sx[tid + kLanes]};
                    fold<KIND, 2>(st, z, x);
                } else if (tid < n) {
                    const uint4 z[1] = {sz[tid]}, x[1] = {sx[tid]};
                    fold<KIND, 1>(st, z, x);
                }
            }
            // what is not kept, from L2 or HBM; the gradient reads it again
            const uint4 *gz = reinterpret_cast<const uint4*>(zr) + sl.begin, *gx = reinterpret_cast<const uint4*>(xr) + sl.begin;
            for (int v = sl.kept + tid; v < sl.end - sl.begin; v += kLanes) {
                const uint4 z[1] = {__ldg(gz + v)};
                if constexpr (KIND == kSampled) {
                    fold<KIND, 1>(st, z, z);
                } else {
                    const uint4 x[1] = {__ldg(gx + v)};
                    fold<KIND, 1>(st, z, x);
                }
            }
            if (odd) {   // a vector whose other columns are both operands' lowest number: they add nothing
                const uint32_t low = 0xff7fff7fu;
                const uint4 z[1] = {make_uint4(0xff7f0000u | zj, low, low, low)}, x[1] = {make_uint4(0xff7f0000u | xj, low, low, low)};
                fold<KIND, 1>(st, z, x);
            }
            __syncwarp();
            st = meet<KIND, 32>(st);
            if (F > 1) {
                if (lane == 0) put(sh.parts[parity][warp], st);
                asm volatile("bar.sync 1, %0;" ::"n"(kLanes) : "memory");
                if (warp == 0) st = meet<KIND, F>(get(sh.parts[parity][lane & (F - 1)]));
                parity ^= 1;
            }
            if (warp == 0 && nct > 1 && lane < nct)
                push_state(sh.states[s.at][rank], &sh.state[s.at], lane, make_float4(st.mz, st.U, st.sz, st.mx),
                           make_float4(st.W, st.sx, st.cross, 0.f));
            if (warp == 0 && nct == 1 && lane == 0) {
                put(sh.states[s.at][0], st);
                mbar_arrive(&sh.state[s.at]);
            }
            __syncwarp();
            s.next();
        }
    }

    __device__ void merge_rows() {
        const int lane = threadIdx.x & 31;
        Ring s(kStates), g(kGrads);
        for (int64_t t = first; t < A.T; t += step) {
            const int a = column_of(A, t);
            if (a < 0) {
                if (rank == 0 && lane == 0) {
                    A.logp[t] = A.token_loss[t] = 0.f;
                    if (A.kl_out) A.kl_out[t] = 0.f;
                    if (!A.mask || A.mask[t]) raise_flag(A.flags, ACRL_FLAG_BAD_ID);
                }
                continue;
            }
            const float za = bf16_to_float(A.z[t * A.ldz + a]), xa = KIND == kSampled ? 0.f : bf16_to_float(A.x[t * A.ldx + a]);
            const float c0 = A.coef ? A.coef[t] : 0.f, kc = A.kl_coef ? A.kl_coef[t] : 0.f;
            const float old = A.old_logp ? A.old_logp[t] : 0.f, ref = A.ref_logp ? A.ref_logp[t] : 0.f;
            if (!wait(&sh.state[s.at], s.phase)) return;
            if (nct > 1) try_wait_cluster(&sh.state[s.at], s.phase);   // completed: for what the other CTAs wrote
            const int k = lane & (kMaxCluster - 1);
            State row = k < nct ? get(sh.states[s.at][k]) : empty_state();
            if (nct > 1) row = meet<KIND, kMaxCluster>(row);
            else row = get(sh.states[s.at][0]);
            RowGrad rg;
            const int what = row_scalars<KIND>(A, t, row, a, za, xa, c0, kc, old, ref, rank == 0 && lane == 0, rg);
            if (!wait(&sh.taken[g.at], g.phase ^ 1u)) return;
            if (lane == 0) {
                sh.grads[g.at] = rg;
                sh.what[g.at] = what;
                mbar_arrive(&sh.ready[g.at]);
            }
            __syncwarp();
            s.next();
            g.next();
        }
    }

    __device__ void write_rows(int warp) {
        const int lane = threadIdx.x & 31, tid = warp * 32 + lane;
        Ring r(A.slots), g(kGrads);
        int next = column_of(A, first);
        for (int64_t t = first; t < A.T; t += step) {
            const int a = next;
            next = column_of(A, t + step);
            acrl_bf16* gr = A.grad + t * A.ldg;
            uint4* out = reinterpret_cast<uint4*>(gr) + sl.begin;
            const int n = sl.end - sl.begin;
            auto fill = [&](uint32_t pair) {
                for (int v = tid; v < n; v += kLanes) st_stream(out + v, make_uint4(pair, pair, pair, pair));
                if (sl.last && tid < (A.V & 7)) gr[(A.V & ~7) + tid] = acrl_bf16(pair & 0xffffu);
            };
            if (a < 0) {
                fill(0u);
                continue;
            }
            if (!wait(&sh.ready[g.at], g.phase)) return;
            const RowGrad rg = sh.grads[g.at];
            const int what = sh.what[g.at];
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.taken[g.at]);
            g.next();
            const int rel0 = a - (sl.begin << 3);
            if (what != kWrite) fill(what == kFillNaN ? 0x7fc07fc0u : 0u);
            for (int c = 0; c < chunks; ++c, r.next()) {
                if (what == kWrite) {
                    if (!wait(&sh.full[r.at], r.phase)) return;   // long since: it makes the copy visible to this warp
                    const uint4 *sz = z_of(r.at), *sx = x_of(r.at);
                    const int end = min(kChunk, sl.kept - c * kChunk);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int v = tid + k * kLanes, at = c * kChunk + v;
                        if (v < end) st_stream(out + at, grad_vec8<KIND>(sz[v], sx[v], rg, rel0 - (at << 3)));
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.empty[r.at]);
            }
            if (what != kWrite) continue;
            const acrl_bf16 *zr = A.z + t * A.ldz, *xr = KIND == kSampled ? zr : A.x + t * A.ldx;
            const uint4 *gz = reinterpret_cast<const uint4*>(zr) + sl.begin, *gx = reinterpret_cast<const uint4*>(xr) + sl.begin;
            for (int v = sl.kept + tid; v < n; v += kLanes) {
                const uint4 z = __ldg(gz + v);
                uint4 x = z;
                if constexpr (KIND != kSampled) x = __ldg(gx + v);
                st_stream(out + v, grad_vec8<KIND>(z, x, rg, rel0 - (v << 3)));
            }
            if (sl.last && tid < (A.V & 7)) {
                const int j = (A.V & ~7) + tid;
                const float z = bf16_to_float(zr[j]), x = KIND == kSampled ? 0.f : bf16_to_float(xr[j]);
                float v, none;
                split(grad_two<KIND>(two(z, z), two(x, x), rg), v, none);
                gr[j] = acrl_bf16(pack_bf16x2(j == a ? rg.target : v, 0.f) & 0xffffu);
            }
            __syncwarp();
        }
    }
};

template <int F>
constexpr int kThreadsOf = (2 * F + 2) * 32;
template <int F>
constexpr int kPerSm = 8 / F;      // CTAs that share an SM

template <Kind KIND, int F>
__global__ void __launch_bounds__(kThreadsOf<F>, kPerSm<F>) policy_kernel(const __grid_constant__ PolicyArgs A) {
    extern __shared__ __align__(16) uint4 ring[];
    __shared__ __align__(16) Shared<F> sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nct = int(cluster_size()), rank = int(cluster_rank());
    if (threadIdx.x == 0) {
        for (int i = 0; i < kMaxSlots; ++i) {
            mbar_init(sh.full + i, 1);
            mbar_init(sh.empty + i, F);
        }
        for (int i = 0; i < kStates; ++i) mbar_init(sh.state + i, uint32_t(nct));
        for (int i = 0; i < kGrads; ++i) {
            mbar_init(sh.ready + i, 1);
            mbar_init(sh.taken + i, F);
        }
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    grid_begin();
    __syncthreads();
    if (nct > 1) cluster_sync();   // every CTA's barriers are there before a state is pushed
    const int nvec = A.V >> 3, per = (nvec + nct - 1) / nct;
    Slice sl;
    sl.begin = min(nvec, rank * per);
    sl.end = min(nvec, sl.begin + per);
    sl.kept = min(sl.end - sl.begin, A.keep);
    sl.last = rank == nct - 1;
    Cta<KIND, F> cta{A, sh, ring, sl, (sl.kept + Cta<KIND, F>::kChunk - 1) / Cta<KIND, F>::kChunk,
                     int64_t(blockIdx.x) / nct, int64_t(gridDim.x) / nct, rank, nct};
    if (warp == 0) {
        if (lane == 0) cta.load();
    } else if (warp == 1) {
        cta.merge_rows();
    } else if (warp < 2 + F) {
        cta.fold_rows(warp - 2);
    } else {
        cta.write_rows(warp - 2 - F);
    }
    __syncwarp();
    if (nct > 1) cluster_sync();   // no CTA leaves while another's state may still be on its way here
}

constexpr int kSmPerBytes = 227 * 1024;

template <Kind KIND, int F>
acrl_status launch_rows(PolicyArgs A, int ctas, cudaStream_t s) {
    using C = Cta<KIND, F>;
    constexpr int slot = C::kOps * C::kChunk * 16;
    const int nvec = A.V >> 3, slice = (nvec + ctas - 1) / ctas;
    const int room = kSmPerBytes / kPerSm<F> - 1024 - int(sizeof(Shared<F>));   // the system takes 1 KB of each CTA's
    A.slots = std::min(kMaxSlots, room / slot);
    // a slice keeps what leaves a quarter of the ring to the next row's
    A.keep = std::min(slice, std::max(1, A.slots * 3 / 4) * C::kChunk);
    const int chunks = std::max(1, (A.keep + C::kChunk - 1) / C::kChunk);
    A.slots = std::min(A.slots, kMaxAhead * chunks);
    const int smem = A.slots * slot;
    auto* kernel = policy_kernel<KIND, F>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmPerBytes - 1024 - int(sizeof(Shared<F>))) !=
        cudaSuccess)
        return launch_status();
    const int64_t most = resident_clusters(reinterpret_cast<const void*>(kernel), kThreadsOf<F>, smem, ctas);
    if (most < 1) return ACRL_ERR_CUDA;
    return launch(kernel, std::min(A.T, most) * ctas, kThreadsOf<F>, size_t(smem), ctas, s, A);
}

template <Kind KIND>
acrl_status launch_policy(const PolicyArgs& A, cudaStream_t s) {
    constexpr int OPS = KIND == kSampled ? 1 : 2;
    const int bytes = (A.V >> 3) * 16 * OPS;
    int ctas = 1;
    while (ctas < kMaxCluster && bytes / ctas > 80 * 1024) ctas *= 2;
    if (bytes <= 12 * 1024) return launch_rows<KIND, 1>(A, 1, s);
    if (bytes <= 24 * 1024) return launch_rows<KIND, 2>(A, 1, s);
    return launch_rows<KIND, 4>(A, ctas, s);
}

}  // namespace
}  // namespace acrl

using namespace acrl;

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
