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
// from memory once.  A cluster of CTAs shares a row: each copies its slice of
// z (and x) into shared memory with bulk copies, folds the running maxima and
// sums as the copies land, exchanges one partial state with the others through
// distributed shared memory, and writes the gradient of its slice from what it
// kept.  So HBM sees every operand once (2 bytes of z, 2 of x, 2 of the
// gradient an element), which bounds it, with the SFU next (three
// exponentials an element pair).  Several such CTAs share an SM, so that one
// loads while another computes and a third stores.
#include <algorithm>
#include <cmath>

#include "acrl_device.cuh"
#include "acrl_host.h"
#include "mbarrier.cuh"
#include "row_lse.cuh"

namespace acrl {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kMaxChunks = 8;

enum Kind { kSampled, kExact, kReverse };   // which sums a row needs

struct PolicyArgs {
    const acrl_bf16 *z, *x;
    int64_t ldz, ldx;
    int V;
    int keep;      // vectors of each operand that a CTA keeps
    int chunk;     // vectors of a bulk copy
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

__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
    f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x);
    f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z);
    f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
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

// Fold N vectors of each operand.  SAFE: a column of probability 0 adds nothing to the cross sum, whatever the
// other side holds there (an infinite difference times 0 is NaN); without it such a row ends with a cross sum
// that is not finite, and is folded again.
template <Kind KIND, int N, bool SAFE>
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
    float sz[2] = {0.f, 0.f}, sx[2] = {0.f, 0.f}, cr[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float a[8], b[8];
        unpack8(z[k], a);
        if (KIND != kSampled) unpack8(x[k], b);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = ex2(fmaf(a[j], kLog2e, -st.U));
            sz[j & 1] += e;
            if constexpr (KIND != kSampled) {
                const float h = ex2(fmaf(b[j], kLog2e, -st.W));
                sx[j & 1] += h;
                const float w = KIND == kExact ? e : h, d = KIND == kExact ? a[j] - b[j] : b[j] - a[j];
                cr[j & 1] = SAFE ? (w > 0.f ? fmaf(w, d, cr[j & 1]) : cr[j & 1]) : fmaf(w, d, cr[j & 1]);
            }
        }
    }
    st.sz += sz[0] + sz[1];
    if (KIND != kSampled) {
        st.sx += sx[0] + sx[1];
        st.cross += cr[0] + cr[1];
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

__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ void st_peer(const float* p, uint32_t rank, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_addr(p, rank)), "f"(v) : "memory");
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

template <Kind KIND, bool SAFE>
__device__ __forceinline__ float grad_at(float z, float x, const RowGrad& g) {
    const float p = ex2(fmaf(z, kLog2e, -g.U));
    if constexpr (KIND == kSampled) return p * g.c;
    if constexpr (KIND == kReverse) return fmaf(p, g.c2, -g.k * ex2(fmaf(x, kLog2e, -g.W)));
    const float v = p * fmaf(g.k, z - x, g.c2);
    return SAFE ? (p > 0.f ? v : 0.f) : v;
}

template <Kind KIND, bool SAFE>
__device__ __forceinline__ uint4 grad_vec8(const uint4& zv, const uint4& xv, const RowGrad& g, int rel) {
    float a[8], b[8], o[8];
    unpack8(zv, a);
    if (KIND != kSampled) unpack8(xv, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = grad_at<KIND, SAFE>(a[j], KIND != kSampled ? b[j] : 0.f, g);
    if (unsigned(rel) < 8u)
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = j == rel ? g.target : o[j];
    return make_uint4(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]), pack_bf16x2(o[4], o[5]), pack_bf16x2(o[6], o[7]));
}

// A slice of a row: vectors [begin, end) of it, the first `kept` of them in shared memory; the last slice also has
// the columns beyond the whole vectors.
struct Slice {
    int begin, end, kept;
    bool last;
};

template <Kind KIND, bool SAFE>
__device__ State sweep(const PolicyArgs& A, const acrl_bf16* zr, const acrl_bf16* xr, const uint4* sz, const uint4* sx,
                       const Slice& sl, uint64_t* bars, bool& landed) {
    State st = empty_state();
    const int tid = threadIdx.x;
    const uint4 *gz = reinterpret_cast<const uint4*>(zr) + sl.begin, *gx = reinterpret_cast<const uint4*>(xr) + sl.begin;
    const int n = sl.end - sl.begin;
    if (sl.last)
        for (int j = (A.V & ~7) + tid; j < A.V; j += kThreads) {
            // one column as a vector whose others are the lowest number of both operands: they add nothing
            const uint32_t lowest = 0xff7fff7fu;
            uint4 a[1] = {make_uint4(0xff7f0000u | zr[j], lowest, lowest, lowest)}, b[1] = {a[0]};
            if (KIND != kSampled) b[0].x = 0xff7f0000u | xr[j];
            fold<KIND, 1, SAFE>(st, a, b);
        }
    for (int v = sl.kept + tid; v < n; v += kThreads) {   // what is not kept: read again by the gradient
        uint4 a[1] = {__ldg(gz + v)}, b[1] = {a[0]};
        if (KIND != kSampled) b[0] = __ldg(gx + v);
        fold<KIND, 1, SAFE>(st, a, b);
    }
    for (int c0 = 0, i = 0; c0 < sl.kept; c0 += A.chunk, ++i) {
        if (!wait_phase(bars + i, 0, nullptr)) landed = false;
        const int end = min(sl.kept, c0 + A.chunk);
        int v = c0 + tid;
        for (; v + kThreads < end; v += 2 * kThreads) {
            const uint4 a[2] = {sz[v], sz[v + kThreads]};
            uint4 b[2] = {a[0], a[1]};
            if (KIND != kSampled) {
                b[0] = sx[v];
                b[1] = sx[v + kThreads];
            }
            fold<KIND, 2, SAFE>(st, a, b);
        }
        if (v < end) {
            uint4 a[1] = {sz[v]}, b[1] = {a[0]};
            if (KIND != kSampled) b[0] = sx[v];
            fold<KIND, 1, SAFE>(st, a, b);
        }
    }
    return st;
}

template <Kind KIND, bool SAFE>
__device__ void write_grad(const PolicyArgs& A, const acrl_bf16* zr, const acrl_bf16* xr, acrl_bf16* gr, const uint4* sz,
                           const uint4* sx, const Slice& sl, const RowGrad& g) {
    const int tid = threadIdx.x;
    const uint4 *gz = reinterpret_cast<const uint4*>(zr) + sl.begin, *gx = reinterpret_cast<const uint4*>(xr) + sl.begin;
    uint4* out = reinterpret_cast<uint4*>(gr) + sl.begin;
    const int n = sl.end - sl.begin, rel0 = g.a - (sl.begin << 3);
    for (int v = tid; v < sl.kept; v += kThreads)
        st_stream(out + v, grad_vec8<KIND, SAFE>(sz[v], KIND != kSampled ? sx[v] : sz[v], g, rel0 - (v << 3)));
    for (int v = sl.kept + tid; v < n; v += kThreads) {
        const uint4 a = __ldg(gz + v);
        st_stream(out + v, grad_vec8<KIND, SAFE>(a, KIND != kSampled ? __ldg(gx + v) : a, g, rel0 - (v << 3)));
    }
    if (sl.last)
        for (int j = (A.V & ~7) + tid; j < A.V; j += kThreads) {
            const float v = grad_at<KIND, SAFE>(bf16_to_float(zr[j]), KIND != kSampled ? bf16_to_float(xr[j]) : 0.f, g);
            gr[j] = acrl_bf16(pack_bf16x2(j == g.a ? g.target : v, 0.f) & 0xffffu);
        }
}

__device__ __forceinline__ void fill_grad(const PolicyArgs& A, acrl_bf16* gr, const Slice& sl, uint32_t pair) {
    uint4* out = reinterpret_cast<uint4*>(gr);
    for (int v = sl.begin + threadIdx.x; v < sl.end; v += kThreads) st_stream(out + v, make_uint4(pair, pair, pair, pair));
    if (sl.last)
        for (int j = (A.V & ~7) + threadIdx.x; j < A.V; j += kThreads) gr[j] = acrl_bf16(pair & 0xffffu);
}

template <Kind KIND>
__global__ void __launch_bounds__(kThreads) policy_kernel(const __grid_constant__ PolicyArgs A) {
    extern __shared__ __align__(16) uint4 kept[];
    __shared__ uint64_t bars[kMaxChunks];
    __shared__ float parts[2][kMaxCluster][8];     // per pass: the CTAs' states
    __shared__ float warps[kWarps][8];
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int nct = int(cluster_size()), rank = int(cluster_rank());
    const int64_t t = int64_t(blockIdx.x) / nct;
    grid_begin();
    const int nvec = A.V >> 3, per = (nvec + nct - 1) / nct;
    Slice sl;
    sl.begin = min(nvec, rank * per);
    sl.end = min(nvec, sl.begin + per);
    sl.kept = min(sl.end - sl.begin, A.keep);
    sl.last = rank == nct - 1;
    acrl_bf16* gr = A.grad + t * A.ldg;
    const bool first = rank == 0 && tid == 0;
    const int a = A.ids[t];
    const bool valid = !(A.mask && A.mask[t] == 0);
    if (!valid || a < 0 || a >= A.V) {     // the same for the whole cluster
        fill_grad(A, gr, sl, 0u);
        if (first) {
            A.logp[t] = A.token_loss[t] = 0.f;
            if (A.kl_out) A.kl_out[t] = 0.f;
            if (valid) raise_flag(A.flags, ACRL_FLAG_BAD_ID);
        }
        return;
    }
    const acrl_bf16 *zr = A.z + t * A.ldz, *xr = KIND == kSampled ? zr : A.x + t * A.ldx;
    uint4 *sz = kept, *sx = kept + A.keep;
    if (tid == 0) {
        for (int i = 0; i < kMaxChunks; ++i) mbar_init(bars + i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        const uint64_t once = policy_evict_first();
        for (int c0 = 0, i = 0; c0 < sl.kept; c0 += A.chunk, ++i) {
            const uint32_t bytes = uint32_t(min(A.chunk, sl.kept - c0)) * 16u;
            mbar_expect_tx(bars + i, (KIND == kSampled ? 1 : 2) * bytes);
            bulk_in(sz + c0, reinterpret_cast<const uint4*>(zr) + sl.begin + c0, bytes, bars + i, once);
            if (KIND != kSampled) bulk_in(sx + c0, reinterpret_cast<const uint4*>(xr) + sl.begin + c0, bytes, bars + i, once);
        }
    }
    const float za = bf16_to_float(zr[a]), xa = KIND == kSampled ? 0.f : bf16_to_float(xr[a]);
    const float c0 = A.coef ? A.coef[t] : 0.f, kc = A.kl_coef ? A.kl_coef[t] : 0.f;
    const float old = A.old_logp ? A.old_logp[t] : 0.f, ref = A.ref_logp ? A.ref_logp[t] : 0.f;
    __syncthreads();                        // the barriers are initialised
    if (nct > 1) cluster_arrive();          // this CTA runs: its shared memory may be written
    bool landed = true, safe = false;
    State row;
    for (int pass = 0;; ++pass) {
        State st = pass == 0 ? sweep<KIND, false>(A, zr, xr, sz, sx, sl, bars, landed)
                             : sweep<KIND, true>(A, zr, xr, sz, sx, sl, bars, landed);
        st = meet<KIND, 32>(st);
        if (pass > 0) __syncthreads();      // the warps have read the first pass's states
        if (lane == 0) {
            float* w = warps[wid];
            w[0] = st.mz; w[1] = st.U; w[2] = st.sz; w[3] = st.mx; w[4] = st.W; w[5] = st.sx; w[6] = st.cross;
        }
        __syncthreads();
        const float* w = warps[lane & (kWarps - 1)];
        row = meet<KIND, kWarps>(State{w[0], w[1], w[2], w[3], w[4], w[5], w[6]});
        if (nct > 1) {
            if (pass == 0) cluster_wait();  // every CTA runs
            if (wid == 0 && lane < nct) {   // lane r hands this CTA's state to CTA r
                const float* mine = parts[pass][rank];
                st_peer(mine + 0, lane, row.mz);
                st_peer(mine + 1, lane, row.U);
                st_peer(mine + 2, lane, row.sz);
                st_peer(mine + 3, lane, row.mx);
                st_peer(mine + 4, lane, row.W);
                st_peer(mine + 5, lane, row.sx);
                st_peer(mine + 6, lane, row.cross);
            }
            cluster_arrive();
            cluster_wait();
            const float* o = parts[pass][lane & (kMaxCluster - 1)];
            const bool there = (lane & (kMaxCluster - 1)) < nct;
            const State e = empty_state();
            row = meet<KIND, kMaxCluster>(there ? State{o[0], o[1], o[2], o[3], o[4], o[5], o[6]} : e);
        }
        if (KIND == kSampled || pass > 0 || isfinite(row.cross) || !isfinite(row.sz) || !isfinite(row.sx)) break;
        safe = true;
    }
    if (!landed) raise_flag(A.flags, ACRL_FLAG_TIMEOUT);

    // the row's scalars, the same in every thread
    const float lz = kLn2 * (log2f(row.sz) - fmaf(row.mz, kLog2e, -row.U));      // lse_z - max z
    const float logp = (za - row.mz) - lz;
    float KL = 0.f, apart = 0.f, logq = 0.f;                                      // apart = lse_z - lse_x
    RowGrad g;
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
    if (first) {
        const float nan = __int_as_float(0x7fc00000);
        A.logp[t] = defined ? logp : nan;
        if (A.kl_out) A.kl_out[t] = defined ? KL : nan;
        A.token_loss[t] = undefined ? nan : loss;
        if (!defined || undefined) raise_flag(A.flags, ACRL_FLAG_NONFINITE);
    }
    if (!carries || undefined) {
        fill_grad(A, gr, sl, undefined ? 0x7fc07fc0u : 0u);
        return;
    }
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
    if (safe)
        write_grad<KIND, true>(A, zr, xr, gr, sz, sx, sl, g);
    else
        write_grad<KIND, false>(A, zr, xr, gr, sz, sx, sl, g);
}

// Shared memory of a CTA's slice.  CTAs of up to kSliceBytes let several share an SM.
constexpr int kSliceBytes = 40 * 1024, kMaxKeepBytes = 192 * 1024;

template <Kind KIND>
acrl_status launch_policy(PolicyArgs A, int64_t T, cudaStream_t s) {
    constexpr int OPS = KIND == kSampled ? 1 : 2;
    const int nvec = A.V >> 3;
    int ctas = 1;
    while (ctas < kMaxCluster && (nvec + ctas - 1) / ctas * 16 * OPS > kSliceBytes) ctas *= 2;
    A.keep = std::min((nvec + ctas - 1) / ctas, kMaxKeepBytes / (16 * OPS));
    constexpr int step = 2 * kThreads;
    A.chunk = std::max(1, (A.keep + kMaxChunks * step - 1) / (kMaxChunks * step)) * step;
    auto* kernel = policy_kernel<KIND>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxKeepBytes) != cudaSuccess)
        return launch_status();
    const int64_t most = kMaxGrid / ctas;
    for (int64_t t = 0; t < T; t += most) {      // a grid's limit
        PolicyArgs B = A;
        auto at = [t](auto* p, int64_t ld = 1) { return p ? p + t * ld : p; };
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
        const acrl_status st = launch(kernel, std::min(most, T - t) * ctas, kThreads, size_t(A.keep) * 16 * OPS, ctas, s, B);
        if (st != ACRL_OK) return st;
    }
    return ACRL_OK;
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
        const acrl_status st = kl == ACRL_KL_EXACT     ? launch_policy<kExact>(A, T, s)
                               : kl == ACRL_KL_REVERSE ? launch_policy<kReverse>(A, T, s)
                                                       : launch_policy<kSampled>(A, T, s);
        if (st != ACRL_OK) return st;
    }
    return acrl_reduce_loss(token_loss, T, loss, stream);
}
