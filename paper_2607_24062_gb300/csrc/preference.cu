// acrl_preference_loss: a loss over pairs of responses of one prompt, and its
// gradient with respect to the tokens' log-probs.
//
//     D_i = sum_t m_t (logp_t - ref_logp_t)   [/ n_i]
//     pairs of a prompt: (i, j) with R_i > R_j, both with valid tokens
//     h = beta (D_i - D_j) - margin
//     L = mean over prompts with pairs of the mean over the prompt's pairs of f(h)
//     coef_t = -dL/dlogp_t
//
// Three kernels: the responses' sums; a prompt's pairs; the tokens' coefficients and the loss.
// The number of prompts with pairs, an integer count, is all that prompts share.
// ~13 bytes per token; latency and the launches bound it.
#include <cmath>

#include "acrl_device.cuh"
#include "acrl_host.h"

namespace acrl {
namespace {

constexpr int kRespThreads = 256, kPairThreads = 128;

// What the kernels hand on, in the caller's workspace.
struct PrefWork {
    double* ratio;    // [S] D_i
    double* slope;    // [S] dL/dD_i times the number of prompts with pairs
    double* loss;     // [Gn] the prompt's mean over its pairs
    int32_t* count;   // [S] n_i
    int32_t* prompts; // [1] prompts with pairs
};

struct PrefForm {
    int form;
    float beta, margin, smooth;
    int mean;
};

__device__ __forceinline__ bool range_of(const int64_t* so, int i, int64_t T, int64_t& lo, int64_t& hi) {
    lo = so[i];
    hi = so[i + 1];
    return lo >= 0 && lo <= hi && hi <= T;
}

// a + b = s + e exactly (Knuth 1969), where nothing overflows.
__device__ __forceinline__ void two_sum(float a, float b, float& s, float& e) {
    const float t = __fadd_rn(a, b), bb = __fsub_rn(t, a);
    e = __fadd_rn(__fsub_rn(a, __fsub_rn(t, bb)), __fsub_rn(b, bb));
    s = t;
}

__global__ void __launch_bounds__(kRespThreads)
    pref_responses(const float* __restrict__ logp, const float* __restrict__ ref, const uint8_t* __restrict__ mask, int64_t T,
                   const int64_t* __restrict__ so, int S, int mean, PrefWork w, float* __restrict__ ratio, int32_t* flags) {
    constexpr int NW = kRespThreads / 32;
    __shared__ double sums[NW];
    __shared__ int counts[NW];
    const int i = blockIdx.x, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    grid_begin();
    int64_t lo, hi;
    bool ok = range_of(so, i, T, lo, hi);
    if (!ok) lo = hi = 0;
    if ((i == 0 && so[0] != 0) || (i == S - 1 && so[S] != T)) ok = false;
    if (threadIdx.x == 0) {
        if (!ok) raise_flag(flags, ACRL_FLAG_BAD_OFFSETS);
        if (i == 0) *w.prompts = 0;
    }
    // Compensated sums: every difference and addition exactly, as a rounded number and what the rounding left, which is added up by
    // itself (in fp32, its own roundings 2^-24 of what was left); then in fp64.  With rounded differences a sum near 0 had lost three
    // digits; with fp64 a token, 2 a cycle and SM, the kernel took 14 us at 512 x 2,048.  Four tokens a thread in flight.
    float high = 0.f, low = 0.f;
    int n = 0;
    for (int64_t t0 = lo + threadIdx.x; t0 < hi; t0 += 4 * kRespThreads) {
        bool in[4];
        float a[4], b[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t t = t0 + k * kRespThreads;
            in[k] = t < hi && !(mask && mask[t] == 0);
            a[k] = t < hi ? logp[t] : 0.f;
            b[k] = t < hi && ref ? ref[t] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (in[k]) {
                float d, e;
                two_sum(a[k], -b[k], d, e);
                low += e;
                two_sum(high, d, high, e);
                low += e;
                ++n;
            }
    }
    // an infinite or undefined sum is that of the high parts
    double sum = warp_sum(isfinite(high) ? double(high) + double(low) : double(high));
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) {
        sums[wid] = sum;
        counts[wid] = n;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < NW; ++k) {
            sum += sums[k];
            n += counts[k];
        }
        if (mean && n > 0) sum /= n;
        if (!isfinite(sum)) raise_flag(flags, ACRL_FLAG_NONFINITE);
        w.ratio[i] = sum;
        w.slope[i] = 0.0;
        w.count[i] = n;
        ratio[i] = float(sum);
    }
}

// f(h) and f'(h).
__device__ __forceinline__ float2 pair_loss(const PrefForm& f, float h) {
    if (!isfinite(h)) return make_float2(__int_as_float(0x7fc00000), __int_as_float(0x7fc00000));
    if (f.form == ACRL_PREF_SIGMOID) {
        const float e = expf(-fabsf(h)), soft = log1pf(e), s = 1.f / (1.f + e);   // s = sigmoid(|h|)
        const float up = h >= 0.f ? s : e * s, down = h >= 0.f ? e * s : s;       // sigmoid(h), sigmoid(-h)
        return make_float2((1.f - f.smooth) * (soft + fmaxf(-h, 0.f)) + f.smooth * (soft + fmaxf(h, 0.f)),
                           -(1.f - f.smooth) * down + f.smooth * up);
    }
    if (f.form == ACRL_PREF_HINGE) return make_float2(fmaxf(1.f - h, 0.f), h < 1.f ? -1.f : 0.f);
    const float d = (h - 0.5f) / f.beta;
    return make_float2(d * d, 2.f * d / f.beta);
}

__global__ void __launch_bounds__(kPairThreads)
    pref_pairs(const float* __restrict__ rewards, const int32_t* __restrict__ go, int Gn, int S, PrefForm f, PrefWork w,
               int32_t* flags) {
    constexpr int NW = kPairThreads / 32;
    __shared__ double sums[NW];
    __shared__ long long pairs[NW];
    __shared__ float their_reward[kPairThreads];
    __shared__ double their_ratio[kPairThreads];
    const int g = blockIdx.x, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    grid_begin();
    int lo = go[g], hi = go[g + 1];
    bool ok = lo >= 0 && lo <= hi && hi <= S;
    if (!ok) lo = hi = 0;
    if ((g == 0 && go[0] != 0) || (g == Gn - 1 && go[Gn] != S)) ok = false;
    if (!ok && threadIdx.x == 0) raise_flag(flags, ACRL_FLAG_BAD_OFFSETS);
    long long n = 0;
    double loss = 0.0;
    // as many lanes a response as there are threads for (whole powers of two up to a warp), its pairs in turn
    int each = 1;
    while (each < 32 && 2 * each * (hi - lo) <= kPairThreads) each *= 2;
    const int part = int(threadIdx.x) & (each - 1), first = lo + int(threadIdx.x) / each;
    const uint32_t together = (each == 32 ? 0xffffffffu : (1u << each) - 1u) << (lane & ~(each - 1));
    // pairs with the responses [j0, j1) of the prompt, which lie in shared memory; kPairThreads of them at a time
    for (int j0 = lo; j0 < hi; j0 += kPairThreads) {
        const int j1 = min(hi, j0 + kPairThreads), mine = j0 + int(threadIdx.x);
        __syncthreads();
        if (mine < j1) {
            const float R = rewards[mine];
            if (isnan(R)) raise_flag(flags, ACRL_FLAG_NONFINITE);
            their_reward[threadIdx.x] = w.count[mine] > 0 ? R : __int_as_float(0x7fc00000);   // NaN: no pair
            their_ratio[threadIdx.x] = w.ratio[mine];
        }
        __syncthreads();
        for (int i = first; i < hi; i += kPairThreads / each) {
            const bool here = i >= j0 && i < j1;
            const float Ri = here ? their_reward[i - j0] : w.count[i] > 0 ? rewards[i] : __int_as_float(0x7fc00000);
            const double Di = here ? their_ratio[i - j0] : w.ratio[i];
            double slope = 0.0;
            for (int j = part; j < j1 - j0; j += each) {
                const float Rj = their_reward[j];
                if (!(Ri > Rj || Rj > Ri)) continue;
                const bool wins = Ri > Rj;
                const double d = Di - their_ratio[j];
                const float2 v = pair_loss(f, float(double(f.beta) * (wins ? d : -d) - double(f.margin)));
                if (wins) {
                    loss += v.x;
                    slope += v.y;
                    ++n;
                } else {
                    slope -= v.y;
                }
            }
            for (int m = each / 2; m >= 1; m >>= 1) slope += __shfl_xor_sync(together, slope, m);
            if (part == 0) w.slope[i] = j0 == lo ? slope : w.slope[i] + slope;
        }
    }
    loss = warp_sum(loss);
    n = warp_sum(n);
    if (lane == 0) {
        sums[wid] = loss;
        pairs[wid] = n;
    }
    __syncthreads();
    n = pairs[0];
    loss = sums[0];
    for (int k = 1; k < NW; ++k) {
        n += pairs[k];
        loss += sums[k];
    }
    const double per = n > 0 ? 1.0 / double(n) : 0.0;
    for (int i = lo + int(threadIdx.x); i < hi; i += kPairThreads) {
        double c = double(f.beta) * w.slope[i] * per;
        if (f.mean && w.count[i] > 0) c /= w.count[i];
        w.slope[i] = n > 0 ? c : 0.0;
    }
    if (threadIdx.x == 0) {
        w.loss[g] = n > 0 ? loss * per : 0.0;
        if (n > 0) atomicAdd(w.prompts, 1);
    }
}

__global__ void __launch_bounds__(kRespThreads)
    pref_tokens(const uint8_t* __restrict__ mask, int64_t T, const int64_t* __restrict__ so, int S, int Gn, PrefWork w,
                float* __restrict__ coef, float* __restrict__ loss) {
    __shared__ double sums[kRespThreads / 32];
    grid_begin();
    const int Q = *w.prompts;
    const int i = blockIdx.x;
    if (i == S) {                     // one CTA for the loss
        double s = 0.0;
        for (int g = threadIdx.x; g < Gn; g += kRespThreads) s += w.loss[g];
        s = warp_sum(s);
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int k = 1; k < kRespThreads / 32; ++k) s += sums[k];
            *loss = Q > 0 ? float(s / Q) : 0.f;
        }
        return;
    }
    int64_t lo, hi;
    if (!range_of(so, i, T, lo, hi)) return;
    float c = 0.f;                    // one fp64 division a warp: one a thread took 4 us at 512 x 2,048
    if ((threadIdx.x & 31) == 0 && Q > 0) c = float(-w.slope[i] / Q);
    c = __shfl_sync(0xffffffffu, c, 0);
#pragma unroll 4
    for (int64_t t = lo + threadIdx.x; t < hi; t += kRespThreads) coef[t] = !mask || mask[t] ? c : 0.f;
}

constexpr int64_t kPrefHead = 16;

int64_t work_bytes(int64_t S, int64_t Gn) { return kPrefHead + 8 * (2 * S + Gn) + 4 * S; }

bool pairs_ok(const float* logp, int64_t T, const float* rewards, const int64_t* seq_offsets, int32_t S, const int32_t* group_offsets,
              int32_t Gn, acrl_preference_form form, float beta, float margin, float label_smoothing, const float* ratio,
              const float* coef, const float* loss) {
    if (T < 0 || S < 0 || Gn < 0 || S == 0x7fffffff || !loss) return false;
    if (form < ACRL_PREF_SIGMOID || form > ACRL_PREF_IPO) return false;
    if (!(beta > 0.f) || !std::isfinite(beta) || !std::isfinite(margin)) return false;
    if (!(label_smoothing >= 0.f && label_smoothing < 0.5f)) return false;
    if (T > 0 && (!logp || !coef)) return false;
    if (S > 0 && (!rewards || !seq_offsets || !ratio)) return false;
    if (Gn > 0 && !group_offsets) return false;
    return !((S == 0 && T > 0) || (Gn == 0 && S > 0));   // offsets that cannot cover
}

}  // namespace
}  // namespace acrl

using namespace acrl;

extern "C" int64_t acrl_preference_workspace_bytes(int32_t S, int32_t Gn) {
    return S < 0 || Gn < 0 ? -1 : work_bytes(S, Gn);
}

extern "C" acrl_status acrl_preference_loss(const float* logp, const float* ref_logp, const uint8_t* mask, int64_t T,
                                            const float* rewards, const int64_t* seq_offsets, int32_t S,
                                            const int32_t* group_offsets, int32_t Gn, acrl_preference_form form, float beta,
                                            float margin, float label_smoothing, int32_t length_norm, float* ratio,
                                            float* coef, float* loss, void* workspace, int64_t workspace_bytes,
                                            int32_t* dev_flags, acrl_stream stream) {
    if (!pairs_ok(logp, T, rewards, seq_offsets, S, group_offsets, Gn, form, beta, margin, label_smoothing, ratio, coef, loss))
        return ACRL_ERR_INVALID_ARG;
    if (!workspace || !aligned16(workspace) || workspace_bytes < work_bytes(S, Gn)) return ACRL_ERR_INVALID_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    char* p = static_cast<char*>(workspace);
    PrefWork w;
    w.prompts = reinterpret_cast<int32_t*>(p);
    w.ratio = reinterpret_cast<double*>(p + kPrefHead);
    w.slope = w.ratio + S;
    w.loss = w.slope + S;
    w.count = reinterpret_cast<int32_t*>(w.loss + Gn);
    const PrefForm f{form, beta, margin, label_smoothing, length_norm != 0};
    if (S == 0)   // no response, no pair
        return cudaMemsetAsync(loss, 0, sizeof(float), s) == cudaSuccess ? ACRL_OK : launch_status();
    acrl_status st = launch(pref_responses, S, kRespThreads, 0, 0, s, logp, ref_logp, mask, T, seq_offsets, S, f.mean, w,
                            ratio, dev_flags);
    if (st != ACRL_OK) return st;
    st = launch(pref_pairs, Gn, kPairThreads, 0, 0, s, rewards, group_offsets, Gn, S, f, w, dev_flags);
    if (st != ACRL_OK) return st;
    return launch(pref_tokens, int64_t(S) + 1, kRespThreads, 0, 0, s, mask, T, seq_offsets, S, Gn, w, coef, loss);
}

// The step's workspace: that of the pairs, then the gradient call's own sums, which nothing reads.
static int64_t step_bytes(int64_t T, int64_t S, int64_t Gn) { return (work_bytes(S, Gn) + 15) / 16 * 16 + 16 + 4 * T; }

extern "C" int64_t acrl_preference_step_workspace_bytes(int64_t T, int32_t S, int32_t Gn) {
    return T < 0 || S < 0 || Gn < 0 ? -1 : step_bytes(T, S, Gn);
}

extern "C" acrl_status acrl_preference_step(const acrl_bf16* logits, int64_t T, int64_t V, int64_t ld, const int32_t* ids,
                                            const uint8_t* mask, const float* ref_logp, const float* rewards,
                                            const int64_t* seq_offsets, int32_t S, const int32_t* group_offsets, int32_t Gn,
                                            acrl_preference_form form, float beta, float margin, float label_smoothing,
                                            int32_t length_norm, float* lse, float* logp, float* ratio, float* coef,
                                            acrl_bf16* grad, float* loss, void* workspace, int64_t workspace_bytes,
                                            int32_t* dev_flags, acrl_stream stream) {
    if (T < 0 || V < 1 || V > kMaxVocab || ld < V || (ld & 7) != 0 || S < 0 || Gn < 0) return ACRL_ERR_INVALID_ARG;
    if (!dev_flags || !workspace || !aligned16(workspace) || workspace_bytes < step_bytes(T, S, Gn)) return ACRL_ERR_INVALID_ARG;
    if (T > 0 && (!logits || !aligned16(logits) || !ids || !lse || !logp || !coef || !grad || !aligned16(grad)))
        return ACRL_ERR_INVALID_ARG;
    const int64_t head = (work_bytes(S, Gn) + 15) / 16 * 16;
    if (!pairs_ok(logp, T, rewards, seq_offsets, S, group_offsets, Gn, form, beta, margin, label_smoothing, ratio, coef, loss))
        return ACRL_ERR_INVALID_ARG;
    if (T > 0) {
        const acrl_status st = acrl_token_logp(logits, T, V, ld, ids, mask, lse, logp, dev_flags, stream);
        if (st != ACRL_OK) return st;
    }
    acrl_status st = acrl_preference_loss(logp, ref_logp, mask, T, rewards, seq_offsets, S, group_offsets, Gn, form, beta, margin,
                                          label_smoothing, length_norm, ratio, coef, loss, workspace, head, dev_flags, stream);
    if (st != ACRL_OK || T == 0) return st;
    float* scratch = reinterpret_cast<float*>(static_cast<char*>(workspace) + head);
    return acrl_loss_grad_logits(logits, T, V, ld, ids, mask, lse, nullptr, coef, nullptr, nullptr, 0.f, grad, scratch + 4, scratch,
                                 dev_flags, stream);
}
