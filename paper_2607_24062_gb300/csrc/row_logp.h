// The statistics pass of the preference step, in policy_loss.cu beside the sums it shares.
#pragma once

#include "acrl_host.h"

namespace acrl {

// lse and logp of T rows as acrl_token_stats defines them, without the entropy; checked arguments, T >= 1.
acrl_status row_logp(const acrl_bf16* logits, int64_t T, int64_t V, int64_t ld, const int32_t* ids, const uint8_t* mask, float* lse,
                     float* logp, int32_t* flags, cudaStream_t s);

}  // namespace acrl
