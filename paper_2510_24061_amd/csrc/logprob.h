// Token log-probabilities and the preference loss (logprob.hip): arguments as include/falqon.h describes them.
#pragma once
#include "falqon_internal.h"

namespace falqon {

int token_splits(int64_t T, int64_t V);   // parts of a row; with more than one, partial has T times as many elements

struct TokenLogprob {
    const void* logits; int64_t ld;
    const int64_t* labels;
    int64_t T, V;
    float *logp, *lse, *lse_low;                 // lse_low may be null
    float2* partial;
};
hipError_t launch_token_logprob(const TokenLogprob& a, bool f32, hipStream_t stream);

struct TokenLogprobBwd {
    const float* d_logp;
    const void* logits; int64_t ld;
    const int64_t* labels;
    const float *lse, *lse_low;
    int64_t T, V;
    void* out; int64_t ld_out;
};
hipError_t launch_token_logprob_bwd(const TokenLogprobBwd& a, bool f32, hipStream_t stream);

hipError_t launch_preference_loss(const float* logp, const float* ref, const int64_t* offsets, int64_t T, int64_t P, float beta, float smoothing, float* pair_loss,
                                  float* loss, float* rewards, float* d_logp, hipStream_t stream);

}  // namespace falqon
