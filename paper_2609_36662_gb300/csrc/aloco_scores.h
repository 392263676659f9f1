// Internal interface of the token scores: what aloco_losses.cpp checks and
// fills in, and what the kernels of aloco_scores.cu take by value.
#pragma once

#include "aloco_logits.h"

namespace aloco {

struct ScoresArgs {
    Rows x, g;                       // logits; gradient
    int64_t n;                       // rows
    int vocab, bf16;
    const void *target;
    int target_bytes;
    float scale;                     // log2(e) / tau
    float tilt;                      // what scale's rounding does to a sum of terms, to
                                     // its powers times their terms: ln 2 (exact / scale - 1)
    float inv_temp;                  // 1 / tau
    int top;
    float *logp, *entropy, *top_logp;
    int *top_ids;
    float2 *stats;
    // gradient
    const float2 *stats_in;
    const float *entropy_in, *d_logp, *d_entropy, *d_top;
    const int *ids_in;
};

cudaError_t launch_token_scores(const ScoresArgs &a, int sm_count, cudaStream_t stream);
cudaError_t launch_token_scores_grad(const ScoresArgs &a, int sm_count, cudaStream_t stream);

}  // namespace aloco
