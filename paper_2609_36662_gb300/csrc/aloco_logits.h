// Internal interface of the post-training losses: what aloco_losses.cpp checks
// and fills in, and what the kernels of aloco_logits.cuh take by value.
#pragma once

#include "aloco_internal.h"

namespace aloco {

// Rows of a [batch, rows, vocab] array with strides (elements).
struct Rows {
    char *data;
    int64_t per_batch;               // rows of one sequence
    int64_t batch_stride, row_stride;
};

// Sums of the policy loss besides L itself.
constexpr int kTerms = 3;

// One cluster's share of them (scratch), and the mark that it has come.
struct PolicyPart {
    float term[kTerms];
    float unused;
    unsigned long long mark;
};

struct LogitsArgs {
    Rows x, g;                       // logits; gradient (g.data null: none)
    int64_t n;                       // rows
    int vocab;
    const void *target;
    int target_bytes, cu_bytes;
    float inv_temp;                  // 1 / tau
    float scale, scale_lo;           // log2(e) / tau as a sum, scale_lo > 0
    float *logp;                     // [n]
    // policy loss
    const float *adv, *old, *ref, *w;
    float lo, hi, kl;                // 1 - clip_low, 1 + clip_high, kl_coef
    PolicyPart *parts;               // [at most n clusters of the row kernel]
    unsigned long long mark;         // this call's, never 0
    int finish;                      // 1: the row kernel's last cluster adds them
                                     // (preference loss: works out the pairs)
    float *terms_out;                // [kTerms + 1]
    // preference loss (ref as above)
    const void *cu;
    int64_t pairs;
    float beta, eps, per_pair;       // per_pair: beta / pairs
    float2 *stats;                   // [n] row maximum and 1 / sum (scratch)
    float *coef;                     // [n] dL/dlogp (scratch)
    unsigned int *ticket;            // blocks of the pairs' kernel that are done (scratch)
    unsigned long long *claim;       // of the sum in a small call (scratch)
    float *loss, *ratios;
    int stages, cluster, per;        // the row kernel: ring slots, CTAs of a
                                     // cluster, units of a CTA's part at most
    int64_t test_stall1;             // testing only: 1 + the number of the slot
                                     // whose copy block 0 leaves out; below 0:
                                     // its first copy comes so many cycles late
};

cudaError_t token_logprobs_f32(const LogitsArgs &a, int sm_count, cudaStream_t stream);
cudaError_t token_logprobs_bf16(const LogitsArgs &a, int sm_count, cudaStream_t stream);
cudaError_t policy_loss_f32(const LogitsArgs &a, int sm_count, cudaStream_t stream);
cudaError_t policy_loss_bf16(const LogitsArgs &a, int sm_count, cudaStream_t stream);
cudaError_t preference_loss_f32(const LogitsArgs &a, int sm_count, cudaStream_t stream);
cudaError_t preference_loss_bf16(const LogitsArgs &a, int sm_count, cudaStream_t stream);

}  // namespace aloco
