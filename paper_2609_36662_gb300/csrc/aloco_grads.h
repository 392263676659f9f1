// Internal interface of the gradient-list operators (norm, clipping).
#pragma once

#include "aloco_internal.h"

namespace aloco {

// A stretch of one tensor, of a multiple of 4096 elements but at the tensor's
// end: its start lies to the 16-byte boundaries as the tensor's does.
struct GradChunk {
    void *p;
    int64_t at;     // its first element's place in the flat vector
    int32_t n;
    int32_t bf16;
};

constexpr int kGradBlock = 256;

// A block's sum of squares: fp32, what its additions rounded away, and what
// only fp64 holds.
struct __align__(16) GradPartial {
    float s, rest;
    double wide;
};

struct GradArgs {
    const GradChunk *chunks;
    int n_chunks;
    GradPartial *partials;  // [grid] (scratch, as the next two)
    unsigned int *ticket;   // 0 between launches
    float *factor;          // clipping factor
    float *norm;
    float max_norm;         // 0 where only the norm is wanted
    void *out;              // null: in place
    int out_bf16;
};

// Blocks of the norm pass on a device of that many SMs (partials' length).
int grad_norm_blocks(int sm_count, int n_chunks);
cudaError_t launch_grad_norm(const GradArgs &a, int sm_count, cudaStream_t stream);
cudaError_t launch_grad_scale(const GradArgs &a, int sm_count, cudaStream_t stream);

}  // namespace aloco
