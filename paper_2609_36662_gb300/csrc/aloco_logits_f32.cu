// The post-training losses on fp32 logits.
#include "aloco_logits.cuh"

namespace aloco {

cudaError_t token_logprobs_f32(const LogitsArgs &a, int sm_count, cudaStream_t stream) {
    int used;
    return launch_rows<false, kFwd>(a, sm_count, stream, &used);
}

cudaError_t policy_loss_f32(const LogitsArgs &a, int sm_count, cudaStream_t stream) {
    return launch_policy_rows<false>(a, sm_count, stream);
}

cudaError_t preference_loss_f32(const LogitsArgs &a, int sm_count, cudaStream_t stream) {
    return launch_preference_rows<false>(a, sm_count, stream);
}

}  // namespace aloco
