// The post-training losses on bf16 logits.
#include "aloco_logits.cuh"

namespace aloco {

cudaError_t token_logprobs_bf16(const LogitsArgs &a, int sm_count, cudaStream_t stream) {
    int used;
    return launch_rows<true, kFwd>(a, sm_count, stream, &used);
}

cudaError_t policy_loss_bf16(const LogitsArgs &a, int sm_count, cudaStream_t stream) {
    return launch_policy_rows<true>(a, sm_count, stream);
}

cudaError_t preference_loss_bf16(const LogitsArgs &a, int sm_count, cudaStream_t stream) {
    return launch_preference_rows<true>(a, sm_count, stream);
}

}  // namespace aloco
