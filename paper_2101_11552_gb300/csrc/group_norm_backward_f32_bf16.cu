// The backward of the group norm for fp32 features and bf16 gradients.
#include "group_norm_backward.cuh"

namespace tfg {

cudaError_t launch_group_norm_backward_f32_bf16(const NormArgs &p, int act, float *grad_gamma, float *grad_beta, cudaStream_t s) {
    return launch_back<float, uint16_t>(p, act, grad_gamma, grad_beta, s);
}

}  // namespace tfg
