// The backward of the group norm for fp32 features and fp32 gradients.
#include "group_norm_backward.cuh"

namespace tfg {

cudaError_t launch_group_norm_backward_f32_f32(const NormArgs &p, int act, float *grad_gamma, float *grad_beta, cudaStream_t s) {
    return launch_back<float, float>(p, act, grad_gamma, grad_beta, s);
}

}  // namespace tfg
