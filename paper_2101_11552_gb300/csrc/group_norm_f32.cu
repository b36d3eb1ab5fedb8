// The forward of the group norm for fp32 features.
#include "group_norm_forward.cuh"

namespace tfg {

cudaError_t launch_group_norm_f32(const NormArgs &p, int act, bool out_bf16, cudaStream_t s) {
    return launch_vec<float>(p, act, out_bf16, s);
}

}  // namespace tfg
