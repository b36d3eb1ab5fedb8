// The forward of the group norm for bf16 features.
#include "group_norm_forward.cuh"

namespace tfg {

cudaError_t launch_group_norm_bf16(const NormArgs &p, int act, bool out_bf16, cudaStream_t s) {
    return launch_vec<uint16_t>(p, act, out_bf16, s);
}

}  // namespace tfg
