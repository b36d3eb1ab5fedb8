// The gated recurrence, backward, for f32 inputs.
#include "gated_recurrence_backward.cuh"

namespace tfg {

cudaError_t launch_scan_backward_f32(const ScanArgs &p, int vec, int kind, cudaStream_t s) {
    if (vec == 4) return launch_backward_grad<float, 4>(p, kind, s);
    return launch_backward_grad<float, 1>(p, kind, s);
}

}  // namespace tfg
