// The gated recurrence, backward, for bf16 inputs.
#include "gated_recurrence_backward.cuh"

namespace tfg {

cudaError_t launch_scan_backward_bf16(const ScanArgs &p, int vec, int kind, cudaStream_t s) {
    if (vec == 8) return launch_backward_grad<uint16_t, 8>(p, kind, s);
    return launch_backward_grad<uint16_t, 1>(p, kind, s);
}

}  // namespace tfg
