// The gated recurrence, backward, for bf16 inputs.
#include "gated_recurrence_backward.cuh"

namespace tfg {

cudaError_t launch_scan_backward_bf16(const ScanArgs &p, const ScanMaps &maps, int vec, int kind, cudaStream_t s) {
    if (vec == 4) return launch_backward_grad<uint16_t, 4>(p, maps, kind, s);
    return launch_backward_grad<uint16_t, 1>(p, maps, kind, s);
}

}  // namespace tfg
