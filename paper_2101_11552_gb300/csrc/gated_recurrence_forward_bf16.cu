// The gated recurrence, forward, for bf16 inputs.
#include "gated_recurrence_forward.cuh"

namespace tfg {

cudaError_t launch_scan_forward_bf16(const ScanArgs &p, const ScanMaps &maps, int vec, int kind, cudaStream_t s) {
    if (vec == 4) return launch_forward_kind<uint16_t, 4>(p, maps, kind, s);
    return launch_forward_kind<uint16_t, 1>(p, maps, kind, s);
}

}  // namespace tfg
