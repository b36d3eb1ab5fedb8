// The backward of the layer norm for a stream in bf16 and output gradients in bf16.
#include "layer_norm_backward.cuh"

namespace tfg {

cudaError_t launch_row_back_bf16_bf16(const RowBackArgs &p, cudaStream_t s) { return launch_row_back<uint16_t, uint16_t>(p, s); }

}  // namespace tfg
