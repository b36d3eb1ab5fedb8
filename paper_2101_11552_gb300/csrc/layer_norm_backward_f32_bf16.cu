// The backward of the layer norm for a stream in f32 and output gradients in bf16.
#include "layer_norm_backward.cuh"

namespace tfg {

cudaError_t launch_row_back_f32_bf16(const RowBackArgs &p, cudaStream_t s) { return launch_row_back<float, uint16_t>(p, s); }

}  // namespace tfg
