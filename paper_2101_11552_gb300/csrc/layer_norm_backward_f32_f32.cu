// The backward of the layer norm for a stream in f32 and output gradients in f32.
#include "layer_norm_backward.cuh"

namespace tfg {

cudaError_t launch_row_back_f32_f32(const RowBackArgs &p, cudaStream_t s) { return launch_row_back<float, float>(p, s); }

}  // namespace tfg
