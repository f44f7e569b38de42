// Layer norm of rows of 32-bit floats.
#include "layer_norm_dev.cuh"

namespace ivk {

template cudaError_t layer_norm_typed<float, float>(const LayerNormArgs &, int, cudaStream_t);
template cudaError_t layer_norm_typed<float, __half>(const LayerNormArgs &, int, cudaStream_t);
template cudaError_t layer_norm_typed<float, __nv_bfloat16>(const LayerNormArgs &, int, cudaStream_t);

}  // namespace ivk
