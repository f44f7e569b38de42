// Layer norm of rows of 16-bit floats.
#include "layer_norm_dev.cuh"

namespace ivk {

template cudaError_t layer_norm_typed<__half, __half>(const LayerNormArgs &, int, cudaStream_t);
template cudaError_t layer_norm_typed<__half, float>(const LayerNormArgs &, int, cudaStream_t);

}  // namespace ivk
