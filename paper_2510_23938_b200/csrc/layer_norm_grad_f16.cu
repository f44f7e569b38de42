// Gradient of layer norm of rows of 16-bit floats.
#include "layer_norm_grad_dev.cuh"

namespace ivk {

template cudaError_t layer_norm_grad_typed<__half, __half>(const LayerNormGradArgs &, float *, uint32_t, int, cudaStream_t);
template cudaError_t layer_norm_grad_typed<__half, float>(const LayerNormGradArgs &, float *, uint32_t, int, cudaStream_t);

}  // namespace ivk
