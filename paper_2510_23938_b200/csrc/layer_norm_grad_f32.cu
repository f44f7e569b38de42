// Gradient of layer norm of rows of 32-bit floats.
#include "layer_norm_grad_dev.cuh"

namespace ivk {

template cudaError_t layer_norm_grad_typed<float, float>(const LayerNormGradArgs &, float *, uint32_t, int, cudaStream_t);
template cudaError_t layer_norm_grad_typed<float, __half>(const LayerNormGradArgs &, float *, uint32_t, int, cudaStream_t);
template cudaError_t layer_norm_grad_typed<float, __nv_bfloat16>(const LayerNormGradArgs &, float *, uint32_t, int, cudaStream_t);

}  // namespace ivk
