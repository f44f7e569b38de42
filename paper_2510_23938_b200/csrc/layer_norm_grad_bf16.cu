// Gradient of layer norm of rows of 16-bit brain floats.
#include "layer_norm_grad_dev.cuh"

namespace ivk {

template cudaError_t layer_norm_grad_typed<__nv_bfloat16, __nv_bfloat16>(const LayerNormGradArgs &, float *, uint32_t, int, cudaStream_t);
template cudaError_t layer_norm_grad_typed<__nv_bfloat16, float>(const LayerNormGradArgs &, float *, uint32_t, int, cudaStream_t);

}  // namespace ivk
