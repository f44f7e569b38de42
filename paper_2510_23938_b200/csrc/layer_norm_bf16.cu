// Layer norm of rows of 16-bit brain floats.
#include "layer_norm_dev.cuh"

namespace ivk {

template cudaError_t layer_norm_typed<__nv_bfloat16, __nv_bfloat16>(const LayerNormArgs &, int, cudaStream_t);
template cudaError_t layer_norm_typed<__nv_bfloat16, float>(const LayerNormArgs &, int, cudaStream_t);

}  // namespace ivk
