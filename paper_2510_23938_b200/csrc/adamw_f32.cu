// AdamW step of weights of 32-bit floats.
#include "adamw_dev.cuh"

namespace ivk {

template cudaError_t adamw_typed<float, float>(const AdamwArgs &, uint32_t *, uint32_t *, int, cudaStream_t);
template cudaError_t adamw_typed<float, __half>(const AdamwArgs &, uint32_t *, uint32_t *, int, cudaStream_t);
template cudaError_t adamw_typed<float, __nv_bfloat16>(const AdamwArgs &, uint32_t *, uint32_t *, int, cudaStream_t);

}  // namespace ivk
