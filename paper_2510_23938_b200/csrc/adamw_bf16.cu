// AdamW step of weights of 16-bit brain floats.
#include "adamw_dev.cuh"

namespace ivk {

template cudaError_t adamw_typed<__nv_bfloat16, __nv_bfloat16>(const AdamwArgs &, uint32_t *, uint32_t *, int, cudaStream_t);
template cudaError_t adamw_typed<__nv_bfloat16, float>(const AdamwArgs &, uint32_t *, uint32_t *, int, cudaStream_t);

}  // namespace ivk
