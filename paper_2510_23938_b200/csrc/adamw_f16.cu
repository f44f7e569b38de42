// AdamW step of weights of 16-bit floats.
#include "adamw_dev.cuh"

namespace ivk {

template cudaError_t adamw_typed<__half, __half>(const AdamwArgs &, uint32_t *, uint32_t *, int, cudaStream_t);
template cudaError_t adamw_typed<__half, float>(const AdamwArgs &, uint32_t *, uint32_t *, int, cudaStream_t);

}  // namespace ivk
