// AdamW step: dispatch by types.  The instances lie in a file for each type of the weights, so that they compile side by side.
#include "element_dev.cuh"
#include "iv_internal.h"

namespace ivk {

template <typename Tw, typename Tg>
cudaError_t adamw_typed(const AdamwArgs &a, uint32_t *arrived, uint32_t *d_status, int sm_count, cudaStream_t stream);

cudaError_t launch_adamw(const AdamwArgs &a, uint32_t *d_arrived, uint32_t *d_status, int sm_count, cudaStream_t stream, uint64_t *launches) {
    ++*launches;
    return by_types(a.set.type, a.grad_type, [&](auto weight, auto grad) {
        return adamw_typed<typename decltype(weight)::type, typename decltype(grad)::type>(a, d_arrived, d_status, sm_count, stream);
    });
}

}  // namespace ivk
