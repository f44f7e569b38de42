// Layer norm: dispatch by types.  The instances lie in a file for each input type, so that they compile side by side.
#include "element_dev.cuh"
#include "iv_internal.h"

namespace ivk {

template <typename Tx, typename Ty>
cudaError_t layer_norm_typed(const LayerNormArgs &a, int sm_count, cudaStream_t stream);

cudaError_t launch_layer_norm(const LayerNormArgs &a, int sm_count, cudaStream_t stream, uint64_t *launches) {
    if (a.n == 0 || a.dim == 0) return cudaSuccess;
    ++*launches;
    return by_types(a.x_type, a.y_type, [&](auto in, auto out) {
        return layer_norm_typed<typename decltype(in)::type, typename decltype(out)::type>(a, sm_count, stream);
    });
}

}  // namespace ivk
