// Gradient of layer norm: dispatch by types, and the last additions of the sums over rows.  The instances lie in a file for each type of
// the rows, so that they compile side by side.
#include "element_dev.cuh"
#include "iv_internal.h"
#include "layer_norm_grad.h"
#include "row_dev.cuh"

namespace ivk {

template <typename Tx, typename Ty>
cudaError_t layer_norm_grad_typed(const LayerNormGradArgs &a, float *partial, uint32_t parts, int sm_count, cudaStream_t stream);

namespace {

using namespace rows;

// The parts' sums of 32 columns: a warp adds up every 32nd part, then the warps' sums are added first to last.
constexpr uint32_t kSlices = 32, kEachSlice = (kMostParts + kSlices - 1) / kSlices;
__global__ void __launch_bounds__(32 * kSlices)
norm_grad_columns_kernel(const float *partial, uint32_t parts, uint32_t dim, void *dw, void *db, int type, bool accumulate) {
    __shared__ float sums[kSlices][33];
    const uint32_t lane = threadIdx.x & 31u, slice = threadIdx.x >> 5;
    const uint32_t c = blockIdx.x * 32u + lane, width = 2u * dim;
    void *out = c < dim ? dw : c < width ? db : nullptr;
    allow_next_kernel();
    wait_for_previous_kernel();
    float part[kEachSlice], sum = 0.f;                   // all on their way at once
#pragma unroll
    for (uint32_t i = 0; i < kEachSlice; ++i) {
        const uint32_t p = slice + i * kSlices;
        part[i] = out && p < parts ? __ldcg(partial + (uint64_t)p * width + c) : 0.f;
    }
#pragma unroll
    for (uint32_t i = 0; i < kEachSlice; ++i) sum += part[i];
    sums[slice][lane] = sum;
    __syncthreads();
    if (slice || !out) return;
    sum = 0.f;
#pragma unroll
    for (uint32_t s = 0; s < kSlices; ++s) sum += sums[s][lane];
    const uint32_t i = c < dim ? c : c - dim;
    if (accumulate) sum += param_at(out, type, i);
    if (type == IV_F32) static_cast<float *>(out)[i] = sum;
    else if (type == IV_F16) static_cast<__half *>(out)[i] = elem::from_float<__half>(sum);
    else static_cast<__nv_bfloat16 *>(out)[i] = elem::from_float<__nv_bfloat16>(sum);
}

}  // namespace

uint64_t layer_norm_grad_scratch_bytes(uint64_t n, uint64_t dim) {
    return 8u * dim * parts_for(n, dim) + (dim > kWidest ? 8u * n : 0u);
}

cudaError_t launch_layer_norm_grad(const LayerNormGradArgs &a, float *d_partial, int sm_count, cudaStream_t stream, uint64_t *launches) {
    if (a.dim == 0 || (a.n == 0 && !a.d_dw && !a.d_db)) return cudaSuccess;
    const uint32_t parts = a.n ? (uint32_t)parts_for(a.n, a.dim) : 0u;
    if (a.n) {
        cudaError_t e = by_types(a.x_type, a.y_type, [&](auto in, auto out) {
            return layer_norm_grad_typed<typename decltype(in)::type, typename decltype(out)::type>(a, d_partial, parts, sm_count, stream);
        });
        if (e != cudaSuccess) return e;
        *launches += a.dim > kWidest ? 2u : 1u;
    }
    if (!a.d_dw && !a.d_db) return cudaSuccess;
    ++*launches;
    const uint32_t dim = (uint32_t)a.dim;
    return launch_overlapping(norm_grad_columns_kernel, dim3((2u * dim + 31u) / 32u), dim3(32 * kSlices), 0, stream,
                              d_partial, parts, dim, a.d_dw, a.d_db, a.dw_type, a.accumulate);
}

}  // namespace ivk
