// Layer norm of rows, and its root-mean-square form:
//     mu = mean(x) (rms: 0),  r = 1 / sqrt(mean((x - mu)^2) + eps),  y = round((x - mu) r w + b)
//
// Bound by memory: a row is read once, held in registers for both sums (the mean first, then the squares of what is left,
// so nothing cancels) and written once.  the threads of a row, 8 to 512 with one to four
// vectors of eight elements each, follow from its width and type alone, and so does the order of its sums: a row's bits do not depend on the other rows, on the
// launch or on the alignment.  Weight and bias are widened into shared memory once per CTA.
#include "element_dev.cuh"
#include "iv_internal.h"
#include "row_dev.cuh"

namespace ivk {

namespace {

using namespace rows;
using elem::Pair;

constexpr uint32_t kThreads = 512;

// Aligned rows: the next row is on its way while one is worked on.
template <typename Tx, typename Ty, uint32_t T, int NV, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, NV * sizeof(Tx) > 8 ? 1 : 2)
layer_norm_kernel(const __grid_constant__ LayerNormArgs a) {
    constexpr uint32_t kGroups = kThreads / T;
    extern __shared__ float4 params[];                   // weight, then bias: two planes each
    __shared__ float slots[2][kThreads / 32];
    const uint32_t t = threadIdx.x % T, group = threadIdx.x / T;
    const uint32_t dim = (uint32_t)a.dim, vectors = (dim + 7u) / 8u;
    const Tx *x = static_cast<const Tx *>(a.d_x);
    Ty *y = static_cast<Ty *>(a.d_y);
    RowVector<Tx, ALIGNED> next[NV];
    const uint64_t step = (uint64_t)gridDim.x * kGroups;
    // a row that is not there is a row without elements: all groups of a warp stay together
    auto fetch = [&](uint64_t row) {
        const Tx *p = x + (row < a.n ? row * a.x_stride : 0u);
#pragma unroll
        for (int j = 0; j < NV; ++j) next[j].load(p, t + j * T, row < a.n ? dim : 0u);
    };
    uint64_t base = (uint64_t)blockIdx.x * kGroups;
    if (ALIGNED) fetch(base + group);
    if (a.d_weight) widen_params(a.d_weight, a.param_type, dim, params);
    float4 *bias = params + (a.d_weight ? 2u * vectors : 0u);
    if (a.d_bias) widen_params(a.d_bias, a.param_type, dim, bias);
    __syncthreads();
    const float scale = 1.f / (float)dim;
    for (; base < a.n; base += step) {
        const uint64_t row = base + group;
        const bool live = row < a.n;
        elem::Packed<Tx, 8> raw[NV];
        if (!ALIGNED) fetch(row);
        const uint32_t off = ALIGNED ? 0u : elem::misalignment(x + (live ? row * a.x_stride : 0u));
#pragma unroll
        for (int j = 0; j < NV; ++j) raw[j] = next[j].get(off, t + j * T, live ? dim : 0u);
        if (ALIGNED && base + step < a.n) fetch(row + step);
        float mean = 0.f;
        if (!a.rms) {
            float sum[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                Pair v[4];
                elem::unpack8(raw[j], v);
                sum[j] = ((v[0] + v[1]) + (v[2] + v[3])).sum();
            }
            mean = group_sum<T>(sum_of<NV>(sum), slots[0]) * scale;
        }
        const Pair shift(-mean);
        float squares[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            Pair v[4], s(0.f);
            elem::unpack8(raw[j], v);
            const uint32_t left = left_of(t + j * T, dim);
            if (!ALIGNED && left < 8u && left) {             // zeros behind the row's end that are not the mean away from it
#pragma unroll
                for (uint32_t i = 0; i < 4u; ++i) {
                    float lo, hi;
                    v[i].get(lo, hi);
                    v[i] = Pair(2u * i < left ? lo : mean, 2u * i + 1u < left ? hi : mean);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Pair d = v[i] + shift;
                s = fma2(d, d, s);
            }
            squares[j] = left ? s.sum() : 0.f;
        }
        const float rstd = 1.f / sqrtf(group_sum<T>(sum_of<NV>(squares), slots[1]) * scale + a.eps);
        Ty *out = y + (live ? row * a.y_stride : 0u);
        const Pair by(rstd);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t v = t + j * T, at = v < vectors ? v : 0u;
            Pair e[4], w[4];
            elem::unpack8(raw[j], e);
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = (e[i] + shift) * by;
            if (a.d_weight) {
                read_params(params, at, vectors, w);
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = e[i] * w[i];
            }
            if (a.d_bias) {
                read_params(bias, at, vectors, w);
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = e[i] + w[i];
            }
            store_row_vector<Ty, ALIGNED, T>(out, v, live ? dim : 0u, e);
        }
        if (live && t == 0u) {
            if (a.d_mean) a.d_mean[row] = mean;
            if (a.d_rstd) a.d_rstd[row] = rstd;
        }
    }
}

// Rows too wide for that: one CTA per row, which reads it three times (from the L2 cache the second and third time).
constexpr uint32_t kWideThreads = 1024;
template <typename Tx, typename Ty>
__global__ void __launch_bounds__(kWideThreads)
layer_norm_wide_kernel(LayerNormArgs a) {
    __shared__ float slots[2][kWideThreads / 32];
    const uint32_t dim = (uint32_t)a.dim, vectors = (dim + 7u) / 8u;
    const float scale = 1.f / (float)dim;
    for (uint64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const Tx *in = static_cast<const Tx *>(a.d_x) + row * a.x_stride;
        Ty *out = static_cast<Ty *>(a.d_y) + row * a.y_stride;
        const uint32_t off = elem::misalignment(in);
        auto each = [&](auto f) {
            for (uint32_t base = 0; base < vectors; base += kWideThreads) {      // whole warps
                const uint32_t v = base + threadIdx.x;
                RowVector<Tx, false> raw;
                Pair e[4];
                raw.load(in, v, dim);
                elem::unpack8(raw.get(off, v, dim), e);
                f(v, e);
            }
        };
        float mean = 0.f, sum = 0.f;
        if (!a.rms) {
            each([&](uint32_t, Pair (&e)[4]) { sum += ((e[0] + e[1]) + (e[2] + e[3])).sum(); });
            mean = group_sum<kWideThreads>(sum, slots[0]) * scale;
        }
        sum = 0.f;
        each([&](uint32_t v, Pair (&p)[4]) {
            const uint32_t left = left_of(v, dim);
            float e[8], part = 0.f;
            unpair(p, e);
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) part = i < left ? fmaf(e[i] - mean, e[i] - mean, part) : part;
            sum += part;
        });
        const float rstd = 1.f / sqrtf(group_sum<kWideThreads>(sum, slots[1]) * scale + a.eps);
        each([&](uint32_t v, Pair (&p)[4]) {
            const uint32_t left = left_of(v, dim);
            float e[8];
            unpair(p, e);
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) {
                e[i] = (e[i] - mean) * rstd;
                if (i < left && a.d_weight) e[i] *= param_at(a.d_weight, a.param_type, v * 8u + i);
                if (i < left && a.d_bias) e[i] += param_at(a.d_bias, a.param_type, v * 8u + i);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = Pair(e[2 * i], e[2 * i + 1]);
            store_row_vector<Ty, false, kWideThreads>(out, v, dim, p);
        });
        if (threadIdx.x == 0) {
            if (a.d_mean) a.d_mean[row] = mean;
            if (a.d_rstd) a.d_rstd[row] = rstd;
        }
    }
}

template <typename Tx, typename Ty, uint32_t T, int NV, bool ALIGNED>
cudaError_t launch_instance(const LayerNormArgs &a, int sm_count, cudaStream_t stream) {
    auto kernel = layer_norm_kernel<Tx, Ty, T, NV, ALIGNED>;
    const uint64_t vectors = (a.dim + 7u) / 8u;
    const size_t shared = 32u * vectors * ((a.d_weight ? 1u : 0u) + (a.d_bias ? 1u : 0u));
    static bool done[kMaxDevices] = {};
    if (shared > 47u << 10) {                               // with the sums' slots beyond what a kernel has without asking
        cudaError_t e = ensure_dynamic_smem(kernel, 2u * 32u * T * NV, done);
        if (e != cudaSuccess) return e;
    }
    const uint64_t blocks = (a.n + kThreads / T - 1) / (kThreads / T), most = (uint64_t)sm_count * 2u;
    kernel<<<(uint32_t)(blocks < most ? blocks : most), kThreads, shared, stream>>>(a);
    return cudaGetLastError();
}

template <typename Tx, typename Ty, bool ALIGNED>
cudaError_t launch_width(const LayerNormArgs &a, int sm_count, cudaStream_t stream) {
    const uint64_t v = (a.dim + 7u) / 8u;
    if (v <= 8u) return launch_instance<Tx, Ty, 8, 1, ALIGNED>(a, sm_count, stream);
    if (v <= 16u) return launch_instance<Tx, Ty, 16, 1, ALIGNED>(a, sm_count, stream);
    if (v <= 32u) return launch_instance<Tx, Ty, 32, 1, ALIGNED>(a, sm_count, stream);
    if (v <= 64u) return launch_instance<Tx, Ty, 32, 2, ALIGNED>(a, sm_count, stream);
    // 64 bytes of a row per thread, or 128 where the row needs them
    constexpr int NV = 8 / (int)sizeof(Tx);
    if (v <= 32u * NV) return launch_instance<Tx, Ty, 32, NV, ALIGNED>(a, sm_count, stream);
    if (v <= 64u * NV) return launch_instance<Tx, Ty, 64, NV, ALIGNED>(a, sm_count, stream);
    if (v <= 128u * NV) return launch_instance<Tx, Ty, 128, NV, ALIGNED>(a, sm_count, stream);
    if (v <= 256u * NV) return launch_instance<Tx, Ty, 256, NV, ALIGNED>(a, sm_count, stream);
    if (v <= 512u * NV) return launch_instance<Tx, Ty, 512, NV, ALIGNED>(a, sm_count, stream);
    return launch_instance<Tx, Ty, 512, 4, ALIGNED>(a, sm_count, stream);
}

}  // namespace

cudaError_t launch_layer_norm(const LayerNormArgs &a, int sm_count, cudaStream_t stream, uint64_t *launches) {
    if (a.n == 0 || a.dim == 0) return cudaSuccess;
    ++*launches;
    return by_types(a.x_type, a.y_type, [&](auto in, auto out) {
        using Tx = typename decltype(in)::type;
        using Ty = typename decltype(out)::type;
        if (a.dim > 8u * kThreads * 4u) {
            const uint64_t most = (uint64_t)sm_count * 2u;
            layer_norm_wide_kernel<Tx, Ty><<<(uint32_t)(a.n < most ? a.n : most), kWideThreads, 0, stream>>>(a);
            return cudaGetLastError();
        }
        return rows_aligned<Tx>(a.d_x, a.x_stride, a.n, a.dim) && rows_aligned<Ty>(a.d_y, a.y_stride, a.n, a.dim)
                   ? launch_width<Tx, Ty, true>(a, sm_count, stream)
                   : launch_width<Tx, Ty, false>(a, sm_count, stream);
    });
}

}  // namespace ivk
