// Rows taken by groups of threads, eight consecutive elements at a time: loads and stores at any element alignment, sums
// over a group, weights widened into shared memory (layer norm and its gradient).
#pragma once
#include "element_dev.cuh"

namespace ivk {
namespace rows {

// Elements of vector v that are in a row of `dim`.
__device__ __forceinline__ uint32_t left_of(uint32_t v, uint32_t dim) { return v * 8u < dim ? (dim - v * 8u < 8u ? dim - v * 8u : 8u) : 0u; }

// Elements 8 v .. 8 v + 7 of a row as they lie in memory; zeros behind the row's end.
template <typename T, bool ALIGNED>
struct RowVector {
    elem::Vector<T, 8, ALIGNED ? 16 : elem::kAny> raw;
    bool whole;
    __device__ __forceinline__ void load(const T *row, uint32_t v, uint32_t dim) {
        const uint32_t left = left_of(v, dim);
        whole = left == 8u;
        if (whole) raw.load(row + v * 8u, elem::misalignment(row + v * 8u));
        else {
            // single elements, packed as get() gives them
            elem::Packed<T, 8> some;
            float e[8];
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) e[i] = i < left ? elem::to_float(row[v * 8u + i]) : 0.f;
            some.pack(e);
            raw.zero();
#pragma unroll
            for (int i = 0; i < elem::Packed<T, 8>::kWords; ++i) raw.w[i] = some.w[i];
        }
    }
    // row_off: the row's bytes from a 16-byte boundary (of a vector too: 8 elements are 16 or 32 bytes)
    __device__ __forceinline__ void get(uint32_t row_off, float (&e)[8]) const { raw.get(ALIGNED || !whole ? 0u : row_off).unpack(e); }
};

template <typename T, bool ALIGNED>
__device__ __forceinline__ void store_row_vector(T *row, uint32_t v, uint32_t dim, const float (&e)[8]) {
    const uint32_t left = left_of(v, dim);
    T *p = row + v * 8u;
    if (left == 8u) {
        elem::Packed<T, 8> out;
        out.pack(e);
        constexpr int W = elem::Packed<T, 8>::kWords;
        if (ALIGNED || elem::misalignment(p) == 0u) {
#pragma unroll
            for (int i = 0; i < W; i += 4) elem::store_aligned<4>(reinterpret_cast<uint32_t *>(p) + i, out.w + i);
        } else if ((elem::misalignment(p) & 7u) == 0u) {
#pragma unroll
            for (int i = 0; i < W; i += 2) elem::store_aligned<2>(reinterpret_cast<uint32_t *>(p) + i, out.w + i);
        } else if ((elem::misalignment(p) & 3u) == 0u) {
#pragma unroll
            for (int i = 0; i < W; ++i) reinterpret_cast<uint32_t *>(p)[i] = out.w[i];
        } else {
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int i = 0; i < 8; ++i) reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)(out.w[i / 2] >> (16 * (i & 1)));
            }
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i)
            if (i < left) p[i] = elem::from_float<T>(e[i]);
    }
}

template <int N>
__device__ __forceinline__ float sum_of(float (&x)[N]) {
#pragma unroll
    for (int d = N / 2; d; d >>= 1)
#pragma unroll
        for (int i = 0; i < d; ++i) x[i] += x[i + d];
    return x[0];
}

// Waits for the T threads (64 or more, whole warps) of this thread's group.
template <uint32_t T>
__device__ __forceinline__ void group_barrier() {
    asm volatile("bar.sync %0, %1;" ::"r"(threadIdx.x / T + 1u), "n"(T) : "memory");
}

// Sum over a group of T threads, in a fixed order; every thread gets it.  `slots`: one float per warp of the CTA, which the
// group may write again once it has met at another barrier of its own (two alternating arrays need no other).
template <uint32_t T>
__device__ __forceinline__ float group_sum(float x, float *slots) {
#pragma unroll
    for (uint32_t d = (T < 32u ? T : 32u) / 2u; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    if constexpr (T > 32u) {
        constexpr uint32_t kWarps = T / 32u;
        const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
        if (lane == 0u) slots[warp] = x;
        group_barrier<T>();
        x = slots[(warp & ~(kWarps - 1u)) + (lane & (kWarps - 1u))];
#pragma unroll
        for (uint32_t d = kWarps / 2u; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    }
    return x;
}

__device__ __forceinline__ float param_at(const void *p, int type, uint32_t i) {
    if (type == IV_F32) return static_cast<const float *>(p)[i];
    if (type == IV_F16) return elem::to_float(static_cast<const __half *>(p)[i]);
    return elem::to_float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

// `dim` weights in 32 bits, by the whole CTA: the first halves of all vectors of eight, then the second halves, so that a
// warp's 16-byte reads of consecutive vectors touch every bank once.
__device__ __forceinline__ void widen_params(const void *p, int type, uint32_t dim, float4 *out) {
    const uint32_t vectors = (dim + 7u) / 8u;
    float *o = reinterpret_cast<float *>(out);
    for (uint32_t i = threadIdx.x; i < vectors * 8u; i += blockDim.x)
        o[((i >> 2 & 1u) * vectors + (i >> 3)) * 4u + (i & 3u)] = i < dim ? param_at(p, type, i) : 0.f;
}
__device__ __forceinline__ void read_params(const float4 *params, uint32_t v, uint32_t vectors, float (&w)[8]) {
    const float4 lo = params[v], hi = params[vectors + v];
    w[0] = lo.x; w[1] = lo.y; w[2] = lo.z; w[3] = lo.w;
    w[4] = hi.x; w[5] = hi.y; w[6] = hi.z; w[7] = hi.w;
}

}  // namespace rows

// Whether every row starts at a 16-byte boundary.
template <typename T>
inline bool rows_aligned(const void *p, uint64_t stride, uint64_t n) {
    return ((reinterpret_cast<uintptr_t>(p) | (n > 1 ? stride * sizeof(T) : 0u)) & 15u) == 0u;
}

}  // namespace ivk
