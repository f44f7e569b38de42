// Rows taken by groups of threads, eight consecutive elements at a time: loads and stores at any element alignment, sums
// over a group, weights widened into shared memory (layer norm and its gradient).
#pragma once
#include "element_dev.cuh"

namespace ivk {
namespace rows {

using elem::Pair;
using elem::unpair;

// Elements of vector v that are in a row of `dim`.
__device__ __forceinline__ uint32_t left_of(uint32_t v, uint32_t dim) { return v * 8u < dim ? (dim - v * 8u < 8u ? dim - v * 8u : 8u) : 0u; }

// Elements 8 v .. 8 v + 7 of a row as they lie in memory.  ALIGNED: rows start at 16-byte boundaries and are whole vectors.
template <typename T, bool ALIGNED>
struct RowVector {
    elem::Vector<T, 8, ALIGNED ? 16 : elem::kAny> raw;
    __device__ __forceinline__ void load(const T *row, uint32_t v, uint32_t dim) {
        const uint32_t left = left_of(v, dim);
        const T *p = row + v * 8u;
        if (ALIGNED ? left : left == 8u) raw.load(p, ALIGNED ? 0u : elem::misalignment(p));
        else {
            raw.zero();
            if constexpr (!ALIGNED) {                     // single elements, where get() looks for them when it shifts nothing
                if (left) {
                    float e[8];
#pragma unroll
                    for (uint32_t i = 0; i < 8u; ++i) e[i] = i < left ? elem::to_float(p[i]) : 0.f;
                    elem::Packed<T, 8> some;
                    some.pack(e);
#pragma unroll
                    for (int i = 0; i < elem::Packed<T, 8>::kWords; ++i) raw.w[i] = some.w[i];
                }
            }
        }
    }
    // The elements, zeros behind the row's end.  row_off: the row's bytes from a 16-byte boundary (and a vector's: it is 16 or 32 bytes)
    __device__ __forceinline__ elem::Packed<T, 8> get(uint32_t row_off, uint32_t v, uint32_t dim) const {
        return raw.get(ALIGNED || left_of(v, dim) < 8u ? 0u : row_off);
    }
};

// Vectors of eight elements by consecutive lanes, `width` lanes to a row, to consecutive places at any element alignment: a lane
// stores the aligned pieces that begin in its elements, with its neighbour's first bytes behind its own, and what no lane's piece
// covers (a row's first and last elements, those between two warps) goes one by one.  `count`: how many of the lane's elements
// there are; by whole warps.
template <typename T>
__device__ __forceinline__ void store_pieces(T *p, const elem::Packed<T, 8> &own, uint32_t count, uint32_t width) {
    constexpr int W = elem::Packed<T, 8>::kWords;
    const uint32_t lane = threadIdx.x & (width - 1u), off = elem::misalignment(p);
    uint32_t x[W + 4];
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = own.w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[W + i] = __shfl_down_sync(0xffffffffu, own.w[i], 1);
    const bool next = __shfl_down_sync(0xffffffffu, count, 1) == 8u && lane != width - 1u;
    const uint32_t skip = (16u - off) & 15u;             // bytes of this lane before its first piece
    if (skip & 8u) {
#pragma unroll
        for (int i = 0; i < W + 2; ++i) x[i] = x[i + 2];
    }
    if (skip & 4u) {
#pragma unroll
        for (int i = 0; i < W + 1; ++i) x[i] = x[i + 1];
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = __funnelshift_r(x[i], x[i + 1], (skip & 2u) * 8u);
    }
    uint32_t *pieces = reinterpret_cast<uint32_t *>(reinterpret_cast<uint8_t *>(p) + skip);
    const bool last = next || off == 0u;                 // the last piece is there
#pragma unroll
    for (int i = 0; i < W; i += 4)
        if (count == 8u && (i + 4 < W || last)) elem::store_aligned<4>(pieces + i, x + i);
    const uint32_t head = count < 8u ? count : lane == 0u ? skip / (uint32_t)sizeof(T) : 0u;
    const uint32_t tail = count < 8u || last ? 8u : (uint32_t)(sizeof(T) * 8u - off) / (uint32_t)sizeof(T);
    if (head == 0u && tail == 8u) return;
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i)
        if (i < head || i >= tail) {
            if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(p)[i] = own.w[i];
            else reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)(own.w[i / 2] >> (16u * (i & 1u)));
        }
}

// A lane's vector v of a row; T threads to a row, by whole warps; `dim` is 0 for a row that is not there.
template <typename T, bool ALIGNED, uint32_t THREADS>
__device__ __forceinline__ void store_row_vector(T *row, uint32_t v, uint32_t dim, const Pair (&pairs)[4]) {
    float e[8];
    unpair(pairs, e);
    elem::Packed<T, 8> out;
    out.pack(e);
    T *p = row + v * 8u;
    if constexpr (ALIGNED) {
        if (v * 8u < dim) {
#pragma unroll
            for (int i = 0; i < elem::Packed<T, 8>::kWords; i += 4) elem::store_aligned<4>(reinterpret_cast<uint32_t *>(p) + i, out.w + i);
        }
    } else {
        store_pieces<T>(p, out, left_of(v, dim), THREADS < 32u ? THREADS : 32u);
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
__device__ __forceinline__ void read_params(const float4 *params, uint32_t v, uint32_t vectors, Pair (&w)[4]) {
    const float4 lo = params[v], hi = params[vectors + v];
    w[0] = Pair(lo.x, lo.y);
    w[1] = Pair(lo.z, lo.w);
    w[2] = Pair(hi.x, hi.y);
    w[3] = Pair(hi.z, hi.w);
}

}  // namespace rows

// Whether every row starts at a 16-byte boundary and consists of whole vectors of eight elements.
template <typename T>
inline bool rows_aligned(const void *p, uint64_t stride, uint64_t n, uint64_t dim) {
    return ((reinterpret_cast<uintptr_t>(p) | (n > 1 ? stride * sizeof(T) : 0u)) & 15u) == 0u && dim % 8u == 0u;
}

}  // namespace ivk
