// Rows taken by groups of threads, eight consecutive elements at a time: loads and stores at any element alignment, sums
// over a group, copies of rows into shared memory (layer norm and its gradient).
#pragma once
#include "element_dev.cuh"

namespace ivk {
namespace rows {

using elem::Pair;
using elem::unpair;

// How rows lie: anywhere; at 16-byte boundaries and in whole vectors of eight elements; so that all threads of a row's group
// have the same number of vectors too; or so, but anywhere.
enum Rows { kAnyRows = 0, kAlignedRows = 1, kExactRows = 2, kShiftedRows = 3 };

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
// covers (a row's first and last elements, those between two warps) goes in smaller ones.  `count`: how many of the lane's elements
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
    uint8_t *bytes = reinterpret_cast<uint8_t *>(p);
    if (count == 8u && lane == 0u && skip) {             // the elements before the first piece: 2, 4 and 8 bytes of them
        if (sizeof(T) == 2 && (skip & 2u)) *reinterpret_cast<uint16_t *>(bytes) = (uint16_t)own.w[0];
        if (skip & 4u) *reinterpret_cast<uint32_t *>(bytes + (skip & 2u)) = __funnelshift_r(own.w[0], own.w[1], (skip & 2u) * 8u);
        if (skip & 8u) {
            const bool word = skip & 4u;
            const uint32_t a = word ? own.w[1] : own.w[0], b = word ? own.w[2] : own.w[1], c = word ? own.w[3] : own.w[2];
            *reinterpret_cast<uint2 *>(bytes + (skip & 6u)) = make_uint2(__funnelshift_r(a, b, (skip & 2u) * 8u), __funnelshift_r(b, c, (skip & 2u) * 8u));
        }
    }
    if (count == 8u && !last) {                          // those behind the last whole piece: 8, 4 and 2 bytes
        bytes += sizeof(T) * 8u - off;
        if (off & 8u) *reinterpret_cast<uint2 *>(bytes) = make_uint2(x[W - 4], x[W - 3]);
        const uint32_t c = off & 8u ? x[W - 2] : x[W - 4], d = off & 8u ? x[W - 1] : x[W - 3];
        if (off & 4u) *reinterpret_cast<uint32_t *>(bytes + (off & 8u)) = c;
        if (sizeof(T) == 2 && (off & 2u)) *reinterpret_cast<uint16_t *>(bytes + (off & 12u)) = (uint16_t)(off & 4u ? d : c);
    }
    if (count < 8u) {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i)
            if (i < count) {
                if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(p)[i] = own.w[i];
                else reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)(own.w[i / 2] >> (16u * (i & 1u)));
            }
    }
}

// A lane's vector v of a row; T threads to a row, by whole warps; `live`: the row is there.
template <typename T, int MODE, uint32_t THREADS>
__device__ __forceinline__ void store_row_vector(T *row, uint32_t v, uint32_t dim, bool live, const Pair (&pairs)[4]) {
    float e[8];
    unpair(pairs, e);
    elem::Packed<T, 8> out;
    out.pack(e);
    T *p = row + v * 8u;
    if constexpr (MODE != kAnyRows) {
        if (live && (MODE == kExactRows || v * 8u < dim)) {
            if (sizeof(T) == 4 && (reinterpret_cast<uintptr_t>(row) & 16u) == 0u) elem::store_32_bytes(p, out.w);
            else {
#pragma unroll
                for (int i = 0; i < elem::Packed<T, 8>::kWords; i += 4) elem::store_aligned<4>(reinterpret_cast<uint32_t *>(p) + i, out.w + i);
            }
        }
    } else {
        store_pieces<T>(p, out, live ? left_of(v, dim) : 0u, THREADS < 32u ? THREADS : 32u);
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

// sum / count, `inverse` being 1 / count rounded.  Times that alone the mean of equal numbers can be off in its last place, which
// 1 / sqrt(eps) then multiplies; what the product leaves of the sum, times it again, mends that: right to the last place
// wherever the quotient is a 32-bit float.  (A division instead changes nothing but the code around it: norm of 131072 x 4096, root-mean-square
// form, 388 us for 338, gradient of 32768 x 8192 307 for 281, but norm of 32768 x 16384 406 for 446.)
__device__ __forceinline__ float mean_of(float sum, float count, float inverse) {
    const float q = sum * inverse;
    return fabsf(q) < __uint_as_float(0x7f800000u) ? fmaf(fmaf(-q, count, sum), inverse, q) : q;
}

__device__ __forceinline__ float param_at(const void *p, int type, uint32_t i) {
    if (type == IV_F32) return static_cast<const float *>(p)[i];
    if (type == IV_F16) return elem::to_float(static_cast<const __half *>(p)[i]);
    return elem::to_float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

__device__ __forceinline__ void copy_async16(void *shared, const void *global) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(shared)), "l"(global) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// f of the sums of N values (a power of two, at most 8) over a group of T threads; every thread gets all.  The order is that of a
// tree over the threads' numbers, upper bits first, whatever N.  Lanes halve the values among them before they halve themselves,
// so that eight values take nine exchanges.  `slots`: a float per value and warp; a call writes them while others may still read
// those of the call before, so calls alternate between two arrays.
template <uint32_t T, int N, typename F>
__device__ __forceinline__ void group_sums(float (&v)[N], float *slots, F f) {
    constexpr uint32_t kWidth = T < 32u ? T : 32u, L = kWidth / N;      // L lanes end up with one value
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    uint32_t d = kWidth / 2u;
#pragma unroll
    for (int n = N; n > 1; n /= 2, d /= 2u) {
        const bool upper = lane & d;
#pragma unroll
        for (int i = 0; i < n / 2; ++i) {
            const float send = upper ? v[i] : v[i + n / 2], keep = upper ? v[i + n / 2] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, d);
        }
    }
    float x = v[0];
#pragma unroll
    for (; d; d /= 2u) x += __shfl_xor_sync(0xffffffffu, x, d);
    if constexpr (T > 32u) {
        constexpr uint32_t kWarps = T / 32u, kEach = kWarps > L ? kWarps / L : 1u, kLanes = kWarps > L ? L : kWarps;
        const uint32_t value = lane / L, q = lane & (kLanes - 1u);
        constexpr uint32_t kAll = T > 512u ? 32u : 16u;                 // warps of a CTA
        if (lane % L == 0u) slots[value * kAll + warp] = x;
        group_barrier<T>();
        float part[kEach];
#pragma unroll
        for (uint32_t e = 0; e < kEach; ++e) part[e] = slots[value * kAll + (warp & ~(kWarps - 1u)) + q + e * kLanes];
        x = sum_of<(int)kEach>(part);
#pragma unroll
        for (uint32_t k = kLanes / 2u; k; k /= 2u) x += __shfl_xor_sync(0xffffffffu, x, k);
    }
    x = f(x);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, x, i * L, kWidth);
}

// The vectors of WIDTH consecutive lanes in a row, as the lanes bring them into shared memory with asynchronous copies of 16 bytes,
// each the pieces in its turn: every piece of the row comes once, whatever its alignment.  The lanes read them after
// wait_copies and a __syncwarp.
template <typename T, uint32_t WIDTH, int MODE>
struct Segment {
    static constexpr bool kAligned = MODE == kAlignedRows || MODE == kExactRows, kWhole = MODE == kExactRows || MODE == kShiftedRows;
    static constexpr uint32_t kEach = sizeof(T) / 2u, kPieces = WIDTH * kEach + (kAligned ? 0u : 1u);
    // v: this lane's vector, `lane` its number among the WIDTH
    static __device__ __forceinline__ void fetch(uint4 *to, const T *row, uint32_t v, uint32_t lane, uint32_t dim) {
        const uint32_t first = (v - lane) * 8u;
        const uint8_t *p = reinterpret_cast<const uint8_t *>(row + first);
        if constexpr (MODE == kExactRows) {
#pragma unroll
            for (uint32_t i = 0; i < kEach; ++i) copy_async16(to + i * WIDTH + lane, p + 16u * (i * WIDTH + lane));
        } else if constexpr (MODE == kShiftedRows) {
            const uint32_t off = elem::misalignment(p);
            p -= off;
#pragma unroll
            for (uint32_t i = 0; i < kEach; ++i) copy_async16(to + i * WIDTH + lane, p + 16u * (i * WIDTH + lane));
            if (lane == 0u && off) copy_async16(to + WIDTH * kEach, p + 16u * WIDTH * kEach);
        } else {
            if (first >= dim) return;
            const uint32_t off = kAligned ? 0u : elem::misalignment(p), bytes = off + (dim - first) * (uint32_t)sizeof(T);
            p -= off;
#pragma unroll
            for (uint32_t i = 0; i < kEach; ++i) {
                const uint32_t c = i * WIDTH + lane;
                if (16u * c < bytes) copy_async16(to + c, p + 16u * c);
            }
            if constexpr (!kAligned)
                if (lane == 0u && off && 16u * WIDTH * kEach < bytes) copy_async16(to + WIDTH * kEach, p + 16u * WIDTH * kEach);
        }
    }
    // This lane's elements, zeros behind the row's end or if it is not there.  row_off: the row's bytes from a 16-byte boundary.
    static __device__ __forceinline__ elem::Packed<T, 8> get(const uint4 *from, uint32_t row_off, uint32_t v, uint32_t lane, uint32_t dim, bool live) {
        elem::Vector<T, 8, kAligned ? 16 : elem::kAny> raw;
        const bool some = live && (kWhole || v * 8u < dim);
#pragma unroll
        for (uint32_t i = 0; i < kEach + (kAligned ? 0u : 1u); ++i) {
            const uint4 x = some ? from[lane * kEach + i] : make_uint4(0u, 0u, 0u, 0u);
            raw.w[4 * i] = x.x; raw.w[4 * i + 1] = x.y; raw.w[4 * i + 2] = x.z; raw.w[4 * i + 3] = x.w;
        }
        elem::Packed<T, 8> out = raw.get(kAligned ? 0u : row_off);
        if constexpr (MODE == kAnyRows) {
            const uint32_t left = left_of(v, dim);
            if (left < 8u) {
#pragma unroll
                for (uint32_t i = 0; i < elem::Packed<T, 8>::kWords; ++i) {
                    const uint32_t bytes = left * (uint32_t)sizeof(T);
                    out.w[i] = 4u * i + 4u <= bytes ? out.w[i] : 4u * i < bytes ? out.w[i] & 0xffffu : 0u;
                }
            }
        }
        return out;
    }
};

// Eight weights of a row's vector v, `otherwise` where there is none; zeros behind the row's end.
__device__ __forceinline__ void params_of(const void *p, int type, uint32_t v, uint32_t dim, float otherwise, Pair (&w)[4]) {
    float e[8];
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) e[i] = v * 8u + i >= dim ? 0.f : p ? param_at(p, type, v * 8u + i) : otherwise;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = Pair(e[2 * i], e[2 * i + 1]);
}

}  // namespace rows

// Whether every row starts at a 16-byte boundary and consists of whole vectors of eight elements.
template <typename T>
inline bool rows_aligned(const void *p, uint64_t stride, uint64_t n, uint64_t dim) {
    return ((reinterpret_cast<uintptr_t>(p) | (n > 1 ? stride * sizeof(T) : 0u)) & 15u) == 0u && dim % 8u == 0u;
}

}  // namespace ivk
