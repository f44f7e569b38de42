// Global gradient norm over a ragged tensor set, and clipping by it.
//     s_k = sum of squares of tensor k,  norm = sqrt(sum_k s_k),  scale = norm <= max_norm ? 1 : max_norm / norm,
//     out_k = round(scale * tensor_k)
//
// Both passes are bound by memory: two (four) operations per element read.  Tensors of very different sizes are cut
// into pieces of one size, a power of two that the total size alone decides; a CTA adds up one piece, so the order of
// every sum is a function of the lengths and not of the launch, the alignment or the GPU: the same gradients give the
// same norm bit for bit.  Squares are added in 32 bits inside a thread's share of a piece (64 of them in one accumulator
// for every 2^16 elements of 32 bits or 2^17 of 16), everything above that in 64 bits.  A piece whose 32-bit sum overflowed or came out so
// small that squares may have been lost below the smallest 32-bit number is added up again in 64 bits, so any finite
// gradient has a right norm.
//
//   1. plan_kernel     pieces of each tensor and their running sum; ill-formed tensors are left out (device status 2)
//   2. norm_kernel     one sum per piece
//   3. finish_kernel   per-tensor sums, the norm, the scale
//   4. scale_kernel    clipping: piece by piece
#include "element_dev.cuh"
#include "iv_internal.h"

namespace ivk {

namespace {

constexpr uint32_t kNormThreads = 256;
constexpr uint32_t kMinShift = 12, kMaxShift = 31;      // pieces of 4,096 elements and more
constexpr uint64_t kPieceTarget = 65536;                // a set has at most this many pieces and one more per tensor

// Scratch: header, running number of pieces before each tensor (n + 1), one sum per piece.
struct PlanHeader {
    uint64_t pieces;
    uint64_t elements;
    uint32_t shift;
    uint32_t pad;
};

__device__ __forceinline__ int type_of(const TensorSet &set, uint64_t k) { return set.d_types ? (int)set.d_types[k] : set.type; }

// Elements of tensor k, 0 for one that is ill-formed (unknown type, offset or length not a multiple of the element).
__device__ __forceinline__ uint64_t elements_of(const TensorSet &set, uint64_t k, uint32_t *status) {
    const int type = type_of(set, k);
    const uint64_t bytes = set.d_lengths[k];
    const uint64_t size = type == IV_F32 ? 4u : 2u;
    const uint64_t address = reinterpret_cast<uint64_t>(set.d_base) + set.d_offsets[k];
    if (type > IV_BF16 || type < 0 || ((bytes | address) & (size - 1u)) != 0u) {
        atomicMax(status, (uint32_t)IVK_DEV_BOUNDS);
        return 0;
    }
    return bytes / size;
}

constexpr uint32_t kPlanThreads = 1024;

__device__ __forceinline__ uint64_t block_exclusive64(uint64_t v, uint64_t *scan, uint64_t &total) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    uint64_t x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= (uint32_t)d) x += y;
    }
    if (lane == 31u) scan[warp] = x;
    __syncthreads();
    uint64_t before = 0;
    total = 0;
    for (uint32_t w = 0; w < kPlanThreads / 32; ++w) {
        if (w == warp) before = total;
        total += scan[w];
    }
    __syncthreads();
    return before + x - v;
}

__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(TensorSet set, PlanHeader *header, uint64_t *first, uint32_t *status) {
    __shared__ uint64_t scan[kPlanThreads / 32];
    uint64_t elements = 0;
    for (uint64_t k = threadIdx.x; k < set.n; k += kPlanThreads) elements += elements_of(set, k, status);
    uint64_t total;
    block_exclusive64(elements, scan, total);
    uint32_t shift = kMinShift;
    while (shift < kMaxShift && (total >> shift) > kPieceTarget) ++shift;
    uint64_t before = 0;
    for (uint64_t k0 = 0; k0 < set.n; k0 += kPlanThreads) {
        const uint64_t k = k0 + threadIdx.x;
        const uint64_t pieces = k < set.n ? (elements_of(set, k, status) + (1ull << shift) - 1) >> shift : 0;
        uint64_t here;
        const uint64_t at = block_exclusive64(pieces, scan, here);
        if (k < set.n) first[k] = before + at;
        before += here;
    }
    if (threadIdx.x == 0) {
        first[set.n] = before;
        header->pieces = before;
        header->elements = total;
        header->shift = shift;
    }
}

// The tensor that piece p belongs to: first[k] <= p < first[k + 1].
__device__ __forceinline__ uint64_t tensor_of(const uint64_t *first, uint64_t n, uint64_t p) {
    uint64_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint64_t mid = (lo + hi) / 2;
        if (first[mid] <= p) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Sum of squares of `count` elements by the CTA; the result is in thread 0.  An element's place in the piece decides
// which thread and accumulator it goes to, whatever the alignment.
template <typename T>
__device__ double piece_squares(const T *p, uint32_t count, double *shared) {
    constexpr int V = 16 / (int)sizeof(T);
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    uint32_t bits = 0;
    const uint32_t vecs = count / V;
    constexpr uint32_t kUnroll = 4;
    for (uint32_t v0 = threadIdx.x; v0 < vecs; v0 += kNormThreads * kUnroll) {
        elem::Packed<T, V> raw[kUnroll];
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u) {
            const uint32_t v = v0 + u * kNormThreads;
            if (v < vecs) elem::load_any<T, V>(p + (uint64_t)v * V, raw[u]);
            else raw[u].zero();
        }
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u) {
            float x[V];
            raw[u].unpack(x);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] = fmaf(x[i], x[i], acc[i]);
#pragma unroll
            for (int i = 0; i < elem::Packed<T, V>::kWords; ++i) bits |= raw[u].w[i];
        }
    }
    float tail = 0.f;
    if (threadIdx.x < count - vecs * V) {
        tail = elem::to_float(p[vecs * V + threadIdx.x]);
        bits |= __float_as_uint(tail);
    }
    double sum = (double)tail * (double)tail;
#pragma unroll
    for (int i = 0; i < V; ++i) sum += (double)acc[i];
    // fine: a finite 32-bit sum that is large against what rounding below the smallest normal number may have cost
    // (each square off by at most 2^-150), or nothing but zeros
    bits &= sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    auto reduce = [&](double x) {
#pragma unroll
        for (int d = 16; d; d >>= 1) x += __shfl_down_sync(0xffffffffu, x, d);
        if ((threadIdx.x & 31u) == 0u) shared[threadIdx.x >> 5] = x;
        __syncthreads();
        double total = 0.0;
#pragma unroll
        for (uint32_t w = 0; w < kNormThreads / 32; ++w) total += shared[w];
        return total;
    };
    const double total = reduce(sum);
    const bool fine = total < 3e38 && total > 0x1p-90;
    const int some = __syncthreads_or(bits != 0u);          // also: everybody has read `shared`
    if (fine || !some) return some ? total : 0.0;
    double slow = 0.0;
    for (uint32_t i = threadIdx.x; i < count; i += kNormThreads) {
        const double x = (double)elem::to_float(p[i]);
        slow = fma(x, x, slow);
    }
    const double exact = reduce(slow);
    __syncthreads();
    return exact;
}

__global__ void __launch_bounds__(kNormThreads)
norm_kernel(TensorSet set, const PlanHeader *header, const uint64_t *first, double *sums) {
    __shared__ double shared[kNormThreads / 32];
    const uint64_t pieces = header->pieces;
    const uint32_t shift = header->shift;
    for (uint64_t p = blockIdx.x; p < pieces; p += gridDim.x) {
        const uint64_t k = tensor_of(first, set.n, p);
        const uint64_t e0 = (p - first[k]) << shift;
        const int type = type_of(set, k);
        const uint64_t total = set.d_lengths[k] >> (type == IV_F32 ? 2 : 1);
        const uint32_t count = (uint32_t)(total - e0 < (1ull << shift) ? total - e0 : (1ull << shift));
        const uint8_t *base = set.d_base + set.d_offsets[k];
        double sum;
        if (type == IV_F32) sum = piece_squares(reinterpret_cast<const float *>(base) + e0, count, shared);
        else if (type == IV_F16) sum = piece_squares(reinterpret_cast<const __half *>(base) + e0, count, shared);
        else sum = piece_squares(reinterpret_cast<const __nv_bfloat16 *>(base) + e0, count, shared);
        if (threadIdx.x == 0) sums[p] = sum;
    }
}

constexpr uint32_t kFinishThreads = 1024;

// One warp per tensor adds up its pieces (lane l takes pieces l, l + 32, ...), then the tensors are added up likewise.
__global__ void __launch_bounds__(kFinishThreads)
finish_kernel(uint64_t n, const PlanHeader *header, const uint64_t *first, const double *sums, bool clip, float max_norm,
              float *norms, iv_norm_result *result, const uint32_t *status) {
    __shared__ double shared[kFinishThreads / 32];
    __shared__ uint32_t bad;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    double mine = 0.0;                                   // of the tensors warp, warp + 32, ...
    for (uint64_t k = warp; k < n; k += kFinishThreads / 32) {
        double s = 0.0;
        for (uint64_t p = first[k] + lane; p < first[k + 1]; p += 32u) s += sums[p];
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        if (lane == 0) {
            if (norms) norms[k] = (float)sqrt(s);
            if (!isfinite(s)) atomicAdd(&bad, 1u);
        }
        mine += s;
    }
    if (lane == 0) shared[warp] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        double total = 0.0;
        for (uint32_t w = 0; w < kFinishThreads / 32; ++w) total += shared[w];
        const double norm = sqrt(total);
        result->status = *status;
        result->n_nonfinite = bad;
        result->norm = (float)norm;
        result->scale = !clip || norm <= (double)max_norm ? 1.f : (float)((double)max_norm / norm);
        result->sum_squares = total;
        result->n_elements = header->elements;
    }
}

template <typename Tin, typename Tout>
__device__ __forceinline__ void scale_piece(const uint8_t *in, uint8_t *out, uint64_t e0, uint32_t count, float scale) {
    elem::map_span<Tin, Tout, 4>(reinterpret_cast<const Tin *>(in) + e0, reinterpret_cast<Tout *>(out) + e0, count, threadIdx.x,
                                 kNormThreads, [scale](float x) { return x * scale; });
}

__global__ void __launch_bounds__(kNormThreads)
scale_kernel(TensorSet set, const PlanHeader *header, const uint64_t *first, const float *scale_at, uint8_t *out_base,
             const uint64_t *out_offsets, int out_type, uint32_t *status) {
    const uint64_t pieces = header->pieces;
    const uint32_t shift = header->shift;
    const float scale = *scale_at;
    if (scale == 1.f && out_base == set.d_base && out_offsets == set.d_offsets) return;   // in place, nothing to change
    for (uint64_t q = blockIdx.x; q < pieces; q += gridDim.x) {
        const uint64_t p = pieces - 1 - q;               // backwards: the norm's last pieces are still in the L2 cache
        const uint64_t k = tensor_of(first, set.n, p);
        const uint64_t e0 = (p - first[k]) << shift;
        const int type = type_of(set, k);
        const int to = out_type < 0 ? type : out_type;
        const uint64_t total = set.d_lengths[k] >> (type == IV_F32 ? 2 : 1);
        const uint32_t count = (uint32_t)(total - e0 < (1ull << shift) ? total - e0 : (1ull << shift));
        const uint8_t *in = set.d_base + set.d_offsets[k];
        uint8_t *out = out_base + out_offsets[k];
        if ((reinterpret_cast<uintptr_t>(out) & (to == IV_F32 ? 3u : 1u)) != 0u) {
            if (threadIdx.x == 0) atomicMax(status, (uint32_t)IVK_DEV_BOUNDS);
            continue;
        }
        switch (type * 3 + to) {
            case IV_F32 * 3 + IV_F32: scale_piece<float, float>(in, out, e0, count, scale); break;
            case IV_F32 * 3 + IV_F16: scale_piece<float, __half>(in, out, e0, count, scale); break;
            case IV_F32 * 3 + IV_BF16: scale_piece<float, __nv_bfloat16>(in, out, e0, count, scale); break;
            case IV_F16 * 3 + IV_F32: scale_piece<__half, float>(in, out, e0, count, scale); break;
            case IV_F16 * 3 + IV_F16: scale_piece<__half, __half>(in, out, e0, count, scale); break;
            case IV_BF16 * 3 + IV_F32: scale_piece<__nv_bfloat16, float>(in, out, e0, count, scale); break;
            case IV_BF16 * 3 + IV_BF16: scale_piece<__nv_bfloat16, __nv_bfloat16>(in, out, e0, count, scale); break;
            default:
                if (threadIdx.x == 0) atomicMax(status, (uint32_t)IVK_DEV_BOUNDS);   // one 16-bit type to the other
        }
    }
}

uint64_t round256(uint64_t x) { return (x + 255u) & ~255ull; }

struct Plan {
    PlanHeader *header;
    uint64_t *first;
    double *sums;
};
Plan plan_at(void *scratch, uint64_t n) {
    uint8_t *p = static_cast<uint8_t *>(scratch);
    return {reinterpret_cast<PlanHeader *>(p), reinterpret_cast<uint64_t *>(p + 256),
            reinterpret_cast<double *>(p + 256 + round256(8u * (n + 1u)))};
}

}  // namespace

uint64_t grad_norm_scratch_bytes(uint64_t n) { return 256u + round256(8u * (n + 1u)) + 8u * (kPieceTarget + n); }

cudaError_t launch_grad_norm(const TensorSet &set, bool clip, float max_norm, float *d_norms, iv_norm_result *d_result,
                             void *d_scratch, uint32_t *d_status, int sm_count, cudaStream_t stream, uint64_t *launches) {
    const Plan plan = plan_at(d_scratch, set.n);
    plan_kernel<<<1, kPlanThreads, 0, stream>>>(set, plan.header, plan.first, d_status);
    norm_kernel<<<sm_count * 8, kNormThreads, 0, stream>>>(set, plan.header, plan.first, plan.sums);
    finish_kernel<<<1, kFinishThreads, 0, stream>>>(set.n, plan.header, plan.first, plan.sums, clip, max_norm, d_norms,
                                                    d_result, d_status);
    *launches += 3;
    return cudaGetLastError();
}

cudaError_t launch_grad_scale(const TensorSet &set, bool with_plan, const float *d_scale, uint8_t *d_out,
                              const uint64_t *d_out_offsets, int out_type, void *d_scratch, uint32_t *d_status, int sm_count,
                              cudaStream_t stream, uint64_t *launches) {
    if (set.n == 0) return cudaSuccess;
    const Plan plan = plan_at(d_scratch, set.n);
    if (with_plan) {
        plan_kernel<<<1, kPlanThreads, 0, stream>>>(set, plan.header, plan.first, d_status);
        ++*launches;
    }
    scale_kernel<<<sm_count * 8, kNormThreads, 0, stream>>>(set, plan.header, plan.first, d_scale, d_out, d_out_offsets, out_type,
                                                            d_status);
    ++*launches;
    return cudaGetLastError();
}

}  // namespace ivk
