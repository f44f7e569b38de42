// Global gradient norm over a ragged tensor set, and clipping by it.
//     s_k = sum of squares of tensor k,  norm = sqrt(sum_k s_k),  scale = norm <= max_norm ? 1 : max_norm / norm,
//     out_k = round(scale * tensor_k)
//
// Both passes are bound by memory: two (four) operations per element read.  Tensors of very different sizes are cut
// into pieces of one size, a power of two that the number of elements (and whether all are of 16-bit types) decides.  A CTA adds
// up a piece, each of its eight warps every eighth run of 32 vectors, without waiting for the others; the warps' sums are
// collected in shared memory and written for up to 256 pieces at a time.  So the order of every sum is a function of
// the lengths and not of the launch, the alignment or the GPU: the same gradients give the same norm bit for bit.
// Squares are added in 32 bits inside a warp's share of a piece (an accumulator takes one in 1,024 elements of 32 bits,
// one in 2,048 of 16: at most 64 for sets of up to 2^31 of either), everything above that in 64 bits.  A piece whose 32-bit sum
// overflowed or came out so small that squares may have been lost below the smallest 32-bit number is added up again
// in 64 bits, so any finite gradient has a right norm.
//
//   1. plan_kernel     sets of more than kSmallSet tensors only: the pieces' running number before each tensor; smaller
//                      sets are laid out by every CTA for itself, in shared memory
//   2. norm_kernel     a CTA takes a run of consecutive pieces; the one that completes a tensor adds up its pieces, the one
//                      that completes the set adds up the tensors
//   3. scale_kernel    clipping: piece by piece, over the whole set at a time (runs of pieces per CTA were no faster)
//
// On one B200: the norm of 194 bf16 tensors (2.6 GB) takes 376 us, 7.0 TB/s; 1000 float32 tensors (6.9 GB) 970 us, 7.1
// TB/s; clipping them into bf16 another 1670 us, 6.2 TB/s; a set that is small enough takes 12 us (norm) and 16 us (clip)
// on a chain of latencies: layout 2, load 1.5, two arrivals 1.5 each, the last sums 2.
#include <type_traits>

#include "element_dev.cuh"
#include "iv_internal.h"

namespace ivk {

namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kWarps = kThreads / 32;
constexpr uint32_t kMaxShift = 31;
constexpr uint32_t kMinShift = 13;                      // pieces of 8,192 elements and more, one shift larger in a set of 16-bit tensors
                                                        // only: 32 KiB, a loop of loads per thread that is long enough against its start
                                                        // (120 MB in 200 tensors, norm: 16-bit 37 us, 45 with half the piece; 32-bit 33, 36)
constexpr uint64_t kPieceTarget = 32768;                // a set has at most this many pieces and one more per tensor
constexpr uint32_t kSmallSet = 1024;                    // laid out by every CTA (200 / 1000 / 2000 small tensors: 12 / 18 / 33 us) or by
                                                        // a kernel before (17 / 21 / 26)
constexpr uint32_t kPending = 256;                       // pieces a CTA adds up between two barriers, one per thread

__device__ __forceinline__ int type_of(const TensorSet &set, uint64_t k) { return set.d_types ? (int)set.d_types[k] : set.type; }

// Elements of tensor k, 0 for one that is ill-formed (unknown type, offset or length not a multiple of the element).
__device__ __forceinline__ uint64_t elements_of(const TensorSet &set, uint64_t k, bool &bad) {
    const int type = type_of(set, k);
    const uint64_t bytes = set.d_lengths[k];
    const uint64_t size = type == IV_F32 ? 4u : 2u;
    const uint64_t address = reinterpret_cast<uint64_t>(set.d_base) + set.d_offsets[k];
    if (type > IV_BF16 || type < 0 || ((bytes | address) & (size - 1u)) != 0u) {
        bad = true;
        return 0;
    }
    return bytes / size;
}

// Exclusive prefix sum over a CTA of THREADS threads, and the total.
template <uint32_t THREADS>
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
#pragma unroll
    for (uint32_t w = 0; w < THREADS / 32; ++w) {
        if (w == warp) before = total;
        total += scan[w];
    }
    __syncthreads();
    return before + x - v;
}

// wide: a tensor with elements is of 32 bits.  However the set is described, the same tensors are cut alike.
__device__ __forceinline__ uint32_t shift_for(bool wide, uint64_t elements) {
    uint32_t shift = kMinShift + (wide ? 0u : 1u);
    while (shift < kMaxShift && (elements >> shift) > kPieceTarget) ++shift;
    return shift;
}

struct Plan {
    uint64_t pieces, elements;
    uint32_t shift;
    uint32_t live;               // tensors that have pieces
};

// The set laid out by one CTA: first[k] = number of pieces before tensor k, first[n] = all.  A thread takes consecutive
// tensors; every thread gets the plan.  T: the tensors' type, void where the set says it.
template <uint32_t THREADS, typename T>
__device__ __forceinline__ Plan lay_out(const TensorSet &set, uint32_t *first, uint64_t *scan, uint32_t *live_shared, uint32_t *status) {
    const uint64_t per = (set.n + THREADS - 1) / THREADS;
    const uint64_t begin = threadIdx.x * per < set.n ? threadIdx.x * per : set.n;
    const uint64_t end = begin + per < set.n ? begin + per : set.n;
    if (threadIdx.x == 0) *live_shared = 0u;
    bool bad = false, wide = false;
    uint64_t elements = 0;
#pragma unroll 4
    for (uint64_t k = begin; k < end; ++k) {
        const uint64_t here = elements_of(set, k, bad);
        elements += here;
        if (std::is_void_v<T> && set.d_types) wide |= here && type_of(set, k) == IV_F32;
    }
    Plan plan;
    block_exclusive64<THREADS>(elements, scan, plan.elements);
    if constexpr (std::is_void_v<T>) wide = set.d_types ? __syncthreads_or(wide) != 0 : set.type == IV_F32;
    else wide = sizeof(T) == 4;
    plan.shift = shift_for(wide, plan.elements);
    auto pieces_of = [&](uint64_t k) { return (elements_of(set, k, bad) + (1ull << plan.shift) - 1) >> plan.shift; };
    uint64_t pieces = 0;
    uint32_t live = 0;
    for (uint64_t k = begin; k < end; ++k) {
        const uint64_t here = pieces_of(k);
        pieces += here;
        live += here ? 1u : 0u;
    }
    live = __reduce_add_sync(0xffffffffu, live);
    if ((threadIdx.x & 31u) == 0u) atomicAdd(live_shared, live);
    uint64_t at = block_exclusive64<THREADS>(pieces, scan, plan.pieces);
    for (uint64_t k = begin; k < end; ++k) {
        first[k] = (uint32_t)at;
        at += pieces_of(k);
    }
    if (bad) atomicMax(status, (uint32_t)IVK_DEV_BOUNDS);
    if (threadIdx.x == 0) first[set.n] = (uint32_t)plan.pieces;
    __syncthreads();
    plan.live = *live_shared;
    return plan;
}

constexpr uint32_t kPlanThreads = 1024;

__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(TensorSet set, Plan *header, uint32_t *first, uint32_t *status) {
    __shared__ uint64_t scan[kPlanThreads / 32];
    __shared__ uint32_t live;
    const Plan plan = lay_out<kPlanThreads, void>(set, first, scan, &live, status);
    if (threadIdx.x == 0) *header = plan;
}

// Where the norm and scale kernels find the plan: in their own shared memory (small sets) or in global memory.
struct PlanAt {
    const Plan *header;          // NULL: lay out in shared memory
    const uint32_t *first;
};

struct Walk {
    Plan plan;
    const uint32_t *first;
};

// The tensor k with first[k] <= p < first[k + 1]; by the whole warp, 32 places at a time.
__device__ __forceinline__ uint64_t tensor_of(const uint32_t *first, uint64_t n, uint64_t p) {
    const uint32_t lane = threadIdx.x & 31u;
    uint64_t lo = 0, count = n;
    while (count > 1) {
        const uint64_t step = (count + 31u) / 32u, at = lane * step;
        const bool before = at < count && first[lo + at] <= p;
        const uint32_t part = __popc(__ballot_sync(0xffffffffu, before)) - 1u;    // true for a first few lanes, lane 0 among them
        lo += part * step;
        count = count - part * step < step ? count - part * step : step;
    }
    return lo;
}

template <typename T>
__device__ __forceinline__ Walk start_walk(const TensorSet &set, const PlanAt &at, uint32_t *shared_first, uint64_t *scan, uint32_t *live, uint32_t *status) {
    Walk w;
    if (at.header) {
        w.plan = *at.header;
        w.first = at.first;
    } else {
        w.plan = lay_out<kThreads, T>(set, shared_first, scan, live, status);
        w.first = shared_first;
    }
    return w;
}

// Sum over the CTA in a fixed order; every thread gets it.  `shared`: kWarps doubles, free again after the next barrier.
__device__ __forceinline__ double block_sum(double x, double *shared) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    if ((threadIdx.x & 31u) == 0u) shared[threadIdx.x >> 5] = x;
    __syncthreads();
    double total = 0.0;
#pragma unroll
    for (uint32_t w = 0; w < kWarps; ++w) total += shared[w];
    return total;
}

// Squares of `vecs` vectors by the CTA, added to acc; the bits that are set anywhere in them added to `bits`.
template <typename T, int V, int ALIGN>
__device__ __forceinline__ void add_squares(const T *p, uint32_t vecs, float (&acc)[V], uint32_t &bits) {
    constexpr uint32_t kUnroll = 4;
    const uint32_t off = elem::misalignment(p);
    for (uint32_t v0 = threadIdx.x; v0 < vecs; v0 += kThreads * kUnroll) {
        elem::Vector<T, V, ALIGN> raw[kUnroll];
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u) {
            const uint32_t v = v0 + u * kThreads;
            if (v < vecs) raw[u].load(p + (uint64_t)v * V, off);
            else raw[u].zero();
        }
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u) {
            const elem::Packed<T, V> w = raw[u].get(off);
            float x[V];
            w.unpack(x);
#pragma unroll
            for (int i = 0; i < V; i += 2) elem::add_squares2(acc[i], acc[i + 1], x[i], x[i + 1]);
#pragma unroll
            for (int i = 0; i < elem::Packed<T, V>::kWords; ++i) bits |= w.w[i];
        }
    }
}

// Sum of squares of this warp's share of `count` elements.  An element's place in the piece decides which thread and
// accumulator it goes to, whatever the alignment.
template <typename T>
__device__ __forceinline__ double piece_squares(const T *p, uint32_t count) {
    constexpr int V = 16 / (int)sizeof(T);
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    uint32_t bits = 0;
    const uint32_t vecs = count / V;
    const uint32_t off = elem::misalignment(p);
    if (off == 0u) add_squares<T, V, 16>(p, vecs, acc, bits);
    else if (off == 8u) add_squares<T, V, 8>(p, vecs, acc, bits);
    else add_squares<T, V, 0>(p, vecs, acc, bits);
    float tail = 0.f;
    if (threadIdx.x < count - vecs * V) {
        tail = elem::to_float(p[vecs * V + threadIdx.x]);
        bits |= __float_as_uint(tail);
    }
    // the thread's accumulators, then the warp's, in 32 bits; from there on in 64
#pragma unroll
    for (int d = V / 2; d; d >>= 1)
#pragma unroll
        for (int i = 0; i < d; ++i) acc[i] += acc[i + d];
    float sum = fmaf(tail, tail, acc[0]);
    bits &= sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    // fine: a finite 32-bit sum that is large against what rounding below the smallest normal number may have cost
    // (each square off by at most 2^-150), or nothing but zeros
    if (sum < 3e38f && sum > 0x1p-90f) return (double)sum;
    if (!__any_sync(0xffffffffu, bits != 0u)) return 0.0;
    double slow = (double)tail * (double)tail;
    for (uint32_t v = threadIdx.x; v < vecs; v += kThreads)
        for (int i = 0; i < V; ++i) {
            const double x = (double)elem::to_float(p[(uint64_t)v * V + i]);
            slow = fma(x, x, slow);
        }
#pragma unroll
    for (int d = 16; d; d >>= 1) slow += __shfl_xor_sync(0xffffffffu, slow, d);
    return slow;
}

// Scratch in global memory: sums[pieces], squares[n] of the tensors, arrived[n] pieces and one word for the set (both
// zero between calls).
struct NormScratch {
    double *sums, *squares;
    uint32_t *arrived, *arrived_set;
};

// T: the tensors' type, void for a set described by d_types (194 bf16 tensors of 2.6 GB: 455 us against 376).
template <typename T>
__global__ void __launch_bounds__(kThreads, std::is_void_v<T> ? 2 : 4)
norm_kernel(TensorSet set, PlanAt at, NormScratch scratch, bool clip, float max_norm, float *norms, iv_norm_result *result,
            uint32_t *status) {
    extern __shared__ uint32_t shared_first[];
    __shared__ uint64_t scan[kWarps];
    __shared__ uint32_t live;
    __shared__ double shared[kWarps];
    __shared__ double pending[kPending][kWarps];     // of pieces this CTA has added up and not written yet
    __shared__ uint32_t flag;
    allow_next_kernel();                                 // the scale kernel may lay out its set
    const Walk w = start_walk<T>(set, at, shared_first, scan, &live, status);
    const uint32_t *first = w.first;
    auto finish_set = [&]() {
        double total = 0.0;
        uint32_t bad = 0;
        for (uint64_t k = threadIdx.x; k < set.n; k += kThreads) {
            const double s = first[k + 1] != first[k] ? __ldcg(&scratch.squares[k]) : 0.0;
            bad += isfinite(s) ? 0u : 1u;
            total += s;
        }
        total = block_sum(total, shared);
        __syncthreads();
        const double bad_tensors = block_sum((double)bad, shared);
        if (threadIdx.x == 0) {
            const double norm = sqrt(total);
            result->status = *reinterpret_cast<volatile uint32_t *>(status);
            result->n_nonfinite = (uint32_t)bad_tensors;
            result->norm = (float)norm;
            result->scale = !clip || norm <= (double)max_norm ? 1.f : (float)((double)max_norm / norm);
            result->sum_squares = total;
            result->n_elements = w.plan.elements;
        }
    };
    if (blockIdx.x == 0) {
        if (norms)
            for (uint64_t k = threadIdx.x; k < set.n; k += kThreads)
                if (first[k] == first[k + 1]) norms[k] = 0.f;
        if (w.plan.pieces == 0) finish_set();
    }
    const uint64_t range_begin = w.plan.pieces * blockIdx.x / gridDim.x;       // this CTA's pieces
    const uint64_t range_end = w.plan.pieces * (blockIdx.x + 1u) / gridDim.x;
    if (range_begin == range_end) return;
    // pieces done of tensor k; true for the CTA whose pieces complete it (and likewise the set)
    auto arrive = [&](uint32_t *counter, uint32_t mine, uint32_t all) {
        __syncthreads();
        if (threadIdx.x == 0) {
            flag = arrive_add(counter, mine) + mine == all ? 1u : 0u;
            if (flag) *counter = 0u;
        }
        __syncthreads();
        const bool last = flag != 0u;
        __syncthreads();
        return last;
    };
    uint32_t completed = 0;                              // tensors this CTA has completed
    // the warps' sums of pieces flushed .. end - 1 added up and written
    uint64_t flushed = 0;
    auto flush = [&](uint64_t end) {
        __syncthreads();
        if (threadIdx.x < (uint32_t)(end - flushed)) {
            double s = 0.0;
#pragma unroll
            for (uint32_t v = 0; v < kWarps; ++v) s += pending[threadIdx.x][v];
            __stcg(&scratch.sums[flushed + threadIdx.x], s);
        }
        flushed = end;
        __syncthreads();
    };
    for (uint64_t p = range_begin, k = tensor_of(first, set.n, range_begin); p < range_end; ++k) {
        const uint64_t from = first[k], next = first[k + 1];
        if (p >= next) continue;
        const int type = type_of(set, k);
        const uint64_t elements = set.d_lengths[k] >> (type == IV_F32 ? 2 : 1);
        const uint8_t *base = set.d_base + set.d_offsets[k];
        const uint64_t stop = next < range_end ? next : range_end, begin = p;
        flushed = p;
        for (; p < stop; ++p) {
            const uint64_t e0 = (p - from) << w.plan.shift;
            const uint32_t count = (uint32_t)(elements - e0 < (1ull << w.plan.shift) ? elements - e0 : (1ull << w.plan.shift));
            double sum;
            if constexpr (!std::is_void_v<T>) sum = piece_squares(reinterpret_cast<const T *>(base) + e0, count);
            else if (type == IV_F32) sum = piece_squares(reinterpret_cast<const float *>(base) + e0, count);
            else if (type == IV_F16) sum = piece_squares(reinterpret_cast<const __half *>(base) + e0, count);
            else sum = piece_squares(reinterpret_cast<const __nv_bfloat16 *>(base) + e0, count);
            if ((threadIdx.x & 31u) == 0u) pending[p - flushed][threadIdx.x >> 5] = sum;
            if (p - flushed + 1u == kPending) flush(p + 1u);
        }
        flush(stop);
        if (stop - begin != next - from) {               // a tensor of several CTAs
            if (!arrive(&scratch.arrived[k], (uint32_t)(stop - begin), (uint32_t)(next - from))) continue;
        }
        double s = 0.0;
#pragma unroll 16
        for (uint64_t q = from + threadIdx.x; q < next; q += kThreads) s += __ldcg(&scratch.sums[q]);
        s = block_sum(s, shared);
        __syncthreads();                                 // everybody has read `shared`
        if (threadIdx.x == 0) {
            __stcg(&scratch.squares[k], s);
            if (norms) norms[k] = (float)sqrt(s);
        }
        ++completed;
    }
    if (completed && arrive(scratch.arrived_set, completed, w.plan.live)) finish_set();
}

template <typename Tin, typename Tout>
__device__ __forceinline__ void scale_piece(const uint8_t *in8, uint8_t *out8, uint64_t e0, uint32_t count, float scale) {
    const Tin *in = reinterpret_cast<const Tin *>(in8) + e0;
    Tout *out = reinterpret_cast<Tout *>(out8) + e0;
    elem::map_any<Tin, Tout, true>(in, out, count, threadIdx.x, kThreads, [scale](float x) { return x * scale; });
}

// Tin, Tout: the types of all tensors, void for a set described by d_types.  Four CTAs per SM: with three the largest sets
// gain 3 %, sets of 120 MB lose 8 %.  The instance for d_types holds the loops of all seven pairs of types and keeps 1.3 KiB a
// thread in local memory at two CTAs per SM: clip of 1000 float32 tensors into bf16 3.7 to 3.9 ms against 2.7, of 200
// packed bf16 tensors 102 us against 81.
template <typename Tin, typename Tout>
__global__ void __launch_bounds__(kThreads, std::is_void_v<Tin> ? 2 : 4)
scale_kernel(TensorSet set, PlanAt at, const float *scale_at, uint8_t *out_base, const uint64_t *out_offsets, int out_type,
             uint32_t *status) {
    extern __shared__ uint32_t shared_first[];
    __shared__ uint64_t scan[kWarps];
    __shared__ uint32_t live;
    const Walk w = start_walk<Tin>(set, at, shared_first, scan, &live, status);
    wait_for_previous_kernel();
    const float scale = *reinterpret_cast<const volatile float *>(scale_at);
    if (scale == 1.f && out_base == set.d_base && out_offsets == set.d_offsets) return;   // in place, nothing to change
    // backwards: some of what the norm read last is still in the L2 cache (120 MB in 200 packed tensors: 80 us against 83)
    for (uint64_t q = blockIdx.x; q < w.plan.pieces; q += gridDim.x) {
        const uint64_t p = w.plan.pieces - 1u - q;
        const uint64_t k = tensor_of(w.first, set.n, p);
        const uint64_t e0 = (p - w.first[k]) << w.plan.shift;
        const int type = type_of(set, k);
        const int to = out_type < 0 ? type : out_type;
        const uint64_t elements = set.d_lengths[k] >> (type == IV_F32 ? 2 : 1);
        const uint32_t count = (uint32_t)(elements - e0 < (1ull << w.plan.shift) ? elements - e0 : (1ull << w.plan.shift));
        const uint8_t *in = set.d_base + set.d_offsets[k];
        uint8_t *out = out_base + out_offsets[k];
        const bool aligned = (reinterpret_cast<uintptr_t>(out) & (to == IV_F32 ? 3u : 1u)) == 0u;
        const bool pair = type == to || type == IV_F32 || to == IV_F32;
        if (!aligned || !pair) {                         // not one 16-bit type to the other
            if (threadIdx.x == 0) atomicMax(status, (uint32_t)IVK_DEV_BOUNDS);
            continue;
        }
        if constexpr (!std::is_void_v<Tin>) scale_piece<Tin, Tout>(in, out, e0, count, scale);
        else switch (type * 3 + to) {
            case IV_F32 * 3 + IV_F32: scale_piece<float, float>(in, out, e0, count, scale); break;
            case IV_F32 * 3 + IV_F16: scale_piece<float, __half>(in, out, e0, count, scale); break;
            case IV_F32 * 3 + IV_BF16: scale_piece<float, __nv_bfloat16>(in, out, e0, count, scale); break;
            case IV_F16 * 3 + IV_F32: scale_piece<__half, float>(in, out, e0, count, scale); break;
            case IV_F16 * 3 + IV_F16: scale_piece<__half, __half>(in, out, e0, count, scale); break;
            case IV_BF16 * 3 + IV_F32: scale_piece<__nv_bfloat16, float>(in, out, e0, count, scale); break;
            default: scale_piece<__nv_bfloat16, __nv_bfloat16>(in, out, e0, count, scale); break;
        }
    }
}

uint64_t round256(uint64_t x) { return (x + 255u) & ~255ull; }

// Plan header | first[n + 1] | sums[kPieceTarget + n] | squares[n]
struct Layout {
    Plan *header;
    uint32_t *first;
    double *sums, *squares;
};
Layout layout_at(void *scratch, uint64_t n) {
    uint8_t *p = static_cast<uint8_t *>(scratch);
    Layout l;
    l.header = reinterpret_cast<Plan *>(p);
    p += 256;
    l.first = reinterpret_cast<uint32_t *>(p);
    p += round256(4u * (n + 1u));
    l.sums = reinterpret_cast<double *>(p);
    p += round256(8u * (kPieceTarget + n));
    l.squares = reinterpret_cast<double *>(p);
    return l;
}

cudaError_t make_plan(const TensorSet &set, const Layout &l, PlanAt *at, size_t *shared, uint32_t *d_status, cudaStream_t stream,
                      uint64_t *launches) {
    if (set.n <= kSmallSet) {
        *at = {nullptr, nullptr};
        *shared = 4u * (set.n + 1u);
        return cudaSuccess;
    }
    *at = {l.header, l.first};
    *shared = 0;
    plan_kernel<<<1, kPlanThreads, 0, stream>>>(set, l.header, l.first, d_status);
    ++*launches;
    return cudaGetLastError();
}

}  // namespace

uint64_t grad_norm_scratch_bytes(uint64_t n) { return 256u + round256(4u * (n + 1u)) + round256(8u * (kPieceTarget + n)) + 8u * n; }
uint64_t grad_norm_arrival_bytes(uint64_t n) { return 4u * (n + 1u); }

cudaError_t launch_grad_norm(const TensorSet &set, bool clip, float max_norm, float *d_norms, iv_norm_result *d_result,
                             void *d_scratch, uint32_t *d_arrivals, uint32_t *d_status, int sm_count, cudaStream_t stream,
                             uint64_t *launches) {
    const Layout l = layout_at(d_scratch, set.n);
    PlanAt at;
    size_t shared;
    cudaError_t e = make_plan(set, l, &at, &shared, d_status, stream, launches);
    if (e != cudaSuccess) return e;
    const NormScratch scratch = {l.sums, l.squares, d_arrivals + 1, d_arrivals};
    const uint32_t grid = (uint32_t)sm_count * 4u;
    if (set.d_types) norm_kernel<void><<<grid, kThreads, shared, stream>>>(set, at, scratch, clip, max_norm, d_norms, d_result, d_status);
    else
        e = by_types(set.type, set.type, [&](auto in, auto) {
            norm_kernel<typename decltype(in)::type><<<grid, kThreads, shared, stream>>>(set, at, scratch, clip, max_norm, d_norms, d_result, d_status);
            return cudaSuccess;
        });
    if (e != cudaSuccess) return e;
    ++*launches;
    return cudaGetLastError();
}

cudaError_t launch_grad_scale(const TensorSet &set, bool planned, const float *d_scale, uint8_t *d_out,
                              const uint64_t *d_out_offsets, int out_type, void *d_scratch, uint32_t *d_status, int sm_count,
                              cudaStream_t stream, uint64_t *launches) {
    if (set.n == 0) return cudaSuccess;
    const Layout l = layout_at(d_scratch, set.n);
    PlanAt at;
    size_t shared;
    if (planned && set.n > kSmallSet) {
        at = {l.header, l.first};
        shared = 0;
    } else {
        cudaError_t e = make_plan(set, l, &at, &shared, d_status, stream, launches);
        if (e != cudaSuccess) return e;
    }
    const uint32_t grid = (uint32_t)sm_count * 4u;
    cudaError_t e = cudaSuccess;
    auto launch = [&](auto kernel) {
        if (planned) return launch_overlapping(kernel, dim3(grid), dim3(kThreads), shared, stream, set, at, d_scale, d_out, d_out_offsets, out_type, d_status);
        kernel<<<grid, kThreads, shared, stream>>>(set, at, d_scale, d_out, d_out_offsets, out_type, d_status);
        return cudaGetLastError();
    };
    if (set.d_types) e = launch(scale_kernel<void, void>);
    else
        e = by_types(set.type, out_type < 0 ? set.type : out_type, [&](auto in, auto out) {
            auto kernel = scale_kernel<typename decltype(in)::type, typename decltype(out)::type>;
            return launch(kernel);
        });
    if (e != cudaSuccess) return e;
    ++*launches;
    return cudaGetLastError();
}

}  // namespace ivk
