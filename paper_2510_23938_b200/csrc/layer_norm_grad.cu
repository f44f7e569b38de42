// Gradient of layer norm:  h = (x - mu) r (rms: x r),  p = dy w,
//     dx = round(r (p - mean(p) - h mean(p h)))  (rms: without mean(p)),   dw = sum over rows of dy h,   db = sum over rows of dy
//
// Bound by memory: x and dy are read once and dx is written once.  A CTA takes a run of consecutive rows; a thread owns
// eight (or sixteen) columns of every T threads' row, so the sums over rows stay in its registers, and only the row's two sums
// cross threads.  Rows come through a ring in shared memory that each thread fills for itself with asynchronous copies of
// 16 bytes (of the aligned pieces its elements lie in), several rows ahead, and reads without any barrier.  At the end each
// CTA leaves its sums over rows in global memory, and norm_grad_columns_kernel adds them up.
// The order of every sum is a function of the number of rows, their width and type alone.
#include "element_dev.cuh"
#include "iv_internal.h"
#include "row_dev.cuh"

namespace ivk {

namespace {

using namespace rows;
using elem::Pair;

constexpr uint32_t kThreads = 512;
constexpr uint64_t kMostParts = 296;      // runs of rows: two for each of a B200's SMs, whatever GPU it is (the sums' order goes by it)
constexpr uint32_t kPartRows = 4;         // and no fewer rows than this per group of threads, if there are that many

// Runs of rows of a gradient over n rows, for groups of T threads.
uint64_t part_count(uint64_t n, uint32_t groups) {
    const uint64_t parts = (n + (uint64_t)groups * kPartRows - 1) / ((uint64_t)groups * kPartRows);
    return parts < kMostParts ? (parts ? parts : 1u) : kMostParts;
}

__device__ __forceinline__ void copy_async16(void *shared, const void *global) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(shared)), "l"(global) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Sums of two values over a group of T threads, in a fixed order; every thread gets both.  `slots`: as group_sum, 32 floats per
// group of 512 threads (two values for each of 16 warps).
template <uint32_t T>
__device__ __forceinline__ void group_sum2(float &a, float &b, float *slots) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    if constexpr (T <= 16u) {
#pragma unroll
        for (uint32_t d = T / 2u; d; d >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, d);
            b += __shfl_xor_sync(0xffffffffu, b, d);
        }
    } else {
        // the lower half-warp adds up a, the upper b
        const bool upper = lane & 16u;
        float x = upper ? b : a;
        x += __shfl_xor_sync(0xffffffffu, upper ? a : b, 16);
#pragma unroll
        for (uint32_t d = 8u; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        if constexpr (T > 32u) {
            constexpr uint32_t kWarps = T / 32u;
            if ((lane & 15u) == 0u) slots[(upper ? kThreads / 32u : 0u) + warp] = x;
            group_barrier<T>();
            x = slots[(upper ? kThreads / 32u : 0u) + (warp & ~(kWarps - 1u)) + (lane & (kWarps - 1u))];
#pragma unroll
            for (uint32_t d = kWarps / 2u; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        }
        a = __shfl_sync(0xffffffffu, x, 0);
        b = __shfl_sync(0xffffffffu, x, 16);
    }
}

// A thread's vector of a row in the ring: the aligned 16-byte pieces it lies in.
template <typename T, bool ALIGNED>
struct Slot {
    static constexpr int kPieces = (int)sizeof(T) / 2 + (ALIGNED ? 0 : 1);
    // pieces[i * kThreads]: this thread's piece i
    static __device__ __forceinline__ void fetch(uint4 *pieces, const T *row, uint32_t v, uint32_t dim) {
        const T *p = row + v * 8u;
        if constexpr (ALIGNED) {
            if (v * 8u < dim) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) copy_async16(pieces + i * kThreads, reinterpret_cast<const uint8_t *>(p) + 16 * i);
            }
        } else {
            const uint32_t left = left_of(v, dim), off = elem::misalignment(p), wanted = left ? off + left * (uint32_t)sizeof(T) : 0u;
            const uint8_t *q = reinterpret_cast<const uint8_t *>(p) - off;
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                if (16u * i < wanted) copy_async16(pieces + i * kThreads, q + 16 * i);
        }
    }
    // zeros behind the row's end
    static __device__ __forceinline__ void get(const uint4 *pieces, uint32_t row_off, uint32_t v, uint32_t dim, Pair (&e)[4]) {
        elem::Vector<T, 8, ALIGNED ? 16 : elem::kAny> raw;
        if (v * 8u < dim) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const uint4 x = pieces[i * kThreads];
                raw.w[4 * i] = x.x; raw.w[4 * i + 1] = x.y; raw.w[4 * i + 2] = x.z; raw.w[4 * i + 3] = x.w;
            }
        } else {
            raw.zero();
        }
        elem::unpack8(raw.get(ALIGNED ? 0u : row_off), e);
        if constexpr (!ALIGNED) {
            const uint32_t left = left_of(v, dim);
            if (left < 8u) {
                float x[8];
                unpair(e, x);
#pragma unroll
                for (uint32_t i = 0; i < 4u; ++i) e[i] = Pair(2u * i < left ? x[2 * i] : 0.f, 2u * i + 1u < left ? x[2 * i + 1] : 0.f);
            }
        }
    }
};

template <typename Tx, typename Ty, bool ALIGNED, int NV>
__host__ __device__ constexpr uint32_t row_bytes() { return 16u * kThreads * NV * (Slot<Tx, ALIGNED>::kPieces + Slot<Ty, ALIGNED>::kPieces); }
// Rows in the ring: what two CTAs can hold in an SM's shared memory, at most eight.
template <typename Tx, typename Ty, bool ALIGNED, int NV>
__host__ __device__ constexpr int stages_of() {
    constexpr uint32_t fit = (96u << 10) / row_bytes<Tx, Ty, ALIGNED, NV>();
    return fit > 8u ? 8 : fit < 2u ? 2 : (int)fit;
}

template <typename Tx, typename Ty, uint32_t T, int NV, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, NV > 1 ? 1 : 2)
norm_grad_kernel(const __grid_constant__ LayerNormGradArgs a, float *partial) {
    constexpr uint32_t kGroups = kThreads / T;
    constexpr int kStages = stages_of<Tx, Ty, ALIGNED, NV>();
    constexpr int kX = Slot<Tx, ALIGNED>::kPieces, kY = Slot<Ty, ALIGNED>::kPieces;
    extern __shared__ uint4 ring[];                      // kStages x (x, dy) x NV x pieces x kThreads
    __shared__ float slots[2][kThreads / 16];
    allow_next_kernel();
    const uint32_t t = threadIdx.x % T, group = threadIdx.x / T;
    const uint32_t dim = (uint32_t)a.dim;
    const uint64_t begin = a.n * blockIdx.x / gridDim.x, end = a.n * (blockIdx.x + 1u) / gridDim.x;
    const Tx *x = static_cast<const Tx *>(a.d_x);
    const Ty *dy = static_cast<const Ty *>(a.d_dy);
    Tx *dx = static_cast<Tx *>(a.d_dx);
    auto slot = [&](int stage, int j) { return ring + (stage * NV + j) * (kX + kY) * kThreads + threadIdx.x; };
    auto fetch = [&](uint64_t base, int stage) {         // the group's row of those from `base` on
        const uint64_t row = base + group;
        if (row < end) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                Slot<Tx, ALIGNED>::fetch(slot(stage, j), x + row * a.x_stride, t + j * T, dim);
                Slot<Ty, ALIGNED>::fetch(slot(stage, j) + kX * kThreads, dy + row * a.dy_stride, t + j * T, dim);
            }
        }
        commit_copies();
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(begin + s * kGroups, s);
    Pair w[NV][4], dw[NV][4], db[NV][4];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) {
            const uint32_t c = (t + j * T) * 8u + 2u * i;
            auto weight = [&](uint32_t at) { return at >= dim ? 0.f : a.d_weight ? param_at(a.d_weight, a.param_type, at) : 1.f; };
            w[j][i] = Pair(weight(c), weight(c + 1u));
            dw[j][i] = db[j][i] = Pair(0.f);
        }
    const float scale = 1.f / (float)dim;
    int stage = 0;
    float *sums = slots[0], *other = slots[1];
    for (uint64_t base = begin; base < end; base += kGroups) {
        fetch(base + (uint64_t)(kStages - 1) * kGroups, stage == 0 ? kStages - 1 : stage - 1);
        wait_copies<kStages - 1>();
        const uint64_t row = base + group;
        const bool live = row < end;
        const float rstd = live ? a.d_rstd[row] : 0.f, mean = live && a.d_mean ? a.d_mean[row] : 0.f;
        const uint32_t x_off = elem::misalignment(x + (live ? row * a.x_stride : 0u)), y_off = elem::misalignment(dy + (live ? row * a.dy_stride : 0u));
        const Pair shift(-mean), by(rstd);
        Pair h[NV][4], p[NV][4], s2(0.f), sh2(0.f);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            Pair e[4];
            Slot<Tx, ALIGNED>::get(slot(stage, j), x_off, t + j * T, live ? dim : 0u, h[j]);
            Slot<Ty, ALIGNED>::get(slot(stage, j) + kX * kThreads, y_off, t + j * T, live ? dim : 0u, e);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[j][i] = (h[j][i] + shift) * by;
                p[j][i] = e[i] * w[j][i];
                db[j][i] = db[j][i] + e[i];
                dw[j][i] = fma2(e[i], h[j][i], dw[j][i]);
                s2 = s2 + p[j][i];
                sh2 = fma2(p[j][i], h[j][i], sh2);
            }
        }
        float s = s2.sum(), sh = sh2.sum();
        group_sum2<T>(s, sh, sums);
        const Pair mp(a.rms ? 0.f : -s * scale), mh(-sh * scale);
        Tx *out = dx + (live ? row * a.dx_stride : 0u);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) h[j][i] = (fma2(h[j][i], mh, p[j][i]) + mp) * by;
            store_row_vector<Tx, ALIGNED, T>(out, t + j * T, live ? dim : 0u, h[j]);
        }
        float *swap = sums;
        sums = other;
        other = swap;
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    if (!a.d_dw && !a.d_db) return;
    // the groups' sums, first to last
    wait_copies<0>();
    float *out = partial + (uint64_t)blockIdx.x * 2u * dim;
    if constexpr (kGroups > 1) {
        __syncthreads();                                 // nobody reads the ring any more
        float *all = reinterpret_cast<float *>(ring);    // [16 NV][kThreads]
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float *to = all + ((2 * j) * 8 + 2 * i) * kThreads + threadIdx.x;
                dw[j][i].get(to[0], to[kThreads]);
                db[j][i].get(to[8 * kThreads], to[9 * kThreads]);
            }
        __syncthreads();
        for (uint32_t q = threadIdx.x; q < 16u * NV * T; q += kThreads) {
            const uint32_t value = q / T, at = q % T;    // value: 16 j + 8 [bias] + i
            float sum = 0.f;
            for (uint32_t g = 0; g < kGroups; ++g) sum += all[value * kThreads + g * T + at];
            const uint32_t c = (at + (value / 16u) * T) * 8u + value % 8u;
            if (c < dim) out[(value & 8u ? dim : 0u) + c] = sum;
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) {
                const uint32_t c = (t + j * T) * 8u + 2u * i;
                float x[2], y[2];
                dw[j][i].get(x[0], x[1]);
                db[j][i].get(y[0], y[1]);
#pragma unroll
                for (uint32_t k = 0; k < 2u; ++k)
                    if (c + k < dim) {
                        out[c + k] = x[k];
                        out[dim + c + k] = y[k];
                    }
            }
    }
}

// Rows too wide for that.  First the two sums of every row, a CTA each; then tiles of 256 columns by runs of rows, a warp
// per row with every lane's eight columns in registers.  The second pass reads x and dy again.
template <typename Tx, typename Ty>
__global__ void __launch_bounds__(kThreads)
norm_grad_wide_rows_kernel(LayerNormGradArgs a, float2 *row_sums) {
    __shared__ float slots[kThreads / 16];
    const uint32_t dim = (uint32_t)a.dim, vectors = (dim + 7u) / 8u;
    for (uint64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const Tx *x = static_cast<const Tx *>(a.d_x) + row * a.x_stride;
        const Ty *dy = static_cast<const Ty *>(a.d_dy) + row * a.dy_stride;
        const float rstd = a.d_rstd[row], mean = a.d_mean ? a.d_mean[row] : 0.f;
        float s = 0.f, sh = 0.f;
        for (uint32_t v = threadIdx.x; v < vectors; v += kThreads) {
            RowVector<Tx, false> rx;
            RowVector<Ty, false> ry;
            Pair pairs[4];
            float h[8], p[8];
            rx.load(x, v, dim);
            ry.load(dy, v, dim);
            elem::unpack8(rx.get(elem::misalignment(x), v, dim), pairs);
            unpair(pairs, h);
            elem::unpack8(ry.get(elem::misalignment(dy), v, dim), pairs);
            unpair(pairs, p);
            const uint32_t left = left_of(v, dim);
#pragma unroll
            for (uint32_t i = 0; i < 8u; ++i) {
                if (i >= left) break;
                const float q = a.d_weight ? p[i] * param_at(a.d_weight, a.param_type, v * 8u + i) : p[i];
                s += q;
                sh = fmaf(q, (h[i] - mean) * rstd, sh);
            }
        }
        group_sum2<kThreads>(s, sh, slots);
        if (threadIdx.x == 0) row_sums[row] = make_float2(s, sh);
        __syncthreads();                                 // before the slots are written again
    }
}

constexpr uint32_t kWideWarps = 8;
template <typename Tx, typename Ty>
__global__ void __launch_bounds__(kWideWarps * 32)
norm_grad_wide_kernel(LayerNormGradArgs a, const float2 *row_sums, float *partial, uint32_t parts) {
    __shared__ float all[16][kWideWarps][32];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, dim = (uint32_t)a.dim;
    const uint32_t tile = blockIdx.x / parts, part = blockIdx.x % parts, v = tile * 32u + lane, left = left_of(v, dim);
    const uint64_t begin = a.n * part / parts, end = a.n * (part + 1u) / parts;
    const float scale = 1.f / (float)dim;
    float w[8], dw[8], db[8];
    for (uint32_t i = 0; i < 8u; ++i) {
        w[i] = i >= left ? 0.f : a.d_weight ? param_at(a.d_weight, a.param_type, v * 8u + i) : 1.f;
        dw[i] = db[i] = 0.f;
    }
    for (uint64_t row = begin + warp; row < end; row += kWideWarps) {
        const Tx *x = static_cast<const Tx *>(a.d_x) + row * a.x_stride;
        const Ty *dy = static_cast<const Ty *>(a.d_dy) + row * a.dy_stride;
        RowVector<Tx, false> rx;
        RowVector<Ty, false> ry;
        rx.load(x, v, dim);
        ry.load(dy, v, dim);
        const float rstd = a.d_rstd[row], mean = a.d_mean ? a.d_mean[row] : 0.f;
        const float2 sums = row_sums[row];
        const float mp = a.rms ? 0.f : sums.x * scale, mh = sums.y * scale;
        Pair pairs[4];
        float h[8], e[8];
        elem::unpack8(rx.get(elem::misalignment(x), v, dim), pairs);
        unpair(pairs, h);
        elem::unpack8(ry.get(elem::misalignment(dy), v, dim), pairs);
        unpair(pairs, e);
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) {
            h[i] = (h[i] - mean) * rstd;
            db[i] += e[i];
            dw[i] = fmaf(e[i], h[i], dw[i]);
            h[i] = rstd * (e[i] * w[i] - mp - h[i] * mh);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) pairs[i] = Pair(h[2 * i], h[2 * i + 1]);
        store_row_vector<Tx, false, 32>(static_cast<Tx *>(a.d_dx) + row * a.dx_stride, v, dim, pairs);
    }
    if (!a.d_dw && !a.d_db) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        all[i][warp][lane] = dw[i];
        all[8 + i][warp][lane] = db[i];
    }
    __syncthreads();
    float *out = partial + (uint64_t)part * 2u * dim;
    for (uint32_t value = warp; value < 16u; value += kWideWarps) {
        float sum = 0.f;
        for (uint32_t g = 0; g < kWideWarps; ++g) sum += all[value][g][lane];
        const uint32_t c = v * 8u + value % 8u;
        if (c < dim) out[(value & 8u ? dim : 0u) + c] = sum;
    }
}

// The parts' sums of 32 columns: a warp adds up every 32nd part, then the warps' sums are added first to last.
constexpr uint32_t kSlices = 32;
__global__ void __launch_bounds__(32 * kSlices)
norm_grad_columns_kernel(const float *partial, uint32_t parts, uint32_t dim, void *dw, void *db, int type, bool accumulate) {
    __shared__ float sums[kSlices][33];
    const uint32_t lane = threadIdx.x & 31u, slice = threadIdx.x >> 5;
    const uint32_t c = blockIdx.x * 32u + lane, width = 2u * dim;
    void *out = c < dim ? dw : c < width ? db : nullptr;
    wait_for_previous_kernel();
    float sum = 0.f;
    if (out) {
#pragma unroll 8
        for (uint32_t p = slice; p < parts; p += kSlices) sum += __ldcg(partial + (uint64_t)p * width + c);
    }
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

template <typename Tx, typename Ty, uint32_t T, int NV, bool ALIGNED>
cudaError_t launch_instance(const LayerNormGradArgs &a, float *partial, uint32_t parts, cudaStream_t stream) {
    auto kernel = norm_grad_kernel<Tx, Ty, T, NV, ALIGNED>;
    constexpr uint32_t rows = row_bytes<Tx, Ty, ALIGNED, NV>() * stages_of<Tx, Ty, ALIGNED, NV>(), sums = 64u * NV * kThreads;
    constexpr uint32_t shared = rows > sums ? rows : sums;
    static bool done[kMaxDevices] = {};
    cudaError_t e = ensure_dynamic_smem(kernel, shared, done);
    if (e != cudaSuccess) return e;
    kernel<<<parts, kThreads, shared, stream>>>(a, partial);
    return cudaGetLastError();
}

constexpr uint64_t kWidest = 8u * kThreads * 2u;      // columns of the kernel that reads its rows once

// Threads of a row's group.
uint32_t threads_for(uint64_t dim) {
    uint32_t t = 8;
    while (t < kThreads && 8u * (uint64_t)t < dim) t *= 2u;
    return t;
}
uint64_t parts_for(uint64_t n, uint64_t dim) {
    if (dim <= kWidest) return part_count(n, kThreads / threads_for(dim));
    const uint64_t tiles = (dim + 255u) / 256u, most = 2368u / tiles ? 2368u / tiles : 1u, parts = part_count(n, kWideWarps);
    return parts < most ? parts : most;                  // 16 CTAs for each of a B200's SMs, all tiles together
}

template <typename Tx, typename Ty, bool ALIGNED>
cudaError_t launch_width(const LayerNormGradArgs &a, float *partial, uint32_t parts, cudaStream_t stream) {
    if (a.dim > 8u * kThreads) return launch_instance<Tx, Ty, kThreads, 2, ALIGNED>(a, partial, parts, stream);
    switch (threads_for(a.dim)) {
        case 8: return launch_instance<Tx, Ty, 8, 1, ALIGNED>(a, partial, parts, stream);
        case 16: return launch_instance<Tx, Ty, 16, 1, ALIGNED>(a, partial, parts, stream);
        case 32: return launch_instance<Tx, Ty, 32, 1, ALIGNED>(a, partial, parts, stream);
        case 64: return launch_instance<Tx, Ty, 64, 1, ALIGNED>(a, partial, parts, stream);
        case 128: return launch_instance<Tx, Ty, 128, 1, ALIGNED>(a, partial, parts, stream);
        case 256: return launch_instance<Tx, Ty, 256, 1, ALIGNED>(a, partial, parts, stream);
        default: return launch_instance<Tx, Ty, 512, 1, ALIGNED>(a, partial, parts, stream);
    }
}

template <typename Tx, typename Ty>
cudaError_t launch_wide(const LayerNormGradArgs &a, float *partial, uint32_t parts, int sm_count, cudaStream_t stream) {
    float2 *row_sums = reinterpret_cast<float2 *>(partial + (uint64_t)parts * 2u * a.dim);
    const uint64_t most = (uint64_t)sm_count * 4u;
    norm_grad_wide_rows_kernel<Tx, Ty><<<(uint32_t)(a.n < most ? a.n : most), kThreads, 0, stream>>>(a, row_sums);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const uint32_t tiles = (uint32_t)((a.dim + 255u) / 256u);
    norm_grad_wide_kernel<Tx, Ty><<<tiles * parts, kWideWarps * 32, 0, stream>>>(a, row_sums, partial, parts);
    return cudaGetLastError();
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
            using Tx = typename decltype(in)::type;
            using Ty = typename decltype(out)::type;
            if (a.dim > kWidest) return launch_wide<Tx, Ty>(a, d_partial, parts, sm_count, stream);
            return rows_aligned<Tx>(a.d_x, a.x_stride, a.n, a.dim) && rows_aligned<Ty>(a.d_dy, a.dy_stride, a.n, a.dim) &&
                           rows_aligned<Tx>(a.d_dx, a.dx_stride, a.n, a.dim)
                       ? launch_width<Tx, Ty, true>(a, d_partial, parts, stream)
                       : launch_width<Tx, Ty, false>(a, d_partial, parts, stream);
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
