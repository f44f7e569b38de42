// Layer norm of rows, and its root-mean-square form:
//     mu = mean(x) (rms: 0),  r = 1 / sqrt(mean((x - mu)^2) + eps),  y = round((x - mu) r w + b)
//
// Bound by memory: a row is read once, held in registers for both sums (the mean first, then the squares of what is left,
// so nothing cancels) and written once.  The threads of a row, 8 to 512 with one, two or four vectors of eight elements each,
// follow from its width alone, and so does the order of its sums: a row's bits do not depend on the other rows, on the
// launch or on the alignment.  Rows come through a ring in shared memory that each warp fills for itself with asynchronous copies,
// several rows ahead; a group of threads works on four (or two) at a time, so that their sums cross threads together.  The kernel may
// start while the one before it ends (8192 x 2048: 18.6 us a call without, 17.2 with).
// On one B200, bf16: 131072 x 4096 350 us, 6.1 TB/s; 65536 x 8192 320 us, 6.7 TB/s; 262144 x 1024 167 us; a single row 2.5 us.  Rows at odd
// places or of odd widths are shifted, which costs instructions: 65536 x 4095 372 us, 2.9 TB/s.
#pragma once
#include <type_traits>

#include "element_dev.cuh"
#include "iv_internal.h"
#include "row_dev.cuh"

namespace ivk {

namespace {

using namespace rows;
using elem::Pair;

constexpr uint32_t kThreads = 512;

// The ring: 16-byte pieces in a row of every group, rows that a group works on at a time, and steps.  One CTA takes an SM's shared
// memory, but for aligned 16-bit rows of 2049 to 4096 columns two share it.  Two and one, us, 1 GB of bf16 rows: 2056 columns 580 and 676,
// 2560 470 and 550, 3584 360 and 436, 4096 350 and 388; root-mean-square form 444 and 522, 367 and 419, 384 and 341, 337 and 340; half as many
// rows to 32 bits 343 and 380, 305 and 318, 272 and 278, 280 and 257: one would be better for a few of them, which no width or
// type sets apart.  Elsewhere two are worse: 262144 x 1024 181 and 166; float32 rows to 16 bits, 65536 x 4096, 279 and 240.
template <typename Tx, uint32_t T, int NV, int MODE>
struct Ring {
    static constexpr uint32_t kWidth = T < 32u ? T : 32u, kSegments = kThreads / kWidth;
    using X = Segment<Tx, kWidth, MODE>;
    static constexpr uint32_t kX = kSegments * X::kPieces, kRow = NV * kX;
    static constexpr int kCtas = NV == 1 && T == kThreads && sizeof(Tx) == 2 && MODE != kAnyRows ? 2 : 1;
    static constexpr uint32_t kRoom = kCtas == 2 ? 6144 : 12288;     // pieces: 96 or 192 KiB
    static constexpr int kRows = 12u * kRow <= kRoom ? 4 : 6u * kRow <= kRoom ? 2 : 1;
    static constexpr int kStages = (int)(kRoom / (kRow * kRows));
    static_assert(kStages >= 2, "a step in flight");
};

template <typename Tx, typename Ty, uint32_t T, int NV, int MODE>
__global__ void __launch_bounds__(kThreads, Ring<Tx, T, NV, MODE>::kCtas)
layer_norm_kernel(const __grid_constant__ LayerNormArgs a) {
    allow_next_kernel();
    wait_for_previous_kernel();
    using Rows = Ring<Tx, T, NV, MODE>;
    using X = typename Rows::X;
    constexpr uint32_t kGroups = kThreads / T, kWidth = Rows::kWidth, kRow = Rows::kRow;
    constexpr int kStages = Rows::kStages, R = Rows::kRows;
    extern __shared__ uint4 ring[];                      // steps x rows x vectors
    __shared__ float slots[2][R * 16];
    const uint32_t t = threadIdx.x % T, group = threadIdx.x / T, lane = threadIdx.x % kWidth;
    const uint32_t dim = (uint32_t)a.dim;
    constexpr uint32_t kStep = R * kGroups;              // rows of a step: row i of the group is number i * kGroups + group of them
    const uint64_t begin = (uint64_t)blockIdx.x * kStep, end = a.n, stride = (uint64_t)gridDim.x * kStep;
    const Tx *x = static_cast<const Tx *>(a.d_x);
    Ty *y = static_cast<Ty *>(a.d_y);
    uint4 *const own = ring + threadIdx.x / kWidth * X::kPieces;
    // this thread's next row to fetch and to work on, and from one row of a step to the next; a CTA takes every gridDim.x-th step, so
    // that all of them read and write in one region of memory (131072 x 4096: 342 us, 387 with a run of rows each)
    const uint64_t row_x = kGroups * a.x_stride, row_y = kGroups * a.y_stride;
    const Tx *fetch_x = x + (begin + group) * a.x_stride, *work_x = fetch_x;
    Ty *work_y = y + (begin + group) * a.y_stride;
    auto fetch = [&](uint64_t base, uint32_t at) {       // at: the step's place in the ring
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (base + i * kGroups + group >= end) break;
#pragma unroll
            for (int j = 0; j < NV; ++j) X::fetch(own + at + (i * NV + j) * Rows::kX, fetch_x + i * row_x, t + j * T, lane, dim);
        }
        commit_copies();
        fetch_x += gridDim.x * R * row_x;
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(begin + s * stride, s * R * kRow);
    Pair w[NV][4], b[NV][4];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        params_of(a.d_weight, a.param_type, t + j * T, dim, 1.f, w[j]);
        params_of(a.d_bias, a.param_type, t + j * T, dim, 0.f, b[j]);
    }
    const float count = (float)dim, scale = 1.f / count;
    uint32_t now = 0, last = (kStages - 1) * R * kRow;
    float *sums = slots[0], *other = slots[1];
    auto turn = [&]() {
        float *used = sums;
        sums = other;
        other = used;
    };
    // `whole`: all rows of the step are there
    auto work = [&](uint64_t base, auto whole) {
        __syncwarp();                                    // the warp has read what is overwritten now
        fetch(base + (kStages - 1) * stride, last);
        last = now;
        wait_copies<kStages - 1>();
        __syncwarp();
        elem::Packed<Tx, 8> raw[R][NV];
        float mean[R], rstd[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const bool live = decltype(whole)::value || base + i * kGroups + group < end;
            const uint32_t off = elem::misalignment(work_x + i * row_x);
#pragma unroll
            for (int j = 0; j < NV; ++j) raw[i][j] = X::get(own + now + (i * NV + j) * Rows::kX, off, t + j * T, lane, dim, live);
            mean[i] = 0.f;
        }
        if (!a.rms) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                Pair sum(0.f);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    Pair v[4];
                    elem::unpack8(raw[i][j], v);
                    sum = sum + ((v[0] + v[1]) + (v[2] + v[3]));
                }
                mean[i] = sum.sum();
            }
            group_sums<T, R>(mean, sums, [count, scale](float sum) { return mean_of(sum, count, scale); });
            turn();
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const Pair shift(-mean[i]);
            Pair squares(0.f);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const uint32_t left = left_of(t + j * T, dim);
                Pair v[4];
                elem::unpack8(raw[i][j], v);
                if (MODE == kAnyRows && left < 8u) {        // zeros behind the row's end are not the mean away from it
#pragma unroll
                    for (uint32_t k = 0; k < 4u; ++k) {
                        float lo, hi;
                        v[k].get(lo, hi);
                        v[k] = Pair(2u * k < left ? lo : mean[i], 2u * k + 1u < left ? hi : mean[i]);
                    }
                }
                if (MODE != kAlignedRows || left) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const Pair d = v[k] + shift;
                        squares = fma2(d, d, squares);
                    }
                }
            }
            rstd[i] = squares.sum();
        }
        group_sums<T, R>(rstd, sums, [&](float sum) { return 1.f / sqrtf(sum * scale + a.eps); });
        turn();
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const uint64_t row = base + i * kGroups + group;
            const bool live = decltype(whole)::value || row < end;
            const Pair shift(-mean[i]), by(rstd[i]);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                Pair e[4];
                elem::unpack8(raw[i][j], e);
#pragma unroll
                for (int k = 0; k < 4; ++k) e[k] = fma2((e[k] + shift) * by, w[j][k], b[j][k]);
                store_row_vector<Ty, MODE, T>(work_y + i * row_y, t + j * T, dim, live, e);
            }
            if (live && t == 0u) {
                if (a.d_mean) a.d_mean[row] = mean[i];
                if (a.d_rstd) a.d_rstd[row] = rstd[i];
            }
        }
        now = now + R * kRow == kStages * R * kRow ? 0u : now + R * kRow;
        work_x += gridDim.x * R * row_x;
        work_y += gridDim.x * R * row_y;
    };
    uint64_t base = begin;
    for (; base + kStep <= end; base += stride) work(base, std::true_type());
    if (base < end) work(base, std::false_type());
}

// Rows too wide for that: one CTA per row, which reads it three times: from the L2 cache the second and third time as long as the rows
// in flight, two for each SM, fit there (on a B200 16-bit rows of some 200,000 columns), from memory beyond.  A row has one SM.
// 1.07e9 bf16 elements: 65,536 columns 1.53 ms, 2.8 TB/s of what must move once; 262,144 1.67 ms; 2^20 1.84 ms; 64 rows of 2^24 4.75 ms.
constexpr uint32_t kWideThreads = 1024;
template <typename Tx, typename Ty, bool ALIGNED>
__global__ void __launch_bounds__(kWideThreads)
layer_norm_wide_kernel(LayerNormArgs a) {
    __shared__ float slots[2][kWideThreads / 32];
    allow_next_kernel();
    wait_for_previous_kernel();
    const uint32_t dim = (uint32_t)a.dim, vectors = (dim + 7u) / 8u;
    const float count = (float)dim, scale = 1.f / count;
    uint32_t turn = 0;
    for (uint64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const Tx *in = static_cast<const Tx *>(a.d_x) + row * a.x_stride;
        Ty *out = static_cast<Ty *>(a.d_y) + row * a.y_stride;
        const uint32_t off = elem::misalignment(in);
        auto each = [&](auto f) {
            for (uint32_t base = 0; base < vectors; base += kWideThreads) {      // whole warps
                const uint32_t v = base + threadIdx.x;
                RowVector<Tx, ALIGNED> raw;
                Pair e[4];
                raw.load(in, v, dim);
                elem::unpack8(raw.get(off, v, dim), e);
                f(v, e);
            }
        };
        float mean = 0.f, sum = 0.f;
        if (!a.rms) {
            each([&](uint32_t, Pair (&e)[4]) { sum += ((e[0] + e[1]) + (e[2] + e[3])).sum(); });
            float all[1] = {sum};
            group_sums<kWideThreads, 1>(all, slots[turn], [count](float s) { return s / count; });
            turn ^= 1u;
            mean = all[0];
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
        float all[1] = {sum};
        group_sums<kWideThreads, 1>(all, slots[turn], [&](float s) { return 1.f / sqrtf(s * scale + a.eps); });
        turn ^= 1u;
        const float rstd = all[0];
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
            store_row_vector<Ty, ALIGNED ? kAlignedRows : kAnyRows, kWideThreads>(out, v, dim, true, p);
        });
        if (threadIdx.x == 0) {
            if (a.d_mean) a.d_mean[row] = mean;
            if (a.d_rstd) a.d_rstd[row] = rstd;
        }
    }
}

template <typename Tx, typename Ty, uint32_t T, int NV, int MODE>
cudaError_t launch_instance(const LayerNormArgs &a, int sm_count, cudaStream_t stream) {
    using Rows = Ring<Tx, T, NV, MODE>;
    auto kernel = layer_norm_kernel<Tx, Ty, T, NV, MODE>;
    constexpr uint32_t shared = 16u * Rows::kRow * Rows::kRows * Rows::kStages;
    static bool done[kMaxDevices] = {};
    cudaError_t e = ensure_dynamic_smem(kernel, shared, done);
    if (e != cudaSuccess) return e;
    const uint64_t blocks = (a.n + kThreads / T * Rows::kRows - 1) / (kThreads / T * Rows::kRows), most = (uint64_t)sm_count * Rows::kCtas;
    return launch_overlapping(kernel, dim3((uint32_t)(blocks < most ? blocks : most)), dim3(kThreads), shared, stream, a);
}

template <typename Tx, typename Ty, uint32_t T, int NV>
cudaError_t launch_mode(const LayerNormArgs &a, int sm_count, cudaStream_t stream) {
    if (!rows_aligned<Tx>(a.d_x, a.x_stride, a.n, a.dim) || !rows_aligned<Ty>(a.d_y, a.y_stride, a.n, a.dim))
        return launch_instance<Tx, Ty, T, NV, kAnyRows>(a, sm_count, stream);
    return a.dim == 8u * T * NV ? launch_instance<Tx, Ty, T, NV, kExactRows>(a, sm_count, stream)
                                : launch_instance<Tx, Ty, T, NV, kAlignedRows>(a, sm_count, stream);
}
template <typename Tx, typename Ty>
cudaError_t launch_width(const LayerNormArgs &a, int sm_count, cudaStream_t stream) {
    const uint64_t v = (a.dim + 7u) / 8u;
    if (v <= 8u) return launch_mode<Tx, Ty, 8, 1>(a, sm_count, stream);
    if (v <= 16u) return launch_mode<Tx, Ty, 16, 1>(a, sm_count, stream);
    if (v <= 32u) return launch_mode<Tx, Ty, 32, 1>(a, sm_count, stream);
    if (v <= 64u) return launch_mode<Tx, Ty, 64, 1>(a, sm_count, stream);
    if (v <= 128u) return launch_mode<Tx, Ty, 128, 1>(a, sm_count, stream);
    if (v <= 256u) return launch_mode<Tx, Ty, 256, 1>(a, sm_count, stream);
    if (v <= 512u) return launch_mode<Tx, Ty, 512, 1>(a, sm_count, stream);
    if (v <= 1024u) return launch_mode<Tx, Ty, 512, 2>(a, sm_count, stream);
    return launch_mode<Tx, Ty, 512, 4>(a, sm_count, stream);
}

}  // namespace

template <typename Tx, typename Ty>
cudaError_t layer_norm_typed(const LayerNormArgs &a, int sm_count, cudaStream_t stream) {
    if (a.dim > 8u * kThreads * 4u) {
        const uint64_t most = (uint64_t)sm_count * 2u;
        const bool aligned = rows_aligned<Tx>(a.d_x, a.x_stride, a.n, a.dim) && rows_aligned<Ty>(a.d_y, a.y_stride, a.n, a.dim);
        auto kernel = aligned ? layer_norm_wide_kernel<Tx, Ty, true> : layer_norm_wide_kernel<Tx, Ty, false>;
        return launch_overlapping(kernel, dim3((uint32_t)(a.n < most ? a.n : most)), dim3(kWideThreads), 0, stream, a);
    }
    return launch_width<Tx, Ty>(a, sm_count, stream);
}

}  // namespace ivk
