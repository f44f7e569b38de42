// Gradient of layer norm:  h = (x - mu) r (rms: x r),  p = dy w,
//     dx = round(r (p - mean(p) - h mean(p h)))  (rms: without mean(p)),   dw = sum over rows of dy h,   db = sum over rows of dy
//
// Bound by memory: x and dy are read once and dx is written once.  A CTA takes a run of consecutive rows; a thread owns
// eight (or sixteen) columns of every T threads' row, so the sums over rows stay in its registers, and only the row's two sums
// cross threads, those of four (or two) rows at a time.  Rows come through a ring in shared memory that each warp fills for itself
// with asynchronous copies of 16 bytes (of the aligned pieces its elements lie in), several rows ahead.  At the end each
// CTA leaves its sums over rows in global memory, and norm_grad_columns_kernel adds them up.
// The order of every sum is a function of the number of rows, their width and type alone.
// On one B200, bf16, with the last additions: 65536 x 4096 250 us, 6.4 TB/s, again and again on the same rows, 284 on three sets in turn;
// 131072 x 1024 145 us; 509 x 2048 7.3 us; rows of odd widths are shifted: 32768 x 4095 250 us, 3.2 TB/s.
#pragma once
#include <type_traits>

#include "element_dev.cuh"
#include "iv_internal.h"
#include "layer_norm_grad.h"
#include "row_dev.cuh"

namespace ivk {

namespace {

using namespace rows;
using elem::Pair;

// The ring: 16-byte pieces of x and of dy in a row of every group, rows that a group works on at a time (four if three such steps
// have room: 8192 x 2048 25.0 us, 27.7 with two), and steps.
template <typename Tx, typename Ty, uint32_t T, int NV, int MODE>
struct Ring {
    static constexpr uint32_t kWidth = T < 32u ? T : 32u, kSegments = kThreads / kWidth;
    using X = Segment<Tx, kWidth, MODE>;
    using Y = Segment<Ty, kWidth, MODE>;
    static constexpr uint32_t kX = kSegments * X::kPieces, kY = kSegments * Y::kPieces, kRow = NV * (kX + kY);
    static constexpr uint32_t kRoom = 12288;             // pieces: 192 KiB
    static constexpr int kRows = NV > 1 ? 1 : 12u * kRow <= kRoom ? 4 : 2;
    static constexpr int kStages = (int)(kRoom / (kRow * kRows));
    static_assert(kStages >= 2 && 2u * kRows <= kWidth, "a step in flight; a lane for each of a step's statistics");
};

// One CTA per SM.
template <typename Tx, typename Ty, uint32_t T, int NV, int MODE>
__global__ void __launch_bounds__(kThreads, 1)
norm_grad_kernel(const __grid_constant__ LayerNormGradArgs a, float *partial) {
    using Rows = Ring<Tx, Ty, T, NV, MODE>;
    using X = typename Rows::X;
    using Y = typename Rows::Y;
    constexpr uint32_t kGroups = kThreads / T, kWidth = Rows::kWidth, kRow = Rows::kRow;
    constexpr int kStages = Rows::kStages, R = Rows::kRows;
    extern __shared__ uint4 ring[];                      // steps x rows x vectors x (x, dy)
    __shared__ float slots[2][2 * R * 16];
    allow_next_kernel();
    wait_for_previous_kernel();
    const uint32_t t = threadIdx.x % T, group = threadIdx.x / T, lane = threadIdx.x % kWidth, segment = threadIdx.x / kWidth;
    const uint32_t dim = (uint32_t)a.dim;
    const uint64_t begin = a.n * blockIdx.x / gridDim.x, end = a.n * (blockIdx.x + 1u) / gridDim.x;
    constexpr uint32_t kStep = R * kGroups;              // rows of a step: row i of the group is number i * kGroups + group of them
    const Tx *x = static_cast<const Tx *>(a.d_x);
    const Ty *dy = static_cast<const Ty *>(a.d_dy);
    Tx *dx = static_cast<Tx *>(a.d_dx);
    uint4 *const own_x = ring + segment * X::kPieces, *const own_y = ring + Rows::kX + segment * Y::kPieces;
    // this thread's next row to fetch and to work on, and from one row of a step, or one step, to the next
    const uint64_t row_x = kGroups * a.x_stride, row_dy = kGroups * a.dy_stride, row_dx = kGroups * a.dx_stride;
    const Tx *fetch_x = x + (begin + group) * a.x_stride, *work_x = fetch_x;
    const Ty *fetch_dy = dy + (begin + group) * a.dy_stride, *work_dy = fetch_dy;
    Tx *work_dx = dx + (begin + group) * a.dx_stride;
    auto fetch = [&](uint64_t base, uint32_t at) {       // at: the step's place in the ring
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (base + i * kGroups + group >= end) break;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const uint32_t place = at + (i * NV + j) * (Rows::kX + Rows::kY);
                X::fetch(own_x + place, fetch_x + i * row_x, t + j * T, lane, dim);
                Y::fetch(own_y + place, fetch_dy + i * row_dy, t + j * T, lane, dim);
            }
        }
        commit_copies();
        fetch_x += R * row_x;
        fetch_dy += R * row_dy;
    };
    // lane i of the group has 1 / deviation of its row i, lane R + i its mean
    auto statistic = [&](uint64_t base) {
        const uint64_t row = base + (lane & (R - 1u)) * kGroups + group;
        const float *from = lane < R ? a.d_rstd : lane < 2u * R ? a.d_mean : nullptr;
        return from && row < end ? from[row] : 0.f;
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(begin + s * kStep, s * R * kRow);
    float next_statistic = statistic(begin);
    Pair w[NV][4], dw[NV][4], db[NV][4];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        params_of(a.d_weight, a.param_type, t + j * T, dim, 1.f, w[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[j][i] = db[j][i] = Pair(0.f);
    }
    const float count = -(float)dim, scale = 1.f / count;
    uint32_t now = 0, last = (kStages - 1) * R * kRow;
    float *sums = slots[0], *other = slots[1];
    // `whole`: all rows of the step are there
    auto work = [&](uint64_t base, auto whole) {
        __syncwarp();                                    // the warp has read what is overwritten now
        fetch(base + (uint64_t)(kStages - 1) * kStep, last);
        last = now;
        const float statistics = next_statistic;
        next_statistic = statistic(base + kStep);
        wait_copies<kStages - 1>();
        __syncwarp();
        Pair h[R][NV][4], p[R][NV][4];
        float s[2 * R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[2 * i] = s[2 * i + 1] = 0.f;
            if (!decltype(whole)::value && base + i * kGroups >= end) continue;      // no group has such a row: 6001 x 1023 21.7 -> 21.1 us
            const bool live = decltype(whole)::value || base + i * kGroups + group < end;
            const uint32_t x_off = elem::misalignment(work_x + i * row_x), y_off = elem::misalignment(work_dy + i * row_dy);
            const float rstd = __shfl_sync(0xffffffffu, statistics, i, kWidth), mean = __shfl_sync(0xffffffffu, statistics, R + i, kWidth);
            // the columns behind the row's end hold 0, which may lie too far from the mean (32768 x 4095: 250 us with and without this
            // test, 262 with zeros in every row; 6001 x 1023: 22.4, 21.8 without, 22.6)
            const bool far = !(fabsf(mean * rstd) < __uint_as_float(0x7f800000u));
            const Pair by(rstd), shift(-mean);
            Pair s2(0.f), sh2(0.f);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                Pair e[4];
                const uint32_t place = now + (i * NV + j) * (Rows::kX + Rows::kY);
                elem::unpack8(X::get(own_x + place, x_off, t + j * T, lane, dim, live), h[i][j]);
                elem::unpack8(Y::get(own_y + place, y_off, t + j * T, lane, dim, live), e);
#pragma unroll
                for (int k = 0; k < 4; ++k) h[i][j][k] = (h[i][j][k] + shift) * by;
                if (MODE != kExactRows && far) {           // no h behind the row's end: an infinite one, times 0, is NaN
                    const uint32_t left = left_of(t + j * T, dim);
#pragma unroll
                    for (uint32_t k = 0; k < 4u; ++k) {
                        float lo, hi;
                        h[i][j][k].get(lo, hi);
                        h[i][j][k] = Pair(2u * k < left ? lo : 0.f, 2u * k + 1u < left ? hi : 0.f);
                    }
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    p[i][j][k] = e[k] * w[j][k];
                    db[j][k] = db[j][k] + e[k];
                    dw[j][k] = fma2(e[k], h[i][j][k], dw[j][k]);
                    s2 = s2 + p[i][j][k];
                    sh2 = fma2(p[i][j][k], h[i][j][k], sh2);
                }
            }
            s[2 * i] = s2.sum();
            s[2 * i + 1] = sh2.sum();
        }
        group_sums<T, 2 * R>(s, sums, [count, scale](float sum) { return mean_of(sum, count, scale); });
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (!decltype(whole)::value && base + i * kGroups >= end) break;
            const bool live = decltype(whole)::value || base + i * kGroups + group < end;
            const Pair by(__shfl_sync(0xffffffffu, statistics, i, kWidth)), mp(a.rms ? 0.f : s[2 * i]), mh(s[2 * i + 1]);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int k = 0; k < 4; ++k) h[i][j][k] = (fma2(h[i][j][k], mh, p[i][j][k]) + mp) * by;
                store_row_vector<Tx, MODE, T>(work_dx + i * row_dx, t + j * T, dim, live, h[i][j]);
            }
        }
        float *swap = sums;
        sums = other;
        other = swap;
        now = now + R * kRow == kStages * R * kRow ? 0u : now + R * kRow;
        work_x += R * row_x;
        work_dy += R * row_dy;
        work_dx += R * row_dx;
    };
    uint64_t base = begin;
    for (; base + kStep <= end; base += kStep) work(base, std::true_type());
    if (base < end) work(base, std::false_type());
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
template <typename Tx, typename Ty, bool ALIGNED>
__global__ void __launch_bounds__(kThreads)
norm_grad_wide_rows_kernel(LayerNormGradArgs a, float2 *row_sums) {
    __shared__ float slots[2 * 16];
    const uint32_t dim = (uint32_t)a.dim, vectors = (dim + 7u) / 8u;
    for (uint64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const Tx *x = static_cast<const Tx *>(a.d_x) + row * a.x_stride;
        const Ty *dy = static_cast<const Ty *>(a.d_dy) + row * a.dy_stride;
        const float rstd = a.d_rstd[row], mean = a.d_mean ? a.d_mean[row] : 0.f;
        float sums[2] = {0.f, 0.f};
        for (uint32_t v = threadIdx.x; v < vectors; v += kThreads) {
            RowVector<Tx, ALIGNED> rx;
            RowVector<Ty, ALIGNED> ry;
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
                sums[0] += q;
                sums[1] = fmaf(q, (h[i] - mean) * rstd, sums[1]);
            }
        }
        group_sums<kThreads, 2>(sums, slots, [](float sum) { return sum; });
        if (threadIdx.x == 0) row_sums[row] = make_float2(sums[0], sums[1]);
        __syncthreads();                                 // before the slots are written again
    }
}

template <typename Tx, typename Ty, bool ALIGNED>
__global__ void __launch_bounds__(kWideWarps * 32)
norm_grad_wide_kernel(LayerNormGradArgs a, const float2 *row_sums, float *partial, uint32_t parts) {
    __shared__ float all[16][kWideWarps][32];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, dim = (uint32_t)a.dim;
    const uint32_t tile = blockIdx.x / parts, part = blockIdx.x % parts, v = tile * 32u + lane, left = left_of(v, dim);
    const uint64_t begin = a.n * part / parts, end = a.n * (part + 1u) / parts;
    const float count = (float)dim;
    float w[8], dw[8], db[8];
    for (uint32_t i = 0; i < 8u; ++i) {
        w[i] = i >= left ? 0.f : a.d_weight ? param_at(a.d_weight, a.param_type, v * 8u + i) : 1.f;
        dw[i] = db[i] = 0.f;
    }
    for (uint64_t row = begin + warp; row < end; row += kWideWarps) {
        const Tx *x = static_cast<const Tx *>(a.d_x) + row * a.x_stride;
        const Ty *dy = static_cast<const Ty *>(a.d_dy) + row * a.dy_stride;
        RowVector<Tx, ALIGNED> rx;
        RowVector<Ty, ALIGNED> ry;
        rx.load(x, v, dim);
        ry.load(dy, v, dim);
        const float rstd = a.d_rstd[row], mean = a.d_mean ? a.d_mean[row] : 0.f;
        const float2 sums = row_sums[row];
        const float mp = a.rms ? 0.f : sums.x / count, mh = sums.y / count;
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
        store_row_vector<Tx, ALIGNED ? kAlignedRows : kAnyRows, 32>(static_cast<Tx *>(a.d_dx) + row * a.dx_stride, v, dim, true, pairs);
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

template <typename Tx, typename Ty, uint32_t T, int NV, int MODE>
cudaError_t launch_instance(const LayerNormGradArgs &a, float *partial, uint32_t parts, cudaStream_t stream) {
    auto kernel = norm_grad_kernel<Tx, Ty, T, NV, MODE>;
    using Rows = Ring<Tx, Ty, T, NV, MODE>;
    constexpr uint32_t rows = 16u * Rows::kRow * Rows::kRows * Rows::kStages, sums = 64u * NV * kThreads;
    constexpr uint32_t shared = rows > sums ? rows : sums;
    static bool done[kMaxDevices] = {};
    cudaError_t e = ensure_dynamic_smem(kernel, shared, done);
    if (e != cudaSuccess) return e;
    return launch_overlapping(kernel, dim3(parts), dim3(kThreads), shared, stream, a, partial);
}

template <typename Tx, typename Ty>
bool all_aligned(const LayerNormGradArgs &a) {
    return rows_aligned<Tx>(a.d_x, a.x_stride, a.n, a.dim) && rows_aligned<Ty>(a.d_dy, a.dy_stride, a.n, a.dim) &&
           rows_aligned<Tx>(a.d_dx, a.dx_stride, a.n, a.dim);
}
template <typename Tx, typename Ty, uint32_t T, int NV>
cudaError_t launch_mode(const LayerNormGradArgs &a, float *partial, uint32_t parts, cudaStream_t stream) {
    if (!all_aligned<Tx, Ty>(a))
        return launch_instance<Tx, Ty, T, NV, kAnyRows>(a, partial, parts, stream);
    return a.dim == 8u * T * NV ? launch_instance<Tx, Ty, T, NV, kExactRows>(a, partial, parts, stream)
                                : launch_instance<Tx, Ty, T, NV, kAlignedRows>(a, partial, parts, stream);
}
template <typename Tx, typename Ty>
cudaError_t launch_width(const LayerNormGradArgs &a, float *partial, uint32_t parts, cudaStream_t stream) {
    if (a.dim > 8u * kThreads) return launch_mode<Tx, Ty, kThreads, 2>(a, partial, parts, stream);
    switch (threads_for(a.dim)) {
        case 8: return launch_mode<Tx, Ty, 8, 1>(a, partial, parts, stream);
        case 16: return launch_mode<Tx, Ty, 16, 1>(a, partial, parts, stream);
        case 32: return launch_mode<Tx, Ty, 32, 1>(a, partial, parts, stream);
        case 64: return launch_mode<Tx, Ty, 64, 1>(a, partial, parts, stream);
        case 128: return launch_mode<Tx, Ty, 128, 1>(a, partial, parts, stream);
        case 256: return launch_mode<Tx, Ty, 256, 1>(a, partial, parts, stream);
        default: return launch_mode<Tx, Ty, 512, 1>(a, partial, parts, stream);
    }
}

template <typename Tx, typename Ty, bool ALIGNED>
cudaError_t launch_wide(const LayerNormGradArgs &a, float *partial, uint32_t parts, int sm_count, cudaStream_t stream) {
    float2 *row_sums = reinterpret_cast<float2 *>(partial + (uint64_t)parts * 2u * a.dim);
    const uint64_t most = (uint64_t)sm_count * 4u;
    norm_grad_wide_rows_kernel<Tx, Ty, ALIGNED><<<(uint32_t)(a.n < most ? a.n : most), kThreads, 0, stream>>>(a, row_sums);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const uint32_t tiles = (uint32_t)((a.dim + 255u) / 256u);
    norm_grad_wide_kernel<Tx, Ty, ALIGNED><<<tiles * parts, kWideWarps * 32, 0, stream>>>(a, row_sums, partial, parts);
    return cudaGetLastError();
}

}  // namespace

template <typename Tx, typename Ty>
cudaError_t layer_norm_grad_typed(const LayerNormGradArgs &a, float *partial, uint32_t parts, int sm_count, cudaStream_t stream) {
    if (a.dim > kWidest)
        return all_aligned<Tx, Ty>(a) ? launch_wide<Tx, Ty, true>(a, partial, parts, sm_count, stream)
                                      : launch_wide<Tx, Ty, false>(a, partial, parts, sm_count, stream);
    return launch_width<Tx, Ty>(a, partial, parts, stream);
}

}  // namespace ivk
