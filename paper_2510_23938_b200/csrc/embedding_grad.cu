// Gradient of the embedding lookup by sorted tokens:
//     grad[r, :] = round( old[r, :] + scale * sum over t with token[t] == r of g[t, :] )
// with the sum in 32 bits and in an order that the tokens alone decide, so that the same step gives the same bits on
// every run and every replica: a row's tokens in ascending order of t, cut into pieces of kPiece terms, the pieces into
// groups of kGroup; terms, pieces and groups are added from the first to the last.  No floating-point atomics.
//
//   1. sort_tokens_kernel      stable radix sort of (token, t) by one cluster, then the list of distinct rows
//   2. sum_rows_kernel         one warp per (8 sorted positions, tile of columns): adds up the pieces that begin there
//   3. fill_tail_kernel        compact form: what lies behind the last distinct row
#include <cooperative_groups.h>

#include "element_dev.cuh"
#include "iv_internal.h"

namespace cg = cooperative_groups;

namespace ivk {

namespace {

// ------------------------------------------------------------------------------------------------- sorted tokens

constexpr uint32_t kSortThreads = 1024;
constexpr uint32_t kSortWarps = kSortThreads / 32;
constexpr uint32_t kItems = 8;                             // keys per thread and tile
constexpr uint32_t kTileKeys = kSortThreads * kItems;
constexpr uint32_t kDigitBits = 9;                         // two passes for tables of up to 262,143 rows
constexpr uint32_t kBins = 1u << kDigitBits;
constexpr uint32_t kMaxCluster = 8;

struct SortShared {
    uint16_t warp_bins[kSortWarps][kBins];   // keys of each digit in a warp's part of the tile, then their prefix over the warps
    uint32_t count[kBins];                   // keys of each digit in this CTA's range (read by the whole cluster)
    uint32_t tile_count[kBins];              // keys of each digit in the current tile
    uint32_t base[kBins];                    // where this CTA's next key of each digit goes
    uint32_t scan[kSortWarps];
    uint32_t heads;                          // distinct rows that begin in this CTA's range (read by the whole cluster)
    uint32_t valid;                          // keys below n_rows in this CTA's range (read by the whole cluster)
};

// Exclusive prefix sum over the CTA; every thread also gets the total.
__device__ __forceinline__ uint32_t block_exclusive(uint32_t v, uint32_t *scan, uint32_t &total) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    uint32_t x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= (uint32_t)d) x += y;
    }
    if (lane == 31u) scan[warp] = x;
    __syncthreads();
    uint32_t w = scan[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, w, d);
        if (lane >= (uint32_t)d) w += y;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const uint32_t before = warp ? __shfl_sync(0xffffffffu, w, (warp - 1u) & 31u) : 0u;
    __syncthreads();
    return before + x - v;
}

template <typename Token>
__device__ __forceinline__ uint32_t key_of(const Token *tokens, uint32_t i, uint64_t n_rows, int64_t padding_row, uint32_t *status) {
    const int64_t t = (int64_t)tokens[i];
    if (t == padding_row) return (uint32_t)n_rows;             // sorts behind every row and is left out
    if ((uint64_t)t >= n_rows) {
        atomicMax(status, (uint32_t)IVK_DEV_BOUNDS);
        return (uint32_t)n_rows;
    }
    return (uint32_t)t;
}

template <typename Token>
__global__ void __launch_bounds__(kSortThreads, 1)
sort_tokens_kernel(const Token *tokens, uint32_t n, uint64_t n_rows, int64_t padding_row, uint32_t passes, SortBuffers b,
                   int64_t *rows_out, uint64_t *count_out, uint32_t *status) {
    extern __shared__ __align__(16) unsigned char raw_smem[];
    SortShared &s = *reinterpret_cast<SortShared *>(raw_smem);
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t ranks = cluster.num_blocks(), me = cluster.block_rank();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t share = ((n + ranks - 1) / ranks + 31u) & ~31u;
    const uint32_t lo = me * share < n ? me * share : n;
    const uint32_t hi = lo + share < n ? lo + share : n;

    for (uint32_t pass = 0; pass < passes; ++pass) {
        const uint32_t shift = pass * kDigitBits;
        const uint32_t *in_key = b.key[(pass + 1) & 1], *in_idx = b.index[(pass + 1) & 1];
        uint32_t *out_key = b.key[pass & 1], *out_idx = b.index[pass & 1];
        // digits of the whole range
        for (uint32_t i = threadIdx.x; i < kBins; i += kSortThreads) s.count[i] = 0;
        __syncthreads();
        for (uint32_t i = lo + threadIdx.x; i < hi; i += kSortThreads) {
            const uint32_t key = pass == 0 ? key_of(tokens, i, n_rows, padding_row, status) : in_key[i];
            atomicAdd(&s.count[(key >> shift) & (kBins - 1)], 1u);
        }
        cluster.sync();
        {
            uint32_t all = 0, before = 0;
            if (threadIdx.x < kBins) {
                for (uint32_t r = 0; r < ranks; ++r) {
                    const uint32_t c = *cluster.map_shared_rank(&s.count[threadIdx.x], r);
                    all += c;
                    before += r < me ? c : 0u;
                }
            }
            uint32_t total;
            const uint32_t start = block_exclusive(all, s.scan, total);
            if (threadIdx.x < kBins) s.base[threadIdx.x] = start + before;
        }
        __syncthreads();
        // stable ranks, tile by tile: a warp owns kItems * 32 consecutive keys
        for (uint32_t t0 = lo; t0 < hi; t0 += kTileKeys) {
            uint32_t key[kItems], idx[kItems], rank[kItems];
            for (uint32_t i = threadIdx.x; i < kSortWarps * kBins / 2; i += kSortThreads)
                reinterpret_cast<uint32_t *>(&s.warp_bins[0][0])[i] = 0u;
            __syncthreads();
#pragma unroll
            for (uint32_t j = 0; j < kItems; ++j) {
                const uint32_t i = t0 + warp * (kItems * 32u) + j * 32u + lane;
                key[j] = 0xffffffffu;
                idx[j] = i;
                if (i < hi) {
                    key[j] = pass == 0 ? key_of(tokens, i, n_rows, padding_row, status) : in_key[i];
                    if (pass) idx[j] = in_idx[i];
                }
            }
#pragma unroll
            for (uint32_t j = 0; j < kItems; ++j) {
                const uint32_t i = t0 + warp * (kItems * 32u) + j * 32u + lane;
                const bool live = i < hi;
                const uint32_t digit = live ? (key[j] >> shift) & (kBins - 1) : kBins + lane;   // dead lanes match nobody
                const uint32_t peers = __match_any_sync(0xffffffffu, digit);
                uint32_t old = 0;
                if (live) old = s.warp_bins[warp][digit];
                __syncwarp();
                const uint32_t below = __popc(peers & ((1u << lane) - 1u));
                if (live && below == 0) s.warp_bins[warp][digit] = (uint16_t)(old + __popc(peers));
                __syncwarp();
                rank[j] = old + below;
            }
            __syncthreads();
            if (threadIdx.x < kBins) {
                uint32_t run = 0;
                for (uint32_t w = 0; w < kSortWarps; ++w) {
                    const uint32_t c = s.warp_bins[w][threadIdx.x];
                    s.warp_bins[w][threadIdx.x] = (uint16_t)run;
                    run += c;
                }
                s.tile_count[threadIdx.x] = run;
            }
            __syncthreads();
#pragma unroll
            for (uint32_t j = 0; j < kItems; ++j) {
                const uint32_t i = t0 + warp * (kItems * 32u) + j * 32u + lane;
                if (i < hi) {
                    const uint32_t digit = (key[j] >> shift) & (kBins - 1);
                    const uint32_t pos = s.base[digit] + s.warp_bins[warp][digit] + rank[j];
                    out_key[pos] = key[j];
                    out_idx[pos] = idx[j];
                }
            }
            __syncthreads();
            if (threadIdx.x < kBins) s.base[threadIdx.x] += s.tile_count[threadIdx.x];
            __syncthreads();
        }
        cluster.sync();                                        // orders this pass's stores before the next pass's loads
    }

    // distinct rows: rank[i] = number of the row among the distinct ones, start[rank] = its first sorted position
    const uint32_t *key = b.key[(passes + 1) & 1];
    if (threadIdx.x == 0) s.heads = s.valid = 0;
    __syncthreads();
    for (uint32_t i = lo + threadIdx.x; i < hi; i += kSortThreads) {
        const uint32_t k = key[i];
        const bool valid = k < n_rows;
        if (valid) atomicAdd(&s.valid, 1u);
        if (valid && (i == 0 || key[i - 1] != k)) atomicAdd(&s.heads, 1u);
    }
    cluster.sync();
    uint32_t before = 0, distinct = 0, valid = 0;
    for (uint32_t r = 0; r < ranks; ++r) {
        const uint32_t h = *cluster.map_shared_rank(&s.heads, r);
        distinct += h;
        before += r < me ? h : 0u;
        valid += *cluster.map_shared_rank(&s.valid, r);
    }
    for (uint32_t t0 = lo; t0 < hi; t0 += kSortThreads) {
        const uint32_t i = t0 + threadIdx.x;
        bool head = false;
        uint32_t k = 0;
        if (i < hi) {
            k = key[i];
            head = k < n_rows && (i == 0 || key[i - 1] != k);
        }
        uint32_t total;
        const uint32_t r = before + block_exclusive(head ? 1u : 0u, s.scan, total);
        if (i < hi && k < n_rows) {
            b.rank[i] = head ? r : r - 1u;
            if (head) {
                b.start[r] = i;
                if (rows_out) rows_out[r] = (int64_t)k;
            }
        }
        before += total;
    }
    if (me == 0 && threadIdx.x == 0) {
        b.start[distinct] = valid;
        b.totals[0] = valid;
        b.totals[1] = distinct;
        if (count_out) *count_out = distinct;
    }
    cluster.sync();                                            // nobody leaves while its shared memory is still read
}

// ------------------------------------------------------------------------------------------------- sums

constexpr uint32_t kWindow = 8;        // sorted positions per warp
constexpr uint32_t kSumWarps = 8;
constexpr uint32_t kTileCols = 256;    // columns per warp: 8 per lane

// 8 columns of one row for this lane, the ones behind the last column as zeros.
template <typename T>
__device__ __forceinline__ void load_cols(const T *p, uint32_t cols, float (&v)[8]) {
    if (cols >= 8u) {
        if constexpr (sizeof(T) == 4) {
            elem::Packed<T, 4> a, b;
            elem::load_any<T, 4>(p, a);
            elem::load_any<T, 4>(p + 4, b);
            float x[4], y[4];
            a.unpack(x);
            b.unpack(y);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = x[i]; v[4 + i] = y[i]; }
        } else {
            elem::Packed<T, 8> a;
            elem::load_any<T, 8>(p, a);
            a.unpack(v);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i) v[i] = i < cols ? elem::to_float(p[i]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store_cols(T *p, uint32_t cols, const float (&v)[8]) {
    if (cols >= 8u && (reinterpret_cast<uintptr_t>(p) & 15u) == 0u) {
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            elem::Packed<T, 8> a;
            a.pack(v);
            elem::store_aligned<4>(p, a.w);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i)
            if (i < cols) p[i] = elem::from_float<T>(v[i]);
    }
}

struct SumArgs {
    const void *grad_out;
    uint64_t grad_stride, dim;
    void *out;
    uint64_t out_stride;
    float scale;
    uint32_t n, tiles;
};

// Adds partial sums slot(first), slot(first + 1), ... in order: pieces begin kPiece positions apart.
__device__ __forceinline__ uint32_t slot_of(uint32_t piece_begin, bool first_of_row) {
    return 2u * (piece_begin / kPiece) + (first_of_row ? 1u : 0u);
}

template <typename Tin, typename Tout, bool COMPACT, bool ADD>
__global__ void __launch_bounds__(kSumWarps * 32)
sum_rows_kernel(SumArgs a, SortBuffers b, uint32_t final_buffer) {
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t unit = (uint64_t)blockIdx.x * kSumWarps + (threadIdx.x >> 5);
    const uint32_t tile = (uint32_t)(unit % a.tiles);
    const uint64_t window64 = unit / a.tiles;
    const uint32_t valid = b.totals[0];
    if (window64 * kWindow >= valid) return;
    const uint32_t w0 = (uint32_t)window64 * kWindow, w1 = w0 + kWindow;
    const uint32_t *key = b.key[final_buffer], *index = b.index[final_buffer];
    const uint32_t col = tile * kTileCols + lane * 8u;
    const uint32_t cols = col < a.dim ? (a.dim - col < 8u ? (uint32_t)(a.dim - col) : 8u) : 0u;
    const Tin *g = static_cast<const Tin *>(a.grad_out) + col;
    Tout *out = static_cast<Tout *>(a.out) + col;

    float acc[8];
    bool open = false;                                  // a piece of ours is being added up
    uint32_t begin = 0, row_rank = 0, row_start = 0, row_end = 0;

    auto write_row = [&](uint32_t rank, uint32_t row, const float (&sum)[8]) {
        if (cols == 0u) return;
        Tout *o = out + (uint64_t)(COMPACT ? rank : row) * a.out_stride;
        float v[8];
        if (ADD) {
            load_cols<Tout>(o, cols, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(a.scale, sum[i], v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = a.scale * sum[i];
        }
        store_cols<Tout>(o, cols, v);
    };
    // partial sums are kept column-major per tile: slot, tile, 8 x 32 columns
    auto partial = [&](uint32_t slot) { return b.partial + ((uint64_t)slot * a.tiles + tile) * kTileCols + lane * 8u; };
    auto put_partial = [&](uint32_t slot, const float (&v)[8]) {
        float4 *p = reinterpret_cast<float4 *>(partial(slot));
        __stcg(p, make_float4(v[0], v[1], v[2], v[3]));
        __stcg(p + 1, make_float4(v[4], v[5], v[6], v[7]));
    };
    auto add_partials = [&](uint32_t first, uint32_t count, uint32_t step, uint32_t start, float (&sum)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = 0.f;
#pragma unroll 4
        for (uint32_t j = 0; j < count; ++j) {
            const uint32_t begin_j = first + j * step;
            const float4 *p = reinterpret_cast<const float4 *>(partial(slot_of(begin_j, begin_j == start)));
            const float4 x = __ldcg(p), y = __ldcg(p + 1);
            sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
            sum[4] += y.x; sum[5] += y.y; sum[6] += y.z; sum[7] += y.w;
        }
    };
    // true for the warp that arrives last of `members`; leaves the counter at zero for the next call
    auto arrive = [&](uint32_t *counter, uint32_t members) {
        __threadfence();
        __syncwarp();
        uint32_t last = 0;
        if (lane == 0) {
            last = atomicAdd(counter, 1u) + 1u == members ? 1u : 0u;
            if (last) *counter = 0u;
        }
        last = __shfl_sync(0xffffffffu, last, 0);
        __threadfence();
        return last != 0u;
    };
    auto flush = [&]() {
        const uint32_t row = key[row_start];
        if (row_end - row_start <= kPiece) {
            write_row(row_rank, row, acc);
            return;
        }
        const uint32_t pieces = (row_end - row_start + kPiece - 1) / kPiece;
        const uint32_t piece = (begin - row_start) / kPiece;
        const uint32_t group = piece / kGroup, groups = (pieces + kGroup - 1) / kGroup;
        const uint32_t first = row_start + group * kGroup * kPiece;      // first position of the group
        const uint32_t members = pieces - group * kGroup < kGroup ? pieces - group * kGroup : kGroup;
        put_partial(slot_of(begin, begin == row_start), acc);
        if (!arrive(b.arrivals + ((uint64_t)slot_of(first, first == row_start) * a.tiles + tile) * 2u, members)) return;
        float sum[8];
        add_partials(first, members, kPiece, row_start, sum);
        if (groups > 1) {
            put_partial(slot_of(first, first == row_start), sum);
            if (!arrive(b.arrivals + ((uint64_t)slot_of(row_start, true) * a.tiles + tile) * 2u + 1u, groups)) return;
            add_partials(row_start, groups, kGroup * kPiece, row_start, sum);
        }
        write_row(row_rank, row, sum);
    };

    for (uint32_t i0 = w0;; i0 += 32u) {
        // 32 sorted positions: token index and row of each, one per lane
        const uint32_t i = i0 + lane;
        const bool live = i < valid;
        const uint32_t my_rank = live ? b.rank[i] : 0u;
        const uint32_t my_index = live ? index[i] : 0u;
        const uint32_t my_start = live ? b.start[my_rank] : 0u;
        const uint32_t my_end = live ? b.start[my_rank + 1] : 0u;
        const bool my_begin = live && (i - my_start) % kPiece == 0u;
        for (uint32_t j = 0; j < 32u; ++j) {
            const uint32_t at = i0 + j;
            const bool piece_begin = __shfl_sync(0xffffffffu, my_begin ? 1u : 0u, j) != 0u;
            if (at >= valid || piece_begin) {
                if (open) flush();
                open = false;
                if (at >= valid || at >= w1) return;
                open = true;
                begin = at;
                row_rank = __shfl_sync(0xffffffffu, my_rank, j);
                row_start = __shfl_sync(0xffffffffu, my_start, j);
                row_end = __shfl_sync(0xffffffffu, my_end, j);
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c] = 0.f;
            }
            if (!open) {
                if (at + 1u >= w1) return;              // no piece begins in this window
                continue;
            }
            const uint32_t t = __shfl_sync(0xffffffffu, my_index, j);
            float v[8];
            load_cols<Tin>(g + (uint64_t)t * a.grad_stride, cols, v);
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[c] += v[c];
        }
    }
}

// Rows behind the last distinct one: number -1, gradient zero.
template <typename Tout>
__global__ void fill_tail_kernel(Tout *out, uint64_t out_stride, uint64_t dim, uint64_t cap, int64_t *rows, const uint32_t *totals) {
    for (uint64_t r = (uint64_t)totals[1] + blockIdx.x; r < cap; r += gridDim.x) {
        if (threadIdx.x == 0) rows[r] = -1;
        for (uint64_t c = threadIdx.x; c < dim; c += blockDim.x) out[r * out_stride + c] = elem::from_float<Tout>(0.f);
    }
}

uint32_t sort_passes(uint64_t n_rows) {
    uint32_t bits = 1;
    while (bits < 32 && (n_rows >> bits) != 0) ++bits;         // keys go up to n_rows itself
    return (bits + kDigitBits - 1) / kDigitBits;
}

template <typename Token>
cudaError_t launch_sort(const EmbeddingGradArgs &a, const SortBuffers &b, uint32_t passes, uint32_t *d_status,
                        cudaStream_t stream) {
    static bool smem_done[kMaxDevices];
    cudaError_t e = ensure_dynamic_smem(sort_tokens_kernel<Token>, sizeof(SortShared), smem_done);
    if (e != cudaSuccess) return e;
    uint32_t ranks = 1;
    while (ranks < kMaxCluster && (uint64_t)ranks * kTileKeys < a.n_tokens) ranks *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ranks);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = sizeof(SortShared);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sort_tokens_kernel<Token>, static_cast<const Token *>(a.d_tokens), (uint32_t)a.n_tokens,
                              a.n_rows, a.padding_row, passes, b, a.d_rows, a.d_count, d_status);
}

template <typename Tin, typename Tout>
cudaError_t launch_sums(const EmbeddingGradArgs &a, const SortBuffers &b, uint32_t final_buffer, cudaStream_t stream,
                        uint64_t *launches) {
    SumArgs s;
    s.grad_out = a.d_grad_out;
    s.grad_stride = a.grad_stride;
    s.dim = a.dim;
    s.out = a.d_grad;
    s.out_stride = a.out_stride;
    s.scale = a.scale;
    s.n = (uint32_t)a.n_tokens;
    s.tiles = (uint32_t)((a.dim + kTileCols - 1) / kTileCols);
    const uint64_t units = (a.n_tokens + kWindow - 1) / kWindow * s.tiles;
    const uint64_t blocks = (units + kSumWarps - 1) / kSumWarps;      // none without tokens or columns
    if (blocks > 0x7fffffffull) return cudaErrorInvalidConfiguration;
    const dim3 grid((uint32_t)blocks), block(kSumWarps * 32);
    if (blocks) {
        ++*launches;
        if (a.d_rows) sum_rows_kernel<Tin, Tout, true, false><<<grid, block, 0, stream>>>(s, b, final_buffer);
        else if (a.accumulate) sum_rows_kernel<Tin, Tout, false, true><<<grid, block, 0, stream>>>(s, b, final_buffer);
        else sum_rows_kernel<Tin, Tout, false, false><<<grid, block, 0, stream>>>(s, b, final_buffer);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !a.d_rows) return e;
    ++*launches;
    fill_tail_kernel<Tout><<<592, 256, 0, stream>>>(static_cast<Tout *>(a.d_grad), a.out_stride, a.dim, a.cap, a.d_rows, b.totals);
    return cudaGetLastError();
}

}  // namespace

// Scratch: two key and two index arrays of n, rank[n], start[n + 1], totals, then the arrival counters and the partial sums of rows with
// more than kPiece tokens (at most two pieces begin in kPiece consecutive sorted positions: the last piece of one row
// and the first of the next).
namespace {
uint64_t round16(uint64_t x) { return (x + 15u) & ~15ull; }
uint64_t slot_count(uint64_t n) { return 2u * (n / kPiece + 1u); }
uint64_t tile_count(uint64_t dim) { return (dim + kTileCols - 1) / kTileCols; }
}  // namespace

uint64_t embedding_grad_sort_bytes(uint64_t n) { return 6u * round16(4u * (n + 1u)) + 64u; }
uint64_t embedding_grad_arrival_bytes(uint64_t n, uint64_t dim) { return round16(8u * slot_count(n) * tile_count(dim)); }
uint64_t embedding_grad_partial_bytes(uint64_t n, uint64_t dim) {
    return n <= kPiece ? 16u : 4u * slot_count(n) * tile_count(dim) * kTileCols;     // one piece at most: no partial sums
}

cudaError_t launch_embedding_grad(const EmbeddingGradArgs &a, void *d_sort, uint32_t *d_arrivals, float *d_partial,
                                  uint32_t *d_status, cudaStream_t stream, uint64_t *launches) {
    const uint64_t out_size = a.out_type == IV_F32 ? 4u : 2u;
    if (!a.d_rows && !a.accumulate && a.n_rows) {
        cudaError_t e = cudaMemset2DAsync(a.d_grad, a.out_stride * out_size, 0, a.dim * out_size, a.n_rows, stream);
        if (e != cudaSuccess) return e;
    }
    if (a.n_tokens == 0 && !a.d_rows) return cudaSuccess;      // the compact form still has its count and its tail to write
    const uint64_t array = round16(4u * (a.n_tokens + 1u));
    uint8_t *p = static_cast<uint8_t *>(d_sort);
    SortBuffers b;
    b.key[0] = reinterpret_cast<uint32_t *>(p);
    b.key[1] = reinterpret_cast<uint32_t *>(p + array);
    b.index[0] = reinterpret_cast<uint32_t *>(p + 2 * array);
    b.index[1] = reinterpret_cast<uint32_t *>(p + 3 * array);
    b.rank = reinterpret_cast<uint32_t *>(p + 4 * array);
    b.start = reinterpret_cast<uint32_t *>(p + 5 * array);
    b.totals = reinterpret_cast<uint32_t *>(p + 6 * array);
    b.arrivals = d_arrivals;
    b.partial = d_partial;
    const uint32_t passes = sort_passes(a.n_rows);
    cudaError_t e = a.token_bytes == 4 ? launch_sort<int32_t>(a, b, passes, d_status, stream)
                                       : launch_sort<int64_t>(a, b, passes, d_status, stream);
    if (e != cudaSuccess) return e;
    ++*launches;
    if (a.dim == 0 && !a.d_rows) return cudaSuccess;
    return by_types(a.grad_type, a.out_type, [&](auto in, auto out) {
        return launch_sums<typename decltype(in)::type, typename decltype(out)::type>(a, b, (passes + 1) & 1, stream, launches);
    });
}

}  // namespace ivk
