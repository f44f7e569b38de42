// Gradient of the embedding lookup by sorted tokens:
//     grad[r, :] = round( old[r, :] + scale * sum over t with token[t] == r of g[t, :] )
// with the sum in 32 bits and in an order that the tokens alone decide, so that the same step gives the same bits on
// every run and every replica: a row's tokens in ascending order of t, cut into pieces of kPiece terms, the pieces into
// groups of kGroup; terms, pieces and groups are added from the first to the last.  No floating-point atomics.
//
//   1. sort_tokens_kernel      stable radix sort of (token, t) by one cluster, then the list of distinct rows
//   2. sum_rows_kernel         one warp per (8 sorted positions, tile of columns): adds up the pieces that begin there
//   3. fill_rows_kernel        fresh table gradient: the rows without a token, beside the other two
//
// The sums are bound by memory (every gradient row read once, every row written once), the sort by latency: its passes
// are chains of shared-memory steps and cluster barriers.  So the sort uses as many SMs as a cluster spans before it gives a
// thread a second key, the sums' CTAs are in place when it ends, and what needs no order (the fill) runs beside it.
// One warp adds up 1 KiB of a row: a row of 8 KiB is eight warps' work, which keeps rows with many tokens from
// becoming the longest path; rows of more than kPiece tokens are cut, and the warp that completes a group of pieces
// adds up their sums.
//
// On one B200, bf16 rows of 8 KiB: 65,536 tokens, whole table of 128,256 rows: 264 to 272 us, 5.9 TB/s of what has to move
// (alone: sort 27, sums 112, fill 145; the last two share the memory); 16,384 tokens, compact: 58 us (sort 15, sums 38 at
// 6 TB/s).  8192 tokens of 4 KiB added to a 32-bit table gradient: 33 us (sort 13, sums 20); 509 tokens: 14 us.  Narrow
// rows wait for the sort and for one latency per row: 131,072 tokens of 64 columns 70 us, where their bytes need 4.
#include <cooperative_groups.h>
#include <type_traits>

#include "element_dev.cuh"
#include "iv_internal.h"
#include "tma_dev.cuh"

namespace cg = cooperative_groups;

namespace ivk {

namespace {

// ------------------------------------------------------------------------------------------------- sorted tokens

constexpr uint32_t kSortThreads = 512;                     // with 1024 the barriers of a pass cost more (8192 tokens added: 35.5 us, 33.6; compact 16,384: 61.3, 58.3)
constexpr uint32_t kSortWarps = kSortThreads / 32;
constexpr uint32_t kMaxItems = 16;                         // keys per thread and tile
constexpr uint32_t kDigitBits = 9;                         // two passes for tables of up to 262,143 rows
constexpr uint32_t kBins = 1u << kDigitBits;
constexpr uint32_t kWarpParts = kSortWarps / 8;            // the prefix over the warps is taken eight at a time
constexpr uint32_t kMaxCluster = 16;                       // 16,384 tokens, compact: 58.5 us with 16, 60.0 with 8 (8192 added: 33.9, 33.1)

struct SortShared {
    union {
        uint32_t peers[kSortWarps][kBins];                 // ranking: lanes of the warp that hold each digit
        uint2 sorted[kSortThreads * kMaxItems];            // afterwards: the tile's keys and indices by digit
    };
    uint2 incoming[kSortThreads * kMaxItems];              // one tile per CTA: the keys at this CTA's positions after the pass
    uint16_t warp_bins[kSortWarps][kBins];                 // keys of each digit in a warp's part of the tile, then their prefix over eight warps
    uint32_t from[kMaxCluster][kBins];                     // keys of each digit in every CTA's share
    uint4 rows_from[kMaxCluster];                          // of every CTA's share: rows that begin, valid keys, 1 + the last place a row begins
    uint32_t parts[kWarpParts][kBins];                     // keys of each digit in every part of the warps, then before it
    uint32_t count[kBins];                                 // keys of each digit in this CTA's share
    uint32_t tile_first[kBins];                            // place of the first key of each digit in the current tile, sorted
    uint32_t base[kBins];                                  // where this CTA's next key of each digit goes
    uint32_t scan[kSortWarps];
    uint32_t warp_heads[kSortWarps], warp_last[kSortWarps];
    uint32_t heads, valid, last_head;                      // of this CTA's share
};

// Exclusive prefix sum over the CTA.
__device__ __forceinline__ uint32_t block_exclusive(uint32_t v, uint32_t *scan) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    uint32_t x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= (uint32_t)d) x += y;
    }
    if (lane == 31u) scan[warp] = x;
    __syncthreads();
    const uint32_t before = __reduce_add_sync(0xffffffffu, lane < warp ? scan[lane] : 0u);
    __syncthreads();
    return before + x - v;
}

// The rows of a fresh table gradient that no token names are set to zero beside the sort: each CTA takes a range of
// rows, marks those with a token (it reads all tokens) and writes the others.
constexpr uint32_t kFillThreads = 1024;
constexpr uint32_t kFillRows = 1u << 18;                   // rows marked at a time: 32 KiB of bits

template <typename Token>
__global__ void __launch_bounds__(kFillThreads)
fill_rows_kernel(const Token *tokens, uint32_t n, uint64_t n_rows, int64_t padding_row, uint8_t *out, uint64_t row_bytes,
                 uint64_t stride_bytes) {
    __shared__ uint32_t marks[kFillRows / 32];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint64_t begin = n_rows * blockIdx.x / gridDim.x, end = n_rows * (blockIdx.x + 1u) / gridDim.x;
    for (uint64_t r0 = begin; r0 < end; r0 += kFillRows) {
        const uint32_t rows = (uint32_t)(end - r0 < kFillRows ? end - r0 : kFillRows);
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < (rows + 31u) / 32u; i += kFillThreads) marks[i] = 0u;
        __syncthreads();
        constexpr uint32_t kAhead = 8;
        for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kFillThreads * kAhead) {
            int64_t t[kAhead];
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) t[u] = i0 + u * kFillThreads < n ? (int64_t)tokens[i0 + u * kFillThreads] : -1;
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) {
                const uint64_t at = (uint64_t)t[u] - r0;
                if (at < rows && t[u] != padding_row) atomicOr(&marks[at >> 5], 1u << (at & 31u));
            }
        }
        __syncthreads();
        for (uint32_t r = warp; r < rows; r += kFillThreads / 32) {
            if (marks[r >> 5] >> (r & 31u) & 1u) continue;
            uint8_t *p = out + (r0 + r) * stride_bytes;
            const uint64_t head = (16u - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u;
            const uint64_t start = head < row_bytes ? head : row_bytes, body = (row_bytes - start) & ~15ull;
            if (lane < start / 2u) reinterpret_cast<uint16_t *>(p)[lane] = 0;
            uint4 *q = reinterpret_cast<uint4 *>(p + start);
#pragma unroll 4
            for (uint64_t i = lane; i < body / 16u; i += 32u) q[i] = make_uint4(0u, 0u, 0u, 0u);
            if (lane < (row_bytes - start - body) / 2u) reinterpret_cast<uint16_t *>(p + start + body)[lane] = 0;
        }
    }
}

// One cluster sorts all tokens; CTA r owns the r-th share of the positions, cut into tiles of kSortThreads * ITEMS keys
// of which each warp owns a consecutive part.  Per pass: digits counted over the share, written into the shared memory
// of every CTA of the cluster, then every key's place = keys of smaller digits + same digit in earlier CTAs, tiles,
// warps and lanes.  With one tile per CTA the keys stay in shared memory, each written into that of the CTA whose
// position it takes; with more they go through global memory.
template <typename Token, uint32_t ITEMS>
__global__ void __launch_bounds__(kSortThreads, 1)
sort_tokens_kernel(const Token *tokens, uint32_t n, uint64_t n_rows, int64_t padding_row, uint32_t passes, SortBuffers b,
                   int64_t *rows_out, uint64_t *count_out, uint32_t *status) {
    constexpr uint32_t kTileKeys = kSortThreads * ITEMS;
    extern __shared__ __align__(16) unsigned char raw_smem[];
    SortShared &s = *reinterpret_cast<SortShared *>(raw_smem);
    allow_next_kernel();
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t ranks = cluster.num_blocks(), me = cluster.block_rank();
    // another CTA's shared memory may be written only once that CTA has started: everybody says so here and waits for the
    // others before the first such write, behind the first tile's loads and its sort (relaxed: nothing has been written yet
    // that they could read; an arrival that publishes writes costs 0.7 us)
    if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t share = ((n + ranks - 1) / ranks + 31u) & ~31u;
    const uint32_t lo = me * share < n ? me * share : n;
    const uint32_t hi = lo + share < n ? lo + share : n;
    const bool one_tile = share <= kTileKeys;
    const uint32_t mine = warp * (ITEMS * 32u) + lane;               // this lane's first key in a tile; the next are 32 apart
    bool bad = false;
    auto all_sync = [&]() {
        if (ranks > 1) cluster.sync();
        else __syncthreads();
    };
    // padding and rows that are not there sort behind every row and are left out; a padding row of -1 is none, not token -1
    auto to_key = [&](Token token) {
        const int64_t t = (int64_t)token;
        const bool there = (uint64_t)t < n_rows, padding = t == padding_row && t >= 0;
        bad |= !there && !padding;
        return there && !padding ? (uint32_t)t : (uint32_t)n_rows;
    };

    for (uint32_t pass = 0; pass < passes; ++pass) {
        const uint32_t shift = pass * kDigitBits;
        const uint32_t *in_key = b.key[(pass + 1) & 1], *in_idx = b.index[(pass + 1) & 1];
        uint32_t *out_key = b.key[pass & 1], *out_idx = b.index[pass & 1];
        uint32_t key[ITEMS], idx[ITEMS], rank[ITEMS];

        // counters of the warps that have keys to zero, while the tile's loads are under way
        auto clear = [&](uint32_t t0) {
            const uint32_t keys = hi - t0 < kTileKeys ? hi - t0 : kTileKeys;
            const uint32_t warps = (keys + ITEMS * 32u - 1) / (ITEMS * 32u);
            for (uint32_t i = threadIdx.x; i < warps * (kBins / 8); i += kSortThreads)
                reinterpret_cast<uint4 *>(&s.warp_bins[0][0])[i] = make_uint4(0u, 0u, 0u, 0u);
            for (uint32_t i = threadIdx.x; i < warps * (kBins / 4); i += kSortThreads)
                reinterpret_cast<uint4 *>(&s.peers[0][0])[i] = make_uint4(0u, 0u, 0u, 0u);
        };
        auto load_tile = [&](uint32_t t0, bool clearing) {
            if (pass == 0) {
                Token token[ITEMS];
#pragma unroll
                for (uint32_t j = 0; j < ITEMS; ++j) {
                    const uint32_t i = t0 + mine + j * 32u;
                    token[j] = i < hi ? tokens[i] : Token(0);
                    idx[j] = i;
                }
                if (clearing) clear(t0);
#pragma unroll
                for (uint32_t j = 0; j < ITEMS; ++j) key[j] = idx[j] < hi ? to_key(token[j]) : 0u;
            } else if (one_tile) {
                const uint2 *from = ranks > 1 ? s.incoming : s.sorted;
#pragma unroll
                for (uint32_t j = 0; j < ITEMS; ++j) {
                    const uint2 k = t0 + mine + j * 32u < hi ? from[mine + j * 32u] : make_uint2(0u, 0u);
                    key[j] = k.x;
                    idx[j] = k.y;
                }
                if (ranks == 1) __syncthreads();               // the counters lie where the sorted keys were
                if (clearing) clear(t0);
            } else {
#pragma unroll
                for (uint32_t j = 0; j < ITEMS; ++j) {
                    const uint32_t i = t0 + mine + j * 32u;
                    key[j] = i < hi ? in_key[i] : 0u;
                    idx[j] = i < hi ? in_idx[i] : 0u;
                }
                if (clearing) clear(t0);
            }
            if (clearing) __syncthreads();
        };
        // The tile sorted by this pass's digit into s.sorted; returns the tile's keys of digit threadIdx.x.
        auto sort_tile = [&](uint32_t t0) {
            const uint32_t keys = hi - t0 < kTileKeys ? hi - t0 : kTileKeys;
            const uint32_t warps = (keys + ITEMS * 32u - 1) / (ITEMS * 32u);          // that have keys
#pragma unroll
            for (uint32_t j = 0; j < ITEMS; ++j) {
                rank[j] = 0;
                if (warp * (ITEMS * 32u) + j * 32u < keys) {                           // the same for the whole warp
                    const bool live = mine + j * 32u < keys;
                    const uint32_t digit = (key[j] >> shift) & (kBins - 1);
                    uint32_t *mask = &s.peers[warp][digit];
                    if (live) atomicOr(mask, 1u << lane);
                    __syncwarp();
                    const uint32_t peers = live ? *mask : 0u, old = s.warp_bins[warp][digit];
                    const uint32_t below = __popc(peers & ((1u << lane) - 1u));
                    rank[j] = old + below;
                    __syncwarp();
                    if (live && below == 0) {
                        s.warp_bins[warp][digit] = (uint16_t)(old + __popc(peers));
                        *mask = 0u;
                    }
                    __syncwarp();
                }
            }
            __syncthreads();
            // prefix over the warps, two digits (16 bits each) and eight of the warps per thread
            static_assert(kWarpParts * (kBins / 2) == kSortThreads, "a thread for every pair of digits and eight warps");
            {
                const uint32_t pair = threadIdx.x % (kBins / 2), part = threadIdx.x / (kBins / 2);
                uint32_t run = 0;
#pragma unroll
                for (uint32_t w = part * 8u; w < (part + 1u) * 8u; ++w) {
                    uint32_t *p = reinterpret_cast<uint32_t *>(&s.warp_bins[w][0]) + pair;
                    const uint32_t c = w < warps ? *p : 0u;
                    if (w < warps) *p = run;
                    run += c;
                }
                reinterpret_cast<uint2 *>(&s.parts[part][0])[pair] = make_uint2(run & 0xffffu, run >> 16);
            }
            __syncthreads();
            uint32_t total = 0;
            if (threadIdx.x < kBins) {
#pragma unroll
                for (uint32_t part = 0; part < kWarpParts; ++part) {
                    const uint32_t c = s.parts[part][threadIdx.x];
                    s.parts[part][threadIdx.x] = total;
                    total += c;
                }
            }
            const uint32_t first = block_exclusive(total, s.scan);
            if (threadIdx.x < kBins) s.tile_first[threadIdx.x] = first;
            __syncthreads();
            // by digit in shared memory first: keys of one digit then leave for consecutive addresses
#pragma unroll
            for (uint32_t j = 0; j < ITEMS; ++j) {
                if (mine + j * 32u < keys) {
                    const uint32_t digit = (key[j] >> shift) & (kBins - 1);
                    const uint32_t at = s.tile_first[digit] + s.parts[warp / 8u][digit] + s.warp_bins[warp][digit] + rank[j];
                    s.sorted[at] = make_uint2(key[j], idx[j]);
                }
            }
            return total;
        };

        uint32_t digits = 0;                                   // of digit threadIdx.x: keys in the share
        if (one_tile) {
            load_tile(lo, true);
            digits = sort_tile(lo);
            if (ranks == 1) {                                  // sorted by this digit as a whole
                __syncthreads();
                continue;
            }
        } else {
            for (uint32_t i = threadIdx.x; i < kBins; i += kSortThreads) s.count[i] = 0;
            __syncthreads();
            for (uint32_t t0 = lo; t0 < hi; t0 += kTileKeys) {
                load_tile(t0, false);
#pragma unroll
                for (uint32_t j = 0; j < ITEMS; ++j)
                    if (t0 + mine + j * 32u < hi) atomicAdd(&s.count[(key[j] >> shift) & (kBins - 1)], 1u);
            }
            __syncthreads();
            if (threadIdx.x < kBins) digits = s.count[threadIdx.x];
        }
        if (ranks > 1) {
            if (pass == 0) cluster.barrier_wait();
            if (threadIdx.x < kBins)
                for (uint32_t r = 0; r < ranks; ++r) *cluster.map_shared_rank(&s.from[me][threadIdx.x], r) = digits;
            cluster.sync();
            uint32_t all = 0, before = 0;
            if (threadIdx.x < kBins) {
                for (uint32_t r = 0; r < ranks; ++r) {
                    const uint32_t c = s.from[r][threadIdx.x];
                    all += c;
                    before += r < me ? c : 0u;
                }
            }
            const uint32_t start = block_exclusive(all, s.scan);
            if (threadIdx.x < kBins) s.base[threadIdx.x] = start + before;
        } else {
            const uint32_t start = block_exclusive(digits, s.scan);
            if (threadIdx.x < kBins) s.base[threadIdx.x] = start;
        }
        __syncthreads();
        for (uint32_t t0 = lo; t0 < hi; t0 += kTileKeys) {
            uint32_t tile_count = 0;
            if (!one_tile) {
                load_tile(t0, true);
                tile_count = sort_tile(t0);
                __syncthreads();
            }
            const uint32_t keys = hi - t0 < kTileKeys ? hi - t0 : kTileKeys;
#pragma unroll
            for (uint32_t j = 0; j < ITEMS; ++j) {
                const uint32_t at = j * kSortThreads + threadIdx.x;
                if (at < keys) {
                    const uint2 k = s.sorted[at];
                    const uint32_t digit = (k.x >> shift) & (kBins - 1);
                    const uint32_t pos = s.base[digit] + at - s.tile_first[digit];
                    if (one_tile) {
                        const uint32_t r = pos / share;
                        *cluster.map_shared_rank(&s.incoming[pos - r * share], r) = k;
                    } else {
                        out_key[pos] = k.x;
                        out_idx[pos] = k.y;
                    }
                }
            }
            if (!one_tile) {
                __syncthreads();
                if (threadIdx.x < kBins) s.base[threadIdx.x] += tile_count;
                __syncthreads();
            }
        }
        all_sync();                                            // orders this pass's stores before the next pass's loads
    }
    if (bad) atomicMax(status, (uint32_t)IVK_DEV_BOUNDS);

    // distinct rows: each sorted position's record {token, first position of its row, number of its row among the
    // distinct ones, row}, and start[number] = the first position
    const uint32_t *key = b.key[(passes + 1) & 1], *index = b.index[(passes + 1) & 1];
    uint32_t k[ITEMS], idx[ITEMS], heads[ITEMS];               // heads: where rows begin among the warp's 32 positions
    uint32_t my_heads, my_last, my_valid;                      // of the warp: rows that begin, 1 + the last such place, valid keys
    auto load_sorted = [&](uint32_t t0) {
        uint32_t prev[ITEMS];
#pragma unroll
        for (uint32_t j = 0; j < ITEMS; ++j) {
            const uint32_t i = t0 + mine + j * 32u;
            k[j] = prev[j] = 0xffffffffu;
            idx[j] = 0;
            if (i < hi) {
                if (one_tile) {
                    const uint2 *from = ranks > 1 ? s.incoming : s.sorted;
                    const uint2 x = from[i - lo];
                    k[j] = x.x;
                    idx[j] = x.y;
                    if (i > lo) prev[j] = from[i - lo - 1u].x;
                    else if (i) prev[j] = cluster.map_shared_rank(&s.incoming[share - 1u], me - 1u)->x;
                } else {
                    k[j] = key[i];
                    idx[j] = index[i];
                    if (i) prev[j] = key[i - 1];
                }
            }
        }
        my_heads = my_last = my_valid = 0;
#pragma unroll
        for (uint32_t j = 0; j < ITEMS; ++j) {
            heads[j] = __ballot_sync(0xffffffffu, k[j] < n_rows && prev[j] != k[j]);
            my_valid += __popc(__ballot_sync(0xffffffffu, k[j] < n_rows));
            my_heads += __popc(heads[j]);
            if (heads[j]) my_last = t0 + warp * (ITEMS * 32u) + j * 32u + 32u - __clz(heads[j]);
        }
    };
    if (threadIdx.x == 0) s.heads = s.valid = s.last_head = 0;
    __syncthreads();
    uint32_t sum_heads = 0, sum_valid = 0, max_last = 0;
    for (uint32_t t0 = lo; t0 < hi; t0 += kTileKeys) {
        load_sorted(t0);
        sum_heads += my_heads;
        sum_valid += my_valid;
        max_last = max(max_last, my_last);
    }
    if (lane == 0 && sum_valid) {
        atomicAdd(&s.heads, sum_heads);
        atomicAdd(&s.valid, sum_valid);
        atomicMax(&s.last_head, max_last);
    }
    __syncthreads();
    uint32_t before = 0, distinct = s.heads, valid = s.valid, last = 0;
    if (ranks > 1) {                                           // nothing is read from or written to another CTA after this
        if (threadIdx.x < ranks)
            *cluster.map_shared_rank(&s.rows_from[me], threadIdx.x) = make_uint4(s.heads, s.valid, s.last_head, 0u);
        cluster.sync();
        const uint4 x = lane < ranks ? s.rows_from[lane] : make_uint4(0u, 0u, 0u, 0u);
        distinct = __reduce_add_sync(0xffffffffu, x.x);
        valid = __reduce_add_sync(0xffffffffu, x.y);
        before = __reduce_add_sync(0xffffffffu, lane < me ? x.x : 0u);
        last = __reduce_max_sync(0xffffffffu, lane < me ? x.z : 0u);
    }
    for (uint32_t t0 = lo; t0 < hi; t0 += kTileKeys) {
        if (!one_tile) load_sorted(t0);
        if (lane == 0) {
            s.warp_heads[warp] = my_heads;
            s.warp_last[warp] = my_last;
        }
        __syncthreads();
        const uint32_t h = lane < kSortWarps ? s.warp_heads[lane] : 0u, p = lane < kSortWarps ? s.warp_last[lane] : 0u;
        uint32_t number = before + __reduce_add_sync(0xffffffffu, lane < warp ? h : 0u);
        uint32_t start = max(last, __reduce_max_sync(0xffffffffu, lane < warp ? p : 0u));
        before += __reduce_add_sync(0xffffffffu, h);
        last = max(last, __reduce_max_sync(0xffffffffu, p));
        __syncthreads();
#pragma unroll
        for (uint32_t j = 0; j < ITEMS; ++j) {
            const uint32_t i0 = t0 + warp * (ITEMS * 32u) + j * 32u, i = i0 + lane;
            const uint32_t upto = heads[j] & (0xffffffffu >> (31u - lane));            // rows that begin here or before
            const uint32_t my_number = number + __popc(upto) - 1u;
            const uint32_t my_start = upto ? i0 + 31u - __clz(upto) : start - 1u;
            if (k[j] < n_rows) {
                if (my_start == i) {
                    b.start[my_number] = i;
                    if (rows_out) rows_out[my_number] = (int64_t)k[j];
                }
                b.record[i] = make_uint4(idx[j], my_start, my_number, k[j]);
            }
            number += __popc(heads[j]);
            if (heads[j]) start = i0 + 32u - __clz(heads[j]);
        }
    }
    if (me == 0 && threadIdx.x == 0) {
        b.start[distinct] = valid;
        b.totals[0] = valid;
        b.totals[1] = distinct;
        if (count_out) *count_out = distinct;
    }
}

// ------------------------------------------------------------------------------------------------- sums

constexpr uint32_t kWindow = 8;        // sorted positions per warp (8192 tokens added / whole table of 65,536: 4 33.0 / 284 us, 8 33.9 / 266, 16 39.2 / 266)
constexpr uint32_t kSumWarps = 4;

// A lane holds PARTS vectors of 16 bytes of a row, a warp 512 * PARTS bytes of it: two for rows in general; one, and twice
// the rows in flight, for rows that fit (131,072 tokens of 64 columns: 72 us, 80 with two).
template <typename T, uint32_t PARTS> struct Tile {
    static constexpr uint32_t V = 16 / sizeof(T);                 // columns of a vector
    static constexpr uint32_t kCols = PARTS * 32 * V;             // columns per warp
    static constexpr uint32_t kStageRows = 8 / PARTS;             // rows per stage of the ring, which has two
};

// V columns of type T of which from .. to - 1 are there: the rest reads as zero and is not written.
template <typename T, uint32_t V>
__device__ __forceinline__ void load_cols(const T *p, uint32_t from, uint32_t to, float (&v)[V]) {
    constexpr uint32_t W = 16 / sizeof(T);                               // 16 bytes at a time
    if (V % W == 0 && to - from == V) {
#pragma unroll
        for (uint32_t i = 0; i + W <= V; i += W) {
            elem::Packed<T, (int)W> x;
            float y[W];
            elem::load_any<T, (int)W>(p + i, x);
            x.unpack(y);
#pragma unroll
            for (uint32_t j = 0; j < W; ++j) v[i + j] = y[j];
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < V; ++i) v[i] = i >= from && i < to ? elem::to_float(p[i]) : 0.f;
    }
}
template <typename T, uint32_t V>
__device__ __forceinline__ void store_cols(T *p, uint32_t from, uint32_t to, const float (&v)[V]) {
    constexpr uint32_t W = 16 / sizeof(T) < V ? 16 / sizeof(T) : V;
    const bool whole = to - from == V;
    if (V * sizeof(T) == 32 && whole && (reinterpret_cast<uintptr_t>(p) & 31u) == 0u) {         // whole sectors at once
        elem::Packed<T, (int)V> x;
        x.pack(v);
        elem::store_32_bytes(p, x.w);
    } else if (whole && (reinterpret_cast<uintptr_t>(p) & (W * sizeof(T) - 1u)) == 0u) {
#pragma unroll
        for (uint32_t i = 0; i < V; i += W) {
            elem::Packed<T, (int)W> x;
            float y[W];
#pragma unroll
            for (uint32_t j = 0; j < W; ++j) y[j] = v[i + j];
            x.pack(y);
            elem::store_aligned<elem::Packed<T, (int)W>::kWords>(p + i, x.w);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < V; ++i)
            if (i >= from && i < to) p[i] = elem::from_float<T>(v[i]);
    }
}

// Asynchronous copy of 16 bytes into shared memory, the last 16 - bytes of them zeros; both addresses 16-byte aligned.
template <int SHARED_OFFSET, int GLOBAL_OFFSET>
__device__ __forceinline__ void copy_async16(uint32_t shared, uint64_t global, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0+%3], [%1+%4], 16, %2;" ::"r"(shared), "l"(global), "r"(bytes), "n"(SHARED_OFFSET),
                 "n"(GLOBAL_OFFSET) : "memory");
}
// (x0, x1) += (y0, y1), each rounded as a 32-bit addition of its own
__device__ __forceinline__ void add2(float &x0, float &x1, float y0, float y1) {
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "+f"(x0), "+f"(x1) : "f"(y0), "f"(y1));
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

struct SumArgs {
    const void *grad_out;
    uint64_t grad_stride, dim;
    void *out;
    uint64_t out_stride;
    float scale;
    uint32_t tiles, tile_shift;
    uint64_t positions;    // records there are
    int64_t *rows;         // compact form: row numbers and how many rows there is room for
    uint64_t cap;
};

// Where the partial sum of a piece lies: at most two pieces of rows with several pieces begin in kPiece consecutive
// sorted positions, the last one of a row and the first one of the next.
__device__ __forceinline__ uint32_t slot_of(uint32_t piece_begin, bool first_of_row) {
    return 2u * (piece_begin / kPiece) + (first_of_row ? 1u : 0u);
}

// ALIGNED: every row of grad_out and of the output starts at a 16-byte boundary (16,384 rows of 4096 bf16 columns: 64 us;
// of 4095 columns, through the other instance: 83).  Otherwise a lane's columns are moved
// back to where the output row has one, so that stores stay whole vectors, and the input is staged in its own
// 16-byte pieces, from which a lane picks its bytes.
template <typename Tin, typename Tout, bool COMPACT, bool ADD, bool ALIGNED, uint32_t PARTS>
// Five CTAs per SM: the instances with two vectors of 16-bit columns a lane keep 16 bytes in local memory.  8192 tokens added /
// 16,384 compact / whole table of 65,536: four CTAs 35.0 / 57.0 / 278 us, five 33.9 / 58.5 / 266, six 41.9 / 62.0 / 274.
__global__ void __launch_bounds__(kSumWarps * 32, 5)
sum_rows_kernel(SumArgs a, SortBuffers b) {
    constexpr uint32_t V = Tile<Tin, PARTS>::V, kCols = Tile<Tin, PARTS>::kCols, kParts = PARTS, kStageRows = Tile<Tin, PARTS>::kStageRows;
    constexpr uint32_t kRowPieces = ALIGNED ? kParts * 32u : kParts * 32u + 4u;            // 16-byte pieces of a staged row
    __shared__ __align__(16) uint4 ring[kSumWarps][2][kStageRows][kRowPieces];
    // a CTA's warps take consecutive tiles of one window, or, where a row has fewer tiles, several windows
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint64_t unit = (uint64_t)blockIdx.x * kSumWarps + warp, window = unit >> a.tile_shift;
    const uint32_t tile = (blockIdx.y << a.tile_shift) + ((uint32_t)unit & ((1u << a.tile_shift) - 1u));
    if (tile >= a.tiles) return;
    wait_for_previous_kernel();
    const uint4 *records = b.record + window * kWindow + lane;
    uint4 ahead = make_uint4(0u, 0u, 0u, 0u);           // the first record, before it is known whether there is one
    if (window * kWindow + lane < a.positions) ahead = __ldcg(records);
    const uint32_t valid = __ldcg(b.totals);
    Tout *out = static_cast<Tout *>(a.out);

    // this lane's columns in part q: V from col(q), of which [from(q), to(q)) are there; back: how far they are moved
    constexpr uint32_t kUnit = V * sizeof(Tout) < 16u ? V * (uint32_t)sizeof(Tout) : 16u;  // bytes of an aligned store
    uint32_t back = 0;
    auto moved = [&](const Tout *row) { return ALIGNED ? 0u : ((uint32_t)reinterpret_cast<uintptr_t>(row) & (kUnit - 1u)) / (uint32_t)sizeof(Tout); };
    auto col = [&](uint32_t q) { return (int32_t)(tile * kCols + (q * 32u + lane) * V) - (int32_t)back; };
    auto from = [&](uint32_t q) { return !ALIGNED && col(q) < 0 ? (uint32_t)-col(q) : 0u; };
    auto to = [&](uint32_t q) {
        const int32_t left = (int32_t)a.dim - col(q);
        return left >= (int32_t)V ? V : left > 0 ? (uint32_t)left : 0u;
    };

    if (COMPACT) {                                      // what lies behind the last distinct row: number -1, gradient zero
        const float zero[V] = {};
        const uint64_t distinct = b.totals[1];
        for (uint64_t r = window * kWindow > distinct ? window * kWindow : distinct; r < (window + 1) * kWindow && r < a.cap; ++r) {
            if (tile == 0 && lane == 0) a.rows[r] = -1;
            Tout *o = out + r * a.out_stride;
            back = moved(o);
#pragma unroll
            for (uint32_t q = 0; q < kParts; ++q)
                if (to(q) > from(q)) store_cols<Tout, V>(o + col(q), from(q), to(q), zero);
        }
    }
    if (window * kWindow >= valid) return;
    const uint32_t w0 = (uint32_t)window * kWindow, w1 = valid - w0 < kWindow ? valid : w0 + kWindow;
    const Tin *g = static_cast<const Tin *>(a.grad_out);

    uint4 *stages = &ring[warp][0][0][0];
    float acc[kParts][V];
    bool open = false;                                  // a piece of ours is being added up
    uint32_t begin = 0, row_start = 0, row_number = 0, row = 0;

    auto write_row = [&](const float (&sum)[kParts][V]) {
        Tout *o = out + (uint64_t)(COMPACT ? row_number : row) * a.out_stride;
#pragma unroll
        for (uint32_t q = 0; q < kParts; ++q) {
            if (to(q) <= from(q)) continue;
            float v[V];
            if (ADD) {
                load_cols<Tout, V>(o + col(q), from(q), to(q), v);
#pragma unroll
                for (uint32_t i = 0; i < V; ++i) v[i] = fmaf(a.scale, sum[q][i], v[i]);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < V; ++i) v[i] = a.scale * sum[q][i];
            }
            store_cols<Tout, V>(o + col(q), from(q), to(q), v);
        }
    };
    auto partial = [&](uint32_t slot, uint32_t q) {
        return reinterpret_cast<float4 *>(b.partial + ((uint64_t)slot * a.tiles + tile) * kCols + (q * 32u + lane) * V);
    };
    auto put_partial = [&](uint32_t slot, const float (&v)[kParts][V]) {
#pragma unroll
        for (uint32_t q = 0; q < kParts; ++q)
#pragma unroll
            for (uint32_t i = 0; i < V; i += 4) __stcg(partial(slot, q) + i / 4, make_float4(v[q][i], v[q][i + 1], v[q][i + 2], v[q][i + 3]));
    };
    auto add_partials = [&](uint32_t first, uint32_t count, uint32_t step) {
#pragma unroll
        for (uint32_t q = 0; q < kParts; ++q)
#pragma unroll
            for (uint32_t i = 0; i < V; ++i) acc[q][i] = 0.f;
#pragma unroll 4
        for (uint32_t j = 0; j < count; ++j) {
            const uint32_t at = first + j * step, slot = slot_of(at, at == row_start);
#pragma unroll
            for (uint32_t q = 0; q < kParts; ++q)
#pragma unroll
                for (uint32_t i = 0; i < V; i += 4) {
                    const float4 x = __ldcg(partial(slot, q) + i / 4);
                    acc[q][i] += x.x; acc[q][i + 1] += x.y; acc[q][i + 2] += x.z; acc[q][i + 3] += x.w;
                }
        }
    };
    // true for the warp that arrives last of `members`; leaves the counter at zero for the next call
    auto arrive = [&](uint32_t *counter, uint32_t members) {
        __syncwarp();
        uint32_t last = 0;
        if (lane == 0) {
            last = arrive_add(counter, 1u) + 1u == members ? 1u : 0u;
            if (last) *counter = 0u;
        }
        last = __shfl_sync(0xffffffffu, last, 0);
        __syncwarp();
        return last != 0u;
    };
    auto counter = [&](uint32_t slot, uint32_t level) { return b.arrivals + ((uint64_t)slot * a.tiles + tile) * 2u + level; };
    // the open piece is complete; row_ends: and no further piece of its row follows
    auto flush = [&](bool row_ends) {
        if (begin != row_start || !row_ends) {
            const uint32_t terms = b.start[row_number + 1] - row_start;
            const uint32_t pieces = (terms + kPiece - 1) / kPiece, piece = (begin - row_start) / kPiece;
            const uint32_t group = piece / kGroup, groups = (pieces + kGroup - 1) / kGroup;
            const uint32_t first = row_start + group * (kGroup * kPiece);    // first position of the group
            const uint32_t members = pieces - group * kGroup < kGroup ? pieces - group * kGroup : kGroup;
            put_partial(slot_of(begin, begin == row_start), acc);
            if (!arrive(counter(slot_of(first, first == row_start), 0u), members)) return;
            add_partials(first, members, kPiece);
            if (groups > 1) {
                put_partial(slot_of(first, first == row_start), acc);
                if (!arrive(counter(slot_of(row_start, true), 1u), groups)) return;
                add_partials(row_start, groups, kGroup * kPiece);
            }
        }
        write_row(acc);
    };

    for (uint32_t i0 = w0;; i0 += 32u) {
        // 32 sorted positions, one per lane; behind the last one everything begins anew
        const uint32_t i = i0 + lane;
        uint4 rec = make_uint4(0u, i, 0u, 0u);
        if (i < valid) rec = i0 == w0 ? ahead : __ldcg(b.record + i);
        const uint32_t begins = __ballot_sync(0xffffffffu, (i - rec.y) % kPiece == 0u);
        const uint32_t row_begins = __ballot_sync(0xffffffffu, i == rec.y);
        // ours: from the first piece that begins in the window to the first that begins behind it
        uint32_t first = 0, last = 32u;
        if (!open) {
            first = begins ? __ffs(begins) - 1u : 32u;
            if (i0 + first >= w1) return;
        }
        const uint32_t inside = w1 > i0 ? w1 - i0 : 0u;
        const uint32_t behind = inside < 32u ? begins >> inside << inside : 0u;
        if (behind) last = __ffs(behind) - 1u;
        // rows j .. j + kStageRows - 1 of them into a stage of the ring
        const uint64_t my_row = reinterpret_cast<uint64_t>(g) + (uint64_t)rec.x * a.grad_stride * sizeof(Tin);
        auto fetch = [&](uint32_t j, uint32_t stage) {
            uint4 *dst = stages + stage * (kStageRows * kRowPieces) + lane;
            if (!ALIGNED) __syncwarp();                 // everybody has read what lies there
#pragma unroll
            for (uint32_t u = 0; u < kStageRows; ++u) {
                const uint64_t src = __shfl_sync(0xffffffffu, my_row, (j + u) & 31u);
                if (j + u < last) {
                    const uint32_t shared = tma::smem_u32(dst + u * kRowPieces);
                    if constexpr (ALIGNED) {
                        if (to(0)) copy_async16<0, 0>(shared, src + col(0) * (int32_t)sizeof(Tin), to(0) * (uint32_t)sizeof(Tin));
                        if (kParts > 1 && to(1)) copy_async16<512, 512>(shared, src + col(0) * (int32_t)sizeof(Tin), to(1) * (uint32_t)sizeof(Tin));
                    } else {
                        // pieces from the one before the tile's first on, as far as they hold something of the row
                        const uint64_t row_end = src + a.dim * sizeof(Tin);
                        const uint64_t piece = (src & ~15ull) + tile * (kParts * 512u) + lane * 16u - 16u;
                        if (piece + 16u > src && piece < row_end) copy_async16<0, 0>(shared, piece, 16u);
                        if (kParts > 1 && piece + 528u > src && piece + 512u < row_end) copy_async16<512, 512>(shared, piece, 16u);
                        if (lane < 4u && piece + kParts * 512u < row_end) copy_async16<kParts * 512, kParts * 512>(shared, piece, 16u);
                    }
                }
            }
            copy_commit();
        };
        uint32_t stage = 0;
        fetch(first, 0u);
        for (uint32_t j0 = first; j0 < last; j0 += kStageRows) {
            fetch(j0 + kStageRows, stage ^ 1u);
            copy_wait<1>();
            if (!ALIGNED) __syncwarp();                 // the other lanes' copies
            const uint4 *src = stages + stage * (kStageRows * kRowPieces) + lane;
            const uint32_t end = last < j0 + kStageRows ? last : j0 + kStageRows;
#pragma unroll 1
            for (uint32_t j = j0; j < end; ++j, src += kRowPieces) {
                if (begins >> j & 1u) {
                    if (open) flush(row_begins >> j & 1u);
                    open = true;
                    begin = i0 + j;
                    row_start = __shfl_sync(0xffffffffu, rec.y, j);
                    row_number = __shfl_sync(0xffffffffu, rec.z, j);
                    row = __shfl_sync(0xffffffffu, rec.w, j);
                    const Tout *o = out + (uint64_t)(COMPACT ? row_number : row) * a.out_stride;
                    back = moved(o);
                    if (ADD && begin == row_start) {    // the old row on its way while its terms are added up (36 us without)
#pragma unroll
                        for (uint32_t q = 0; q < kParts; ++q)
                            if (to(q) > from(q)) asm volatile("prefetch.global.L2 [%0];" ::"l"(o + col(q) + from(q)));
                    }
#pragma unroll
                    for (uint32_t q = 0; q < kParts; ++q)
#pragma unroll
                        for (uint32_t c = 0; c < V; ++c) acc[q][c] = 0.f;
                }
                // where this lane's first column lies behind the first staged piece
                uint32_t at = 0;
                if constexpr (!ALIGNED) at = (__shfl_sync(0xffffffffu, (uint32_t)my_row, j) & 15u) + 16u - back * (uint32_t)sizeof(Tin);
#pragma unroll
                for (uint32_t q = 0; q < kParts; ++q) {
                    elem::Packed<Tin, (int)V> c;
                    if constexpr (ALIGNED) {
                        const uint4 x = src[q * 32u];
                        c.w[0] = x.x; c.w[1] = x.y; c.w[2] = x.z; c.w[3] = x.w;
                    } else {
                        const uint4 x = src[q * 32u + (at >> 4)], y = src[q * 32u + (at >> 4) + 1u];
                        elem::Vector<Tin, (int)V, 0> both;
                        both.w[0] = x.x; both.w[1] = x.y; both.w[2] = x.z; both.w[3] = x.w;
                        both.w[4] = y.x; both.w[5] = y.y; both.w[6] = y.z; both.w[7] = y.w;
                        c = both.get(at & 15u);
                    }
                    float v[V];
                    c.unpack(v);
#pragma unroll
                    for (uint32_t k = 0; k < V; k += 2) add2(acc[q][k], acc[q][k + 1], v[k], v[k + 1]);
                }
            }
            stage ^= 1u;
        }
        copy_wait<0>();                                 // nothing but empty groups is left
        if (last < 32u) {
            flush(row_begins >> last & 1u);
            return;
        }
    }
}

uint32_t sort_passes(uint64_t n_rows) {
    uint32_t bits = 1;
    while (bits < 32 && (n_rows >> bits) != 0) ++bits;         // keys go up to n_rows itself
    return (bits + kDigitBits - 1) / kDigitBits;
}

template <typename Token, uint32_t ITEMS>
cudaError_t launch_sort(const EmbeddingGradArgs &a, const SortBuffers &b, uint32_t passes, uint32_t *d_status,
                        cudaStream_t stream) {
    static bool smem_done[kMaxDevices], cluster_done[kMaxDevices];
    cudaError_t e = ensure_dynamic_smem(sort_tokens_kernel<Token, ITEMS>, sizeof(SortShared), smem_done);
    if (e == cudaSuccess) e = ensure_large_clusters(sort_tokens_kernel<Token, ITEMS>, cluster_done);
    if (e != cudaSuccess) return e;
    uint32_t ranks = 1;
    while (ranks < kMaxCluster && (uint64_t)ranks * kSortThreads * ITEMS < a.n_tokens) ranks *= 2;
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
    return cudaLaunchKernelEx(&cfg, sort_tokens_kernel<Token, ITEMS>, static_cast<const Token *>(a.d_tokens), (uint32_t)a.n_tokens,
                              a.n_rows, a.padding_row, passes, b, a.d_rows, a.d_count, d_status);
}

template <typename Token>
cudaError_t launch_sort_sized(const EmbeddingGradArgs &a, const SortBuffers &b, uint32_t passes, uint32_t *d_status,
                              cudaStream_t stream) {
    // first all CTAs of a cluster, then more keys per thread: what a pass costs is the keys of ONE multiprocessor
    // (8192 tokens added: 33.8 us with sixteen CTAs of one key a thread, 42.0 with one CTA of sixteen)
    const uint64_t row = (uint64_t)kMaxCluster * kSortThreads;
    if (a.n_tokens <= row) return launch_sort<Token, 1>(a, b, passes, d_status, stream);
    if (a.n_tokens <= 2 * row) return launch_sort<Token, 2>(a, b, passes, d_status, stream);
    if (a.n_tokens <= 4 * row) return launch_sort<Token, 4>(a, b, passes, d_status, stream);
    if (a.n_tokens <= 8 * row) return launch_sort<Token, 8>(a, b, passes, d_status, stream);
    return launch_sort<Token, kMaxItems>(a, b, passes, d_status, stream);
}

template <typename Tin, typename Tout>
cudaError_t launch_sums(const EmbeddingGradArgs &a, const SortBuffers &b, cudaStream_t stream, uint64_t *launches) {
    SumArgs s;
    s.grad_out = a.d_grad_out;
    s.grad_stride = a.grad_stride;
    s.dim = a.dim;
    s.out = a.d_grad;
    s.out_stride = a.out_stride;
    s.scale = a.scale;
    s.rows = a.d_rows;
    s.cap = a.cap;
    s.positions = a.n_tokens;
    const uint64_t out_rows = a.d_rows ? a.cap : a.n_rows;
    const uintptr_t ends = reinterpret_cast<uintptr_t>(a.d_grad_out) | (a.n_tokens > 1 ? a.grad_stride * sizeof(Tin) : 0u) |
                           reinterpret_cast<uintptr_t>(a.d_grad) | (out_rows > 1 ? a.out_stride * sizeof(Tout) : 0u);
    const bool aligned = (ends & 15u) == 0u || a.dim == 0;                          // without columns no row is touched
    const uint64_t columns = a.dim + (aligned ? 0u : Tile<Tin, 1>::V);               // columns that are moved back need more room
    const bool narrow = columns <= Tile<Tin, 1>::kCols;
    s.tiles = narrow ? 1u : (uint32_t)((columns + Tile<Tin, 2>::kCols - 1) / Tile<Tin, 2>::kCols);   // without columns: the row numbers alone
    const uint64_t positions = a.n_tokens > a.cap ? a.n_tokens : a.cap;
    s.tile_shift = s.tiles >= 4u ? 2u : s.tiles >= 2u ? 1u : 0u;
    const uint64_t windows = (positions + kWindow - 1) / kWindow;
    const uint64_t blocks = ((windows << s.tile_shift) + kSumWarps - 1) / kSumWarps;
    const uint64_t groups = (s.tiles + (1u << s.tile_shift) - 1) >> s.tile_shift;
    if (blocks == 0) return cudaSuccess;
    if (blocks > 0x7fffffffull || groups > 65535u) return cudaErrorInvalidConfiguration;   // refused at the entry points
    ++*launches;
    const dim3 grid((uint32_t)blocks, (uint32_t)groups), block(kSumWarps * 32);
    auto launch = [&](auto kernel, bool overlapping) {
        if (overlapping) return launch_overlapping(kernel, grid, block, 0, stream, s, b);
        kernel<<<grid, block, 0, stream>>>(s, b);
        return cudaGetLastError();
    };
    auto pick = [&](auto compact, auto add, bool overlapping) {
        constexpr bool C = decltype(compact)::value, A = decltype(add)::value;
        if (narrow)
            return aligned ? launch(sum_rows_kernel<Tin, Tout, C, A, true, 1>, overlapping) : launch(sum_rows_kernel<Tin, Tout, C, A, false, 1>, overlapping);
        return aligned ? launch(sum_rows_kernel<Tin, Tout, C, A, true, 2>, overlapping) : launch(sum_rows_kernel<Tin, Tout, C, A, false, 2>, overlapping);
    };
    if (a.d_rows) return pick(std::true_type{}, std::false_type{}, true);
    if (a.accumulate) return pick(std::false_type{}, std::true_type{}, true);
    return pick(std::false_type{}, std::false_type{}, false);                            // the fill needs the SMs meanwhile
}

}  // namespace

// Scratch: a record for each sorted position, two key and two index arrays, start[n + 1], totals; then the arrival
// counters and the partial sums of rows with more than kPiece tokens.
namespace {
uint64_t round16(uint64_t x) { return (x + 15u) & ~15ull; }
uint64_t slot_count(uint64_t n) { return 2u * (n / kPiece + 1u); }
constexpr uint64_t kLeastCols = Tile<float, 2>::kCols, kMostCols = Tile<__half, 2>::kCols;
uint64_t tile_count(uint64_t dim) { return (dim + 8u + kLeastCols - 1) / kLeastCols; }
}  // namespace

uint64_t embedding_grad_sort_bytes(uint64_t n) { return 16u * (n + 1u) + 5u * round16(4u * (n + 1u)) + 64u; }
uint64_t embedding_grad_arrival_bytes(uint64_t n, uint64_t dim) { return round16(8u * slot_count(n) * tile_count(dim)); }
uint64_t embedding_grad_partial_bytes(uint64_t n, uint64_t dim) {
    return n <= kPiece ? 16u : 4u * slot_count(n) * ((dim + 8u + kMostCols - 1) / kMostCols * kMostCols);     // one piece at most: no partial sums
}

namespace {
SortBuffers sort_buffers(const EmbeddingGradArgs &a, const EmbeddingGradScratch &scratch) {
    const uint64_t array = round16(4u * (a.n_tokens + 1u));
    uint8_t *p = static_cast<uint8_t *>(scratch.d_sort);
    SortBuffers b;
    b.record = reinterpret_cast<uint4 *>(p);
    p += 16u * (a.n_tokens + 1u);
    b.key[0] = reinterpret_cast<uint32_t *>(p);
    b.key[1] = reinterpret_cast<uint32_t *>(p + array);
    b.index[0] = reinterpret_cast<uint32_t *>(p + 2 * array);
    b.index[1] = reinterpret_cast<uint32_t *>(p + 3 * array);
    b.start = reinterpret_cast<uint32_t *>(p + 4 * array);
    b.totals = reinterpret_cast<uint32_t *>(p + 5 * array);
    b.arrivals = scratch.d_arrivals;
    b.partial = scratch.d_partial;
    return b;
}

template <typename Token>
cudaError_t launch_fill(const EmbeddingGradArgs &a, int sm_count, cudaStream_t stream) {
    const uint64_t size = a.out_type == IV_F32 ? 4u : 2u;
    const uint32_t grid = (uint32_t)(sm_count > 2 * (int)kMaxCluster ? sm_count - (int)kMaxCluster : sm_count);   // the SMs the sort leaves
    fill_rows_kernel<Token><<<grid, kFillThreads, 0, stream>>>(static_cast<const Token *>(a.d_tokens), (uint32_t)a.n_tokens, a.n_rows,
                                                               a.padding_row, static_cast<uint8_t *>(a.d_grad), a.dim * size,
                                                               a.out_stride * size);
    return cudaGetLastError();
}
}  // namespace

cudaError_t launch_embedding_grad_sort(const EmbeddingGradArgs &a, const EmbeddingGradScratch &scratch, uint32_t *d_status,
                                       cudaStream_t stream, uint64_t *launches) {
    const SortBuffers b = sort_buffers(a, scratch);
    const uint32_t passes = sort_passes(a.n_rows);
    ++*launches;
    return a.token_bytes == 4 ? launch_sort_sized<int32_t>(a, b, passes, d_status, stream)
                              : launch_sort_sized<int64_t>(a, b, passes, d_status, stream);
}

cudaError_t launch_embedding_grad_fill(const EmbeddingGradArgs &a, int sm_count, cudaStream_t stream, uint64_t *launches) {
    ++*launches;
    return a.token_bytes == 4 ? launch_fill<int32_t>(a, sm_count, stream) : launch_fill<int64_t>(a, sm_count, stream);
}

cudaError_t launch_embedding_grad_sums(const EmbeddingGradArgs &a, const EmbeddingGradScratch &scratch, cudaStream_t stream,
                                       uint64_t *launches) {
    const SortBuffers b = sort_buffers(a, scratch);
    return by_types(a.grad_type, a.out_type, [&](auto in, auto out) {
        return launch_sums<typename decltype(in)::type, typename decltype(out)::type>(a, b, stream, launches);
    });
}

}  // namespace ivk
