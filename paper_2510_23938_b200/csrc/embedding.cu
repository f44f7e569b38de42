// Embedding lookup with scaling: out[t, :] = round(scale * table[token[t], :]), the product in 32 bits, rounded once.
//
// A gather of rows: what bounds it is memory (the distinct rows read once, every output row written once), for a few
// tokens the latency of the chain token -> row -> store.  A warp takes one tile of kTile columns of one token, so that
// a single token's row is spread over several warps and every lane has four vector loads in flight; rows of few
// columns are taken by a half or a quarter of a warp (65,536 rows of 64 columns: 7 us, 13 with whole warps).
//
// On one B200, the kernel alone: 131,072 rows of 4096 bf16 columns 232 us, 5.8 TB/s of what has to move; the memory itself
// runs at 6.4 TB/s, because the stream of output rows pushes table rows out of the L2 cache that are wanted again (468 MB read
// for 270 MB of distinct rows; hints to keep them cost more than they saved).  8192 rows out of a weight file, 8 bytes
// off a 16-byte boundary: 16 us, 6.2 TB/s (20.5 us from one pass to the next).  One row: 3.6 us.
#include "element_dev.cuh"
#include "iv_internal.h"

namespace ivk {

namespace {

constexpr uint32_t kTile = 1024;      // columns per warp: 4 vectors of 8 (16-bit types) or 8 of 4 (32-bit) per lane
constexpr uint32_t kWarps = 8;

// ALIGN: every row of the output starts at a 16-byte boundary and every row of the table at one of ALIGN (16 or 8) bytes;
// 0: anywhere.  65,536 rows of 4096 bf16 columns take 117 us at 16, 119 at 8, and 136 and 141 through the instance for
// any alignment.
template <typename Tin, typename Tout, typename Token, int ALIGN>
__global__ void __launch_bounds__(kWarps * 32, ALIGN ? 6 : 8)
embedding_kernel(const Tin *table, uint64_t n_rows, uint64_t dim, uint64_t row_stride, const Token *tokens, uint64_t n_tokens,
                 float scale, Tout *out, uint64_t out_stride, uint32_t tiles, uint32_t lanes, uint32_t *status) {
    const uint32_t lane = threadIdx.x & (lanes - 1u), teams = kWarps * 32u / lanes;
    const uint64_t units = n_tokens * tiles;
    for (uint64_t unit = (uint64_t)blockIdx.x * teams + threadIdx.x / lanes; unit < units; unit += (uint64_t)gridDim.x * teams) {
        uint64_t t = unit, c0 = 0;
        if (tiles > 1u) {
            t = unit / tiles;
            c0 = (unit - t * tiles) * kTile;
        }
        const uint32_t cols = (uint32_t)(dim - c0 < kTile ? dim - c0 : kTile);
        const uint64_t row = (uint64_t)(int64_t)tokens[t];       // a negative token becomes a large number
        Tout *o = out + t * out_stride + c0;
        if (row < n_rows) {
            const Tin *in = table + row * row_stride + c0;
            auto scaled = [scale](float x) { return x * scale; };
            if constexpr (ALIGN != 0) elem::map_aligned<Tin, Tout, ALIGN>(in, o, cols, lane, lanes, scaled);
            else elem::map_any<Tin, Tout, false>(in, o, cols, lane, lanes, scaled);
        } else {
            for (uint32_t i = lane; i < cols; i += lanes) o[i] = elem::from_float<Tout>(0.f);
            if (lane == 0 && c0 == 0) atomicMax(status, (uint32_t)IVK_DEV_BOUNDS);
        }
    }
}

template <typename Tin, typename Tout, typename Token, int ALIGN>
cudaError_t launch_instance(const EmbeddingArgs &a, uint32_t *d_status, cudaStream_t stream) {
    const uint32_t tiles = (uint32_t)((a.dim + kTile - 1) / kTile);
    const uint64_t vectors = a.dim / elem::MapShape<Tin, Tout>::V;
    const uint32_t lanes = vectors <= 8u ? 8u : vectors <= 16u ? 16u : 32u;      // at least 8: single elements at a row's ends
    const uint32_t teams = kWarps * 32u / lanes;
    const uint64_t blocks = (a.n_tokens * tiles + teams - 1) / teams;
    const uint32_t grid = (uint32_t)(blocks < (1u << 30) ? blocks : (1u << 30));
    embedding_kernel<Tin, Tout, Token, ALIGN><<<grid, kWarps * 32, 0, stream>>>(
        static_cast<const Tin *>(a.d_table), a.n_rows, a.dim, a.row_stride, static_cast<const Token *>(a.d_tokens), a.n_tokens,
        a.scale, static_cast<Tout *>(a.d_out), a.out_stride, tiles, lanes, d_status);
    return cudaGetLastError();
}

template <typename Tin, typename Tout, typename Token>
cudaError_t launch_typed(const EmbeddingArgs &a, uint32_t *d_status, cudaStream_t stream) {
    const uintptr_t table = reinterpret_cast<uintptr_t>(a.d_table) | (a.n_rows > 1 ? a.row_stride * sizeof(Tin) : 0u);
    const uintptr_t out = reinterpret_cast<uintptr_t>(a.d_out) | (a.n_tokens > 1 ? a.out_stride * sizeof(Tout) : 0u);
    if ((out & 15u) || (table & 7u)) return launch_instance<Tin, Tout, Token, 0>(a, d_status, stream);
    return table & 15u ? launch_instance<Tin, Tout, Token, 8>(a, d_status, stream)
                       : launch_instance<Tin, Tout, Token, 16>(a, d_status, stream);
}

template <typename Tin, typename Tout>
cudaError_t launch_token(const EmbeddingArgs &a, uint32_t *d_status, cudaStream_t stream) {
    return a.token_bytes == 4 ? launch_typed<Tin, Tout, int32_t>(a, d_status, stream)
                              : launch_typed<Tin, Tout, int64_t>(a, d_status, stream);
}

}  // namespace

cudaError_t launch_embedding(const EmbeddingArgs &a, uint32_t *d_status, cudaStream_t stream, uint64_t *launches) {
    if (a.n_tokens == 0 || a.dim == 0) return cudaSuccess;
    ++*launches;
    return by_types(a.table_type, a.out_type, [&](auto in, auto out) {
        return launch_token<typename decltype(in)::type, typename decltype(out)::type>(a, d_status, stream);
    });
}

}  // namespace ivk
