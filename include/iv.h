/*
 * iv.h -- C ABI of libiv: GPU-resident integrity verification of model-weight
 * bytes on NVIDIA B200 (sm_100a).
 *
 * The library computes, entirely in CUDA kernels, the data-parallel path of the
 * paper "Scalable GPU-Based Integrity Verification for Large Machine Learning
 * Models": FIPS 180-4 SHA-256 digests of fixed-size chunks of a byte blob, a
 * binary Merkle reduction of those digests to a root, and the comparison of
 * digests and root with an expected manifest (Algorithm 1, "Streaming Model
 * Verification", and the section "Memory Scalability Considerations").
 *
 * Conventions
 *  - Pointers named d_* are DEVICE pointers owned by the caller; the library
 *    neither frees nor keeps them beyond the work it enqueues.  Pointers named
 *    h_* are HOST pointers.  Everything else is passed by value.
 *  - A digest is 32 bytes: the eight 32-bit words H0..H7 of FIPS 180-4
 *    section 6.2.2, each stored big-endian.  Digest arrays are contiguous
 *    records in index order.
 *  - Every call enqueues its GPU work on `cuda_stream` (a cudaStream_t passed
 *    as void*, NULL = the legacy default stream) and returns without waiting,
 *    except where stated.  Results in device memory are valid once the stream
 *    has reached that point.
 *  - Return value: IV_OK (0) or a negative iv_status.  Finding a mismatch is
 *    NOT an error: verification calls return IV_OK and report it in the result.
 *  - There is no CPU fallback: without a usable CUDA device iv_create fails.
 *  - A context may be used by one host thread at a time.  Calls on the same
 *    context that overlap on the GPU (different streams) share its scratch
 *    memory and therefore race; serialise them or use one context per stream.
 */
#ifndef IV_H
#define IV_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum iv_status {
    IV_OK = 0,
    IV_ERR_INVALID_ARG = -1, /* null pointer, zero chunk size, capacity too small, inconsistent manifest */
    IV_ERR_NOMEM = -2,       /* a device or host allocation for scratch failed */
    IV_ERR_CUDA = -3,        /* a CUDA runtime call failed; see iv_last_cuda_error */
    IV_ERR_NO_DEVICE = -4,   /* no CUDA device, or not a compute-capability-10.x device */
    IV_ERR_TOO_LARGE = -5    /* the size exceeds a fixed limit of the entry point (iv_merkle_root_noalloc) */
} iv_status;

/* Opaque context.  Owns scratch memory (Merkle level buffers, tickets, the
 * digest array used by verification, streaming windows), sized lazily. */
typedef struct iv_ctx iv_ctx;

/* Creates a context on CUDA device `cuda_device`.  Synchronous.  *out is set
 * to NULL on failure. */
int iv_create(iv_ctx **out, int cuda_device);

/* Waits for the device, frees all scratch, destroys the context.  NULL is allowed. */
int iv_destroy(iv_ctx *ctx);

/* Static, human-readable text for a status code. */
const char *iv_strerror(int code);

/* The cudaError_t (as int) of the last failed CUDA call on this context, 0 if none. */
int iv_last_cuda_error(const iv_ctx *ctx);

/* Device-side status of the kernels this context has run: 0 = all completed,
 * 1 = a kernel gave up on a bounded wait for a bulk copy (its outputs are then
 * invalid), 2 = an index check failed.  Waits for the device (synchronous),
 * writes the word to *h_status and clears it.  Verification calls also copy it
 * into iv_verify_result::status. */
int iv_device_status(iv_ctx *ctx, uint32_t *h_status);

/* Number of kernels this context has launched so far (a host-side counter). */
uint64_t iv_kernel_launches(const iv_ctx *ctx);

/* Name of the leaf-hashing kernel the last hashing or verification call on this context launched
 * (the library picks one of several by chain count, chunk size and alignment); "" before any call.
 * Static text, never freed. */
const char *iv_last_leaf_kernel(const iv_ctx *ctx);

/* Where that kernel has several launch shapes (the many-chain kernel: workers per SM; the SHA-384/512
 * two-warp kernel: pairs per SM), the one the last call ran in; "" otherwise.  Static text. */
const char *iv_last_leaf_instance(const iv_ctx *ctx);

/* Self-test of the bounded waits (a diagnostic; the paper has no counterpart).  Every wait inside the
 * library's kernels -- for a bulk copy, for a hand-over between warps -- gives up after a fixed number of
 * SM clocks (about two seconds), sets the device status to 1 and lets the kernel return, so that a lost
 * copy can never hang the GPU.  This call runs that path on purpose: one warp waits, with the same wait
 * routine and a limit of limit_cycles SM clocks (1 .. 4e9), on a barrier that nobody arrives at, gives
 * up, sets the status word and returns.  Afterwards iv_device_status reports 1 (and clears it), and the
 * context works as before.
 *   h_waited_cycles   optional host pointer; when given, the call waits for the stream and stores the
 *                     SM clocks the warp spent waiting (>= limit_cycles) */
int iv_selftest_wait_timeout(iv_ctx *ctx, uint64_t limit_cycles, uint64_t *h_waited_cycles, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Leaf hashing -- Algorithm 1, "chunk_count <- ceil(|M| / C)" and
 * "H_i = GPU_HASH(M_i)" with GPU_HASH = SHA-256 (FIPS 180-4 section 6.2).
 *
 *   d_data        nbytes bytes of device memory, any alignment
 *   chunk_bytes   C > 0; chunk i covers bytes [i*C, min((i+1)*C, nbytes)); the
 *                 last chunk is hashed at its true length (no zero fill)
 *   d_digests     receives n = ceil(nbytes / C) records of 32 bytes
 *   digests_cap   capacity of d_digests in records; n > digests_cap is an error
 *   h_n_chunks    optional host pointer, receives n (written before returning)
 *
 * nbytes == 0 gives n == 0 and launches nothing.  Streaming (the loop of
 * Algorithm 1) needs no other entry point: call once per resident window,
 * each window a multiple of C except the last, with d_digests advanced by
 * 32 * (chunks before the window).
 */
int iv_hash_chunks(iv_ctx *ctx, const void *d_data, uint64_t nbytes, uint64_t chunk_bytes,
                   uint8_t *d_digests, uint64_t digests_cap, uint64_t *h_n_chunks,
                   void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Merkle reduction -- Algorithm 1, "Construct Merkle tree from leaf_hashes
 * using GPU".  Binary tree over n_leaves digests in index order; a parent is
 * SHA-256(left || right) of exactly 64 bytes (no domain-separation prefix); an
 * unpaired last node of a level moves up unchanged; one leaf is its own root;
 * zero leaves give SHA-256 of the empty string.
 *
 *   d_leaves   n_leaves * 32 bytes (may be NULL when n_leaves == 0)
 *   d_root     receives 32 bytes
 */
int iv_merkle_root(iv_ctx *ctx, const uint8_t *d_leaves, uint64_t n_leaves, uint8_t *d_root,
                   void *cuda_stream);

/* `levels` levels of the same reduction without going all the way to the root:
 * d_nodes[n] -> d_out[n_out], n_out = n halved (rounding up) `levels` times.  Node j
 * of the result is the root of the aligned run of 2^levels inputs starting at
 * j * 2^levels, which is also a node of the whole tree -- the building block for
 * the paper's multi-GPU scheme (section "Multi-GPU Deployment Architectures",
 * a global tree built from the hashes computed on each device): every GPU
 * reduces its aligned range of leaves to such nodes, the nodes are gathered, and
 * iv_merkle_root over them gives the global root.
 *   d_out, out_cap   receives n_out records; out_cap (in records) must be >= n_out;
 *                    must not overlap d_nodes
 *   h_n_out          optional host pointer, receives n_out
 */
int iv_merkle_levels(iv_ctx *ctx, const uint8_t *d_nodes, uint64_t n, uint32_t levels,
                     uint8_t *d_out, uint64_t out_cap, uint64_t *h_n_out, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Incremental re-verification -- the paper's hierarchical / differential
 * verification (section "Version Management and Incremental Verification": when fine-tuning
 * or an update touches some chunks, only those leaves and their paths to the
 * root are recomputed).
 *
 * A retained tree holds every level of the tree over n leaves in one device
 * array of iv_tree_records(n) records of 32 bytes: the n leaves first, then
 * ceil(n/2) parents, and so on; the LAST record is the root (for n == 0 the
 * single record is SHA-256 of the empty string).  d_tree must be 16-byte aligned.
 *
 * iv_tree_build   fills the array from n leaf digests (d_leaves 16-byte aligned).
 * iv_tree_update  re-hashes the chunks listed in d_dirty (n_dirty uint64 chunk
 *                 indices in DEVICE memory, any order, repeats allowed, each
 *                 < ceil(nbytes / chunk_bytes)) from the current bytes of d_data,
 *                 stores their digests in the leaf level and recomputes only the
 *                 ancestors of those leaves.  Work is n_dirty chunk hashes plus
 *                 n_dirty * ceil(log2 n) node hashes.  An index outside the tree
 *                 is skipped and sets the device status to 2 (iv_device_status).
 */
uint64_t iv_tree_records(uint64_t n_leaves);
int iv_tree_build(iv_ctx *ctx, const uint8_t *d_leaves, uint64_t n_leaves, uint8_t *d_tree,
                  uint64_t tree_cap, void *cuda_stream);
int iv_tree_update(iv_ctx *ctx, const void *d_data, uint64_t nbytes, uint64_t chunk_bytes,
                   const uint64_t *d_dirty, uint64_t n_dirty, uint8_t *d_tree, uint64_t tree_cap,
                   void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Verification -- Algorithm 1, "Compare root hash with expected value", plus
 * the per-chunk comparison that locates the damage.
 *
 * The manifest is the publisher's expected value: the blob's size, the chunk
 * size, the chunk digests and their Merkle root.
 */
typedef struct iv_manifest {
    uint64_t total_bytes;     /* must equal nbytes of the call */
    uint64_t chunk_bytes;     /* C */
    uint64_t n_chunks;        /* must equal ceil(total_bytes / chunk_bytes) */
    const uint8_t *d_digests; /* DEVICE: n_chunks * 32 bytes (may be NULL when n_chunks == 0) */
    uint8_t root[32];         /* expected Merkle root (host bytes inside this struct) */
} iv_manifest;

/* Written by the GPU into DEVICE memory supplied by the caller. */
typedef struct iv_verify_result {
    uint32_t status;     /* device-side status: 0 = completed */
    uint32_t root_ok;    /* 1 iff the recomputed root equals manifest root */
    uint64_t n_mismatch; /* exact number of chunks whose digest differs, even if > idx_cap */
    uint8_t root[32];    /* the recomputed root */
} iv_verify_result;

/*   d_data, nbytes    the blob to verify (device)
 *   h_manifest        host struct (read before returning), digests on the device
 *   d_result          device memory for one iv_verify_result
 *   d_mismatch_idx    device array of idx_cap uint64: the indices of mismatching
 *                     chunks in ASCENDING order, the first min(n_mismatch, idx_cap)
 *                     of them; may be NULL when idx_cap == 0
 * The recomputed chunk digests stay in the context (iv_ctx_digests). */
int iv_verify_manifest(iv_ctx *ctx, const void *d_data, uint64_t nbytes,
                       const iv_manifest *h_manifest, iv_verify_result *d_result,
                       uint64_t *d_mismatch_idx, uint64_t idx_cap, void *cuda_stream);

/* Batch verification -- the paper's batch processing (section "Scalability Analysis"): n_blobs blobs of
 * the same size (copies, replicas, variants that share a manifest) are verified against ONE manifest in
 * one pass; all their chunks are independent chains of a single hashing launch, which is what fills the
 * GPU when one blob alone has few chunks.
 *   h_d_blobs        HOST array of n_blobs DEVICE pointers (read before returning), at most 64
 *   d_results        DEVICE array of n_blobs iv_verify_result, one per blob
 *   d_mismatch_idx   DEVICE array of n_blobs * idx_cap uint64: blob b's ascending list starts at b * idx_cap
 * Everything else as for iv_verify_manifest. */
int iv_verify_manifest_batch(iv_ctx *ctx, const void *const *h_d_blobs, uint64_t n_blobs, uint64_t nbytes,
                             const iv_manifest *h_manifest, iv_verify_result *d_results,
                             uint64_t *d_mismatch_idx, uint64_t idx_cap, void *cuda_stream);

/* Device pointer of the digest array the last iv_verify_manifest /
 * iv_verify_streamed on this context wrote (n_chunks * 32 bytes), NULL if none. */
const uint8_t *iv_ctx_digests(const iv_ctx *ctx);

/* ---------------------------------------------------------------------------
 * Two-level leaves -- a SEPARATELY NAMED mode whose digests differ from
 * iv_hash_chunks (the paper's hierarchical verification at several
 * granularities).  The digest of chunk i is the Merkle root (this library's tree
 * rule) over the SHA-256 digests of its sub_bytes-sized pieces:
 *     D_i = root( SHA-256(piece_0), SHA-256(piece_1), ... )   pieces of chunk i.
 * A chunk is then no longer one serial SHA-256 chain but chunk_bytes/sub_bytes
 * independent ones, which is what fills a GPU when a blob has few large chunks.
 * chunk_bytes must be sub_bytes times a power of two (else IV_ERR_INVALID_ARG);
 * with that, the root over the D_i equals the root over all pieces' digests, so
 * a manifest at chunk granularity and one at piece granularity share one root.
 * sub_bytes == chunk_bytes gives iv_hash_chunks / iv_verify_manifest exactly.
 * Other arguments as for iv_hash_chunks / iv_verify_manifest; the manifest's
 * digests and root must have been made in the same mode.
 */
int iv_hash_chunks_two_level(iv_ctx *ctx, const void *d_data, uint64_t nbytes, uint64_t chunk_bytes,
                             uint64_t sub_bytes, uint8_t *d_digests, uint64_t digests_cap,
                             uint64_t *h_n_chunks, void *cuda_stream);
int iv_verify_manifest_two_level(iv_ctx *ctx, const void *d_data, uint64_t nbytes,
                                 const iv_manifest *h_manifest, uint64_t sub_bytes,
                                 iv_verify_result *d_result, uint64_t *d_mismatch_idx,
                                 uint64_t idx_cap, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Streamed verification -- the whole of Algorithm 1 for a blob that lives in
 * HOST memory ("Load model chunk M_i into GPU memory ... Free GPU memory"):
 * the blob is copied window by window into two device windows owned by the
 * context, the copy of window w+1 overlapping the hashing of window w on a
 * second stream, then the tree is built and compared as in iv_verify_manifest.
 * A window with few large chunks is copied and hashed in column parts (part s of
 * every chunk while part s+1 is in flight), so that its hashing ends shortly
 * after its last byte arrives; the results are the same.
 *
 *   h_windows      host array of n_windows HOST pointers; window w holds bytes
 *                  [w*window_bytes, min((w+1)*window_bytes, nbytes)) of the blob.
 *                  The windows need not be adjacent in memory (file shards,
 *                  mapped pieces) and may repeat.  Page-locked memory is needed
 *                  for the copies to overlap (pageable memory works, slowly).
 *   n_windows      must equal ceil(nbytes / window_bytes)
 *   window_bytes   > 0, a multiple of h_manifest->chunk_bytes
 * The pointer array is read before the call returns; the window contents must
 * stay valid until the enqueued copies have run.  The call returns when all
 * work is ENQUEUED on cuda_stream and the context's copy stream; cuda_stream
 * reaches completion only after both are done.
 */
int iv_verify_streamed(iv_ctx *ctx, const void *const *h_windows, uint64_t n_windows,
                       uint64_t window_bytes, uint64_t nbytes, const iv_manifest *h_manifest,
                       iv_verify_result *d_result, uint64_t *d_mismatch_idx, uint64_t idx_cap,
                       void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Phase timing (the paper's result record carries a verification time).  When
 * switched on, iv_verify_manifest and iv_verify_streamed bracket their three
 * phases -- leaf hashing, tree reduction, comparison -- with CUDA events on
 * cuda_stream.  The context keeps the events of the most recent
 * IV_TIMING_RING verification calls.  Independently of this switch the three
 * phases are NVTX ranges ("iv: leaf hashing", "iv: Merkle reduction",
 * "iv: manifest compare") around the launches of each phase, for profilers.
 *
 * iv_phase_times waits for the events of the call made `calls_back` calls ago
 * (0 = the most recent) and writes the three durations in milliseconds to
 * h_ms[0..2].  Returns IV_ERR_INVALID_ARG if timing was off for that call or
 * calls_back >= IV_TIMING_RING.
 */
#define IV_TIMING_RING 64
int iv_set_timing(iv_ctx *ctx, int enabled);
int iv_phase_times(iv_ctx *ctx, uint32_t calls_back, float *h_ms);

/* ---------------------------------------------------------------------------
 * Per-tensor digests -- the paper's batch verification (section "Scalability
 * Analysis": many payloads per launch, one digest per payload): digest k =
 * SHA-256(d_base[offset_k .. offset_k + length_k)).
 *
 *   d_offsets, d_lengths   n uint64 each, DEVICE memory; any byte alignment of
 *                          offsets, any length including 0
 *   d_digests              receives n * 32 bytes
 * The caller guarantees that every range lies inside the d_base allocation.
 */
int iv_hash_ragged(iv_ctx *ctx, const void *d_base, const uint64_t *d_offsets,
                   const uint64_t *d_lengths, uint64_t n, uint8_t *d_digests,
                   void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Resumable per-tensor digests -- the paper's multi-pass processing (section
 * "Memory Scalability Considerations", the hash state carried from pass to pass): a tensor
 * that is larger than a resident window, or that spans two windows, is hashed
 * part by part.
 *
 * d_states holds one iv_sha_state per tensor in DEVICE memory, zero-filled by
 * the caller before a tensor's first part.  Each call hashes, for every k, the
 * next length_k bytes of tensor k found at d_base + offset_k and advances state
 * k.  With finish == 0 every length must be a multiple of 64 bytes (a remainder
 * is left unhashed and the device status is set to 2); the call with finish != 0
 * takes the last part (any length, 0 allowed), applies the padding for the
 * TOTAL length and writes digest k to d_digests + 32 k (d_digests may be NULL
 * when finish == 0).  At most 32,768 tensors per call (IV_ERR_TOO_LARGE beyond).
 */
typedef struct iv_sha_state {
    uint32_t h[8];     /* chaining value after the bytes hashed so far */
    uint64_t bytes;    /* bytes hashed so far (0 = fresh) */
    uint64_t reserved; /* keeps the record at 48 bytes */
} iv_sha_state;

int iv_hash_ragged_update(iv_ctx *ctx, const void *d_base, const uint64_t *d_offsets,
                          const uint64_t *d_lengths, uint64_t n, iv_sha_state *d_states,
                          int finish, uint8_t *d_digests, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * SHA-384 and SHA-512 variants -- SHA-384 is the digest of the paper's own kernel
 * listings (FIPS 180-4 section 6.5).  Chunking and tree rule as above with 48-byte records: digest i
 * = SHA-384(chunk i); parent = SHA-384(left || right) over exactly 96 bytes, an
 * unpaired last node moves up unchanged, one leaf is its own root, zero leaves
 * give SHA-384 of the empty string.  The SHA-512 entry points (FIPS 180-4 section
 * 6.4, initial value of section 5.3.5, no truncation) are the same with 64-byte
 * records and SHA-512(left || right) over exactly 128 bytes as the parent.
 * 16-byte aligned blobs with up to about 131,000 chunks of 16 KiB or more (a
 * multiple of 16 bytes) run through a kernel in the design of the SHA-256 path
 * (tiled bulk copies, the compression split between two warps, chains migrating
 * between workers); other shapes through a plain one-chain-per-lane kernel,
 * which is the faster one when chains are plentiful.
 */
int iv_hash_chunks_sha384(iv_ctx *ctx, const void *d_data, uint64_t nbytes, uint64_t chunk_bytes,
                          uint8_t *d_digests, uint64_t digests_cap, uint64_t *h_n_chunks,
                          void *cuda_stream);
int iv_merkle_root_sha384(iv_ctx *ctx, const uint8_t *d_leaves, uint64_t n_leaves, uint8_t *d_root,
                          void *cuda_stream);

int iv_hash_chunks_sha512(iv_ctx *ctx, const void *d_data, uint64_t nbytes, uint64_t chunk_bytes,
                          uint8_t *d_digests, uint64_t digests_cap, uint64_t *h_n_chunks,
                          void *cuda_stream);
int iv_merkle_root_sha512(iv_ctx *ctx, const uint8_t *d_leaves, uint64_t n_leaves, uint8_t *d_root,
                          void *cuda_stream);

/* iv_verify_manifest for the SHA-384 variant: the same steps over 48-byte records.  The manifest holds the
 * SHA-384 chunk digests (device) and the root of the SHA-384 tree; fields, index list, errors and
 * asynchrony as for iv_manifest / iv_verify_result / iv_verify_manifest. */
typedef struct iv_manifest_sha384 {
    uint64_t total_bytes;
    uint64_t chunk_bytes;
    uint64_t n_chunks;
    const uint8_t *d_digests; /* DEVICE: n_chunks * 48 bytes */
    uint8_t root[48];
} iv_manifest_sha384;
typedef struct iv_verify_result_sha384 {
    uint32_t status;
    uint32_t root_ok;
    uint64_t n_mismatch;
    uint8_t root[48];
} iv_verify_result_sha384;
int iv_verify_manifest_sha384(iv_ctx *ctx, const void *d_data, uint64_t nbytes,
                              const iv_manifest_sha384 *h_manifest, iv_verify_result_sha384 *d_result,
                              uint64_t *d_mismatch_idx, uint64_t idx_cap, void *cuda_stream);

/* The same for SHA-512: 64-byte records. */
typedef struct iv_manifest_sha512 {
    uint64_t total_bytes;
    uint64_t chunk_bytes;
    uint64_t n_chunks;
    const uint8_t *d_digests; /* DEVICE: n_chunks * 64 bytes */
    uint8_t root[64];
} iv_manifest_sha512;
typedef struct iv_verify_result_sha512 {
    uint32_t status;
    uint32_t root_ok;
    uint64_t n_mismatch;
    uint8_t root[64];
} iv_verify_result_sha512;
int iv_verify_manifest_sha512(iv_ctx *ctx, const void *d_data, uint64_t nbytes,
                              const iv_manifest_sha512 *h_manifest, iv_verify_result_sha512 *d_result,
                              uint64_t *d_mismatch_idx, uint64_t idx_cap, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * RFC 6962 section 2.1 mode -- the Merkle Tree Hash the paper cites for its tree,
 * with that RFC's domain separation, over SHA-256 with the chunks as entries:
 * leaf hash i = SHA-256(0x00 || chunk i); node = SHA-256(0x01 || left || right)
 * (65 bytes); the list is split at the largest power of two below n, one entry
 * is its own leaf hash, no entry gives SHA-256 of the empty string.  Digests
 * and root differ from the default (unprefixed) path by construction.
 * Arguments, layout and errors as iv_hash_chunks / iv_merkle_root.
 */
int iv_hash_chunks_rfc6962(iv_ctx *ctx, const void *d_data, uint64_t nbytes, uint64_t chunk_bytes,
                           uint8_t *d_digests, uint64_t digests_cap, uint64_t *h_n_chunks,
                           void *cuda_stream);
int iv_merkle_root_rfc6962(iv_ctx *ctx, const uint8_t *d_leaves, uint64_t n_leaves, uint8_t *d_root,
                           void *cuda_stream);
/* iv_verify_manifest in this mode: the manifest holds the prefixed leaf hashes and the root of the
 * prefixed tree; result record, index list, errors and asynchrony as iv_verify_manifest. */
int iv_verify_manifest_rfc6962(iv_ctx *ctx, const void *d_data, uint64_t nbytes,
                               const iv_manifest *h_manifest, iv_verify_result *d_result,
                               uint64_t *d_mismatch_idx, uint64_t idx_cap, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Merkle root without allocation (the paper has no counterpart; this exists
 * for callers of this library, see below).
 *
 * Same result as iv_merkle_root, for callers that cannot allocate device
 * memory: code running inside a framework whose memory pool already owns the
 * whole GPU, a serving loop that must never block on the allocator, a process
 * that may only use buffers handed to it.  It needs no iv_ctx (creating one
 * allocates) and calls no cudaMalloc, cudaFree or other allocating routine.
 * Its scratch -- 512 intermediate digests and a ticket word -- lives in a
 * fixed 16.25 KiB array inside the library image, which every GPU that loads
 * the library holds until the process exits.
 *
 *   d_leaves, d_root   as for iv_merkle_root; the caller supplies both
 *   n_leaves           at most IV_NOALLOC_MAX_LEAVES (512 * 512); more returns
 *                      IV_ERR_TOO_LARGE and launches nothing
 * Work is enqueued on cuda_stream for the CURRENT device.  The first call on
 * a device looks up the device address of the array (once per device); make
 * that first call before starting any stream capture.  All calls share the
 * one array, which keeps the previous call's contents (the entry point clears
 * the one word that must start at zero): calls that overlap on the GPU --
 * two streams, two threads -- race and give wrong roots; serialise them.
 */
#define IV_NOALLOC_MAX_LEAVES (512ull * 512ull)
int iv_merkle_root_noalloc(const uint8_t *d_leaves, uint64_t n_leaves, uint8_t *d_root,
                           void *cuda_stream);

/* ---------------------------------------------------------------------------
 * A training step on verified weights -- the paper verifies a model before and
 * between the steps of a training pipeline and, after an update that "touches
 * some chunks", re-verifies only those (iv_tree_update).  The calls below are
 * the parts of such a step that touch few rows or all gradients at once: the
 * embedding lookup, its gradient, the global gradient norm and clipping; the
 * norms in front of its products with their gradient; and the update itself.
 * Results are functions of the inputs alone, bit for bit: no floating-point
 * atomics, every sum in an order fixed by the data, so replicas that make the
 * same step keep the same digests and root.
 *
 * Element types; 16-bit values are widened to 32 bits, sums and products are
 * taken in 32 bits or more and rounded once (to nearest, ties to even).  An
 * input and an output type may be the same, or one of them IV_F32.  Tensors may
 * start at any multiple of their element size (a tensor inside a weight file
 * rarely starts at a multiple of 16 bytes); sizes and strides are in elements.
 *
 * The calls may be captured into a CUDA graph once the context has made a call
 * of the same kind and at least that size outside a capture.  A call under
 * capture that would have to enlarge the context's scratch is refused with
 * IV_ERR_CUDA (iv_last_cuda_error: cudaErrorStreamCaptureUnsupported) before
 * anything is recorded.  Scratch that a captured call uses stays until
 * iv_destroy, also when later calls need more and get their own: replay such
 * graphs only while the context lives, and not beside its other calls.
 */
typedef enum iv_dtype { IV_F32 = 0, IV_F16 = 1, IV_BF16 = 2 } iv_dtype;

/* Embedding lookup with scaling: out[t, :] = round(scale * table[token[t], :]).
 *   d_table      n_rows rows of dim elements, row r at d_table + r * row_stride
 *                (row_stride >= dim when there is more than one row)
 *   d_tokens     n_tokens row numbers of token_bytes (4 or 8) bytes, signed
 *   d_out        n_tokens rows of dim elements, out_stride apart; must not
 *                overlap the table
 * A token outside [0, n_rows) gives a row of zeros and sets the device status
 * to 2.  n_tokens == 0 or dim == 0 launches nothing. */
int iv_embedding(iv_ctx *ctx, const void *d_table, int table_type, uint64_t n_rows, uint64_t dim, uint64_t row_stride,
                 const void *d_tokens, int token_bytes, uint64_t n_tokens, float scale, void *d_out, int out_type,
                 uint64_t out_stride, void *cuda_stream);

/* Its gradient: grad[r, :] = round(old + scale * sum of grad_out[t, :] over the tokens t of row r), old = grad[r, :]
 * when accumulate != 0 (rows without a token are then left alone) and 0 otherwise (they are set to zero).
 * The sum of a row runs over its tokens in ascending order of t: 32 terms make
 * a piece, 32 pieces a group; terms, pieces and groups are added first to last
 * in 32 bits, then scaled.
 *   d_grad_out    n_tokens rows of dim elements, grad_stride apart
 *   padding_row   tokens equal to it give no gradient; -1 for none
 *   d_grad        n_rows rows of dim elements, out_stride apart; must not overlap
 *                 grad_out or the tokens (also the compact form's outputs)
 * Tokens outside [0, n_rows) give no gradient and set the device status to 2 (a
 * padding row outside the table does not; a token of -1 always does).
 * IV_ERR_TOO_LARGE for n_tokens or cap > 2^30, n_rows > 2^31 or dim > 2^24 (also
 * the other calls of this section). */
int iv_embedding_grad(iv_ctx *ctx, const void *d_grad_out, int grad_type, uint64_t grad_stride, uint64_t dim,
                      const void *d_tokens, int token_bytes, uint64_t n_tokens, uint64_t n_rows, int64_t padding_row,
                      float scale, int accumulate, void *d_grad, int out_type, uint64_t out_stride, void *cuda_stream);

/* The same gradient with only the rows that have a token, for a table of which a
 * step touches little (the touched rows are also what makes chunks dirty):
 *   d_rows     receives the distinct rows in ascending order, then -1
 *   d_grad     receives row d_rows[i]'s gradient as row i, then zeros (so norms
 *              over the whole array are right)
 *   cap        rows of both arrays, all written; >= min(n_tokens, n_rows)
 *   d_count    receives the number of distinct rows (device memory) */
int iv_embedding_grad_rows(iv_ctx *ctx, const void *d_grad_out, int grad_type, uint64_t grad_stride, uint64_t dim,
                           const void *d_tokens, int token_bytes, uint64_t n_tokens, uint64_t n_rows,
                           int64_t padding_row, float scale, int64_t *d_rows, void *d_grad, int out_type,
                           uint64_t out_stride, uint64_t cap, uint64_t *d_count, void *cuda_stream);

/* Global gradient norm over a ragged tensor set.  The set is given as for
 * iv_hash_ragged: tensor k is the d_lengths[k] BYTES at d_base + d_offsets[k]
 * (modulo 2^64, so a tensor of another allocation has the offset address -
 * d_base).
 *   d_types    one byte per tensor, its iv_dtype; NULL: all are of `type`
 *   d_norms    optional: n floats, the norm of each tensor
 *   d_result   device memory for one record:
 *     norm = sqrt(sum of squares over all tensors); scale = 1;
 *     n_nonfinite = tensors that hold an infinity or a NaN.
 * Finite gradients of any size have a right norm (squares that leave the range
 * of 32 bits are taken in 64).  A tensor whose offset or length is not a
 * multiple of its element size, or whose type is unknown, is left out and sets
 * the device status to 2.  n == 0 gives norm 0.
 * For gradients sharded over several GPUs, add up sum_squares over them. */
typedef struct iv_norm_result {
    uint32_t status;      /* device-side status, as iv_device_status */
    uint32_t n_nonfinite; /* tensors with an infinity or a NaN */
    float norm;
    float scale;          /* what the gradients are multiplied by (1 for iv_grad_norm) */
    double sum_squares;
    uint64_t n_elements;
} iv_norm_result;
int iv_grad_norm(iv_ctx *ctx, const void *d_base, const uint64_t *d_offsets, const uint64_t *d_lengths,
                 const uint8_t *d_types, int type, uint64_t n, float *d_norms, iv_norm_result *d_result,
                 void *cuda_stream);

/* Clipping: the norm as above, scale = norm <= max_norm ? 1 : max_norm / norm
 * (so an infinite norm gives 0 and NaN gives NaN: n_nonfinite tells to skip the
 * step), then every tensor times scale, rounded once.
 *   max_norm        >= 0, not NaN
 *   d_out           NULL: in place.  Otherwise tensor k goes to d_out +
 *                   d_out_offsets[k] (bytes) as out_type, or as its own type when
 *                   out_type < 0; the output must not overlap the input.  A
 *                   tensor whose output starts at no multiple of its element, or
 *                   would go from one 16-bit type to the other, is not written
 *                   and sets the device status to 2
 * The same tensors give the same bits whether their type is given as `type` or
 * one by one; a set described by d_types takes up to 45 % longer. */
int iv_grad_clip(iv_ctx *ctx, void *d_base, const uint64_t *d_offsets, const uint64_t *d_lengths, const uint8_t *d_types,
                 int type, uint64_t n, float max_norm, void *d_out, const uint64_t *d_out_offsets, int out_type,
                 float *d_norms, iv_norm_result *d_result, void *cuda_stream);

/* Its second half alone, with a factor from device memory (gradients sharded over several GPUs, whose norm is known
 * after a reduction).  Arguments as iv_grad_clip. */
int iv_grad_scale(iv_ctx *ctx, void *d_base, const uint64_t *d_offsets, const uint64_t *d_lengths, const uint8_t *d_types,
                  int type, uint64_t n, const float *d_scale, void *d_out, const uint64_t *d_out_offsets, int out_type,
                  void *cuda_stream);

/* Layer norm of rows:  y[r, :] = round((x[r, :] - mu) * s * weight + bias),
 *   mu = mean of x[r, :],  s = 1 / sqrt(mean of (x[r, :] - mu)^2 + eps);
 * with rms != 0 the root-mean-square form, mu = 0.
 *   d_x        n_rows rows of dim elements, x_stride apart
 *   d_weight   dim elements of param_type (any of the three), NULL: ones;
 *   d_bias     the same, NULL: zeros
 *   d_y        n_rows rows, y_stride apart; must not overlap the inputs
 *   d_mean, d_rstd   optional: n_rows floats each, mu and s (for the gradient)
 *   eps        >= 0, not NaN
 * A row's result does not depend on the other rows, nor on strides or
 * alignment.  mu is a sum of 32 bits over dim: what it is off, some of its last
 * places, is multiplied by s (nothing in a row of equal numbers the sum of which
 * is exact in 24 bits).  Sums of squares are taken in 32 bits: a row whose squares leave
 * that range has s = 0.  IV_ERR_TOO_LARGE for n_rows > 2^30, dim > 2^24. */
int iv_layer_norm(iv_ctx *ctx, const void *d_x, int x_type, uint64_t x_stride, uint64_t n_rows, uint64_t dim,
                  const void *d_weight, const void *d_bias, int param_type, float eps, int rms, void *d_y, int y_type,
                  uint64_t y_stride, float *d_mean, float *d_rstd, void *cuda_stream);

/* Its gradient, from d_dy (of the result's type), the inputs and the stored mu and s:  with h = (x - mu) s and
 * p = dy * weight,
 *   dx[r, :] = round(s (p - mean(p) - h mean(p h)))     (rms: without mean(p))
 *   d_weight_grad = round(old + sum over rows of dy h),  d_bias_grad = round(old + sum over rows of dy)
 * old being what is there when accumulate != 0 and 0 otherwise.  The sums over
 * rows are taken in 32 bits in an order that n_rows, dim and the types alone decide.
 *   x_type, y_type  as in the forward call: dx is of x_type
 *   d_mean          not read when rms != 0
 *   d_weight_grad, d_bias_grad   dim elements of sum_type (any), NULL: not wanted
 * Without rows dx is empty and both sums are 0 (or old).  Outputs must not
 * overlap inputs or each other. */
int iv_layer_norm_grad(iv_ctx *ctx, const void *d_dy, int y_type, uint64_t dy_stride, const void *d_x, int x_type,
                       uint64_t x_stride, uint64_t n_rows, uint64_t dim, const void *d_weight, int param_type,
                       const float *d_mean, const float *d_rstd, int rms, void *d_dx, uint64_t dx_stride,
                       void *d_weight_grad, void *d_bias_grad, int sum_type, int accumulate, void *cuda_stream);

/* One AdamW step over a ragged tensor set, t being the number of this step (*d_step + 1):
 *   g = c * gradient,   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *   w = w (1 - lr weight_decay) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps),
 * in 32 bits, w rounded once (the moments' products and sums are rounded one by
 * one; the root and the quotient are within 2^-23 of themselves, with 8-bit
 * moments the quotient within 2^-22, and an eps below 2^-126 counts as 0).  The weights are given as for iv_grad_norm, all
 * of one type, and updated in place (in the bytes of a weight file: the chunks
 * they lie in are then dirty); they must not overlap one another, the gradients
 * or the state.
 *   d_grads, d_grad_offsets   tensor k's gradient, as many elements of
 *                    grad_type, starts at d_grads + d_grad_offsets[k] (bytes,
 *                    modulo 2^64).  The types are equal or one of them is IV_F32
 *   d_state_offsets  n places in the state, in ELEMENTS, ascending multiples of
 *                    IV_ADAMW_BLOCK: element i of tensor k has its moments at
 *                    d_state_offsets[k] + i
 *   state_size       elements of the state, a multiple of IV_ADAMW_BLOCK
 *   state_bits       32: d_m, d_v are state_size floats, 32-byte aligned.
 *                    8: d_m, d_v are state_size codes (e4m3: sign, four bits of
 *                    exponent with bias 7, three digits; 0x7f is NaN), 8-byte
 *                    aligned, and d_m_scales, d_v_scales one float for each
 *                    block: m = code * scale, sqrt(v) = code * scale.  All
 *                    zero: no moments yet.  What lies between tensors is left alone
 *   d_master         optional, for 16-bit weights: state_size floats, 32-byte
 *                    aligned, the weights in 32 bits; they are updated, and
 *                    the weights receive them rounded
 *   d_lr             optional: the learning rate in device memory, instead of lr
 *   d_norm           optional: the record of iv_grad_norm over all gradients;
 *                    c = norm <= max_norm ? 1 : max_norm / norm (c = 1 without a
 *                    record).  When its n_nonfinite is not 0 the call
 *                    changes nothing, the number of steps included
 *   d_step           the number of steps taken, counted up by the call
 * stochastic != 0 rounds 16-bit weights up with the probability that the lost
 * bits give (to nearest otherwise); 8-bit moments are always rounded so, a
 * root that is not 0 to no less than the smallest code.  The random words are
 * a function of (seed, t, place in the state):  with
 *   mix(x): x ^= x >> 16; x *= 0x6A09E667; x ^= x >> 15; x *= 0xBB67AE85; x ^= x >> 16,
 *   K0 = mix(mix(mix(low(seed) + G) + high(seed)) + low(t)),  K1 = mix(K0 + high(t) + G),
 *   G = 0x9E3779B9,  q = place / 8,  b = mix(q ^ K0),  a = mix(b + K1)
 * word k is b + (k + 1) a, and k = place % 8 rounds m, 8 + place % 8 the root, 16 +
 * place % 8 the weight, each by the word's upper bits, as many as are lost (16 at
 * most for weights, 20 for codes).
 * A block's scale is its largest finite magnitude / 447.9995; an infinite or NaN
 * moment becomes a NaN code and leaves the other elements of its block alone.
 * A tensor that is ill-formed (a length, address or place at no multiple of its
 * unit, no room before the next tensor's place) is left out and sets the device status
 * to 2.  IV_ERR_TOO_LARGE for n > 2^30 or state_size > 2^34. */
#define IV_ADAMW_BLOCK 256
typedef struct iv_adamw_options {
    double lr, beta1, beta2, eps, weight_decay; /* all >= 0 and finite, the betas < 1 */
    float max_norm;                             /* >= 0; read with d_norm only */
    uint32_t stochastic;
    uint64_t seed;
} iv_adamw_options;
int iv_adamw_step(iv_ctx *ctx, void *d_base, const uint64_t *d_offsets, const uint64_t *d_lengths, int type, uint64_t n,
                  const void *d_grads, const uint64_t *d_grad_offsets, int grad_type, const uint64_t *d_state_offsets,
                  uint64_t state_size, int state_bits, void *d_m, void *d_v, float *d_m_scales, float *d_v_scales,
                  float *d_master, const iv_adamw_options *h_options, const float *d_lr, const iv_norm_result *d_norm,
                  uint64_t *d_step, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Roofline probe (a measurement aid; the paper has no counterpart).  Runs a
 * register-only microbenchmark on every SM and reports, from the SM cycle
 * counter, how many lane-operations of one instruction kind an SM retires per
 * clock -- the denominator of the integer roofline -- or, for the kinds that run
 * SHA-256 (6, 7, 13, 14), how many message bytes per clock per SM that part of the
 * compression function alone sustains.  Synchronous; allocates and frees a few KB of device memory.
 *
 *   warps_per_block, blocks_per_sm   launch shape (blocks = blocks_per_sm * SM count)
 *   active_lanes                     1..32 lanes of each warp that do work
 *   iters                            loop trips (128 operations each; one 64-byte block
 *                                    each for the SHA-256 kinds)
 *   h_out[0]                         lane-ops (or bytes) per clock per SM
 *   h_out[1]                         mean cycles per block
 */
typedef enum iv_probe_kind {
    IV_PROBE_IADD3 = 0,  /* three-input integer add */
    IV_PROBE_LOP3 = 1,   /* three-input logic op */
    IV_PROBE_SHF = 2,    /* funnel shift (rotate) */
    IV_PROBE_PRMT = 3,   /* byte permute */
    IV_PROBE_IMAD = 4,   /* integer multiply-add */
    IV_PROBE_MIXED = 5,  /* LOP3 and IMAD interleaved 1:1 */
    IV_PROBE_SHA256 = 6,     /* full SHA-256 compressions, registers only */
    IV_PROBE_SHA256_SCHED_FMA = 7, /* the same with the message schedule's additions as multiply-adds (FMA pipe) */
    IV_PROBE_LAT_IADD3 = 8,  /* kinds 8..11: ONE dependent chain per thread; with one warp per SM,   */
    IV_PROBE_LAT_LOP3 = 9,   /* 32 / h_out[0] is the dependent-issue latency of the instruction in   */
    IV_PROBE_LAT_SHF = 10,   /* clocks                                                               */
    IV_PROBE_LAT_IMAD = 11,
    IV_PROBE_LAT_CROSS = 12, /* one chain alternating LOP3 (ALU pipe) and IMAD (FMA pipe) */
    IV_PROBE_ROUNDS = 13,    /* the 64 rounds alone, W + K from shared memory: the consumer half of the two-warp kernel */
    IV_PROBE_SCHEDULE = 14   /* the message schedule + round constants alone: its producer half */
} iv_probe_kind;
int iv_probe_alu(iv_ctx *ctx, int kind, uint32_t warps_per_block, uint32_t blocks_per_sm,
                 uint32_t active_lanes, uint32_t iters, double *h_out);

#ifdef __cplusplus
}
#endif
#endif /* IV_H */
