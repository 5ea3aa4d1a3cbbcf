/*
 * lora_b200 -- unmerged multi-adapter LoRA forward for NVIDIA B200 (sm_100a).
 *
 *     y[t, :] = y_base[t, :] + s_i * (x[t, :] . A_i) . B_i ,      i = slot_idx[t]
 *
 * A LoRA adapter is a pair of low-rank matrices per adapted projection whose
 * activations are added to the output of the backbone projection (paper
 * Section 2.2).  Serving systems keep the adapters unmerged so that hundreds of
 * them share one backbone, run several of them inside one batch, hold them in a
 * statically reserved GPU region of A_max slots with one uniform footprint
 * S_max each, and swap missing ones in from CPU memory (paper Sections 1, 2.2
 * and the adapter-cache / Lat_load stage of Section 5, Eq. 1).  This library is
 * that per-projection computation and the slot pool around it:
 *
 *   lora_pool_create      the A_max x S_max slot pool in caller-owned device memory
 *   lora_pool_load_slot   side-stream swap-in of one adapter from pinned host memory
 *   lora_build_segments   integer metadata: tokens grouped by adapter slot, cut in tiles
 *   lora_bgmv_apply       decode batches (one token per request)
 *   lora_sgmv_apply       prefill / chunked-prefill batches (per-adapter segments)
 *
 * and what a served batch needs between two such projections, on a cache that leaves the GPU's
 * memory to adapter slots (4 bits a value):
 *
 *   lora_kv_create        a paged key/value cache in caller-owned device memory
 *   lora_kv_build_tables  block tables, positions and slot maps from the requests' lengths
 *   lora_qk_norm_rope     per-head norm and rotation of queries and keys in one pass
 *   lora_kv_append        the same pass, with the keys and values going to the cache as 4-bit rows
 *   lora_kv_attention     attention of a batch (single tokens and prompts together) over the cache
 *
 * Conventions
 *  - plain C ABI; every call returns a lora_status_t; nothing aborts, traps or resets a device;
 *  - "dev" pointers are device memory, "host" pointers are host memory; all buffers are owned
 *    by the caller and must stay valid until the work queued on the stream has finished;
 *  - streams are cudaStream_t values passed as void*; all GPU work is asynchronous on the
 *    stream given; the library never synchronises a device and never allocates device memory;
 *  - bf16 tensors are row-major with a leading dimension in ELEMENTS; base pointers must be
 *    16-byte aligned and every d_in, d_out and leading dimension a multiple of 8;
 *  - arithmetic: bf16 inputs, fp32 accumulation, one round-to-nearest-even to bf16 at the store;
 *  - a pool handle keeps host-side state (slot table copy, events, tensor maps, the shapes of the
 *    metadata tables built through it) and is not thread-safe: calls on one pool come from one
 *    host thread at a time.  Different pools are independent.
 */
#ifndef LORA_B200_H
#define LORA_B200_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LORA_OK = 0,
    LORA_ERR_INVALID_ARG = 1,      /* null pointer, bad enum, misaligned or overlapping buffers */
    LORA_ERR_SHAPE = 2,            /* dimension not a multiple of 8, negative sizes */
    LORA_ERR_SLOT_RANGE = 3,       /* slot >= num_slots or < 0 */
    LORA_ERR_RANK = 4,             /* rank < 1 or rank > r_max */
    LORA_ERR_NOT_LOADED = 5,       /* operation needs an occupied slot (slot policy calls) */
    LORA_ERR_BUSY = 6,             /* every candidate slot is pinned by an in-flight batch */
    LORA_ERR_BUFFER_TOO_SMALL = 7, /* caller buffer smaller than the matching *_bytes query */
    LORA_ERR_NOT_PINNED = 8,       /* host adapter memory is pageable */
    LORA_ERR_CUDA = 9,             /* a CUDA runtime call failed: see lora_last_cuda_error() */
    LORA_ERR_TIMEOUT = 10          /* a bounded device-side wait expired (lora_pool_check_status) */
} lora_status_t;

const char *lora_status_string(lora_status_t s);
/* cudaError_t value of the most recent failing runtime call made by this thread's last call. */
int32_t lora_last_cuda_error(void);
/* Number of kernels this library has launched since it was loaded (all pools, all threads). */
int64_t lora_launch_count(void);

/* ----------------------------------------------------------------------------------------
 * Slot pool (paper Section 2.2: a fixed region for adapter weights, at most A_max adapters
 * loaded at once, every adapter given the same maximum footprint S_max).
 * num_slots = A_max; r_max = the rank that S_max is sized for.
 * -------------------------------------------------------------------------------------- */
typedef struct lora_pool lora_pool_t;

typedef struct {
    int32_t d_in;    /* input width of the adapted projection  (multiple of 8) */
    int32_t d_out;   /* output width of the adapted projection (multiple of 8) */
} lora_target_t;

typedef struct {
    int32_t device;               /* CUDA device ordinal the pool lives on */
    int32_t num_slots;            /* A_max, 1 .. 8192 */
    int32_t r_max;                /* largest rank a slot can hold, 1 .. 64 */
    int32_t num_targets;          /* adapted projections (e.g. 7 per layer x 32 layers) */
    const lora_target_t *targets; /* host, [num_targets]; copied */
    void *device_buf;             /* dev, 256-byte aligned, >= lora_pool_bytes(); caller-owned */
    size_t device_buf_bytes;
} lora_pool_desc_t;

/* Bytes of device memory a pool of this shape needs (control block with the slot table and the
 * targets' tensor maps + transpose staging + num_slots slots of r_max rows for every target's
 * A and B).  device_buf is ignored. */
lora_status_t lora_pool_bytes(const lora_pool_desc_t *desc, size_t *bytes);

/* Creates the host handle and clears the pool's control block (slot table: all slots empty;
 * status words: zero).  Synchronous: returns after the clear has completed.  The handle is
 * owned by the library; the device memory stays the caller's and must outlive the handle. */
lora_status_t lora_pool_create(const lora_pool_desc_t *desc, lora_pool_t **out);
lora_status_t lora_pool_destroy(lora_pool_t *pool);

enum { LORA_A_DIN_MAJOR = 0,   /* A given as [d_in, rank] row-major (the formula's orientation) */
       LORA_A_RANK_MAJOR = 1,  /* A given as [rank, d_in] row-major (already in slot layout)    */
       LORA_PACKED = 2         /* A[0] is ONE pinned buffer (16-byte aligned) holding, for every
                                  target in order, A as [rank, d_in] then B as [rank, d_out]; the
                                  other pointers are ignored.  With rank == r_max this is the slot's
                                  own layout and the swap-in is a single DMA. */ };

typedef struct {
    int32_t rank;            /* 1 .. r_max */
    float scale;             /* s_i */
    const void *const *A;    /* host, [num_targets] pointers to pinned bf16 matrices, see a_layout */
    const void *const *B;    /* host, [num_targets] pointers to pinned bf16 [rank, d_out] row-major */
    int32_t a_layout;        /* LORA_A_DIN_MAJOR, LORA_A_RANK_MAJOR or LORA_PACKED */
    int32_t trust_pinned;    /* non-zero: skip the per-pointer pinned-memory check */
} lora_adapter_host_t;

/*
 * Swap one adapter into a slot (paper Section 5: the adapter-cache stage loads missing
 * adapters from CPU memory; its cost is Lat_load in Eq. 1).  Queues on load_stream:
 *   wait until everything queued so far on compute_stream has finished (the slot may still be
 *   read), mark the slot empty, copy A and B for every target, zero the padding rows
 *   rank .. r_max - 1, mark the slot occupied with (rank, scale), record the slot's ready event.
 * Inside a slot every matrix is stored rank-major: A as [r_max, d_in], B as [r_max, d_out],
 * rows 0 .. rank-1 meaningful, the rest zero.  LORA_A_DIN_MAJOR input is transposed on the device.
 * Host matrices must stay valid until the ready event has fired (lora_pool_acquire + stream
 * completion, or a synchronise on load_stream).  compute_stream may be NULL when no reader
 * can be in flight.  All loads of one pool go through ONE load stream (LORA_A_DIN_MAJOR input
 * passes through a staging area of the pool that consecutive loads reuse in stream order).
 * On an argument error (every code below but CUDA) the slot is left untouched; after a CUDA error
 * in the middle of the sequence the slot is empty on the device and in the host's view.
 * Errors: INVALID_ARG, SLOT_RANGE, RANK, NOT_PINNED, CUDA.
 */
lora_status_t lora_pool_load_slot(lora_pool_t *pool, int32_t slot, const lora_adapter_host_t *adapter,
                                  void *load_stream, void *compute_stream);

/* Marks a slot empty (same ordering as a load: waits for compute_stream's queued readers). */
lora_status_t lora_pool_evict_slot(lora_pool_t *pool, int32_t slot, void *load_stream,
                                   void *compute_stream);

/* Makes compute_stream wait for the ready events of these slots (host array of n slot ids).
 * Slots that were never loaded are skipped.  Errors: SLOT_RANGE, CUDA. */
lora_status_t lora_pool_acquire(lora_pool_t *pool, const int32_t *slots_host, int32_t n,
                                void *compute_stream);

/* Copies one slot's stored matrices of one target back to host memory (A_host: [r_max, d_in],
 * B_host: [r_max, d_out], bf16) on `stream`; either pointer may be NULL.  For inspection. */
lora_status_t lora_pool_read_slot(lora_pool_t *pool, int32_t slot, int32_t target,
                                  void *A_host, void *B_host, void *stream);

/* Host-side view of a slot as of the last load/evict call: rank (0 when empty) and scale. */
lora_status_t lora_pool_slot_info(const lora_pool_t *pool, int32_t slot, int32_t *rank, float *scale);

/* Device status words, copied asynchronously to host_out[4] (pinned host memory) on `stream`:
 * [0] tokens whose slot id was neither -1 nor an occupied slot (accumulated; such tokens are
 * treated as -1), [1] expired device-side waits, [2..3] reserved. */
lora_status_t lora_pool_poll_status(lora_pool_t *pool, int32_t *host_out, void *stream);
lora_status_t lora_pool_reset_status(lora_pool_t *pool, void *stream);

/* The one call that waits: copies the status words back on `stream`, synchronises that stream and
 * returns LORA_ERR_TIMEOUT when word 1 is non-zero (some block of some kernel gave up a bounded
 * wait and stored no result for its rows: the outputs of the applies queued since the last reset
 * are not to be trusted), LORA_OK otherwise.  words_out (host, [4]) may be NULL.  The apply calls
 * themselves are asynchronous and cannot report this; call it wherever a step's results are
 * consumed on the host, or once per step in a server loop. */
lora_status_t lora_pool_check_status(lora_pool_t *pool, void *stream, int32_t *words_out);

/* Exercises the time-out path without disturbing anything: launches ONE block that polls an
 * mbarrier nobody completes, `polls` times (1 .. 2^20), then records the expiry in status word 1
 * exactly as the apply kernels do and returns without writing *witness_dev (dev int32, may be
 * NULL; it is written only if the wait had succeeded).  For tests and for monitoring code that
 * wants to see its own alarm fire. */
lora_status_t lora_pool_selftest_wait_expiry(lora_pool_t *pool, int32_t polls, int32_t *witness_dev,
                                             void *stream);

/* Tuning knobs, for measurement (0 = the default behaviour for every key):
 *   key 0  apply path: 1 = two-phase CUDA-core kernels with the fp32 workspace
 *   key 1  fused kernel: blocks per cluster (1, 2, 4, 8)
 *   key 2  programmatic dependent launch of the fused kernel: 2 = never
 *   key 3  fused kernel: upper bound on the clusters in the grid
 *   key 4  tensor-core kernels of lora_sgmv_apply: 1 = never, 2 = whenever they apply (read by
 *          lora_build_segments, which writes their tile list, and by the apply)
 *   key 5  fused kernel: stages of the shared-memory ring (2 .. 4)
 *   key 6  lora_sgmv_apply: 1 = the tiles the tensor-core kernels leave over run after them on the
 *          caller's stream, not beside them on the pool's own stream
 *   key 7  segment builder: 1 = one warp per slot also for long batches
 *   key 8  tensor-core expand of lora_sgmv_apply: blocks per SM in its grid (0 = the default, 8)
 *   key 9  fused kernel: share (1 .. 99 %) of the resident clusters one launch may take
 *   key 10 1 = decode batches take the general fused kernel, not the decode kernel
 *   key 11 when a fused kernel lets its successor on the stream become resident: 1 = only at its
 *          end, 2 = at its start (default: at its start for launches of fewer than four projections)
 * Keys outside 0 .. 15 -> INVALID_ARG. */
lora_status_t lora_pool_set_tuning(lora_pool_t *pool, int32_t key, int32_t value);

/* ----------------------------------------------------------------------------------------
 * Slot policy and pool sizing (paper Section 1: adapters move between CPU and GPU memory
 * according to their usage; Section 2.2: A_max slots of one footprint S_max; Section 5: the
 * adapter-cache stage of a step loads what the scheduled batch needs).  Host-side bookkeeping
 * only: no CUDA call is made, and a policy object is independent of any pool.  Adapter ids are
 * the caller's non-negative 64-bit keys.  "Least recently used" follows a logical clock advanced
 * by every use, so decisions are a deterministic function of the call sequence.  A pinned slot
 * (pin count > 0: an in-flight batch's metadata references it) is never chosen as a victim.
 * Not thread-safe.
 * -------------------------------------------------------------------------------------- */
typedef struct lora_policy lora_policy_t;
lora_status_t lora_policy_create(int32_t num_slots, lora_policy_t **out);
lora_status_t lora_policy_destroy(lora_policy_t *policy);
/* *slot_out = the slot holding the adapter, or -1. */
lora_status_t lora_policy_lookup(const lora_policy_t *policy, int64_t adapter, int32_t *slot_out);
/* What a slot holds (-1: empty) and its pin count; either pointer may be NULL. */
lora_status_t lora_policy_slot(const lora_policy_t *policy, int32_t slot, int64_t *adapter_out,
                               int32_t *pins_out);
/* Marks the slot most recently used.  Errors: SLOT_RANGE, NOT_LOADED (empty slot). */
lora_status_t lora_policy_touch(lora_policy_t *policy, int32_t slot);
/* Pin / unpin the n slots of a host array (a slot named twice is pinned twice).  All or nothing.
 * Errors: SLOT_RANGE, NOT_LOADED (pin of an empty slot), INVALID_ARG (unpin below zero). */
lora_status_t lora_policy_pin(lora_policy_t *policy, const int32_t *slots_host, int32_t n);
lora_status_t lora_policy_unpin(lora_policy_t *policy, const int32_t *slots_host, int32_t n);
/* The slot to fill next: the lowest empty unpinned slot, else the unpinned slot used longest ago
 * (ties: lowest index); *evicted_out (may be NULL) = the adapter it holds now, or -1.  Changes
 * nothing.  Errors: BUSY (every slot is pinned). */
lora_status_t lora_policy_choose_victim(const lora_policy_t *policy, int32_t *slot_out,
                                        int64_t *evicted_out);
/* Records that `adapter` now lives in `slot` (after lora_pool_load_slot), replacing what was
 * there, and marks it used.  Errors: SLOT_RANGE, BUSY (slot pinned), INVALID_ARG (the adapter is
 * resident in another slot). */
lora_status_t lora_policy_assign(lora_policy_t *policy, int32_t slot, int64_t adapter);
/* Records that the slot is empty (after lora_pool_evict_slot).  Errors: NOT_LOADED, BUSY. */
lora_status_t lora_policy_release(lora_policy_t *policy, int32_t slot);
/* The adapter-cache stage for one batch: adapters[i] is request i's adapter (-1: none).
 * Writes slot_idx_out[i] (host, [n]; -1 for requests without adapter) and the loads the caller
 * has to queue with lora_pool_load_slot before the batch's metadata is built: miss_slots_out[k],
 * miss_adapters_out[k], k < *n_miss_out, in order of first appearance in the batch.  Victims are
 * chosen as by lora_policy_choose_victim among slots the batch itself does not use; every slot of
 * the batch is marked used.  On error nothing has changed.
 * Errors: BUSY (more distinct adapters than slots that are free or may be evicted: the scheduler
 * has to defer requests, the A_max limit of paper Section 5), BUFFER_TOO_SMALL (miss_cap). */
lora_status_t lora_policy_admit(lora_policy_t *policy, const int64_t *adapters, int32_t n,
                                int32_t *slot_idx_out, int32_t *miss_slots_out,
                                int64_t *miss_adapters_out, int32_t miss_cap, int32_t *n_miss_out);
/* Counters since creation: distinct resident adapters found per batch, loads asked for, adapters
 * displaced.  Any pointer may be NULL. */
lora_status_t lora_policy_stats(const lora_policy_t *policy, int64_t *hits, int64_t *misses,
                                int64_t *evictions);

/* Sizing: the largest num_slots (A_max) whose pool fits in bytes_budget for these targets at this
 * r_max (S_max), and the bytes one more slot costs.  Errors: BUFFER_TOO_SMALL (not even one slot),
 * plus those of lora_pool_bytes. */
lora_status_t lora_pool_plan(size_t bytes_budget, const lora_target_t *targets, int32_t num_targets,
                             int32_t r_max, int32_t *num_slots_out, size_t *bytes_per_slot_out);

/* ----------------------------------------------------------------------------------------
 * Segment metadata (several adapters are served inside one batch, paper Section 2.2; each
 * request names its adapter, Section 5): a stable group-by-slot of the batch's tokens.
 *
 * Output buffer `meta_dev`, all int32, in this order (N = num_slots,
 * cap_seg = min(T, N), cap_tile = cap_seg + T / tile_m):
 *   header[16]   {T, n_active, n_invalid, n_seg, n_tile, tile_m, long_min, N, cap_seg, cap_tile, 0..}
 *   perm[T]      active tokens ordered by (slot, token id), then the other tokens ascending
 *   seg_slot[cap_seg], seg_start[cap_seg + 1], seg_rank[cap_seg], seg_flags[cap_seg]
 *                flags bit0: the segment's tokens are consecutive ids; bit1: length >= long_min
 *   tile_seg[cap_tile], tile_row0[cap_tile], tile_rows[cap_tile]
 *                each segment cut into pieces of at most tile_m rows (positions in perm)
 *   (then words private to the library: one flag word per tile, and from the next 16-byte
 *    boundary a 4-word record per
 *    tile, a 4-word record plus 16 row ids per piece of at most 16 rows of a tile, and the
 *    list of the tiles lora_sgmv_apply gives to its tensor-core kernels (written by a second
 *    small launch when the batch qualifies for them); lora_segments_bytes counts them)
 * Unused entries are -1.  A token is active iff its slot id names an occupied slot; a token
 * that is neither active nor -1 is invalid (counted in header and in the pool's status word 0).
 * The result is an exact integer function of its inputs.
 * -------------------------------------------------------------------------------------- */
lora_status_t lora_segments_bytes(int32_t T, int32_t num_slots, int32_t tile_m, size_t *bytes);

/* slot_idx_dev: dev int32 [T]; meta_dev: dev, 16-byte aligned, meta_bytes >= lora_segments_bytes.
 * tile_m in 1 .. 128, long_min >= 1.  T == 0 writes an empty table.  Uses the slot table as it is
 * on the device when the kernel runs.  Errors: INVALID_ARG, SHAPE, BUFFER_TOO_SMALL, CUDA. */
lora_status_t lora_build_segments(lora_pool_t *pool, const int32_t *slot_idx_dev, int32_t T,
                                  int32_t tile_m, int32_t long_min,
                                  void *meta_dev, size_t meta_bytes, void *stream);

/* ----------------------------------------------------------------------------------------
 * The forward itself.  x: bf16 [T, d_in]; y_base: bf16 [T, d_out] (the backbone projection's
 * output, computed by the caller); y: bf16 [T, d_out], either exactly y_base (in place) or
 * not overlapping it.  Tokens without an active slot get y = y_base bit for bit.  Row t of y
 * depends only on row t of x and y_base, the token's slot and the pool.
 * workspace: dev scratch of >= lora_workspace_bytes(pool, T) bytes (fp32 partial products
 * v = x . A_i between the two phases of the tensor-core and two-phase kernels; the fused
 * kernels keep v on chip), contents undefined afterwards; calls sharing a workspace must be ordered on
 * one stream.
 * Ordering: every apply is ordered behind the lora_build_segments call that wrote its table.
 * Later applies on the same table may start reading the table and the pool (never x or y_base)
 * while the kernel queued before them on the stream is still running, so nothing queued between
 * two applies may write the table or the pool without an event or a rebuild in between (slot
 * loads go through lora_pool_load_slot / lora_pool_acquire, which order themselves).
 * T == 0 returns LORA_OK without launching.
 * Errors: INVALID_ARG, SHAPE, SLOT_RANGE (target), BUFFER_TOO_SMALL, CUDA.
 * -------------------------------------------------------------------------------------- */
lora_status_t lora_workspace_bytes(const lora_pool_t *pool, int32_t T_max, size_t *bytes);

/* Decode batches.  meta_dev_or_null: metadata built from the same slot_idx_dev (tile_m <= 16)
 * so that each adapter's matrices are fetched once per group of tokens; NULL = index per token. */
lora_status_t lora_bgmv_apply(lora_pool_t *pool, int32_t target,
                              const void *x, int64_t ldx,
                              const void *y_base, int64_t ldyb,
                              void *y, int64_t ldy,
                              const int32_t *slot_idx_dev, int32_t T,
                              const void *meta_dev_or_null,
                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * Several projections of ONE decode batch in one launch (paper Section 2.2: the adapters of a
 * batch are served together through kernel-level work; Section 8.1: the models carry LoRA on all
 * their attention and MLP projections): q/k/v, or gate/up, or all seven adapted projections of a
 * layer when the caller has their inputs ready.  Every item is what one lora_bgmv_apply call would
 * take; all items share the batch (slot_idx_dev, T) and its grouped metadata, which is required.
 * The items must be independent: no item's y may overlap another item's x, y_base or y (an item's
 * own y may equal its y_base); items may share x.  The launch walks the units of item 0 first,
 * then item 1, ...: list wide projections first for the best balance.  Results are bit-identical
 * to n_items separate lora_bgmv_apply calls.
 * n_items in 1 .. LORA_MULTI_MAX.  Errors: those of lora_bgmv_apply, per item.
 */
#define LORA_MULTI_MAX 8
typedef struct {
    int32_t target;
    const void *x;       int64_t ldx;    /* dev bf16 [T, d_in]  */
    const void *y_base;  int64_t ldyb;   /* dev bf16 [T, d_out] */
    void *y;             int64_t ldy;    /* dev bf16 [T, d_out] */
} lora_apply_item_t;
lora_status_t lora_bgmv_apply_multi(lora_pool_t *pool, const lora_apply_item_t *items, int32_t n_items,
                                    const int32_t *slot_idx_dev, int32_t T, const void *meta_dev,
                                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * lora_bgmv_apply for callers that cannot hand over a workspace (the paper has no counterpart;
 * this is a convenience of the library).  Some hosts of this code may not allocate device
 * memory at the point where they call it: a serving engine that has already given all free HBM
 * to its KV cache and adapter pool, a plug-in running inside another framework's memory
 * manager, code on a latency path where an allocation (or the implicit synchronisation of a
 * free) is not acceptable.  For them the fp32 scratch between the shrink and expand phases is a
 * fixed array of LORA_STATIC_SCRATCH_BYTES inside the library image; every GPU that loads the
 * library holds that much memory until the process exits.
 *  - Same arguments and results as lora_bgmv_apply minus the workspace; it always runs the
 *    two-phase CUDA-core kernels.  It allocates and frees nothing.
 *  - Limit: 32 * T * bucket(r_max) <= LORA_STATIC_SCRATCH_BYTES, bucket = r_max rounded up to
 *    8, 16, 32 or 64 (T <= 4096 at r_max 16, T <= 1024 at r_max 64); beyond it the call returns
 *    LORA_ERR_BUFFER_TOO_SMALL and launches nothing.
 *  - The first call on each device looks up the array's device address; make that call before
 *    starting any stream capture.
 *  - All calls on a device share the one array, and it keeps whatever the last call left there
 *    (the kernels overwrite every entry they later read, so nothing is cleared).  Two calls
 *    that can overlap on the GPU (different streams without an ordering between them) race on
 *    it: keep such calls on one stream or order them with events.
 */
#define LORA_STATIC_SCRATCH_BYTES (2u * 1024u * 1024u)
lora_status_t lora_bgmv_apply_static(lora_pool_t *pool, int32_t target,
                                     const void *x, int64_t ldx,
                                     const void *y_base, int64_t ldyb,
                                     void *y, int64_t ldy,
                                     const int32_t *slot_idx_dev, int32_t T,
                                     const void *meta_dev_or_null, void *stream);

/* Prefill / chunked-prefill batches.  meta_dev: metadata built for this batch (any tile_m).
 * With tile_m = 128 and a batch of at least 4096 tokens, tiles that are runs of 32 .. 128
 * consecutive tokens take the tcgen05 kernels (split-K partials in `workspace`); every other tile,
 * and every tile of a shorter batch, takes the fused kernel that also serves lora_bgmv_apply.
 * When both kinds are present the fused kernel runs on a stream the pool owns, forked from
 * `stream` by an event at the call and joined back into it before the call returns, so work
 * enqueued on `stream` afterwards is ordered behind all of it (this also holds inside a stream
 * capture: the pool's stream joins the capture and leaves it within the call). */
lora_status_t lora_sgmv_apply(lora_pool_t *pool, int32_t target,
                              const void *x, int64_t ldx,
                              const void *y_base, int64_t ldyb,
                              void *y, int64_t ldy,
                              const void *meta_dev, int32_t T,
                              void *workspace, size_t workspace_bytes, void *stream);

/* ----------------------------------------------------------------------------------------
 * One layer step from HOST buffers: copies x, y_base and slot_idx (pinned host memory) to the
 * caller's device staging buffers, builds the metadata, applies, and copies y back, all on
 * `stream`.  kind: 0 = BGMV, 1 = SGMV.  y_host is complete when the stream has drained.
 * -------------------------------------------------------------------------------------- */
typedef struct {
    void *x_dev;            /* >= T * d_in  bf16 */
    void *y_base_dev;       /* >= T * d_out bf16 */
    void *y_dev;            /* >= T * d_out bf16 (may equal y_base_dev) */
    int32_t *slot_idx_dev;  /* >= T int32 */
    void *meta_dev;         size_t meta_bytes;
    void *workspace;        size_t workspace_bytes;
} lora_step_buffers_t;

lora_status_t lora_apply_host(lora_pool_t *pool, int32_t target, int32_t kind,
                              const void *x_host, const void *y_base_host, void *y_host,
                              const int32_t *slot_idx_host, int32_t T,
                              int32_t tile_m, int32_t long_min,
                              const lora_step_buffers_t *dev, void *stream);

/* ----------------------------------------------------------------------------------------
 * Paged key/value cache in 4 bits.
 *
 * Adapter slots and the cache of running requests share one GPU's memory (paper Section 2.2: the
 * A_max x S_max region is taken from what the requests' keys and values could use), so a row of
 * head_dim values is kept as head_dim 4-bit codes with one scale and one low value:
 *     value_i = low + scale * code_i ,  code_i in 0 .. 15 ,
 *     low = bf16(min x) , scale = bf16((max x - low) * fl(1/15)) ,
 *     code_i = clamp(rint((x_i - low) * (1 / scale)), 0, 15)      (all in fp32, IEEE rounding;
 *     a scale below the smallest normal number counts as 0, and then every code is 0;
 *     a row with a value that is not finite, or whose scale is not, reads back as NaN throughout)
 * in head_dim / 2 + 4 bytes: 3.76 times less than bf16 at head_dim 128.
 *
 * A page holds page_size tokens of every key/value head of one layer; pages are numbered alike in
 * all layers.  Memory order: layer, page, head, cell of 16 tokens; a cell is
 *     [16 x head_dim/2 K codes][16 x head_dim/2 V codes][16 x (scale, low) K][16 x (scale, low) V]
 * with scale and low as bf16 and, in each 32-bit word of codes, nibble n (from the low end) holding
 * element {0,2,4,6,1,3,5,7}[n] of the word's eight.
 *
 * A token's place is its slot: page * page_size + offset.  The handle keeps host-side state only
 * and is not thread-safe (as lora_pool_t).
 * -------------------------------------------------------------------------------------- */
typedef struct lora_kv lora_kv_t;

typedef struct {
    int32_t device;
    int32_t num_layers;       /* >= 1 */
    int32_t num_pages;        /* per layer; num_pages * page_size < 2^31 */
    int32_t page_size;        /* tokens: 16, 32, 64 or 128 */
    int32_t num_q_heads;      /* a multiple of num_kv_heads; at most 128 per key/value head */
    int32_t num_kv_heads;
    int32_t head_dim;         /* 64 or 128 */
    void *device_buf;         /* dev, 256-byte aligned, >= lora_kv_bytes(); caller-owned */
    size_t device_buf_bytes;
} lora_kv_desc_t;

/* Bytes of device memory the cache needs (a control block, then the layers).  device_buf is
 * ignored.  Errors: INVALID_ARG, SHAPE. */
lora_status_t lora_kv_bytes(const lora_kv_desc_t *desc, size_t *bytes);
/* Byte offset of a layer's first page inside device_buf, and the bytes of one layer. */
lora_status_t lora_kv_layer_range(const lora_kv_desc_t *desc, int32_t layer, size_t *offset, size_t *bytes);
/* Creates the handle and clears the control block (synchronous).  The pages are left as they are:
 * nothing reads a row that was not written.  Errors: INVALID_ARG, SHAPE, BUFFER_TOO_SMALL, CUDA. */
lora_status_t lora_kv_create(const lora_kv_desc_t *desc, lora_kv_t **out);
lora_status_t lora_kv_destroy(lora_kv_t *kv);

/* Device status words since creation: [0] new tokens whose slot, position or page was outside its range (they
 * are not stored or not rotated), and pages that a release could not put back (attention does not see keys in
 * pages outside the cache, and counts nothing); [1] expired device-side waits (that call's outputs are not to be
 * trusted), [2..3] reserved.  Synchronises `stream`; returns LORA_ERR_TIMEOUT when word 1 is non-zero.
 * words_out (host, [4]) may be NULL. */
lora_status_t lora_kv_check_status(lora_kv_t *kv, void *stream, int32_t *words_out);

/*
 * Tables of one batch of R requests that bring T new tokens in all, request r's q_len[r] tokens
 * after the kv_len[r] it has in the cache (either may be 0).  Takes the pages that the new tokens
 * need from a stack of free pages and writes, in `tables`, all int32, in this order:
 *   header[16]    {R, T, sum of q_len, failed requests, negative lengths, pages taken, 0 ..}
 *   start[R + 1]  first token of each request; start[R] = sum of q_len (no entry exceeds T)
 *   kv_len[R]     lengths after the batch
 *   position[T]   a token's position in its request (0 behind the last request's tokens)
 *   slot[T]       its place in the cache, -1: none
 *   (then words private to the library; lora_kv_tables_bytes counts them)
 * Page k of the batch (k = 0, 1, .. in request order) is free_pages[*free_count - 1 - k]; block_table
 * [r, i] (row r at r * ld_table, i = page number inside the request) is written for new pages and
 * read for old ones.  A request gets all the pages it needs or fails: a request that needs pages
 * fails once the pages needed up to and including it exceed the stack; so does one that needs more
 * than ld_table pages, has more than max_q new tokens or tokens past T (so do all behind that one, idle ones
 * too).  A failed request keeps its
 * length, its slots are -1 and its attention is zero.  A negative length counts as 0.
 * kv_len_out [R] and free_count_out [1] may be the inputs themselves or NULL.  window: 0, or how many
 * keys a query sees, itself included (for the attention calls on these tables).  max_q bounds the
 * batch's q_len; batches of single tokens (max_q = 1) skip what only prompts need.  0 = T.
 * R <= 4096.  The result is an exact integer function of its inputs.
 * Errors: INVALID_ARG, SHAPE, BUFFER_TOO_SMALL, CUDA.
 */
lora_status_t lora_kv_tables_bytes(const lora_kv_t *kv, int32_t R, int32_t T, size_t *bytes);
lora_status_t lora_kv_build_tables(lora_kv_t *kv, const int32_t *kv_len, const int32_t *q_len,
                                   int32_t R, int32_t T, int32_t max_q, int32_t window,
                                   const int32_t *free_pages, const int32_t *free_count,
                                   int32_t *block_table, int64_t ld_table,
                                   int32_t *kv_len_out, int32_t *free_count_out,
                                   void *tables, size_t tables_bytes, void *stream);

/* Gives the pages of n requests (dev int32 ids; an id outside 0 .. R - 1, a second mention and a page
 * outside the cache are skipped) back to the stack: request by request in the order of the list, each
 * one's pages in their order.  Their kv_len becomes 0 and their block-table entries -1.  A stack that
 * would pass num_pages entries is cut there (a page was given back twice) and counted in status word 0.
 * n <= 4096. */
lora_status_t lora_kv_release(lora_kv_t *kv, const int32_t *requests, int32_t n, int32_t R,
                              int32_t *kv_len, int32_t *block_table, int64_t ld_table,
                              int32_t *free_pages, int32_t *free_count, void *stream);

/*
 * Norm and rotation of the queries and keys of T tokens, per head h of head_dim values x:
 *     y_i = x_i * (1 / sqrt(mean(x^2) + eps)) * weight_i            (skipped where weight is NULL)
 *     (y_a, y_b) -> (y_a c - y_b s, y_b c + y_a s)                  (skipped where cos_sin is NULL)
 * in fp32, every operation rounded by itself (no fused multiply-add), the sum of squares taken as a
 * tree: x_i^2 + x_{i + head_dim/2}^2 first, then neighbours with neighbours; so the result, and the
 * 4-bit code of a key, does not depend on how the work is split.  Rounded once to bf16 at the store.
 * cos_sin: fp32 [num_positions, rot_dim], rot_dim/2 cosines, then rot_dim/2 sines; pair p is elements
 * (p, p + rot_dim/2), or (2p, 2p + 1) when interleaved; elements from rot_dim on are not rotated.
 * q, k, v rows start at t * ld (elements) and hold heads * head_dim values each; they may be parts of
 * one fused projection's rows.  q_out may be q and k_out may be k (same leading dimension).
 */
typedef struct {
    int32_t device;
    int32_t num_q_heads, num_kv_heads, head_dim;   /* head_dim 64 or 128; either count may be 0 */
    int32_t rot_dim, interleaved;                  /* rot_dim: a multiple of 16, <= head_dim */
    float eps;
    int32_t num_positions;
    const void *q;  int64_t ldq;                   /* dev bf16 */
    const void *k;  int64_t ldk;
    const void *v;  int64_t ldv;                   /* read by lora_kv_append only */
    const void *q_weight, *k_weight;               /* dev bf16 [head_dim] or NULL */
    const float *cos_sin;                          /* dev or NULL */
    const int32_t *positions;                      /* dev [T]; needed with cos_sin */
    void *q_out;    int64_t ldqo;                  /* dev bf16, or NULL with num_q_heads = 0 */
    void *k_out;    int64_t ldko;                  /* may be NULL in lora_kv_append */
} lora_qk_args_t;
/* A token whose position is outside 0 .. num_positions - 1 is not rotated.
 * Errors: INVALID_ARG, SHAPE, CUDA. */
lora_status_t lora_qk_norm_rope(const lora_qk_args_t *args, int32_t T, void *stream);
/* The same pass; the keys (before their rounding to bf16) and the values also go to their slots of
 * `layer` as 4-bit rows.  slots: dev int32 [T], -1 = not stored; two tokens with one slot leave that
 * row undefined.  The heads must be the cache's.  Errors: INVALID_ARG, SHAPE, SLOT_RANGE (layer), CUDA. */
lora_status_t lora_kv_append(lora_kv_t *kv, int32_t layer, const lora_qk_args_t *args,
                             const int32_t *slots, int32_t T, void *stream);
/* Rows of the cache as bf16, one per slot (zeros for a slot that is -1 or outside the cache): k_out
 * and v_out are [n, num_kv_heads * head_dim] with leading dimensions; either may be NULL. */
lora_status_t lora_kv_read(lora_kv_t *kv, int32_t layer, const int32_t *slots, int32_t n,
                           void *k_out, int64_t ldk, void *v_out, int64_t ldv, void *stream);

/*
 * Attention of a batch over one layer of the cache: for token t of request r at position p and query
 * head h, over the keys j in [max(0, p + 1 - window), p] of r that key/value head h / (num_q_heads /
 * num_kv_heads) holds,
 *     out[t, h] = sum_j softmax_j(scale * q[t, h] . k_j) v_j ,   lse[t, h] = log sum_j exp(scale * q . k_j)
 * with k and v the values that the cache's rows stand for.  Call it after the batch's keys have been
 * appended.  Queries of tokens without a request, of a failed request or without a key give zeros and lse =
 * -inf; a key in a page outside the cache is not seen.  q, out: dev bf16 [T, num_q_heads * head_dim] with
 * leading dimensions; rows of out may lie beside rows of q (one leading dimension), but not on them; lse:
 * dev fp32 [T, num_q_heads] or NULL.  tables: as written by lora_kv_build_tables for this R and T (and
 * through this handle, which knows the 256 buffers that it wrote tables to last), block_table the one it
 * was given.  A row of the cache that is not finite makes the outputs that see it NaN and no others.
 * Statistics and sums are fp32.  Both products run on tensor cores with fp16 operands and fp32 sums:
 * queries, codes and scales enter exactly (what is 2^-17 of its row's, of its request's largest so far, or
 * smaller loses bits below 2^-25 of that), a probability times its value row's scale is rounded to 11 bits,
 * or to 2^-33 of the largest probability times the largest scale (or |low| / 16) where that is more; in
 * requests with more than 64 rows (q_len * num_q_heads / num_kv_heads) a probability is rounded to 11 bits,
 * or to 2^-33 of the largest where that is more, and the values to 11 bits, or to 2^-23 of the request's
 * largest scale or |low| so far.  The other requests' codes enter as subnormal numbers, which costs their
 * sums bits: a score is good to about 2^-14 of the row's largest |q| times the key's scale (times scale;
 * 2^-17 is usual), an output to about 2^-13 of the largest probability times its scale (2^-19 is usual).
 * Queries beyond 2^110 count as infinite.  The result does not depend on timing.  scale is finite, and so
 * is scale * log2(e).  Calls on one workspace must be ordered on one stream; the workspace's contents are
 * undefined afterwards.
 * Errors: INVALID_ARG, SHAPE, SLOT_RANGE (layer), BUFFER_TOO_SMALL (workspace), CUDA.
 */
lora_status_t lora_kv_workspace_bytes(const lora_kv_t *kv, size_t *bytes);
lora_status_t lora_kv_attention(lora_kv_t *kv, int32_t layer, const void *q, int64_t ldq,
                                void *out, int64_t ldo, float *lse, float scale,
                                const void *tables, int32_t R, int32_t T,
                                const int32_t *block_table, int64_t ld_table,
                                void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LORA_B200_H */
