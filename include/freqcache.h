/* freqcache -- C ABI of the MI355X (gfx950) frequency-aware software cache for large
 * embedding tables, after arXiv:2208.05321 ("A Frequency-aware Software Cache for Large
 * Recommendation System Embeddings").
 *
 * The library keeps the whole embedding table in pinned host memory, re-ordered by
 * descending id frequency ("CPU Weight", paper Section 4.2), and `cache_rows` of its rows
 * in HBM ("CUDA Cached Weight", Section 4.3).  Once per training iteration the caller
 * turns the batch's ids into row indices of the cached weight (Algorithm 1,
 * PrepareCache), runs the EmbeddingBag-sum forward on the cached rows and applies the
 * sparse SGD update to them (Section 4.3, last step of the workflow; synchronous
 * updates, Section 2.2).  Every step runs in hand-written HIP kernels, on the caller's
 * stream unless stated otherwise: three library-owned streams carry the write-back of
 * evicted rows, the sort the backward pass needs, and -- with cache_plan_next or
 * cache_prepare_next -- the next batch's index work and row fetch beside the current batch.
 *
 * Conventions
 *   - every function returns FC_OK (0) or a negative FC_ERR_* code; nothing throws or aborts;
 *   - pointers named *_dev are device pointers owned by the caller (e.g. PyTorch tensors),
 *     pointers named *_host are ordinary host pointers owned by the caller;
 *   - one handle = one table = one GPU (the device current at cache_create); a handle is
 *     not thread-safe and calls on one handle must not overlap;
 *   - ids are already offset into the single concatenated table (Section 5.1);
 *   - int32 row indices internally: num_rows < 2^31 - 2^16, n < 2^31 - 2^16.
 *
 * There is no CPU fallback: if no HIP device is usable the calls fail with FC_ERR_HIP.
 */
#ifndef FREQCACHE_H
#define FREQCACHE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct fc_cache fc_cache; /* opaque, owned by the library */

/* Observables of the most recent successful cache_prepare (Algorithm 1). */
typedef struct fc_stats {
    int64_t n_ids;        /* ids in the batch                                            */
    int64_t n_unique;     /* distinct rows the batch touches (|unique(idx_map[ids])|)    */
    int64_t n_hit_unique; /* of those, already resident                                  */
    int64_t n_hit_ids;    /* ids whose row was already resident (access-level hits)      */
    int64_t n_miss;       /* rows moved host -> HBM                                      */
    int64_t n_evict;      /* rows evicted (all written to the host table unless FC_DIRTY_TRACK) */
    int64_t bytes_h2d;    /* n_miss  * dim * 4                                           */
    int64_t bytes_d2h;    /* n_evict * dim * 4 (FC_DIRTY_TRACK: dirty victims * dim * 4)  */
} fc_stats;

enum {
    FC_OK = 0,
    FC_ERR_INVALID_ARG = -1,
    FC_ERR_ID_OUT_OF_RANGE = -2,     /* an id outside [0, num_rows)                               */
    FC_ERR_BAD_OFFSETS = -3,         /* offsets[0] != 0, offsets[num_bags] != n, or not monotone  */
    FC_ERR_BATCH_EXCEEDS_CACHE = -4, /* more distinct rows in the batch than cache_rows           */
    FC_ERR_NOT_PERMUTATION = -5,     /* freq_rank is not a permutation of [0, num_rows)           */
    FC_ERR_OOM_DEVICE = -6,
    FC_ERR_OOM_PINNED = -7,
    FC_ERR_HIP = -8,                 /* a HIP runtime call failed, or no usable device            */
    FC_ERR_NOT_PINNED = -9,          /* host_weight given but not page-locked, GPU-mapped memory  */
    FC_ERR_BAD_SLOT = -10,           /* a slot index outside [0, cache_rows) reached fwd / bwd     */
    FC_ERR_SCRATCH_EXCEEDED = -11,   /* embedding_bag_bwd_sgd_noalloc: the batch needs more than its fixed scratch */
    FC_ERR_COUNT_OVERFLOW = -12      /* freq_add: more than 2^31 - 1 ids in all would overflow the 32-bit counters */
};

/* Limits of embedding_bag_bwd_sgd_noalloc (below). */
#define FC_NOALLOC_MAX_IDS 524288                 /* lookups per call                                     */
#define FC_NOALLOC_SCRATCH_BYTES (20 * 1048576)   /* size of the library's fixed scratch array, per GPU   */

/* cache_create flags */
enum {
    FC_WARM = 1,            /* preload the cache_rows highest-frequency rows (Section 4.3, "cache warm-up") */
    FC_TRANSMIT_STAGED = 2, /* move rows the way the paper's data transmitter does (Section 4.3):
                               gather into a contiguous block on the source side, one bulk
                               hipMemcpyAsync over the host link, scatter on the target side.
                               Default (flag clear): kernels read / write the mapped pinned table
                               directly, one row-group of lanes per row.  Results are identical. */
    FC_EVICT_DMA = 4,       /* evicted rows only: the block leaves HBM by hipMemcpyAsync on the side stream (DMA
                               engine, full duplex with the miss fill, no compute units involved; the few rows of a small
                               batch are stored into the pinned block by the kernel that gathers them) and library-owned
                               host threads scatter it into the host table in the background (block transmitter of
                               Section 4.3 for the device -> host direction).  Misses are still read by kernels.
                               The host table is complete after cache_flush (or cache_check).  Number of threads:
                               environment variable FC_SCATTER_THREADS (default 8).  Not with FC_TRANSMIT_STAGED.
                               Results are identical. */
    FC_NO_PRESORT = 8,      /* By default cache_prepare also enqueues the sort of the batch's (slot, bag) pairs that
                               embedding_bag_bwd_sgd needs (cache_prepare_next and cache_plan_next on a library-owned
                               stream); it reads slots_dev and offsets_dev until it is done.  Set this flag when
                               no backward pass follows (inference) or those buffers are reused at once. */
    FC_INPUTS_READY = 32,   /* A promise about cache_plan_next's inputs: ids_dev / offsets_dev are complete when the call is made
                               (resident batches, or uploads the caller has waited for), not merely enqueued on the caller's
                               stream.  The library then starts the index work of the planned batch without waiting for the
                               caller's stream at all (only the slot write-out and the sort still wait for the backward pass
                               that last read those buffers), which puts the planned batch's index decisions and row fetch a
                               whole step ahead of cache_advance, and lets the sort's later passes run on the stream of the
                               evicted-row block instead of holding up the next batch's index kernels.  That pays where HBM
                               binds the step (large batches, high hit ratio); where the host link binds it, the extra overlap
                               slows the link transfers down, so the library runs ahead only while the previous batch missed
                               at most FC_AHEAD_MISS_PCT (default 2) rows per 100 of (lookups + bags) / 2, the point where
                               the link's bytes take as long as HBM's.  Results are unchanged.  Ignored with FC_DIRTY_TRACK. */
    FC_MISS_DMA = 64,       /* cache_plan_next only, with FC_EVICT_DMA or the default transmitter: the planned batch's missing rows
                               cross the link the way the paper's transmitter moves them (Section 4.3), pipelined: their list
                               is copied to the host, library-owned host threads (FC_GATHER_THREADS, default 6) gather the
                               rows from the host table into a pinned block chunk by chunk, and each chunk goes into the
                               arrival block in HBM by hipMemcpyAsync (DMA engine) on the fetch stream; no compute unit reads
                               host memory.  cache_advance waits on the host until the last chunk has been handed over.
                               Memory: two more pinned blocks of staging_rows * dim * 4 bytes.  Results are identical.
                               Ignored with FC_DIRTY_TRACK. */
    FC_DIRTY_TRACK = 16     /* Variant beyond the paper (Algorithm 1 always calls move_to_cpu): a resident row is
                               dirty once embedding_bag_bwd_sgd has updated it since it was loaded; only dirty
                               victims are written back, clean ones are dropped (their copy in the host table is
                               current), and cache_flush writes dirty rows only.  bytes_d2h counts the rows written.
                               Every other result is unchanged.  The call that moves the rows (cache_prepare,
                               cache_prepare_next, or cache_advance after cache_plan_next: what is dirty is only
                               known after the current batch's backward pass) then waits on the host once more, for
                               the number of dirty victims (cache_prepare does not with the default transmitter, nor
                               with FC_EVICT_DMA while victims come out clean and no block is on its way; rows then
                               change places in one kernel, and cache_last_stats waits for the number); after cache_plan_next, bytes_d2h of
                               cache_last_stats is final only once cache_advance has returned. */
};

/* Static module + dynamic module set-up (Sections 4.2, 4.3).
 *   num_rows, dim   table shape; fp32; 1 <= dim <= 1024.
 *   cache_rows      rows of the cached weight, 0 < cache_rows <= num_rows (the paper's cache ratio
 *                   times num_rows; 1.5% by default there).
 *   freq_rank_host  "idx_map": id -> row of the frequency-ordered table (0 = most frequent).
 *                   Host pointer, length num_rows, must be a permutation; copied.
 *   host_weight     the frequency-ordered table, num_rows*dim fp32, row r = embedding of the id with
 *                   rank r.  Either NULL -- the library allocates pinned memory, the caller fills it
 *                   through cache_host_weight() BEFORE the first cache_prepare (and before
 *                   cache_create's warm-up if FC_WARM is wanted: then create cold, fill, and call
 *                   cache_warm) -- or a pointer to page-locked, GPU-mapped memory
 *                   (hipHostMalloc / a pinned torch tensor) that outlives the handle.  The table is
 *                   the store of record: evictions and cache_flush write into it.
 *   staging_rows    bound, in rows, of the transmitter's block buffers (Section 4.3 keeps the transmitter's
 *                   memory footprint bounded); larger transfers are
 *                   done in several rounds.  0 = default (min(cache_rows, 524288)).  Memory, in blocks of
 *                   staging_rows * dim * 4 bytes: one in HBM by default; with FC_TRANSMIT_STAGED two in
 *                   HBM and one pinned; with FC_EVICT_DMA four in HBM and four pinned; cache_plan_next
 *                   adds two in HBM on first use.
 *   flags           any of FC_WARM, FC_TRANSMIT_STAGED, FC_EVICT_DMA, FC_NO_PRESORT, FC_DIRTY_TRACK, FC_INPUTS_READY, FC_MISS_DMA.
 *   hip_stream      hipStream_t on which all per-batch work is enqueued (NULL = default stream).
 *   out             receives the handle.
 * Errors: INVALID_ARG, NOT_PERMUTATION, NOT_PINNED, OOM_DEVICE, OOM_PINNED, HIP.  Synchronous (it also runs a few
 * sub-millisecond test kernels on hip_stream to find library streams that run beside it; and with FC_EVICT_DMA and blocks of 1 MB or
 * more, the first handle of a process on a device copies a few dozen blocks of up to 4 MB, about 20 ms, so that the runtime sets up
 * its copy engines here and not among the first training steps).
 * Tuning knobs, read from the environment at this call (defaults suit an MI355X on a PCIe Gen5 x16 link):
 *   FC_FILL_BLOCKS        workgroups of the miss fill (40 with FC_EVICT_DMA, else 256), also where cache_plan_next fetches few rows (1.5 MB in
 *                         the batch before, 3 MB at most) on its index stream (there up to 200 for rows that leave lanes idle)
 *   FC_FILL_BLOCKS_EARLY  workgroups of cache_plan_next's early row fetch on a stream of its own, fixed (default: starts at 32 and follows the
 *                         measured fetch / block-copy durations); FC_FILL_BLOCKS_EARLY_START only moves the start
 *   FC_EVICT_BLOCKS, FC_EVICT_EARLY   width and start of the host-table store kernel (without FC_EVICT_DMA: after cache_plan_next,
 *                         or cache_prepare_next with FC_DIRTY_TRACK, otherwise rows change places in the miss fill; with it: more victims than staging_rows)
 *   FC_SCATTER_THREADS    host threads of FC_EVICT_DMA (8)
 *   FC_GATHER_THREADS     host threads of FC_MISS_DMA (6)
 *   FC_AHEAD_MISS_PCT     threshold of FC_INPUTS_READY (see there); 0 = never run ahead, 100 = always
 *   FC_SORT_TAIL          0: with FC_INPUTS_READY the whole sort stays on the index stream (default 1: passes after the first
 *                         on the side stream)
 *   FC_FWD_SORTED         0: batches with one lookup per bag are always pooled in bag order (default 1: in slot order, from
 *                         the pairs cache_prepare has sorted ahead of time for the backward pass, when those are at hand)
 *   FC_FWD_BAGS           bags per row-group of the bag-order forward kernel for one-lookup bags: 1, 2 or 4 (4); batches of
 *                         fewer than 768 workgroups take one
 *   FC_SORT_BITS          most key bits per pass of the backward's sort (4..11; default: passes of up to 9 bits without a
 *                         scan kernel); FC_SORT_FUSED=0 keeps the scan kernel
 *   FC_FETCH_CU_MASK      experiment: number of compute units the early fetch's stream may use (default: all)
 *   FC_MARK_BYTES         0: marks are bits, as they are where device memory has no room for a byte per row (see cache_reserve)
 *   FC_MARK_DENSE         ranks per id of a batch whose marks are read one and all, not chunk by chunk (4)
 *   FC_PLAN_FOLD_TILES    most tiles of 32768 ranks for which the emitting kernel has eight workgroups to a tile (1024), else one
 *   FC_SMALL_INDEX        0: small batches (up to 4096 ids, 2^20 rows, 2^16 slots) are indexed by the general kernels, too
 *   FC_TUNE_REPORT        if set, cache_destroy prints where the early-fetch workgroup count settled
 *   FC_TIMELINE           file that receives, whenever profiling totals are collected, one line "name start_us end_us"
 *                         per timed kernel or copy (read at every collection, not here) */
int cache_create(int64_t num_rows, int32_t dim, int64_t cache_rows, const int32_t* freq_rank_host,
                 float* host_weight, int64_t staging_rows, int32_t flags, void* hip_stream, fc_cache** out);

/* Allocate now everything the per-batch calls would otherwise allocate when they first meet a batch of that size:
 * the per-id rank buffer of cache_prepare and its byte marks (num_rows * 257 / 256
 * bytes, which a batch allocates that is not indexed by one workgroup; where there is no room for them the marks are bits, and no
 * call fails for it), the
 * sort scratch and partial-sum rows of embedding_bag_bwd_sgd for batches of up to max_ids lookups (three sort sets of 16 * max_ids bytes), and, if pipelined != 0 (a handle that will plan ahead), the two arrival blocks of
 * cache_plan_next (staging_rows * dim * 4 bytes each).  The transmitter's memory stays bounded by staging_rows
 * (Section 4.3); this call only moves the allocations out of the training loop.  Optional: without it (or for a larger
 * batch later) the buffers grow on demand, which costs a hipMalloc and a device-wide synchronisation in that step.
 * Synchronous.  Errors: INVALID_ARG, OOM_DEVICE, HIP. */
int cache_reserve(fc_cache* c, int64_t max_ids, int32_t pipelined);

/* Cache warm-up (Section 4.3): empty the cache and load rows 0..cache_rows-1 of the host table into
 * slots 0..cache_rows-1.  cache_create(FC_WARM) calls this.  Synchronous.  Does not write back
 * resident rows first (call cache_flush if they carry updates). */
int cache_warm(fc_cache* c);

/* Algorithm 1 (PrepareCache + PrepareCPURowIdxOnGPU): make every row the batch needs resident and
 * return, per input id, its row index in the cached weight.
 *   ids_dev      int64[n], device.           offsets_dev  int64[num_bags+1], device, bag b = ids
 *   slots_dev    int32[n], device, output.                [offsets[b], offsets[b+1]) (EmbeddingBag).
 * Steps, all on the GPU: ids -> frequency rank; distinct ranks; split into resident / missing; if the
 * missing rows outnumber the empty slots, evict that many resident rows not used by this batch,
 * largest rank (least frequent) first, writing them back to the host table; assign the i-th smallest
 * missing rank to the i-th smallest empty slot and load it from the host table.
 * On return the index decisions are final and the error code is known (the call waits for the
 * planning kernels, a few microseconds of GPU work); row movement and the slot write-out are enqueued
 * on the stream, so later work on the same stream sees every needed row resident.
 * Errors: INVALID_ARG, BAD_OFFSETS, ID_OUT_OF_RANGE, BATCH_EXCEEDS_CACHE (in this order of precedence),
 * OOM_DEVICE, HIP.  On any error the cache state is unchanged and slots_dev is unspecified. */
int cache_prepare(fc_cache* c, const int64_t* ids_dev, int64_t n, const int64_t* offsets_dev, int64_t num_bags,
                  int32_t* slots_dev);

/* Look-ahead (the paper's Future Work section proposes prefetching on the ids of coming batches): Algorithm 1 for the
 * NEXT batch, issued while the batch of the latest cache_prepare / cache_prepare_next is still being trained on.
 * Same arguments, results and errors as cache_prepare, with two differences:
 *   - the rows of that previous batch are protected from eviction as well (the backlist of Algorithm 1 is the union
 *     of both batches), so the forward / backward calls of the previous batch may be enqueued after this call; if too
 *     few evictable rows remain the call fails with FC_ERR_BATCH_EXCEEDS_CACHE and changes nothing (the caller then
 *     finishes the current batch and uses cache_prepare);
 *   - the work is enqueued on a library-owned stream and overlaps the caller's stream; ids_dev / offsets_dev must be
 *     complete on the caller's stream at the time of the call and stay untouched until cache_advance.
 * Usage:  cache_prepare(batch 0);  loop { cache_prepare_next(batch t+1, slots_next); fwd(t); bwd(t); cache_advance(); } */
int cache_prepare_next(fc_cache* c, const int64_t* ids_dev, int64_t n, const int64_t* offsets_dev, int64_t num_bags,
                       int32_t* slots_dev);
/* Software pipelining WITHOUT a change of policy: the index half of cache_prepare for the NEXT batch (ids -> ranks,
 * unique rows, misses, victims, slot assignment, the slots of the batch, the sort for its backward pass), enqueued on
 * a library-owned stream beside whatever the caller's stream still runs for the current batch: the arrival of its
 * missing rows, its forward and its backward pass.  None of these decisions depends on embedding values, so the
 * results (slots, statistics, lists, maps) are exactly those of cache_prepare called after the current batch's
 * backward pass.  No row is moved: cache_advance does that, on the caller's stream, i.e. after the backward pass the
 * caller enqueued in between.
 * Same arguments and errors as cache_prepare; not available with FC_TRANSMIT_STAGED.
 * Ordering (without FC_INPUTS_READY): the index work is ordered behind the caller's stream as of the ENTRY of the latest
 * cache_prepare / cache_advance call, not as of this call.  ids_dev / offsets_dev must therefore be complete by then (written by work
 * enqueued on the caller's stream before that call, or finished altogether) and stay untouched until cache_advance;
 * slots_dev must not be the buffer the current batch's forward / backward read.  cache_copy_rows / cache_host_weight
 * reflect the planned batch only after cache_advance.  (The first call of this kind on a handle, unless cache_reserve has announced
 * it with pipelined != 0, is ordered behind everything on the caller's stream instead: until then plain calls mark no place there.)
 * Usage:  cache_prepare(batch 0);  loop { fwd(t); bwd(t); cache_plan_next(batch t+1, slots_next); cache_advance(); }
 * (forward / backward are asynchronous and best enqueued first, since this call waits on the host for its planning
 * kernels; those do not wait for them.  Calling it before them is equally correct.  With FC_EVICT_DMA it also waits for the last
 * evicted block if that is long overdue, which keeps a program with several handles from getting many steps ahead of the link.)
 * The call also starts fetching the planned batch's missing rows, on another library-owned stream, into a block in
 * device memory (allocated on first use, staging_rows rows per list set); cache_advance then writes the evicted
 * rows out and copies the fetched rows into their slots. */
int cache_plan_next(fc_cache* c, const int64_t* ids_dev, int64_t n, const int64_t* offsets_dev, int64_t num_bags,
                    int32_t* slots_dev);
/* Makes the batch of the latest cache_prepare_next / cache_plan_next the current one (for cache_plan_next this is
 * where its evicted rows leave and its missing rows arrive): work enqueued on the caller's stream after this
 * call sees its rows resident and its slots written.  Asynchronous (a stream-to-stream dependency). */
int cache_advance(fc_cache* c);

/* EmbeddingBag, mode "sum", on the cached weight (Section 4.3: the framework's embedding op runs on the
 * cached weight after the cache step):  out[b, :] = sum_{i in bag b} cached_weight[slots[i], :], summed
 * in position order; an empty bag gives zeros.
 *   slots_dev int32[n] as returned by the latest cache_prepare; out_dev fp32[num_bags*dim], device.
 * Asynchronous on the stream.  A slot outside [0, cache_rows) contributes nothing and raises a sticky
 * FC_ERR_BAD_SLOT reported by cache_check. */
int embedding_bag_fwd(fc_cache* c, const int32_t* slots_dev, int64_t n, const int64_t* offsets_dev,
                      int64_t num_bags, float* out_dev);

/* Backward of the sum-bag fused with the SGD step (synchronous update, Section 2.2): for every distinct
 * slot s, g = sum over the lookups i with slots[i] == s of grad_out[bag(i), :] (a row looked up k times
 * receives k gradients), then cached_weight[s, :] -= lr * g.  Deterministic: no floating-point atomics;
 * lookups of a slot are summed in position order within fixed blocks of consecutive lookups (8 or 32, by the size of the batch), the
 * blocks' sums in levels.
 *   grad_out_dev fp32[num_bags*dim], device.  Asynchronous on the stream; BAD_SLOT as above. */
int embedding_bag_bwd_sgd(fc_cache* c, const int32_t* slots_dev, int64_t n, const int64_t* offsets_dev,
                          int64_t num_bags, const float* grad_out_dev, float lr);

/* embedding_bag_bwd_sgd for callers that cannot allocate device memory: code under HIP graph capture, tight serving
 * or training loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and bit-identical results, but the
 * call allocates nothing (no hipMalloc / hipFree, no event creation): the sort buffers, radix histograms and partial
 * rows it needs live in a fixed array of FC_NOALLOC_SCRATCH_BYTES bytes of device memory that is part of the library's
 * code object (every GPU the library runs on holds one copy until the process ends; cache_create looks its address up).
 * Limits: n <= FC_NOALLOC_MAX_IDS lookups, and 10.5 MB + blocks * (16 + 8 * dim) bytes <= FC_NOALLOC_SCRATCH_BYTES, where
 * blocks = ceil(n / 256) for dim <= 128 and ceil(n * lanes / 8192) with lanes = min(64, dim / 4) for wider rows (dim 256:
 * n <= 524288; dim 1024: n <= 150000 or so); beyond them the call returns FC_ERR_SCRATCH_EXCEEDED and does nothing.  (Batches of up to
 * min(2048, 2^20 / dim) blocks of a quarter of that many lookups are cut into those; they always fit.)
 * It never uses a sort started ahead of time by cache_prepare (create the handle with FC_NO_PRESORT to spare that work)
 * and is not covered by cache_profile_*.  All calls on one GPU, from any handle, share the one array: calls that overlap
 * on a GPU (two handles on different streams) race; the array keeps the previous call's contents, none of which the
 * next call reads before writing.  Errors: INVALID_ARG, SCRATCH_EXCEEDED, HIP; BAD_SLOT as embedding_bag_bwd_sgd. */
int embedding_bag_bwd_sgd_noalloc(fc_cache* c, const int32_t* slots_dev, int64_t n, const int64_t* offsets_dev,
                                  int64_t num_bags, const float* grad_out_dev, float lr);

/* Write every resident row back to the host table (the host table is the store of record, Section 3);
 * residency is unchanged.  Returns after the host table is complete. */
int cache_flush(fc_cache* c);

/* Wait for all enqueued work of this handle and return the sticky asynchronous error, if any
 * (then clears it). */
int cache_check(fc_cache* c);

/* Waits for outstanding work, frees everything the library allocated.  Does NOT flush. */
int cache_destroy(fc_cache* c);

/* ---- introspection (parity checks, reports) ---- */
int cache_last_stats(const fc_cache* c, fc_stats* out);
/* Copies of the two index maps (paper's cache_idx_map in both directions): slot_rank_host int32[cache_rows]
 * (-1 = empty slot), rank_slot_host int32[num_rows] (-1 = not resident); either may be NULL. Synchronous. */
int cache_copy_state(fc_cache* c, int32_t* slot_rank_host, int32_t* rank_slot_host);
/* Lists of the latest cache_prepare, each may be NULL: missing ranks (ascending, n_miss), evicted ranks
 * (ascending, n_evict) with the slots they left, and fill_slots[j] = slot that received miss_ranks[j]. */
int cache_last_lists(fc_cache* c, int32_t* miss_ranks_host, int32_t* evict_ranks_host, int32_t* evict_slots_host,
                     int32_t* fill_slots_host);
/* Copy of the cached weight, fp32[cache_rows*dim]. Synchronous. */
int cache_copy_rows(fc_cache* c, float* rows_host);
/* The pinned, frequency-ordered host table (library- or caller-allocated). */
float* cache_host_weight(fc_cache* c);
const char* cache_strerror(int code);

/* ---- static module (Section 4.2): id frequency statistics -> freq_rank, built on the GPU ---- */
typedef struct fc_freq fc_freq; /* opaque accumulator of per-id occurrence counts */

/* Zeroed counters for ids in [0, num_rows) on the current device; work is enqueued on hip_stream. */
int freq_create(int64_t num_rows, void* hip_stream, fc_freq** out);
/* counts[id] += 1 for each of the n ids (int64, device memory): one scan step over the dataset, or over a sample of
 * it when the dataset is too large (Section 4.2).  Asynchronous; ids outside [0, num_rows) are skipped and make
 * freq_build fail with FC_ERR_ID_OUT_OF_RANGE.  The counters are 32 bits wide: once the ids of all calls together would
 * exceed 2^31 - 1 the call returns FC_ERR_COUNT_OVERFLOW and counts nothing (sample the dataset instead). */
int freq_add(fc_freq* f, const int64_t* ids_dev, int64_t n);
/* Order the rows from high to low occurrence count, equal counts by lower id:
 *   freq_rank_host[id] = position of id in that order (the idx_map cache_create takes), int32[num_rows];
 *   inv_rank_host[r]   = id at position r, int32[num_rows];   counts_host[id] = its count.  Each may be NULL.
 * Synchronous; the counters stay valid (more freq_add / freq_build calls may follow). */
int freq_build(fc_freq* f, int32_t* freq_rank_host, int32_t* inv_rank_host, int32_t* counts_host);
int freq_destroy(fc_freq* f);
/* Re-order an embedding table by frequency: dst[r, :] = src[inv_rank[r], :] for r in [0, num_rows), fp32 rows of `dim`.
 * src_pinned and dst_pinned are distinct page-locked, GPU-mapped host buffers (the rows cross the host link twice);
 * inv_rank_host is an ordinary host array.  Synchronous.  Errors: INVALID_ARG, NOT_PERMUTATION, NOT_PINNED, HIP. */
int table_reorder(const float* src_pinned, float* dst_pinned, const int32_t* inv_rank_host, int64_t num_rows,
                  int32_t dim, void* hip_stream);

/* ---- operators beside the cached table ----
 * A model has small tables and dense layers beside the one behind the cache: positions, item types, words; norms; gradients
 * that are clipped together.  These calls work on the caller's device memory, in the model's types, on the stream of their handle; the
 * results are complete in the order of that stream.  Values are worked out in 32 bits (norms over tensors: 64) and rounded once, to
 * the type they are stored in.  Rows are `dim` neighbouring elements, `stride` elements apart (stride >= dim), and may start at any element.
 * Results are reproducible: no sum depends on the order in which workgroups run.  Rows, tokens: below 2^31 - 2^16; dim: up to 2^20. */
enum {                    /* element types */
    FC_TYPE_F32 = 0,
    FC_TYPE_BF16 = 1,
    FC_TYPE_F16 = 2,
    FC_TYPE_F8E4M3 = 3,   /* 8 bits: 4 of exponent, 3 of mantissa, no infinities, largest 448 (results of rms_norm_fwd) */
    FC_TYPE_I8 = 4,       /* results of rms_norm_fwd */
    FC_TYPE_I32 = 5,      /* ids */
    FC_TYPE_I64 = 6
};

typedef struct fc_dense fc_dense; /* opaque: stream, workspace, sticky error; one per stream, not thread-safe */

/* On the current device; hip_stream: hipStream_t (NULL = default stream) of all its calls. */
int dense_create(void* hip_stream, fc_dense** out);
/* Allocate now what calls up to these sizes need beyond the caller's memory: token_embed_bwd of max_tokens ids and a table of max_rows rows of max_dim
 * columns, rms_norm_bwd of any number of rows of max_dim columns, grad_norm_clip of max_tensors tensors; distill_* and beam_* of any sizes (5 MB) where max_dim > 0.  What token_embed_bwd needs grows with
 * max_tokens * max_dim: a wide norm beside a narrow table is better reserved by a call of its own (max_tokens 0), as the workspace keeps the larger of
 * the two.  Optional: the workspace grows on demand, which costs a hipMalloc and a device-wide
 * synchronisation in that call, and is refused (FC_ERR_HIP) while the stream is captured into a graph; buffers that a captured call uses stay
 * until dense_destroy, and its replays have to be in order with the handle's other work, which uses the same ones.  Synchronous.
 * Errors: INVALID_ARG, OOM_DEVICE, HIP. */
int dense_reserve(fc_dense* d, int64_t max_tokens, int64_t max_rows, int32_t max_dim, int32_t max_tensors);
/* Wait for the handle's stream and return the sticky error, if any (then clears it): FC_ERR_ID_OUT_OF_RANGE. */
int dense_check(fc_dense* d);
/* Waits for the stream, frees the workspace. */
int dense_destroy(fc_dense* d);

/* Token embedding: out[i, :] = scale * table[ids[i], :] for i in [0, n).
 *   table, out types F32, BF16 or F16 each; ids I32 or I64.
 * An id outside [0, num_rows) gives a row of zeros and raises a sticky FC_ERR_ID_OUT_OF_RANGE reported by dense_check. */
int token_embed_fwd(fc_dense* d, const void* table_dev, int32_t table_type, int64_t table_stride, int64_t num_rows, int32_t dim, const void* ids_dev,
                    int32_t id_type, int64_t n, float scale, void* out_dev, int32_t out_type, int64_t out_stride);
/* Its gradient: grad_table[v, :] = scale * sum of grad_out[i, :] over the tokens i with ids[i] == v, for every row v of the table (zeros for one
 * without tokens); with accumulate != 0 that is added to grad_table, and rows without tokens are not touched.
 *   grad_out F32, BF16 or F16; grad_table F32 or grad_out's type; n * dim below 2^36.
 * Tokens with padding_id and, with the sticky error, ids outside the table contribute nothing.  A padding_id of -1 means that there is none: ids of -1
 * are then outside, too.  Another padding_id may lie outside the table, without the error. */
int token_embed_bwd(fc_dense* d, const void* grad_out_dev, int32_t grad_out_type, int64_t grad_out_stride, const void* ids_dev, int32_t id_type, int64_t n,
                    int64_t num_rows, int32_t dim, float scale, int64_t padding_id, void* grad_table_dev, int32_t grad_table_type,
                    int64_t grad_table_stride, int32_t accumulate);

/* Root-mean-square norm of each of n rows, with the residual's addition: h = x + residual (rounded to its type; residual may be NULL),
 * y = h * (mean(h^2) + eps)^-1/2 * weight.
 *   x, residual, h: `type` (F32, BF16, F16); weight: F32 or `type`; h may be NULL (not wanted) and may be x or residual itself (same stride).
 *   y: `type`, or F8E4M3 / I8 with scales: y ~ q * scale, one scale for each `group` columns (32, 64, 128, 256; the last group may be
 *   narrower) or for the row (0): scales_dev fp32[n][ceil(dim / group)] = max |y| / (448 or 127) of the group, q = y / scale rounded to nearest, ties to
 *   even; both quotients are in 32 bits, rounded once.  Where the scale is below 1.18e-38 q = 0.  Where y holds an infinity the scale is infinite, and where it
 *   holds one that is no number the scale is none either; of such a group (row) I8 stores 0 throughout, F8E4M3 0 for finite y beside an infinity and no number
 *   for all else: it is the scale that says so for both. */
int rms_norm_fwd(fc_dense* d, const void* x_dev, int32_t type, int64_t x_stride, const void* residual_dev, int64_t residual_stride, const void* weight_dev,
                 int32_t weight_type, int64_t n, int32_t dim, float eps, void* h_dev, int64_t h_stride, void* y_dev, int32_t y_type, int64_t y_stride,
                 float* scales_dev, int32_t group);
/* Its backward pass: grad_x (the gradient of x and of residual alike) = grad_h + gradient of y's path, with grad_h what arrives at h by other
 * paths (may be NULL), and grad_weight = sum over the rows (zeros for n = 0; not accumulated).
 *   grad_y, h (as the forward pass stored it, or x without a residual), grad_h, grad_x: `type`; grad_weight: F32, BF16 or F16.
 *   grad_x may be grad_y or grad_h itself (same stride). */
int rms_norm_bwd(fc_dense* d, const void* grad_y_dev, int64_t grad_y_stride, const void* h_dev, int32_t type, int64_t h_stride, const void* weight_dev,
                 int32_t weight_type, const void* grad_h_dev, int64_t grad_h_stride, int64_t n, int32_t dim, float eps, void* grad_x_dev,
                 int64_t grad_x_stride, void* grad_weight_dev, int32_t grad_weight_type);

/* Global norm of `count` tensors (sizes[k] contiguous elements of types[k]: F32, BF16, F16), and clipping by it:
 *   norm_dev[0] = N = sqrt(sum of all squares);  out[k] = grads[k] * min(1, max_norm / (N + 1e-6)).
 * grads_dev, out_dev, sizes, types are host arrays, read before the call returns; out_dev NULL: in place (tensors are then
 * left alone where the factor is 1).  Tensors must not overlap, except that out[k] may be grads[k].  max_norm > 0; infinity: nothing is scaled.
 * A norm that is infinite or no number makes the factor 0 or no number, as the formula says. */
int grad_norm_clip(fc_dense* d, const void* const* grads_dev, void* const* out_dev, const int64_t* sizes, const int32_t* types, int32_t count,
                   float max_norm, float* norm_dev);

/* Distillation from a teacher's top logits, with cross entropy beside it.  Row i has logits x (of `type`, dim of them: the vocabulary), `top` entries of the teacher
 * (ids t_k, logits z_k; an id of -1: no entry; 0 <= top <= 1024) and, if targets are given, an id y.  With T = temperature (1/1024 to 1024), a = alpha (0 to 1):
 *   P_k = exp(z_k / T - L), where L = teacher_lse[i] is the logarithm of the sum of exp(z / T) over the teacher's whole vocabulary, and P_0 = max(0, 1 - sum P_k) is what
 *         the entries leave over;  teacher_lse NULL: L is that of the row's entries, and P_0 = 0
 *   Q = softmax(x / T), Q_0 = the sum of Q over the ids that no entry names
 *   loss[i] = a T^2 (sum P_k (log P_k - log Q[t_k]) + P_0 (log P_0 - log Q_0)) + (1 - a) (-log softmax(x)[y])
 * Sums are over the row's entries: an id that is named twice counts twice among P, and once among those that Q_0 leaves out.  Terms with P = 0, and with a factor a or 1 - a of 0, are 0.
 * Of a teacher whose entries hold everything P_0 is what roundings leave over: where Q_0 is 0 in 32 bits a P_0 of no more than 2^-23 (|L| + |max z / T - L| + top / 64 + 16) counts as 0.
 * (A larger one makes the loss infinite where the other ids are masked by -infinity, and as large as the mask where that is finite.)  A row without
 * entries (or, without teacher_lse, with entries of -infinity only) has no first term (and is left out where a is 1).  A target of -1 leaves the row out: its loss and gradient are 0, whatever its
 * logits hold; other ids outside [0, dim) raise the sticky FC_ERR_ID_OUT_OF_RANGE, an entry then does not count, and a row with such a target is left out.
 * Logits of -infinity are ids of probability 0; rows with logits that are +infinity, no number or all -infinity have a loss and a gradient that are no numbers.  Finite logits count wherever they
 * are: ids masked by -1e10 or by the type's lowest value have a probability of 0 too, but where all are that, equal ones; a loss beyond the range of 32 bits is infinite.  targets may be NULL where alpha is 1.
 *   type, teacher_type F32, BF16, F16; id_type (teacher_ids [n][top]) and target_type I32 or I64; loss fp32[n];
 *   stats fp32[n][12]: what distill_bwd needs of the forward pass (of no meaning otherwise). */
int distill_fwd(fc_dense* d, const void* logits_dev, int32_t type, int64_t logits_stride, int64_t n, int32_t dim, const void* teacher_ids_dev, int32_t id_type,
                const void* teacher_dev, int32_t teacher_type, int32_t top, const float* teacher_lse_dev, const void* targets_dev, int32_t target_type,
                float temperature, float alpha, float* loss_dev, float* stats_dev);
/* Its backward pass: grad_logits[i] = grad_loss[i * grad_loss_stride] * the gradient of loss[i], of the logits' type.
 *   grad_loss_stride 1, or 0: one number for all rows.  A row whose grad_loss is 0 gets zeros, whatever its logits hold.  The other arguments are those of the forward call;
 *   grad_logits may be logits itself (same stride). */
int distill_bwd(fc_dense* d, const float* grad_loss_dev, int64_t grad_loss_stride, const void* logits_dev, int32_t type, int64_t logits_stride, int64_t n, int32_t dim,
                const void* teacher_ids_dev, int32_t id_type, const void* teacher_dev, int32_t teacher_type, int32_t top, const void* targets_dev, int32_t target_type,
                float temperature, float alpha, const float* stats_dev, void* grad_logits_dev, int64_t grad_logits_stride);
/* Both in one call, where grad_loss is known beforehand (1 / n for a mean): the same loss and gradient but for the roundings of sums, which are added up in another order for some sizes. */
int distill_grad(fc_dense* d, const float* grad_loss_dev, int64_t grad_loss_stride, const void* logits_dev, int32_t type, int64_t logits_stride, int64_t n, int32_t dim,
                 const void* teacher_ids_dev, int32_t id_type, const void* teacher_dev, int32_t teacher_type, int32_t top, const float* teacher_lse_dev,
                 const void* targets_dev, int32_t target_type, float temperature, float alpha, float* loss_dev, void* grad_logits_dev, int64_t grad_logits_stride);

/* One step of beam search: of the candidates (w, v) of each of `batch` sequences,
 *   c = scores[w] + x[w][v] - log(sum over u of exp(x[w][u])),   of a beam with finished[w] != 0 only (w, eos_id) with c = scores[w],
 * the `keep` largest in descending order: scores_out, parents_out (w), tokens_out (v), [batch][keep] each.  Of equal ones the lower beam comes first, then the larger
 * logit, then the lower id.  Candidates are compared in 64 bits, but the log-sum of a beam, which its candidates share, is made of sums in 32 and is off by some 1e-7 (at most 1e-5), whatever the logits
 * have in common: candidates of different beams that are closer than that may come in either order.  Scores are rounded to 32 bits when stored.
 *   logits of `type` (F32, BF16, F16), batch * beams rows; scores fp32[batch][beams]; beams, keep: 1 to 64; tokens I32 or I64.
 *   finished uint8[batch][beams], may be NULL; finished_out uint8[batch][keep] = (token == eos_id), may be NULL; eos_id -1: none, then both are NULL.
 * A logit of -infinity is no candidate.  A beam whose score is -infinity has none (its logits are not read), nor has one whose score is +infinity or no number or whose
 * logits hold a +infinity or one that is no number.  Finite logits count wherever they are: ids masked by -1e10 or by the type's lowest value are candidates, far down, and where all of a beam's are
 * that, equal ones (a score below the lowest number of 32 bits is stored as -infinity).  Where fewer than `keep` candidates are left the remaining places hold score -infinity, parent 0, token max(eos_id, 0). */
int beam_select(fc_dense* d, const void* logits_dev, int32_t type, int64_t logits_stride, int64_t batch, int32_t beams, int32_t dim, const float* scores_dev,
                const uint8_t* finished_dev, int32_t eos_id, int32_t keep, float* scores_out_dev, int32_t* parents_out_dev, void* tokens_out_dev, int32_t token_type,
                uint8_t* finished_out_dev);
/* A tensor of beam_reorder: rows of `pieces` pieces of piece_bytes bytes each, of any type; row r begins src_row * r bytes from src, piece p of it src_piece * p bytes on
 * (pieces of a row, and rows, do not overlap).  The same for dst. */
typedef struct {
    const void* src;
    void* dst;
    int64_t src_row, dst_row, src_piece, dst_piece;
    int64_t piece_bytes, pieces;
} fc_state;
/* Reordering of the states of beams: for every tensor, row b * keep + j of dst = row b * beams + parents[b][j] of src.  parents [batch][keep], I32 or I64; beams, keep: 1 to 64.
 * dst may be src (then keep == beams, and the strides are the same): rows that are their own parent are not touched.  Tensors do not overlap otherwise, and none that is written overlaps
 * the parents (dst == parents_dev is refused).
 * A parent outside [0, beams) raises the sticky FC_ERR_ID_OUT_OF_RANGE; its row of dst becomes zeros, in place it stays as it was.  `states` is a host array, read before the call
 * returns; pieces and piece_bytes below 2^31, a row below 2^35 bytes. */
int beam_reorder(fc_dense* d, const fc_state* states, int32_t count, int64_t batch, int32_t beams, const void* parents_dev, int32_t parent_type, int32_t keep);

/* ---- per-kernel timing with HIP events on the handle's own streams (for the benchmark) ----
 * Each item stands for one kind of work.  While recording, what shares a launch otherwise is launched by itself: the sort of a small batch
 * ("sort_scatter") apart from its missing rows ("miss_fill"), and with FC_EVICT_DMA the evicted block of a small batch crosses the
 * link as a copy ("d2h_block"), as larger ones do, and not by the stores of its gather ("evict_gather").  Results are identical. */
int cache_profile_enable(fc_cache* c, int32_t on);   /* on=1 starts recording, 0 stops; resets totals when turned on */
int cache_profile_count(void);                        /* number of timed kernels / copies                               */
const char* cache_profile_name(int32_t k);
/* total milliseconds and number of launches of timed item k since profiling was enabled; synchronises */
int cache_profile_get(fc_cache* c, int32_t k, double* total_ms, int64_t* launches);

#ifdef __cplusplus
}
#endif
#endif /* FREQCACHE_H */
