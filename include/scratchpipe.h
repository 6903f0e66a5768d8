/*
 * scratchpipe.h - C ABI of an MI355X embedding-training scratchpad.
 *
 * The library trains embedding tables that live in host memory through a
 * GPU-resident cache (the "scratchpad": Storage plus Hit-Map, Sec. IV-D).
 * Because the sparse IDs of upcoming mini-batches are already known from the
 * training data (Sec. IV-A), every batch is planned before it is trained: its
 * missing rows are brought in and victims are chosen only among slots that no
 * batch of the look-forward window uses (Sec. IV-C), so forward and backward
 * always hit in HBM.  One training step is
 *
 *     sp_plan(window)  ->  sp_forward(ticket)  ->  sp_backward_update(ticket)
 *
 * and sp_flush() makes the host tables authoritative again.
 *
 * Conventions shared by every call:
 *  - Batches are table-major CSR: ids[] holds table 0's row IDs, then table
 *    1's, ...; bag g = t*B + b spans ids[bag_off[g] .. bag_off[g+1]); row IDs
 *    are local to their table; bag_off has T*B+1 entries, bag_off[0] = 0 and
 *    bag_off[T*B] = nnz.
 *  - Pooled outputs and their gradients are fp32 [T][B][D] in device memory
 *    owned by the caller (row g = t*B + b).
 *  - Return value: SP_OK (0) or a negative sp_status.  After SP_ERR_HIP the
 *    context is unusable and only sp_destroy is valid.  sp_last_error()
 *    describes the last failure.
 *  - One context is used from one host thread at a time.
 */
#ifndef SCRATCHPIPE_H
#define SCRATCHPIPE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t sp_status;
#define SP_OK 0
#define SP_ERR_INVALID_ARG (-1) /* bad config, bad IDs or offsets, bad pointer        */
#define SP_ERR_OOM (-2)         /* device or pinned allocation failed                  */
#define SP_ERR_CAPACITY (-3)    /* some table has more misses than unheld slots        */
#define SP_ERR_SEQUENCE (-4)    /* call out of plan -> forward -> backward order       */
#define SP_ERR_HIP (-5)         /* a HIP runtime call failed (sticky)                  */
#define SP_ERR_STATE (-6)       /* context unusable (after SP_ERR_HIP) or null handle  */

/* sp_config.policy: how victims are chosen among unheld slots (Sec. VI-E
 * names LRU as the default and random eviction and LFU as alternatives).
 * Every policy takes the slots with the smallest (priority, slot):
 *   LRU     priority = last plan that used the slot (never used: first)
 *   LFU     priority = plans that used the slot since its current row was
 *           placed there, the placing plan included (never used: 0, first)
 *   RANDOM  priority = 0 for a never-used slot, else 1 + the top 24 bits of
 *           output number u * 2^31 + g + 1 of a SplitMix64 stream started at
 *           sp_config.seed (u = plan index, g = global slot): a fresh uniform
 *           draw per slot and plan */
#define SP_POLICY_LRU 0
#define SP_POLICY_LFU 1
#define SP_POLICY_RANDOM 2

/* sp_config.hold_past at most: earlier batches a plan may hold as well */
#define SP_MAX_HOLD_PAST 4

/* sp_config.prefetch at most: successor batches a plan may fill ahead */
#define SP_MAX_PREFETCH 4

/* sp_config.flags */
#define SP_FLAG_DEBUG_SYNC 0x1u /* synchronise the device at the end of every call     */
#define SP_FLAG_TIMING 0x2u     /* time forward/backward/plan/fill kernels with events */
#define SP_FLAG_EVENT_WAITS 0x4u /* wait on events where the library otherwise waits on
                                    stream values (hipStreamWaitValue64); for tools
                                    that run one dispatch at a time, under which a
                                    value wait would wait for a dispatch held back */
#define SP_FLAG_POISON 0x8u     /* debugging aid, read by sp_create: Storage starts as
                                    NaN instead of zeros, and with the staged fill the
                                    device staging of filled rows is set to NaN once
                                    the fill has used it, so a read of a slot before
                                    its fill landed, or of stale staging, shows up as
                                    NaN in outputs and tables                        */
#define SP_FLAG_DEFER_SORTS 0x10u /* debugging aid, staged fill: batches prepared ahead
                                    are always sorted behind the update of the plan
                                    that received them (sp_backward_update enqueues
                                    them; the allocation-free variant leaves them to
                                    the next sp_plan), as they are by default only
                                    behind a write-back copy above 256 MiB           */

/* sp_config.fill: how missing rows reach the scratchpad (Sec. IV-B) */
#define SP_FILL_MAPPED 0 /* the move kernel reads them straight from pinned,
                            device-mapped host tables over the host link          */
#define SP_FILL_STAGED 1 /* host threads gather them from the tables into pinned
                            staging ([Collect]), copies take them to the device in
                            pieces as they are gathered ([Exchange]) and the move
                            kernel writes them into their slots ([Insert]); the
                            tables may then be any host memory                    */

typedef struct sp_ctx *sp_handle;

typedef struct {
    int32_t num_tables;         /* T, 1..64                                            */
    const int64_t *rows;        /* [T] rows per table, 1 .. 2^25                       */
    int32_t dim;                /* D, fp32 elements per row; multiple of 4, <= 256     */
    const int64_t *slots;       /* [T] scratchpad slots per table, 1 .. rows[t]         */
    int32_t lookahead;          /* L >= 0: successor batches a plan may hold           */
    float *const *host_tables;  /* [T] row-major [rows][D] fp32 host tables, caller-owned,
                                   must outlive the context, each 16-byte aligned; read
                                   on misses, written on evictions and flush.
                                   SP_FILL_MAPPED: pinned,
                                   device-mapped memory from sp_host_alloc (or
                                   hipHostMalloc with the mapped flag); SP_FILL_STAGED:
                                   any host memory                                   */
    int32_t max_batch;          /* largest B any batch will have; T * max_batch * dim * 4
                                   (the bytes of one [T*B][D] gradient) must stay
                                   below 4 GiB                                         */
    int64_t max_ids;            /* largest nnz any batch will have (all tables)        */
    uint32_t flags;             /* SP_FLAG_*                                           */
    int32_t device;             /* HIP device ordinal                                  */
    int32_t policy;             /* SP_POLICY_* (0 = LRU)                               */
    int32_t hold_past;          /* 0..SP_MAX_HOLD_PAST, and lookahead + 1 + hold_past
                                   <= 16: a plan also holds the rows of this many
                                   batches planned before it (the past window of
                                   Sec. IV-C), so no row a recent batch used is
                                   evicted; 0 = look-forward window only          */
    uint64_t seed;              /* SP_POLICY_RANDOM's stream                           */
    int64_t max_table_ids;      /* 0, or the most IDs one table has in any batch: a
                                   batch with a table above it is rejected
                                   (SP_ERR_INVALID_ARG).  With max_table_ids and
                                   max_batch both <= 8192 each table of a batch is
                                   sorted and deduplicated by one workgroup in LDS,
                                   the whole batch in one launch                    */
    int32_t prefetch;           /* depth d in 0 .. SP_MAX_PREFETCH (above lookahead it
                                   acts as lookahead): each plan also fills the rows
                                   of its next d window batches (window[1..d], those
                                   given) that are
                                   neither cached nor in an earlier window batch: the
                                   earlier fill of future misses that the multi-stage
                                   overlap of Sec. IV-C allows.  Per table the planned
                                   batch's misses come first, then window[1]'s rows,
                                   then window[2]'s, ..., each ascending; the capacity
                                   check counts them all, so SP_ERR_CAPACITY can come
                                   earlier than without prefetch.  0 = none        */
    int32_t fill;               /* SP_FILL_MAPPED (0) or SP_FILL_STAGED               */
} sp_config;

typedef struct {
    int32_t batch;              /* B, 0 .. max_batch                                   */
    int64_t nnz;                /* number of IDs, 0 .. max_ids                          */
    const int32_t *ids;         /* [nnz] row IDs, table-major                          */
    const int32_t *bag_off;     /* [T*B+1] bag offsets                                 */
    int32_t on_device;          /* 0: ids/bag_off are host memory, copied before sp_plan
                                   returns; 1: device memory, which must hold the batch
                                   when sp_plan is called (the library reads it on its
                                   own stream, with no order against the caller's
                                   streams: synchronise the stream that wrote it first)
                                   and stay unchanged until an sp_plan call that holds
                                   the batch (window index <= lookahead) has returned */
} sp_batch;

typedef struct {
    int64_t plans;              /* plans committed                                     */
    int64_t updates;            /* backward updates issued                              */
    int64_t lookups;            /* IDs planned (sum of nnz)                             */
    int64_t unique;             /* unique (table,row) keys planned                      */
    int64_t hits, misses;       /* unique keys found / not found in the Hit-Map         */
    int64_t evictions;          /* misses placed in a slot that held a row              */
    int64_t bytes_fill;         /* host -> HBM bytes of miss fills                      */
    int64_t bytes_writeback;    /* HBM -> host bytes of evicted rows                    */
    int64_t hash_rebuilds;      /* of the Hit-Map's hash (0 where it is one entry per row) */
    int64_t chunks;             /* backward work chunks processed                       */
    int64_t min_capacity_margin;/* min over plans and tables of unheld slots - misses  */
    int64_t device_bytes;       /* device memory held by the context                    */
    int64_t pinned_bytes;       /* pinned staging held by the context                   */
    /* SP_FLAG_TIMING only: summed time in ms and number of timed launches.
     * forward, backward (per-chunk kernel) and combine (runs split over several
     * chunks, launched only when there are any) and fill (evicted-row
     * staging and miss fill, plans with misses only) are kernel execution
     * times; plan (the commit sequence: victims, Hit-Map, slot metadata)
     * spans its launch sequence. */
    double ms_forward, ms_backward, ms_combine, ms_plan, ms_fill;
    int64_t timed_forward, timed_backward, timed_combine, timed_plan, timed_fill;
    /* host time spent inside sp_plan, in ms: enqueueing ingest, enqueueing the
     * query, waiting for its counts, enqueueing the commit, and the mover
     * (including waits for the write-back thread) */
    double host_ms_ingest, host_ms_query, host_ms_wait, host_ms_commit, host_ms_mover;
    /* SP_FLAG_TIMING only: ingest of a batch (keys, sort, dedup, backward
     * chunks) and the query of a plan (hold marks and probe, from the moment
     * its stream reaches it, waits for ingests included) */
    double ms_ingest, ms_query;
    int64_t timed_ingest, timed_query;
    /* host time, in ms, that sp_plan spends before returning waiting until its
     * ingests have read the caller's window arrays */
    double host_ms_inputs;
    /* prefetch mode: rows filled for the next batch (included in misses,
     * evictions and bytes_fill, not in hits: hits count the planned batch's
     * keys found cached, prefetched ones included) */
    int64_t prefetched;
    /* SP_FILL_STAGED: host time of the fill thread gathering missing rows into
     * pinned staging, and host time the calling thread spent waiting for the
     * fill thread to enqueue a plan's fill (ms); SP_FLAG_TIMING: the span of a
     * plan's host-to-device copies of gathered rows, first start to last end */
    double host_ms_gather, host_ms_fill_join, ms_h2d;
    int64_t timed_h2d;
} sp_stats;

/* Per-plan decisions copied to the host for checking.  The caller allocates
 * every array with room for the planned batch's nnz entries.  Slots are global
 * (table t's slots follow tables 0..t-1).  Filled fields:
 *   u_table,u_row,hit,slot_u [n_unique]  the batch's unique keys, ascending
 *                                        (table,row); hit=1 if it was cached;
 *                                        slot_u = its slot after the plan
 *   inv,slot_of [nnz]                    index into u_*, slot of ids[j]
 *   m_table,m_row,v_slot,v_old_row,v_old_use [n_miss]
 *                                        misses in ascending (table,row), the
 *                                        slot each one gets, the row evicted
 *                                        from it (-1 if none) and that slot's
 *                                        previous last-use plan index (-1 if
 *                                        never used).  In prefetch mode these
 *                                        hold, per table, the planned batch's
 *                                        misses then the prefetched rows, and
 *                                        need room for the nnz of the planned
 *                                        batch and its d successors together */
typedef struct {
    int32_t *u_table, *u_row, *inv, *m_table, *m_row, *v_slot, *v_old_row, *v_old_use;
    int32_t *slot_u, *slot_of;
    uint8_t *hit;
    int64_t n_unique, n_miss, n_evict, nnz;
} sp_plan_dump;

/*
 * Create a context: allocates Storage (sum(slots) x D fp32), the Hit-Map,
 * per-slot metadata and holds, two int32 per row of every table (sum(rows) x 8
 * bytes: the row index behind the holds of filled rows), the window ring and
 * staging buffers on config->device, and four library streams at default
 * priority (plan, ingest, move and copy).
 * Nothing is cached initially.
 * Errors: SP_ERR_INVALID_ARG (config out of range; with SP_FILL_MAPPED a host
 * table that is not pinned and mapped), SP_ERR_OOM, SP_ERR_HIP.  *out is set
 * only on success; on failure everything allocated so far is freed.  For
 * testing that path, the environment variable SP_FAIL_ALLOC_AFTER=n makes the
 * allocation after the first n of this call fail with SP_ERR_OOM.
 * (Sec. IV-D "GPU scratchpad design": Storage and Hit-Map.)
 */
sp_status sp_create(const sp_config *config, sp_handle *out);

/* Batches after the hold window that sp_plan accepts for early sorting. */
#define SP_MAX_AHEAD 2

/*
 * Plan the next mini-batch.  window[0] is the batch to plan (ticket k = number
 * of plans so far) and window[1..] are the batches that follow it, n of them
 * in all, 1 <= n <= lookahead + 1 + SP_MAX_AHEAD.  The first
 * min(n, lookahead+1) batches form the hold window; any after them are only
 * sorted and deduplicated ahead of time (not held), which takes that work off
 * later plans' paths.  Handing over at least one such batch also lets this
 * plan issue the next plan's query right behind its own commit.  Batches
 * enter the device window
 * ring once, when first seen, and are not read again: the same batch must be
 * passed with the same content every time it appears (after a plan rejected
 * for its IDs, offsets or capacity all of that call's batches are read again
 * on the next call, and may have other content from then on).  Host window
 * buffers may be reused when the call returns; device ones once a call that
 * holds their batch has returned (a batch prepared ahead in device memory is
 * read asynchronously, before the query of the first plan that holds it).
 * The plan queries the Hit-Map
 * for window[0]'s unique keys, holds
 * every cached slot used by any window batch (and by the hold_past batches
 * planned before this one), takes for each table's misses the unheld slots
 * that come first under the policy (smallest priority first, ties by slot;
 * the ascending misses take them in that order), updates Hit-Map, slot keys,
 * last-use and use counts, and enqueues the evicted rows' write-back and the
 * misses' fill (Sec. IV-C "Putting everything together", Sec. IV-D
 * Algorithm 1; policies from Sec. VI-E).  With sp_config.prefetch = d the
 * misses also include the rows of window[1..d] that are neither cached nor in
 * an earlier window batch (after window[0]'s own misses, per table).  The host waits once for
 * per-table counts.
 * Requires the previous ticket's sp_backward_update to have been issued.
 * Transactional: on SP_ERR_INVALID_ARG (ID out of range, bad offsets, sizes
 * above the config) or SP_ERR_CAPACITY (misses > unheld slots in some table)
 * the scratchpad state is unchanged and the same ticket can be planned again.
 */
sp_status sp_plan(sp_handle h, const sp_batch *window, int32_t n, int64_t *ticket);

/*
 * Pooled forward of a planned batch: d_out[t*B+b][:] = sum of the Storage rows
 * of bag (t,b) (Sec. II-B "Forward propagation", sum reduction; empty bag ->
 * zeros).  Enqueued on `stream` (a hipStream_t; NULL = default stream) after
 * the ticket's fill, or, when the batch had no misses of its own (all its
 * rows cached before this plan, as with prefetch), after the ticket's commit
 * and the previous ticket's fill: this plan's fill touches none of its rows.
 * `ticket` must be the latest plan, not yet forwarded.
 * d_out: caller-owned device fp32 [T][B][D].  Errors: SP_ERR_SEQUENCE,
 * SP_ERR_INVALID_ARG (null d_out with B*T > 0).
 */
sp_status sp_forward(sp_handle h, int64_t ticket, float *d_out, void *stream);

/*
 * Backward and update of a forwarded batch: every unique row gets the sum of
 * the gradients of the bags that gathered it, positions in ascending order,
 * and Storage[row] -= lr * sum in place (Sec. II-B "Backpropagation"; plain
 * SGD).  d_grad: device fp32 [T][B][D].  Enqueued on `stream`.
 * Errors: SP_ERR_SEQUENCE, SP_ERR_INVALID_ARG.
 */
sp_status sp_backward_update(sp_handle h, int64_t ticket, const float *d_grad, float lr,
                             void *stream);

/*
 * For callers that cannot allocate device memory at call time or at all
 * outside set-up (code under graph capture, tight serving loops, harnesses
 * that forbid hipMalloc): sp_backward_update with the partial sums of runs
 * split over several backward chunks kept in a fixed device array of 32 MiB
 * instead of the context's buffer.  The array exists once per GPU for the
 * life of the process; its address is taken in sp_create.  It holds the
 * partials of at most 32 MiB / (4 * dim) backward chunks, one chunk per run
 * of up to 16 positions of one key, so a batch with nnz * dim * 4 <= 32 MiB
 * always fits; a ticket above that (with a split run) is rejected with
 * SP_ERR_INVALID_ARG and nothing changes, and sp_backward_update can then be
 * called for it.  Every call on one GPU uses the same array: calls that
 * overlap on one GPU (contexts on different streams) race and must be
 * ordered by the caller.  Otherwise as sp_backward_update; it allocates
 * nothing.
 */
sp_status sp_backward_update_static(sp_handle h, int64_t ticket, const float *d_grad, float lr,
                                    void *stream);

/*
 * Synchronise everything and write every cached row back to its host table;
 * afterwards the host tables hold the trained model.  The scratchpad keeps
 * its contents, so training may continue.  (Evicted entries are dirty and must
 * be written back, Sec. IV-B; flush applies that to all entries.)
 */
sp_status sp_flush(sp_handle h);

/*
 * Wait until every effect of the calls so far is complete: all device work
 * (on the library's streams and the rest of the device) has finished and
 * every row evicted so far has been written back to its host table.  Unlike
 * sp_flush it writes no cached row back.  Training may continue afterwards.
 */
sp_status sp_sync(sp_handle h);

/* Counters since sp_create (synchronises pending timing events). */
sp_status sp_get_stats(sp_handle h, sp_stats *out);

/* Replace the context's SP_FLAG_* bits for the calls that follow, e.g. to
 * time only a sample of the steps.  SP_ERR_INVALID_ARG for unknown bits. */
sp_status sp_set_flags(sp_handle h, uint32_t flags);

/* Copy the decisions of the most recent plan (ticket must equal it) to host
 * arrays; for checking against a reference.  Synchronises the library stream. */
sp_status sp_debug_plan(sp_handle h, int64_t ticket, sp_plan_dump *out);

/* Wait for all work, join the write-back thread, free everything.  NULL is ok. */
void sp_destroy(sp_handle h);

/* Text of the last error on this context (or of the last failed sp_create
 * or call without a context when h is NULL, by this thread).  Valid until the
 * next call on the context. */
const char *sp_last_error(sp_handle h);

/* Pinned, device-mapped host memory for host tables (hipHostMalloc with the
 * mapped and portable flags; exact size).  *ptr is set on SP_OK. */
sp_status sp_host_alloc(size_t bytes, void **ptr);
void sp_host_free(void *ptr);

/*
 * ---------------------------------------------------------------------------
 * Operators on token tables, rows in 8 and 4 bits and scores, on device memory.
 *
 * A table of rows is trained (sp_lookup, sp_lookup_grad, sp_dropout, sp_distill_grad), then kept
 * in 8 bits, read back (sp_cache_write, sp_cache_read) and scored against
 * (sp_product), or in 4 bits (sp_cache4_write, sp_cache4_read, sp_product4); scores are adjusted
 * before tokens are chosen from them (sp_adjust).  These calls take no context.  They enqueue kernels on `stream`
 * of the current device, allocate nothing, keep nothing, wait for nothing (so
 * they can be captured into a graph; numbers given by value, seed and offset among
 * them, are then those of the capture), and may be used from several threads.
 *
 *  - A matrix is a pointer, its element type and `ld`, the elements from the
 *    start of one row to the next (at least its columns); the elements of a row
 *    follow one another.  Rows may start at any multiple of the element's size.
 *  - At most 2^31 - 1 rows of anything, 2^20 columns (sp_dropout 2^30).
 *  - Results do not depend on the order in which the device runs blocks.  Sums
 *    are held in fp32 (sp_product: in 32-bit integers) and rounded once.
 *  - Outputs overlap no input, except where a call says so.
 *  - Errors: SP_ERR_INVALID_ARG (nothing was enqueued), SP_ERR_HIP (a launch
 *    failed); text from sp_last_error(NULL).
 */
#define SP_F32 0
#define SP_BF16 1
#define SP_F16 2
#define SP_I32 3
#define SP_I64 4
#define SP_I8 5
#define SP_F8 6 /* 1 sign, 4 exponent, 3 mantissa bits, no infinities, largest 448 */

/*
 * out[i][:] = scale * table[tokens[i]][:], i < n, with dropout of probability p
 * (0: none) as sp_dropout's, row i being row i of its generator.  tokens: SP_I32 or
 * SP_I64; a token outside 0 .. rows-1 (padding) gives a row of zeros.  table and
 * out: SP_F32, SP_BF16 or SP_F16 each.
 */
sp_status sp_lookup(const void *tokens, int32_t token_type, int64_t n, const void *table,
                    int32_t table_type, int64_t rows, int64_t dim, int64_t table_ld, float scale,
                    float p, uint64_t seed, uint64_t offset, void *out, int32_t out_type,
                    int64_t out_ld, void *stream);

/*
 * The gradient of sp_lookup to its table: out[r][:] = scale * the sum of the
 * gradients of the positions with token r, as the same p, seed and offset let
 * them through, in a fixed order.  Rows without a token become zeros; with
 * accumulate != 0 the sums are added to out, and rows without a token are neither
 * read nor written.  grad [n][dim] and out [rows][dim]: SP_F32, SP_BF16 or SP_F16
 * each.  Gradients of tokens that are no rows count nothing, whatever they hold.
 * workspace: device memory of at least the bytes that sp_lookup_grad_workspace
 * gives for n, rows and dim (0 for few tokens), 16-byte aligned, in use until the
 * call's work is done; its content means nothing before and after.
 */
sp_status sp_lookup_grad_workspace(int64_t n, int64_t rows, int64_t dim, int64_t *bytes);
sp_status sp_lookup_grad(const void *tokens, int32_t token_type, int64_t n, const void *grad,
                         int32_t grad_type, int64_t dim, int64_t grad_ld, float scale, float p,
                         uint64_t seed, uint64_t offset, void *out, int32_t out_type, int64_t rows,
                         int64_t out_ld, int32_t accumulate, void *workspace,
                         int64_t workspace_bytes, void *stream);

/*
 * out = [residual +] x / (1 - p) where kept, [residual + ] 0 where dropped.  The mask
 * is drawn from seed, offset and the element's row and column and stored nowhere:
 * the gradient to x is the same call on the output's gradient without a residual
 * (the residual's is the output's gradient itself).  Give every use its own offset.
 * A captured call keeps its offset: every replay of the graph drops the same places, so
 * a training step that is replayed has its dropout outside the graph, or a graph for
 * each of several offsets.  The same holds for sp_lookup and sp_lookup_grad with p > 0.
 * The generator is Philox 4x32-10 with counter (column / 8, row, offset low, offset
 * high) and key (seed low, seed high); its four words are 16 bits for each of 8
 * columns, the low half of a word first; a column is dropped where they are below
 * 65536 p, rounded to an integer.  1 - p is taken from that integer.
 * x, residual (may be NULL) and out have one type: SP_F32, SP_BF16 or SP_F16.
 * out may be x or residual itself (same pointer and ld).
 */
sp_status sp_dropout(const void *x, int32_t type, int64_t n, int64_t dim, int64_t x_ld,
                     const void *residual, int64_t residual_ld, float p, uint64_t seed,
                     uint64_t offset, void *out, int64_t out_ld, void *stream);

/*
 * A cache of rows in 8 bits: q [slots][dim] (SP_I8 or SP_F8) and fp32 scales
 * [slots][dim / group], a scale for each `group` columns of a slot (group: dim, or a
 * multiple of 8 that divides dim).
 *
 * sp_cache_write quantises row i of x (SP_F32, SP_BF16 or SP_F16) into slot index[i]
 * (SP_I32 or SP_I64; NULL: slot i).  scale = the group's largest magnitude / 127
 * (SP_I8) or / 448 (SP_F8), byte = x / scale rounded to nearest, ties to even.  A
 * group with an infinity or NaN reads back as NaN; one whose scale is below the
 * smallest normal fp32 number is held as zeros.  Rows whose index is no slot are
 * left out.  The slots of one call are distinct: which of two rows, or what mixture
 * of them, one slot gets is not defined.
 *
 * sp_cache_read gives out[i][:] = byte * scale of slot index[i], zeros where the index
 * is no slot.
 */
sp_status sp_cache_write(const void *x, int32_t type, int64_t n, int64_t dim, int64_t x_ld,
                         const void *index, int32_t index_type, int64_t group, void *q,
                         int32_t kind, int64_t slots, int64_t q_ld, float *scales,
                         int64_t scales_ld, void *stream);
sp_status sp_cache_read(const void *q, int32_t kind, int64_t slots, int64_t dim, int64_t q_ld,
                        const float *scales, int64_t scales_ld, int64_t group, const void *index,
                        int32_t index_type, int64_t n, void *out, int32_t out_type, int64_t out_ld,
                        void *stream);

/*
 * out[i][j] = x_scales[i] * w_scales[j] * sum over c < k of x[i][c] * w[j][c], i < m, j < n,
 * of 8-bit integers (-128 .. 127), the sum exact (k: 1 .. 131071).  With x from
 * sp_cache_write (group = dim) the scales are those of its tokens, with w a cache
 * they are those of its rows.  out: SP_F32, SP_BF16 or SP_F16.  Fastest where x and w
 * start at, and their strides are, multiples of 64; where they are multiples of 16 (and
 * strides below 2^23) rows are read in whole aligned 16-byte pieces (what lies beyond k
 * in the last one counts nothing); slower otherwise, rows going through registers.
 * workspace: as for sp_lookup_grad, of the bytes that sp_product_workspace gives for
 * m, n and k.
 */
sp_status sp_product_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes);
sp_status sp_product(const int8_t *x, const float *x_scales, int64_t m, int64_t x_ld,
                     const int8_t *w, const float *w_scales, int64_t n, int64_t w_ld, int64_t k,
                     void *out, int32_t out_type, int64_t out_ld, void *workspace,
                     int64_t workspace_bytes, void *stream);

/*
 * A cache of rows in 4 bits: q [slots][dim / 32 * 16] bytes and scales [slots][dim / 32] bytes,
 * dim rounded up to a multiple of 32.  Blocks of 32 columns share a scale 2^(byte - 127); a value is
 * scale times 0, .5, 1, 1.5, 2, 3, 4 or 6, its code (0 .. 7, the sign in bit 3) in half a byte, the
 * even column's in the low half: the MXFP4 format of the OCP Microscaling Formats specification.
 *
 * sp_cache4_write quantises row i of x (SP_F32, SP_BF16 or SP_F16) into slot index[i] (SP_I32 or
 * SP_I64; NULL: slot i).  With a the block's largest magnitude, scale = 2^(floor(log2 a) - 2), 2^-127
 * at least; code = x / scale rounded to nearest, ties to even codes, above 6 to 6.  Everything but
 * that rounding is exact.  A block with an infinity or NaN gets the byte 255 and reads back as NaN.
 * Columns past dim in the last block are written as zeros.  Rows whose index is no slot are left
 * out.  The slots of one call are distinct, as for sp_cache_write.
 *
 * sp_cache4_read gives the values of slot index[i], zeros where the index is no slot.
 */
sp_status sp_cache4_write(const void *x, int32_t type, int64_t n, int64_t dim, int64_t x_ld,
                          const void *index, int32_t index_type, uint8_t *q, int64_t slots,
                          int64_t q_ld, uint8_t *scales, int64_t scales_ld, void *stream);
sp_status sp_cache4_read(const uint8_t *q, int64_t slots, int64_t dim, int64_t q_ld,
                         const uint8_t *scales, int64_t scales_ld, const void *index,
                         int32_t index_type, int64_t n, void *out, int32_t out_type, int64_t out_ld,
                         void *stream);

/*
 * out[i][j] = sum over c < k of x[i][c] * w[j][c], i < m, j < n, of rows in 4 bits (k: 1 .. 2^20,
 * rounded up to a multiple of 32: what the last block holds past k counts, so zeros).  Products and
 * scales are exact, sums fp32.  A scale byte of 255 gives NaN.  Rows of x, of w and of their scales
 * start at multiples of 16 bytes (x and w best of 128), and are read in whole aligned 16-byte
 * pieces (scales past the row's last count nothing); their strides and the output's are below 2^23.
 * out: SP_F32, SP_BF16 or SP_F16.  workspace: as for sp_lookup_grad, of the bytes that
 * sp_product4_workspace gives for m, n and k.
 */
sp_status sp_product4_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes);
sp_status sp_product4(const uint8_t *x, const uint8_t *x_scales, int64_t m, int64_t x_ld,
                      int64_t x_scales_ld, const uint8_t *w, const uint8_t *w_scales, int64_t n,
                      int64_t w_ld, int64_t w_scales_ld, int64_t k, void *out, int32_t out_type,
                      int64_t out_ld, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * Scores [n][vocab] adjusted before a token is chosen, row by row: for a column v that is c > 0 times
 * among the row's previous tokens
 *     y = (s > 0 ? s / repetition : s * repetition) - (presence + frequency * c),   else y = s;
 * plus the bias of v (of several entries for v the last); -infinity where v is not allowed,
 * whatever s holds.  scores and out have one type (SP_F32, SP_BF16 or SP_F16); out may be scores
 * itself (same pointer and ld).
 *   previous [n][length], SP_I32 or SP_I64: tokens outside 0 .. vocab-1 (padding) count nothing;
 *     length 0: none.
 *   penalties [n][3] fp32: each row's repetition, presence and frequency in place of the numbers
 *     (NULL: the numbers, repetition positive, all finite).
 *   bias_tokens [n][biases], SP_I32 or SP_I64, and bias [n][biases] fp32: entries whose token is
 *     no column count nothing; biases 0: none.
 *   allowed [n][vocab / 32, rounded up]: column v is bit v % 32 of word v / 32 (NULL: all).
 * Strides of these may be 0: one row for all.  vocab and length: at most 2^20; biases: at most 2047.
 */
sp_status sp_adjust(const void *scores, int32_t type, int64_t n, int64_t vocab, int64_t ld,
                    const void *previous, int32_t previous_type, int64_t length, int64_t previous_ld,
                    float repetition, float presence, float frequency, const float *penalties,
                    int64_t penalties_ld, const void *bias_tokens, int32_t bias_type,
                    int64_t bias_tokens_ld, const float *bias, int64_t bias_ld, int64_t biases,
                    const int32_t *allowed, int64_t allowed_ld, void *out, int64_t out_ld,
                    void *stream);

/*
 * Distillation of scores [n][vocab] (SP_F32, SP_BF16 or SP_F16) from a teacher's top logits:
 * tokens [n][k] (SP_I32 or SP_I64) and teacher [n][k] (SP_F32, SP_BF16 or SP_F16), k 1 .. 1024.
 * With T the temperature, p the softmax of teacher / T over the row's entries and q that of
 * scores / T over its columns,
 *     loss[i] = T^2 * sum over entries j of p_j * (log p_j - log q_token(j)).
 * Entries whose token is no column (padding) are none; a token listed several times counts as often.
 * A row without entries, or with none above -infinity, has loss 0, whatever its scores hold.
 * Entries with p = 0 count nothing; a score of -infinity under p > 0 gives a loss of infinity (a row
 * of them alone: q = 0 everywhere), NaN and +infinity a loss of NaN or infinity.
 *
 * sp_distill_grad gives the loss and the gradient of weight * loss[i] to the scores,
 *     grad[i][v] = weight * T * (q_v - sum over j with token(j) = v of p_j),
 * zeros for a row of loss 0 by lack of entries (a row's sums are taken in an order that goes by its
 * sizes and by where its gradient starts in 64 bytes).  weights [n] fp32: each row's in place of the number
 * (NULL: the number).  grad: SP_F32, SP_BF16 or SP_F16; it may be scores itself (same pointer,
 * type and ld).
 * workspace: as for sp_lookup_grad, of the bytes that sp_distill_workspace gives for n, vocab, k and
 * whether the gradient is asked for.
 */
sp_status sp_distill_workspace(int64_t n, int64_t vocab, int64_t k, int32_t grad, int64_t *bytes);
sp_status sp_distill(const void *scores, int32_t type, int64_t n, int64_t vocab, int64_t ld,
                     const void *tokens, int32_t token_type, int64_t tokens_ld, const void *teacher,
                     int32_t teacher_type, int64_t teacher_ld, int64_t k, float temperature,
                     float *loss, void *workspace, int64_t workspace_bytes, void *stream);
sp_status sp_distill_grad(const void *scores, int32_t type, int64_t n, int64_t vocab, int64_t ld,
                          const void *tokens, int32_t token_type, int64_t tokens_ld,
                          const void *teacher, int32_t teacher_type, int64_t teacher_ld, int64_t k,
                          float temperature, float weight, const float *weights, float *loss,
                          void *grad, int32_t grad_type, int64_t grad_ld, void *workspace,
                          int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SCRATCHPIPE_H */
