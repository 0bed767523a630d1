/*
 * scar.h - C ABI of the SCAR checkpoint-and-recover parameter pass on one GPU.
 *
 * The library keeps a running checkpoint z of a caller-owned parameter buffer
 * x in device memory and offers the two strategies of the paper's Section 4:
 *   - prioritized partial checkpoints (Section 4.2, protocol of Section 4.3):
 *     score every block by its distance to the saved copy, take the fraction
 *     r with the largest scores, refresh z on those blocks and emit them as a
 *     contiguous payload;
 *   - partial recovery (Section 4.1): restore only the lost blocks from z and
 *     report the perturbation ||z_S - x_S|| that the iteration-cost bound of
 *     Theorem 3.2 depends on.
 *
 * Terms.  An element is 4 bytes (float32 or int32).  A block is a contiguous
 * element range and is the unit of scoring, selection and loss (the paper's
 * "parameter": a row, a layer or a shard of a layer, Section 5.1).  A shard is
 * a contiguous range of blocks standing for one parameter-server node.
 *
 * Conventions for every call.
 *   - Return value: SCAR_OK (0) or a negative SCAR_ERR_* code; nothing throws.
 *     Arguments are validated before any GPU work is enqueued, so a call that
 *     fails validation leaves every buffer untouched.
 *   - Pointer names say where the memory lives: d_* device, h_* host.
 *   - All GPU work of a context runs on the CUDA stream given at init, in call
 *     order.  A call whose result pointer `out` is NULL only enqueues; with a
 *     non-NULL `out` it also waits for the stream and fills `out`.
 *     Enqueue-only calls use no host synchronisation and read no caller-owned
 *     host memory after they return, so they can be recorded by CUDA stream
 *     capture on the context's stream: saves, recoveries and norms with device
 *     block masks or with shard masks of up to 1024 shards (their flags travel
 *     in launch parameters; a replay uses the mask of the capture), and
 *     scar_ckpt_load.  A shard-mask call on a context with more than 1024
 *     shards waits for the stream and is not capturable.
 *   - One context serves one caller at a time (no internal locking).
 *   - There is no CPU fallback: without a usable CUDA device init fails.
 */
#ifndef SCAR_H
#define SCAR_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct scar_ctx scar_ctx; /* opaque; created by scar_ckpt_init, freed by scar_ckpt_destroy */

/* Element type.  SCAR_F32 scores blocks by the squared l2 distance (the norm of
 * the appendix proofs of Theorems 4.1/4.2); SCAR_I32 by the integer l1 distance
 * (twice the length-scaled total variation that Appendix C uses for LDA).  The
 * 16-bit types are operand types of the training-step operators (scar_xent_*,
 * scar_gnorm_*, scar_linear_*, scar_dropout_*, scar_resnorm_*) only: checkpoint
 * contexts refuse them. */
typedef enum { SCAR_F32 = 0, SCAR_I32 = 1, SCAR_BF16 = 2, SCAR_F16 = 3 } scar_dtype;

/* Which norm measures the distance of a block to its saved copy.  DEFAULT is the
 * one above for the element type.  L1 on SCAR_F32 data scores a block by
 * sum |x_i - z_i| in float32 and reports perturbations as the plain sum (no
 * square root): with per-block weights L_b / 2 this is the total variation of
 * each topic distribution scaled by its document's length, the norm Appendix C
 * uses for LDA.  On SCAR_I32 data L1 is the default already. */
typedef enum { SCAR_NORM_DEFAULT = 0, SCAR_NORM_L1 = 1 } scar_norm;

enum {
    SCAR_OK = 0,
    SCAR_ERR_INVALID_ARG = -1, /* NULL where not allowed, r outside [0,1], k > B, misaligned x ... */
    SCAR_ERR_LAYOUT = -2,      /* inconsistent block geometry */
    SCAR_ERR_ALLOC = -3,       /* device or host allocation failed */
    SCAR_ERR_CUDA = -4,        /* a CUDA runtime call or kernel launch failed */
    SCAR_ERR_STATE = -5,       /* call not valid in the context's current state */
    SCAR_ERR_TIMEOUT = -6,     /* a bounded device-side wait (of the selection, or of the norm reduction) gave
                                  up; the call's outputs are invalid, the context stays usable */
    SCAR_ERR_CAPACITY = -7,    /* problem larger than a fixed-size internal buffer */
    SCAR_ERR_IO = -8           /* a read or write of the stored checkpoint failed or came up short */
};

/* Block geometry of the flat buffer of n_elems elements.
 *   Implicit form (block_offsets == NULL): rows of row_elems elements
 *   (0 = one row of n_elems; otherwise n_elems % row_elems == 0), each cut into
 *   blocks of block_elems; the last block of a row may be shorter; blocks never
 *   cross a row end.  n_blocks is ignored.
 *   Explicit form: block_offsets is a HOST array of n_blocks + 1 non-decreasing
 *   element offsets with block_offsets[0] == 0 and block_offsets[n_blocks] ==
 *   n_elems; it is copied during init.  row_elems / block_elems are ignored.
 * n_shards >= 1; shard s owns blocks [floor(s*B/S), floor((s+1)*B/S)).
 * At most 2^32 - 1 blocks. */
typedef struct {
    uint64_t n_elems;
    uint64_t row_elems;
    uint32_t block_elems;
    uint32_t n_shards;
    const uint64_t *block_offsets;
    uint64_t n_blocks;
} scar_layout;

typedef struct {
    uint64_t k;                /* blocks saved */
    uint64_t payload_elems;    /* elements in the payload = poff[k] */
    uint64_t nonfinite_blocks; /* SCAR_F32: blocks whose score was NaN or +Inf (ranked first) */
} scar_save_info;

typedef struct {
    double l2;            /* SCAR_F32: ||z_S - x_S|| in the context's norm (l2 unless scar_ckpt_set_norm
                             chose another); 0 for SCAR_I32 */
    uint64_t l1;          /* SCAR_I32: sum_{i in S} |z_i - x_i| ; 0 for SCAR_F32 */
    uint64_t lost_blocks; /* |S| in blocks */
    uint64_t lost_elems;  /* |S| in elements */
} scar_norm_info;

/* Creates a context over the caller's device buffer d_x (n_elems elements of
 * type dt, 16-byte aligned, owned by the caller, must stay valid and in place
 * until destroy) and initialises the running checkpoint z := x (Section 4.2:
 * the running checkpoint starts from the initial parameter values).  Allocates
 * z, the score/selection arrays and a payload buffer of n_elems elements on the
 * current CUDA device.  cuda_stream is a cudaStream_t (NULL = default stream).
 * Waits for the stream before returning.  On error *out is NULL. */
int scar_ckpt_init(scar_ctx **out, void *d_x, scar_dtype dt, const scar_layout *layout, void *cuda_stream);

/* Chooses the norm and optional per-block weights for all later scoring,
 * selection and perturbation results of this context.  h_block_weights: HOST
 * array of B finite floats >= 0 (copied before the call returns), or NULL for
 * no weights; SCAR_F32 only (SCAR_ERR_INVALID_ARG with SCAR_I32: integer scores
 * stay exact integers, and for count rows of fixed total the length-scaled
 * total variation is half the plain l1 anyway).  With weights w a block scores
 * w_b * dist(x_b, z_b) (dist = squared l2, or l1), and a perturbation is
 * sqrt(sum_b w_b ||d_b||^2) or sum_b w_b ||d_b||_1, reported in the l2 field of
 * scar_norm_info: a positive combination of block norms, hence a norm
 * (Appendix C).  Waits for the stream. */
int scar_ckpt_set_norm(scar_ctx *ctx, scar_norm norm, const float *h_block_weights);

/* Checkpoint step 1 of Section 4.3 alone: recomputes score_b = dist(x_b, z_b)
 * for every block into the context's score array (float32 squared l2, or
 * uint64 l1).  Enqueue only. */
int scar_ckpt_block_scores(scar_ctx *ctx);

/* One prioritized partial checkpoint (Section 4.2; steps 1, 3, 4 of the
 * checkpoint protocol in Section 4.3): scores all blocks, selects the
 * k = round(r*B) highest (halves away from zero; at least 1 if r > 0; ties to
 * the lowest block id; NaN/Inf scores rank first), writes their ids ascending to
 * sel[k], their payload offsets to poff[k+1], copies x over them into the
 * payload in that order and refreshes z_b := x_b on them.  r = 1 is the
 * traditional full checkpoint.  r outside [0,1] or NaN: SCAR_ERR_INVALID_ARG. */
int scar_ckpt_priority_save(scar_ctx *ctx, double r, scar_save_info *out);

/* The rule that turns the fraction r of Section 4.2 into a block count, as
 * scar_ckpt_priority_save applies it: k = round(r * n_blocks), halves away from
 * zero, at least 1 when r > 0 and n_blocks > 0, at most n_blocks.  For callers
 * that schedule saves themselves (the baseline selectors take k, not r).  Host
 * only.  SCAR_ERR_INVALID_ARG for r outside [0,1], NaN, or k == NULL. */
int scar_k_from_r(double r, uint64_t n_blocks, uint64_t *k);

/* Same with the block count given directly (0 <= k <= B). */
int scar_ckpt_priority_save_k(scar_ctx *ctx, uint64_t k, scar_save_info *out);

/* The multi-GPU form of a prioritized save: the checkpoint protocol of Section
 * 4.3 the way the paper runs it, with one GPU per parameter-server node.  Every
 * node scores its own partition (step 1: scar_ckpt_block_scores), the scores of
 * all nodes are made known to all (step 2: the caller's exchange, e.g. an NCCL
 * all-gather of the score arrays; the library itself has no communication), and
 * every node selects the same global fraction and saves what it owns (steps 3
 * and 4: this call).  Payloads never leave their GPU; recovery stays a local
 * call on whichever context owns the lost blocks.
 *
 * The context covers this rank's partition: its B blocks are blocks
 * [first_block, first_block + B) of a global layout of n_global_blocks blocks.
 *   d_global_scores  DEVICE array of n_global_blocks scores in global block
 *                    order, of the context's score type (float32 / uint64), as
 *                    scar_ckpt_view returns them per rank; read when the
 *                    enqueued work runs
 *   k_global         blocks to save over all ranks (e.g. scar_k_from_r(r,
 *                    n_global_blocks)), 0 <= k_global <= n_global_blocks
 * The k_global highest global scores are selected, ties to the lowest global
 * id; the ones in this rank's range are packed and refreshed exactly as by a
 * single-GPU save: sel holds LOCAL block ids, ascending, out->k is this rank's
 * count, out->nonfinite_blocks counts over all ranks.  The union over ranks of
 * the saved blocks (local id + first_block) is what one context over the
 * concatenated buffer would have saved.  Always waits for the stream (the
 * rank's count crosses to the host once), so `out` must not be NULL and the
 * call cannot be captured. */
int scar_ckpt_priority_save_sharded(scar_ctx *ctx, const void *d_global_scores, uint64_t n_global_blocks,
                                    uint64_t first_block, uint64_t k_global, scar_save_info *out);

/* The two baseline selectors the paper compares the prioritized checkpoint with
 * (Section 5.4).  Both skip the scoring pass (the score array keeps the values
 * of the last scoring) and then pack the chosen blocks and refresh z on them
 * exactly as a prioritized save does: same sel / poff / payload outputs, ids
 * ascending.
 *   round:  "selected in a round-robin manner": the k blocks that follow the
 *           context's cursor, wrapping at the end of the buffer; the cursor
 *           then advances by k (mod B).  It starts at block 0.
 *   random: "selected uniformly at random".  The randomness is the caller's:
 *           d_priorities is a DEVICE array of B uint32 values drawn
 *           independently and uniformly by the caller; the k largest are taken,
 *           ties to the lowest id, which is a uniform k-subset up to those ties.
 *           Read when the enqueued work runs.
 * 0 <= k <= B, otherwise SCAR_ERR_INVALID_ARG. */
int scar_ckpt_save_round(scar_ctx *ctx, uint64_t k, scar_save_info *out);
int scar_ckpt_save_random(scar_ctx *ctx, uint64_t k, const uint32_t *d_priorities, scar_save_info *out);

/* Round-robin cursor: if set != NULL the cursor becomes *set (must be < B, or 0
 * when B == 0); if get != NULL it receives the cursor.  Host state only. */
int scar_ckpt_round_cursor(scar_ctx *ctx, const uint64_t *set, uint64_t *get);

/* Partial recovery (Section 4.1; recovery step 2 of Section 4.3): for every
 * block of every lost shard, accumulates the perturbation of the appendix proof
 * of Theorem 4.1, ||z_S - x_S||, from the values x still holds, then overwrites
 * x_b := z_b.  Blocks outside S and all of z are left untouched.
 * h_lost_shards: HOST array of n_shards bytes, 0 = alive, non-zero = lost. */
int scar_recover_partial(scar_ctx *ctx, const uint8_t *h_lost_shards, scar_norm_info *out);

/* Same with an arbitrary lost set: d_lost_blocks is a DEVICE array of B bytes
 * (0 alive, non-zero lost), read when the enqueued work runs. */
int scar_recover_partial_blocks(scar_ctx *ctx, const uint8_t *d_lost_blocks, scar_norm_info *out);

/* The perturbation a recovery of the given lost set would cause, without
 * writing anything.  NULL mask = every block lost = full recovery, whose
 * perturbation is x^(T) - x^(C) (Example 2.3). */
int scar_perturbation_norm(scar_ctx *ctx, const uint8_t *h_lost_shards, scar_norm_info *out);
int scar_perturbation_norm_blocks(scar_ctx *ctx, const uint8_t *d_lost_blocks, scar_norm_info *out);

/* Perturbation norm without any allocation.  (The paper has no counterpart: it
 * is the same quantity as scar_perturbation_norm_blocks, offered for callers
 * that cannot allocate.)
 *
 * Some callers cannot create a context, because scar_ckpt_init calls cudaMalloc:
 * a failure handler running while memory is exhausted, a latency-critical loop
 * that cannot take the device-wide synchronisation an allocation implies, or a
 * plug-in whose host forbids it to grow its memory.  This call needs no
 * context and calls no cudaMalloc / cudaFree or other allocating routine.  Its
 * partial sums live in a fixed array of about 0.3 MiB inside the library's
 * device image (every GPU that loads the library holds it until the process
 * exits), which caps the problem at SCAR_STATIC_MAX_BLOCKS blocks; larger
 * layouts return SCAR_ERR_CAPACITY and nothing is enqueued.
 *
 *   d_x, d_z       DEVICE buffers of layout->n_elems elements of type dt, both
 *                  16-byte aligned, read only; z is the checkpoint to compare with
 *   layout         implicit form only (block_offsets must be NULL); n_shards ignored
 *   d_lost_blocks  DEVICE array of B bytes, 0 alive / non-zero lost; NULL = all lost
 *   d_out          DEVICE scar_norm_info written by the enqueued work (caller-owned)
 *   cuda_stream    cudaStream_t to enqueue on; the call does not wait
 *
 * The first call on each device looks up the array's device address (once, with
 * that device current), and with CUDA's lazy module loading it is also what
 * brings the array and this call's kernels onto the device, which itself needs
 * a little device memory.  So make the first call at start-up, before memory
 * can run short and before any stream capture: a call with n_elems == 0 does the
 * look-up, one tiny real call loads the kernels.  All calls on a device share
 * the one array (each call first empties the part it uses): calls whose GPU
 * work overlaps (different streams, or different threads) race and give wrong
 * results; calls ordered on one stream are fine.  Results are bit-identical to
 * scar_perturbation_norm_blocks. */
#define SCAR_STATIC_MAX_BLOCKS (1ull << 20)
int scar_perturbation_norm_static(const void *d_x, const void *d_z, scar_dtype dt, const scar_layout *layout,
                                  const uint8_t *d_lost_blocks, scar_norm_info *d_out, void *cuda_stream);

/* Host-buffer forms for callers whose parameters live in host memory.
 * save_host: copies n_elems elements from h_x into the context's x, runs the
 * save, then copies back payload_elems elements to h_payload (capacity n_elems
 * elements), k ids to h_sel (capacity k) and k+1 offsets to h_poff.  Always
 * waits for completion; `out` must not be NULL.
 * recover_host: copies the lost shards' element ranges of h_x (the values the
 * failed nodes last held) into x, runs the recovery, and copies the recovered
 * ranges back into h_x; other ranges of h_x are neither read nor written. */
int scar_ckpt_priority_save_host(scar_ctx *ctx, const void *h_x, double r, void *h_payload, uint32_t *h_sel,
                                 uint64_t *h_poff, scar_save_info *out);
int scar_recover_partial_host(scar_ctx *ctx, void *h_x, const uint8_t *h_lost_shards, scar_norm_info *out);

/* ---- Asynchronous drain of a save's output (Section 4.3) --------------------
 * In the paper's protocol training resumes as soon as the in-memory cache (z)
 * is refreshed, while the saved parameters go to persistent storage in the
 * background, so the checkpoint overhead T_dump is only the prioritisation and
 * the cache refresh.  Here: a save runs on the context's stream as always;
 * scar_ckpt_drain_enqueue then copies that save's ids, offsets and payload to
 * pinned host memory on a second, library-owned stream, ordered after the save
 * by an event, and returns at once.  Two slots alternate, so the next save can
 * run while the previous one is still being copied out.
 *
 *   drain_init     switches the context to drain mode and allocates the second
 *                  device output set plus two pinned host mirrors.  From then
 *                  on every save is limited to max_k blocks and to layouts whose
 *                  k longest blocks together hold at most max_payload_elems
 *                  elements (whatever the save then selects fits; otherwise
 *                  SCAR_ERR_CAPACITY, nothing enqueued).  Waits for
 *                  the context's stream.  Once per context.
 *   drain_enqueue  hands the most recent save (there must be one that was not
 *                  handed over yet: SCAR_ERR_STATE otherwise) to the drain
 *                  stream; *ticket identifies it.  The next save writes to the
 *                  other slot, and fails with SCAR_ERR_STATE, nothing enqueued,
 *                  while that slot's ticket has not been released: at most two
 *                  tickets are out at any time.  Does not wait.
 *   drain_done     1 if the copy of that ticket has finished, 0 if not yet.
 *   drain_wait     waits for the copy and fills *out with HOST pointers into
 *                  the slot's pinned mirror: valid until drain_release.
 *   drain_release  gives the slot back to the library (waits for the copy if it
 *                  is still running).
 * scar_ckpt_view keeps returning the device buffers of the most recent save.
 * A save called with a non-NULL `out` fetches its result record over the same
 * device-to-host path and can queue behind a running drain; to overlap, enqueue
 * saves with out == NULL and read the record from the drained view. */
typedef struct {
    scar_save_info info;
    const uint32_t *h_sel;  /* info.k ids, ascending */
    const uint64_t *h_poff; /* info.k + 1 element offsets */
    const void *h_payload;  /* info.payload_elems elements */
} scar_drain_view;
int scar_ckpt_drain_init(scar_ctx *ctx, uint64_t max_k, uint64_t max_payload_elems);
int scar_ckpt_drain_enqueue(scar_ctx *ctx, uint64_t *ticket);
int scar_ckpt_drain_done(scar_ctx *ctx, uint64_t ticket);
int scar_ckpt_drain_wait(scar_ctx *ctx, uint64_t ticket, scar_drain_view *out);
int scar_ckpt_drain_release(scar_ctx *ctx, uint64_t ticket);

/* ---- The running checkpoint in persistent storage (Sections 4.2, 4.3) --------
 * The paper keeps the running checkpoint in shared persistent storage and z is
 * only the in-memory cache of it: step 4 of a checkpoint saves the selected
 * parameters there, and a recovery re-loads parameters from it.  Here the
 * stored checkpoint is a plain file of n_elems * 4 bytes in element order, given
 * as an open POSIX file descriptor (the caller opens, syncs and closes it); after
 * every store it holds exactly the bytes of z.
 *   store_full     writes all of z (the initial checkpoint x^(0), or after
 *                  scar_ckpt_load).  Waits for the stream.
 *   store_drained  waits for the drain of `ticket` and writes each saved block
 *                  from the pinned host mirror to its place in the file (one
 *                  write per run of consecutive blocks).  The ticket stays
 *                  valid; release it afterwards.  Host work only.
 *   load_stored    z := the file (a restart that lost the in-memory cache, or a
 *                  recovery from storage: follow it with scar_recover_partial).
 *                  Waits for the stream.
 * SCAR_ERR_IO on a failed or short read / write; the file or z may then be
 * partly updated. */
int scar_ckpt_store_full(scar_ctx *ctx, int fd);
int scar_ckpt_store_drained(scar_ctx *ctx, uint64_t ticket, int fd);
int scar_ckpt_load_stored(scar_ctx *ctx, int fd);

/* Replaces the running checkpoint by n_elems elements read from the device
 * buffer d_z_src (e.g. a checkpoint read back from storage).  Enqueue only. */
int scar_ckpt_load(scar_ctx *ctx, const void *d_z_src);

/* Waits for the stream and returns the results of the most recent save and the
 * most recent recover/norm call (either pointer may be NULL). */
int scar_ckpt_last_info(scar_ctx *ctx, scar_save_info *save, scar_norm_info *norm);

/* Borrowed device pointers (any may be NULL to skip): z (n_elems elements),
 * scores (B float32 for SCAR_F32, B uint64 for SCAR_I32; as of the last
 * scoring), sel (k uint32), poff (k+1 uint64), payload.  Valid until destroy;
 * contents change with the next save. */
int scar_ckpt_view(scar_ctx *ctx, const void **d_z, const void **d_scores, const uint32_t **d_sel,
                   const uint64_t **d_poff, const void **d_payload);

/* Geometry as the library resolved it. */
uint64_t scar_ckpt_n_blocks(const scar_ctx *ctx);

/* Kernels this context has launched so far (its own kernels only). */
uint64_t scar_ckpt_launch_count(const scar_ctx *ctx);

/* Optional per-phase device timing.  With enable != 0 every later call brackets
 * its phases with CUDA events on the context's stream.  phase_ms receives the
 * duration of the most recent call's phases, in milliseconds, after waiting for
 * the stream: [0] block scores, [1] selection, [2] pack + cache refresh,
 * [3] restore / norm pass including its reduction (one kernel), [4] the
 * reduction as a kernel of its own (layouts cut into segments only, else 0);
 * phases a call did not run read 0. */
int scar_ckpt_profile(scar_ctx *ctx, int enable);
int scar_ckpt_profile_read(scar_ctx *ctx, float phase_ms[5]);

/* ---- Iteration-cost arithmetic of Section 3 (host only, no GPU work) --------
 * c is the linear convergence rate of the training algorithm, 0 < c < 1
 * (Eq. 5/6); dist0 = ||x^(0) - x*|| > 0.  Every function returns NaN when an
 * argument is outside its domain.
 *
 * baseline_iterations: kappa(x, eps) = log(dist0 / eps) / log(1 / c), the
 *   iterations the unperturbed sequence needs to come within eps (Section 3.1).
 * discounted_perturbation: Delta_T = sum_i c^(-iters[i]) * norms[i] of
 *   Theorem 3.2, for n perturbations of size norms[i] >= 0 met at iteration
 *   iters[i] (HOST arrays).  A single recovery at iteration T with
 *   perturbation norm p gives c^(-T) * p.
 * iteration_cost_bound: Theorem 3.2, log(1 + Delta_T / dist0) / log(1 / c):
 *   the most extra iterations the perturbations can cost.
 * irreducible_error: (c / (1 - c)) * delta_max, the accuracy floor when every
 *   iteration may be perturbed by up to delta_max (Example 3.3, infinite
 *   perturbations). */
double scar_baseline_iterations(double dist0, double eps, double c);
double scar_discounted_perturbation(const double *norms, const uint64_t *iters, uint64_t n, double c);
double scar_iteration_cost_bound(double delta_T, double dist0, double c);
double scar_irreducible_error(double delta_max, double c);

/* Self-test hook for the bounded device-side wait.  The selection kernel's
 * CTAs meet at a few points whose wait gives up after a fixed number of polls
 * (2^19 to 2^20: a quarter of a second at the earliest, about a second in
 * practice) instead of hanging.  This call makes the NEXT prioritized or
 * random save wait for one key, one record or one arrival more than its
 * selection has (host state only), so that its first wait can never
 * complete: that save takes up to about a second,
 * selects and copies nothing, leaves z untouched, and returns SCAR_ERR_TIMEOUT
 * from the call that reads its result (the save itself with a non-NULL out, or
 * scar_ckpt_last_info).  The save after that one works normally.
 * SCAR_ERR_STATE on an empty buffer. */
int scar_ckpt_selftest_arm_timeout(scar_ctx *ctx);

/* ---- Guard bands (debugging aid; no counterpart in the paper) ------------------
 * scar_ckpt_init_guarded is scar_ckpt_init for a context whose every device
 * buffer (running checkpoint, payload, scores, id and offset lists, masks,
 * selection and reduction scratch, segment tables, drain and sharding buffers
 * allocated later) sits between two bands of 256 bytes holding a known pattern,
 * the second band starting at the first byte behind the buffer.
 * scar_ckpt_debug_check_guards waits for the stream and counts, on the device,
 * the band bytes that no longer hold the pattern: any write of the library's
 * kernels just outside one of its buffers shows up as a non-zero count.
 * SCAR_ERR_STATE on a context that was not created guarded.
 * scar_static_debug_check_guard does the same for the band behind the fixed
 * array of scar_perturbation_norm_static on the current device (waits for the
 * device; SCAR_ERR_STATE before that call was ever used there). */
int scar_ckpt_init_guarded(scar_ctx **out, void *d_x, scar_dtype dt, const scar_layout *layout, void *cuda_stream);
int scar_ckpt_debug_check_guards(scar_ctx *ctx, uint64_t *bad_bytes);
int scar_static_debug_check_guard(uint64_t *bad_bytes);

/* Diagnostic builds only (library compiled with -DSCAR_SELECT_STAMPS; otherwise
 * SCAR_ERR_STATE).  Waits for the stream and copies the 32 time stamps of the
 * most recent selection kernel: SM clock cycles of its first CTA at
 *   [0] start, [1] keys loaded, then for digit pass p = 0..5
 *   [2+4p] shared histogram built, [3+4p] flushed to the global histogram
 *   (a selection that one CTA does alone flushes nothing), [4+4p] every CTA
 *   has arrived (only selections with several tiles per CTA meet at a
 *   counter; otherwise the same point as [3+4p]), [5+4p] global histogram
 *   complete and digit resolved,
 *   [26] own counts known, [27] every CTA's record read, [28] output bases
 *   known, [29] ids and offsets written.
 * Stamps of passes that did not run keep the value of an earlier selection (or
 * zero).  No counterpart in the paper: it shows where the selection of
 * checkpoint step 3 spends its time. */
int scar_ckpt_debug_select_stamps(scar_ctx *ctx, int64_t stamps[32]);

/* Waits for the stream, frees everything the context owns (never x). */
int scar_ckpt_destroy(scar_ctx *ctx);

/* ==== The training step the checkpoints are taken between ===========================
 * The paper checkpoints iterative-convergent training (Eq. 1); its first workload is
 * multinomial logistic regression.  The two operators below are the ends of such a
 * step on the GPU: the loss of a linear map followed by a softmax cross entropy with
 * its gradient, and the global norm of a gradient with clipping (which bounds one
 * step, and with it the perturbation a recovery undoes).  Both follow the conventions
 * at the top of this file: a handle owns the workspaces, all work runs on the stream
 * given at init in call order, arguments are checked before anything is enqueued,
 * nothing throws, calls only enqueue (so they can be captured in a CUDA graph) and a *_status call waits.  Operands may be
 * float32, bfloat16 or float16; sums, softmax statistics and norms are float32 or
 * wider whatever the operands are. */

/* ---- Linear softmax cross entropy ------------------------------------------------------
 * With h [T, D] (one row per token or sample), w [V, D] (one row per class) and labels
 * [T]: z = h w^T, lse_t = log sum_v exp(z_tv),
 *   row_loss_t = lse_t - z_{t, label_t}
 *   loss       = sum_t row_loss_t / n     n = rows that count (MEAN; 1 if there are
 *                                         none) or 1 (SUM)
 *   dz_tv      = (grad_scale / n) (exp(z_tv - lse_t) - [v = label_t])
 *   dh = dz w,  dw = dz^T h
 * A row whose label is ignore_label does not count: its row_loss is 0, its row of dh
 * is zero and whatever its row of h holds (NaN, infinities) reaches nothing.  A label
 * outside [0, V) that is not ignore_label is treated the same and counted
 * (scar_xent_status).  Without any row that counts the loss and both gradients are 0.
 * What is stored of the T x V values: the rows go through in pieces, as many at a time
 * as `workspace_bytes` holds (all of them where that is enough).  With gradients a
 * piece's block holds exponentials in float16 that become dz in place; float32 operands
 * have a piece of float32 logits and dz as three bfloat16 planes.  The loss alone keeps
 * two numbers per row and group of 128 classes (float32 operands: a piece of float32
 * logits too).  Products of so few tiles that their sums are cut leave float32 parts of
 * the logits (64 MiB at most).
 * 16-bit operands: dz is rounded once to their type for the two products (the matrix
 * instruction takes operands of one type), dh and dw once to it at the end; sums are
 * float32.  The gradients' error is 1.01 to 1.41 times that of rounding the exact ones
 * (in the mean square, measured).  In float32 an infinity in an operand acts as a NaN. */
typedef struct scar_xent scar_xent; /* opaque; created by scar_xent_init, freed by scar_xent_destroy */

typedef enum { SCAR_MEAN = 0, SCAR_SUM = 1 } scar_reduction;

typedef struct {
    uint64_t max_tokens;  /* most rows of h a call may have, < 2^31 */
    uint64_t n_classes;   /* V, 1 .. 2^31 - 1 */
    uint64_t dim;         /* D, 1 .. 2^31 - 1 */
    int64_t ignore_label;
    uint64_t workspace_bytes; /* bound on the block of dz that is held at a time; 0 = 1 GiB.  At least the
                                 256 rows of one piece are held, and all rows are when that needs less memory
                                 than dw's float32 sums over several pieces would. */
    scar_dtype dtype;         /* of h, w, dh, dw: SCAR_F32, SCAR_BF16 or SCAR_F16 */
    scar_reduction reduction;
    int loss_only;            /* non-zero: no workspace for gradients; scar_xent_loss_grad returns SCAR_ERR_STATE */
} scar_xent_config;

typedef struct {
    float loss;
    uint64_t rows;    /* rows that counted in the most recent call */
    uint64_t ignored; /* rows whose label was ignore_label */
    uint64_t bad;     /* rows whose label was outside [0, V) and not ignore_label */
} scar_xent_info;

/* Creates the operator with its workspaces on the current device.  cuda_stream is a cudaStream_t (NULL = default
 * stream).  Waits for the stream.  On error *out is NULL. */
int scar_xent_init(scar_xent **out, const scar_xent_config *cfg, void *cuda_stream);

/* Loss of n_tokens rows.  d_h, d_w: DEVICE matrices, row-major, rows h_pitch / w_pitch elements apart (>= D), at
 * any address their element type allows.  16-bit rows of w that lie on 16-byte boundaries are read in place, others
 * are copied first (with a dim that is a multiple of 8, the first such call allocates that copy: make it before a
 * stream capture).  d_labels: DEVICE int64.  d_row_loss: DEVICE float[n_tokens] or NULL.  d_loss: DEVICE float or
 * NULL. */
int scar_xent_loss(scar_xent *op, const void *d_h, uint64_t h_pitch, const void *d_w, uint64_t w_pitch,
                   const int64_t *d_labels, uint64_t n_tokens, float *d_row_loss, float *d_loss);

/* The same with the gradients, in one call (a training step knows the scale of its loss beforehand).
 * d_dh [T, D], d_dw [V, D]: DEVICE matrices of the operator's type, overwritten; neither may overlap an input. */
int scar_xent_loss_grad(scar_xent *op, const void *d_h, uint64_t h_pitch, const void *d_w, uint64_t w_pitch,
                        const int64_t *d_labels, uint64_t n_tokens, float grad_scale, float *d_row_loss,
                        float *d_loss, void *d_dh, uint64_t dh_pitch, void *d_dw, uint64_t dw_pitch);

/* Waits for the stream and returns the record of the most recent call.  SCAR_ERR_TIMEOUT if a wait inside one of
 * its kernels gave up (its loss is then NaN, its other outputs are invalid; the operator stays usable). */
int scar_xent_status(scar_xent *op, scar_xent_info *out);
/* Self-test hook: the next call reports a wait that gave up (host state only; none does). */
int scar_xent_selftest_arm_timeout(scar_xent *op);
uint64_t scar_xent_workspace_bytes(const scar_xent *op); /* device memory the operator holds */
uint64_t scar_xent_launch_count(const scar_xent *op);    /* kernels launched so far */
int scar_xent_destroy(scar_xent *op);

/* ---- Global gradient norm and clipping ---------------------------------------------------
 * Over a list of tensors g_1 .. g_k of any lengths (0 included), types and addresses:
 *   norm = sqrt(sum g^2) | sum |g| | max |g|        (scar_gnorm_kind)
 *   coef = min(1, max_norm / norm), 1 when norm is 0
 *   out_i = coef * g_i, rounded once
 * Sums run in float32 over short runs (in double where a sum would leave float32's
 * range, so any finite tensors have a finite norm in scar_gnorm_info; the float32 of it
 * may be infinite) and in double across them, in an order that, on one GPU, depends on
 * the lengths, the types and the addresses modulo 16 alone: equal inputs there give
 * equal bits.  A NaN or an infinity in the tensors gives the IEEE result of these
 * formulas (norm NaN: all outputs NaN; norm infinite: coef 0, NaN where g is infinite)
 * and is reported (scar_gnorm_status), so that a caller can leave the step out. */
typedef struct scar_gnorm scar_gnorm; /* opaque; created by scar_gnorm_init, freed by scar_gnorm_destroy */

typedef enum { SCAR_GNORM_L2 = 0, SCAR_GNORM_L1 = 1, SCAR_GNORM_MAX = 2 } scar_gnorm_kind;

typedef struct {
    const void *d_data; /* DEVICE, n_elems elements of type dtype, aligned to one element */
    void *d_out;        /* DEVICE, same type and length, or NULL: scar_gnorm_clip works in place */
    uint64_t n_elems;
    scar_dtype dtype; /* SCAR_F32, SCAR_BF16 or SCAR_F16 */
} scar_tensor;

typedef struct {
    double norm;
    double coef;        /* 1 after scar_gnorm_norm */
    uint64_t nonfinite; /* 1 when the norm is NaN or infinite, else 0 */
} scar_gnorm_info;

/* Registers the caller's tensors (HOST array, read before the call returns); they must stay valid and in place
 * until scar_gnorm_destroy or until scar_gnorm_bind gives their new addresses.  An output may be its own input
 * (the same as NULL) but may not overlap another tensor.  Waits for the stream. */
int scar_gnorm_init(scar_gnorm **out, const scar_tensor *h_tensors, uint64_t n_tensors, scar_gnorm_kind kind,
                    void *cuda_stream);
/* New addresses for the same lengths and types (SCAR_ERR_LAYOUT otherwise; the tensors registered before then stay).
 * Waits for the stream.  Graphs that hold captured calls work on the new tensors from then on. */
int scar_gnorm_bind(scar_gnorm *op, const scar_tensor *h_tensors, uint64_t n_tensors);
/* The norm alone.  d_norm: DEVICE float or NULL.  Enqueue only. */
int scar_gnorm_norm(scar_gnorm *op, float *d_norm);
/* Norm and scaled outputs; max_norm >= 0 (infinity leaves the values as they are).  Enqueue only. */
int scar_gnorm_clip(scar_gnorm *op, float max_norm, float *d_norm);
/* Waits for the stream and returns the record of the most recent call. */
int scar_gnorm_status(scar_gnorm *op, scar_gnorm_info *out);
/* Short lists are clipped in one launch whose CTAs wait for one another, for a millisecond at most: if a kernel of another
 * stream keeps some of them from starting for longer, the last one to run finishes the call by itself, with the same
 * bits.  scar_gnorm_finished_alone waits for the stream and counts the calls that ended this way;
 * scar_gnorm_selftest_arm_timeout makes the next clipping in one launch end so (host state only). */
int scar_gnorm_finished_alone(scar_gnorm *op, uint64_t *calls);
int scar_gnorm_selftest_arm_timeout(scar_gnorm *op);
uint64_t scar_gnorm_launch_count(const scar_gnorm *op);
int scar_gnorm_destroy(scar_gnorm *op);

/* ==========================================================================
 * Hidden layers
 *
 * What lies between a model's input and its loss: the operators below follow the
 * conventions of the training step above (operand types, float32 or wider sums,
 * streams, capture). */

/* ---- Dropout -------------------------------------------------------------------------
 * A mask that is computed from (seed, offset) wherever it is needed and stored nowhere:
 * forward, backward and a step that is taken again after a recovery have the same one.
 * Value (row t, column c) of a matrix is kept if its 16 bits are at least cut, and then
 * multiplied by 65536 / (65536 - cut):
 *   cut  = p 65536 rounded, between 1 and 65535 unless p is 0 or 1
 *   bits = the (c mod 8)-th 16 bits, low halves first, of Philox 4x32 with ten rounds,
 *          key = seed, counter = (c / 8, t, offset low, offset high)
 * A value that is dropped becomes 0 whatever it was (NaN, infinities).  Calls that are to
 * have masks of their own take different offsets (a step's number times the number of
 * masks a step has, plus which). */
typedef struct {
    double p;          /* 0 .. 1: the share that is dropped */
    uint64_t seed;
    uint64_t offset;
    const uint64_t *d_offset; /* DEVICE, added to offset, or NULL: a captured graph takes another mask at each
                                 replay if the caller changes it in between */
} scar_dropout;

/* y = mask . x (+ residual), rounded once.  DEVICE matrices of rows x cols values of type dtype, rows a pitch of
 * elements apart, at any address their type allows; d_residual may be NULL; y may be x or the residual itself (same
 * address and pitch) and may not overlap them in any other way.  Applied to dy it gives dx.  Holds no workspace and
 * no handle: enqueues on cuda_stream, on the current device.  rows and cols below 2^31. */
int scar_dropout_apply(const scar_dropout *rule, scar_dtype dtype, const void *d_x, uint64_t x_pitch, const void *d_residual,
                       uint64_t residual_pitch, void *d_y, uint64_t y_pitch, uint64_t rows, uint64_t cols, void *cuda_stream);

/* ---- Linear layer --------------------------------------------------------------------
 * With x [T, K], w [N, K], bias [N], residual [T, N]:
 *   z = x w^T + bias,   y = residual + mask . act(z)
 * and from dy [T, N] (the residual's gradient is dy itself):
 *   dz = mask . dy . act'(z),   dx = dz w,   dw = dz^T x,   dbias = sum_t dz
 * act: z; max(z, 0) (derivative 0 at 0); z Phi(z) with the Gaussian's distribution function Phi; z / (1 + exp(-z)).
 * Forward leaves act'(z) in the caller's d_slope, [T][N rounded up to 8] values of float16 beside bfloat16 operands and
 * of float32 beside the others, for backward; the mask is computed again.  16-bit operands: y is rounded once, dz once for the two
 * products (the matrix instruction takes operands of one type; a float16 dz beyond its range is infinite; of up to 16 rows or
 * 2048 values dz goes there as the sum of two values), dx, dw and dbias once; sums are float32.  In float32 an infinity in x, w or dy may act as a NaN in the products. */
typedef struct scar_linear scar_linear; /* opaque; created by scar_linear_init, freed by scar_linear_destroy */

typedef enum { SCAR_ACT_IDENTITY = 0, SCAR_ACT_RELU = 1, SCAR_ACT_GELU = 2, SCAR_ACT_SILU = 3 } scar_activation;

typedef struct {
    uint64_t max_rows;     /* most rows of x a call may have, < 2^31 */
    uint64_t in_features;  /* K, 1 .. 2^31 - 1 */
    uint64_t out_features; /* N, 1 .. 2^31 - 1 */
    scar_dtype dtype;      /* of x, w, bias, residual, y and the gradients: SCAR_F32, SCAR_BF16 or SCAR_F16 */
    scar_activation activation;
    int forward_only;      /* non-zero: no workspace for gradients; scar_linear_backward returns SCAR_ERR_STATE */
} scar_linear_config;

/* Creates the operator with its workspaces on the current device.  Waits for the stream.  On error *out is NULL.
 * Calls of one operator share its workspaces: they may not overlap (other threads, graphs captured from it and run at the same time). */
int scar_linear_init(scar_linear **out, const scar_linear_config *cfg, void *cuda_stream);

/* d_bias, d_residual, dropout (HOST, read before the call returns) and d_slope may be NULL.  DEVICE matrices, row-major,
 * rows a pitch of elements apart, at any address their type allows; d_slope on a 16-byte boundary (NULL with
 * SCAR_ACT_IDENTITY).  16-bit rows of x and w that lie on 16-byte boundaries are read in place, others are copied first
 * (with in_features a multiple of 8, the first such call allocates that copy: make it before a stream capture).  y may
 * be the residual itself (same address and pitch) and may overlap nothing else. */
int scar_linear_forward(scar_linear *op, const void *d_x, uint64_t x_pitch, const void *d_w, uint64_t w_pitch, const void *d_bias,
                        const void *d_residual, uint64_t residual_pitch, const scar_dropout *dropout, uint64_t n_rows, void *d_y,
                        uint64_t y_pitch, void *d_slope);
uint64_t scar_linear_slope_bytes(const scar_linear *op, uint64_t n_rows); /* of d_slope; 0 with SCAR_ACT_IDENTITY */

/* Gradients with the x, w, d_slope and dropout of the forward call.  d_dx, d_dw and d_dbias are overwritten; each may be NULL
 * (d_w is needed for d_dx only, d_x for d_dw).  None may overlap an input or another output.  Of no rows d_dw and d_dbias
 * are zero. */
int scar_linear_backward(scar_linear *op, const void *d_dy, uint64_t dy_pitch, const void *d_x, uint64_t x_pitch, const void *d_w,
                         uint64_t w_pitch, const void *d_slope, const scar_dropout *dropout, uint64_t n_rows, void *d_dx, uint64_t dx_pitch,
                         void *d_dw, uint64_t dw_pitch, void *d_dbias);

/* Waits for the stream.  SCAR_ERR_TIMEOUT if a wait inside a kernel of the calls since the last status gave up (their
 * outputs are invalid; the operator stays usable). */
int scar_linear_status(scar_linear *op);
/* Self-test hook: the next call reports a wait that gave up (none does). */
int scar_linear_selftest_arm_timeout(scar_linear *op);
uint64_t scar_linear_workspace_bytes(const scar_linear *op); /* device memory the operator holds */
uint64_t scar_linear_launch_count(const scar_linear *op);    /* kernels launched so far */
int scar_linear_destroy(scar_linear *op);

/* ---- Norms around a residual block -----------------------------------------------------
 * For the output f [T, D] of a block on the residual stream x [T, D], and the input n of the next block:
 *   u = f, or N(f; w_post, b_post)            (post)
 *   y = x + scale gate u                      (rounded to the operands' type)
 *   n = N(y; w_pre, b_pre)                    (pre; of the rounded y)
 *   N(v; w, b) = (v - mean v) / sqrt(var v + eps) w + b        SCAR_RESNORM_LAYER
 *              = v / sqrt(mean v^2 + eps) w                    SCAR_RESNORM_RMS
 * over each row.  The gate has a row for every rows_per_gate rows of x (1: for each; T: one for all), or is left out
 * (1).  Without f, y is x and is not written.  Backward takes the gradients dy and dn of y and n:
 *   dY = dy + N'(dn),  dx = dY,  dgate = scale sum dY u,  df = N'(scale gate dY),  dw = sum (dout hat),  db = sum dout
 * with sums over the rows (of a gate) in an order that depends on the sizes alone: equal inputs give equal bits.
 * Squares and sums are float32: rows with values above 1.8e19 have an infinite deviation. */
typedef struct scar_resnorm scar_resnorm; /* opaque; created by scar_resnorm_init, freed by scar_resnorm_destroy */

typedef enum { SCAR_RESNORM_RMS = 0, SCAR_RESNORM_LAYER = 1 } scar_resnorm_kind;
#define SCAR_RESNORM_MAX_DIM 16384

typedef struct {
    uint64_t max_rows;  /* most rows a call may have, < 2^31 */
    uint64_t dim;       /* D, 1 .. SCAR_RESNORM_MAX_DIM (SCAR_ERR_CAPACITY beyond) */
    double eps;         /* >= 0 */
    scar_dtype dtype;   /* of all tensors */
    scar_resnorm_kind kind;
    int forward_only;   /* non-zero: no workspace for gradients; scar_resnorm_backward returns SCAR_ERR_STATE */
} scar_resnorm_config;

typedef struct {
    int post, pre;           /* which norms */
    float scale;             /* of the block's output */
    const void *d_gate;      /* DEVICE [T / rows_per_gate rounded up][D], or NULL */
    uint64_t gate_pitch, rows_per_gate;
    const void *d_w_post, *d_b_post, *d_w_pre, *d_b_pre; /* DEVICE [D], NULL: 1 and 0; the b's with SCAR_RESNORM_LAYER only */
} scar_resnorm_block;

/* Creates the operator with its workspace on the current device.  Waits for the stream.  On error *out is NULL.  Calls
 * of one operator share its workspace: they may not overlap (other threads, graphs captured from it and run at the same time). */
int scar_resnorm_init(scar_resnorm **out, const scar_resnorm_config *cfg, void *cuda_stream);
/* block: HOST, read before the call returns.  DEVICE matrices, rows a pitch of elements apart, at any address their type
 * allows.  d_f may be NULL (then no post and no gate, and d_y may be NULL), d_n is needed with pre.  y may be x or f
 * itself (same address and pitch); outputs may overlap nothing in any other way. */
int scar_resnorm_forward(scar_resnorm *op, const scar_resnorm_block *block, const void *d_x, uint64_t x_pitch, const void *d_f, uint64_t f_pitch,
                         uint64_t n_rows, void *d_y, uint64_t y_pitch, void *d_n, uint64_t n_pitch);
/* d_dy may be NULL with pre (y goes nowhere else); d_dn and d_y are needed with pre.  Each gradient may be NULL; one of
 * something that the block does not have is refused.  dx may be dy or dn itself, df may be f; outputs may overlap nothing
 * in any other way. */
int scar_resnorm_backward(scar_resnorm *op, const scar_resnorm_block *block, const void *d_dy, uint64_t dy_pitch, const void *d_dn, uint64_t dn_pitch,
                          const void *d_y, uint64_t y_pitch, const void *d_f, uint64_t f_pitch, uint64_t n_rows, void *d_dx, uint64_t dx_pitch,
                          void *d_df, uint64_t df_pitch, void *d_dgate, uint64_t dgate_pitch, void *d_dw_post, void *d_db_post, void *d_dw_pre,
                          void *d_db_pre);
/* Waits for the stream.  SCAR_ERR_TIMEOUT if a wait inside a kernel of the calls since the last status gave up (their
 * outputs are invalid; the operator stays usable). */
int scar_resnorm_status(scar_resnorm *op);
/* Self-test hook: in the next call that has rows, a warp of the first CTA takes its first wait as one that ran out (the one that
 * copies rows; armed n times, the n-th or the last).  What waits for it runs into the two seconds. */
int scar_resnorm_selftest_arm_timeout(scar_resnorm *op);
uint64_t scar_resnorm_launch_count(const scar_resnorm *op); /* kernels launched so far */
int scar_resnorm_destroy(scar_resnorm *op);

/* Static description of an error code. */
const char *scar_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* SCAR_H */
