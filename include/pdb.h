/*
 * pdb.h -- C ABI of libpdb: serially-equivalent sparse SGD on one GPU.
 *
 * The method is data-centric synchronization (Parameter Database): each
 * training example's sparse SGD update is a transaction whose read and write
 * set is the example's nonzero features.  Examples that share no feature run
 * concurrently; examples that share one run in data order, so the trained
 * weights equal those of sequential SGD over the data in its given order.
 *
 * Paper anchors (the paper's own section, definition and algorithm labels):
 *   Definition 1   parameter database M(Theta, D): D immutable, Theta mutable
 *   Definition 2   chunks (here: single features)
 *   Definition 3   an iteration reads its chunks, then writes them
 *   Algorithm 1,   the sequential computation every result must equal
 *   Definition 4
 *   Algorithm 2a   BSP: read barrier, reads, compute, write barrier, writes
 *   Algorithm 2b   relaxed: per-chunk Read and Write Constraints (Sec. 4.4)
 *   Theorem 2      RC + WC give the sequential result
 *   Theorem 3      BSP executions are a subset of RC/WC executions
 *   Section 5      read protocol: a per-chunk iteration number gates reads
 *   Section 7      admissible delay: reads and writes within delta iterations
 *
 * Conventions for every call:
 *   - Pointers named as device pointers must be device memory of the current
 *     CUDA device; the caller owns them and keeps them alive until the work
 *     queued on `stream` has finished.
 *   - `stream` is a cudaStream_t passed as void*; NULL is the legacy default
 *     stream.  Every call only enqueues work on `stream` (asynchronous),
 *     except where a comment says it synchronizes.
 *   - Return value: PDB_OK or a negative PDB_E* code for errors found on the
 *     host (arguments, allocation, launch).  Errors found by the kernels
 *     (bad CSR contents, expired waits) are recorded in the conflicts
 *     handle's device status word; read it with pdb_status().  Once a handle
 *     holds an error, later kernels that use it return at once and the
 *     handle must be rebuilt.
 *   - Calls that share a handle must be ordered on one stream (the handles
 *     hold device-side counters that a concurrent call would clobber).
 *   - Limits: n_rows, n_cols and nnz below 2^31 (positions and ids are int32).
 *   - Memory: handles allocate stream-ordered from a memory pool the library
 *     creates for each device on first use.  That pool keeps freed blocks for
 *     reuse (its release threshold is raised) until the process exits; the
 *     device's default pool and every other process-wide CUDA setting are left
 *     as they are.
 *   - Host memory: a pinned, device-mapped slab of small words, one per
 *     process (grown in slabs of 64 slots), holds each conflicts handle's info
 *     words and stages pdb_status' read.  The library's kernels store those
 *     words into it directly: a device-to-host copy of a few bytes would queue
 *     behind the caller's large copies on the copy engine.
 *   - Diagnostics: every call opens an NVTX range named after it (seen by
 *     profilers); with the environment variable PDB_LOG set to anything but
 *     "" or "0" each call (but pdb_sgd_epoch_ready_noalloc) prints one line
 *     of pdb_get_stats on stderr afterwards, which synchronizes the device.
 *     PDB_NEAR (pdb_build_conflicts) and PDB_LEVELS (pdb_schedule_build)
 *     are described where they apply.
 */
#ifndef PDB_H
#define PDB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- errors */
#define PDB_OK 0
#define PDB_EINVAL (-1)   /* null pointer, negative size, row_ptr not nondecreasing from 0 to nnz, size mismatch */
#define PDB_ERANGE (-2)   /* a feature id outside [0, n_cols) */
#define PDB_EDUP (-3)     /* a feature id repeated inside one example (read/write sets are sets, Def. 3) */
#define PDB_ENOMEM (-4)   /* device allocation failed */
#define PDB_ECUDA (-5)    /* a CUDA runtime call or launch failed */
#define PDB_ETIMEOUT (-6) /* a bounded device-side wait expired (the kernel stopped, the GPU stays usable) */
#define PDB_EFAULT (-7)   /* an internal invariant failed on the device */
#define PDB_ESTATE (-8)   /* wrong handle for this call (e.g. a READY schedule where levels are needed) */
#define PDB_ETOOBIG (-9)  /* beyond a fixed limit: the scratch of pdb_sgd_epoch_ready_noalloc, CHAIN's
                             row length, or a feature occurring 2^29 times or more */

/* ---------------------------------------------------------------- types */

/* The data D of the parameter database M(Theta, D) (Definition 1): n_rows
 * examples in CSR form over n_cols features.  Example t holds the features
 * col[row_ptr[t] .. row_ptr[t+1]) with values val[...] (val == NULL means
 * every value is 1.0, binary features).  Device pointers, caller-owned,
 * never written by the library.  Example order is the data order that the
 * result must reproduce.  Rows may be empty; ids in a row must be distinct
 * (any order). */
typedef struct {
    int64_t n_rows, n_cols, nnz;
    const int64_t *row_ptr; /* [n_rows + 1] */
    const int32_t *col;     /* [nnz] */
    const float *val;       /* [nnz] or NULL */
} pdb_csr;

/* Loss term f_t of example t as a function of its margin m = w . x_t
 * (Eq. 2's data terms; the regularizer g is not supported).
 *   LOGISTIC  f = log(1 + exp(-y m)),  y in {-1, +1}
 *   SQUARED   f = (m - y)^2 / 2
 *   HINGE     f = max(0, 1 - y m), subgradient 0 at y m = 1 */
typedef enum { PDB_LOSS_LOGISTIC = 0, PDB_LOSS_SQUARED = 1, PDB_LOSS_HINGE = 2 } pdb_loss;

/* How pdb_sgd_epoch keeps conflicting examples in data order.
 *   LEVELS  dependency levels: level-synchronous execution, one grid barrier
 *           per level (each level is one BSP step over disjoint examples,
 *           Theorem 3)
 *   READY   per-feature ready counters: an occurrence of feature j with rank
 *           r reads w_j once the iteration number of j equals r and
 *           publishes r + 1 with its write (the read protocol of Section 5
 *           with the iteration number counted per feature); no barrier at
 *           all.  The number lives in the same 64-bit word as the weight,
 *           counted on from epoch to epoch: all epochs run in one pipelined launch,
 *           each feature's next-epoch occurrences starting as soon as its
 *           last occurrence of the epoch has written.
 *   CHAIN   for conflict graphs that are close to one chain (a feature in
 *           most examples): one thread block runs the examples strictly in
 *           data order (Algorithm 1 itself), prefetching ids, values and
 *           weights ahead and forwarding each new weight whose next
 *           occurrence is among the next 40 examples through shared memory,
 *           so a dependency hop costs a few hundred cycles (examples of at
 *           most 256 ids).  Longer examples run with all n_cols weights
 *           resident in shared memory instead, when they fit (about 55,000
 *           features; dense examples of ~1000 features); else PDB_ETOOBIG.
 *   WINDOW  for conflict graphs whose consecutive occurrences of a feature
 *           mostly lie far apart: w stays a plain float array.  A position
 *           whose previous occurrence lies at least `near` positions back
 *           (a distance fixed by the build, >= 2^22) reads w_j once the
 *           completion watermark -- every example before it finished --
 *           has passed that occurrence; a nearer one takes the weight from
 *           its previous occurrence through feature j's 64-bit record,
 *           bits(w_j) | tag << 32, written only by positions whose next
 *           occurrence is near, the tag being the reader's occurrence rank
 *           with an epoch stamp (the read protocol of Section 5 on the near
 *           pairs only).
 *   AUTO    CHAIN when the longest per-feature chain exceeds n_rows / 20 and
 *           CHAIN takes the rows (see above); else WINDOW when at most 1/8
 *           of the positions have a near next occurrence; else READY (waits
 *           on the host for the conflict build to read those numbers). */
typedef enum {
    PDB_SCHED_LEVELS = 0,
    PDB_SCHED_READY = 1,
    PDB_SCHED_CHAIN = 2,
    PDB_SCHED_AUTO = 3,
    PDB_SCHED_WINDOW = 4
} pdb_sched_mode;

/* Gates of pdb_ssp_epoch (Section 7; iterations counted per feature, the
 * occurrence of feature j with rank r being iteration r of j). */
typedef enum {
    PDB_SSP_COUNT = 1,  /* counters: rank r reads once r - delay writes of j are done and writes once
                         * r - delay + 1 occurrences of j have read (the default) */
    PDB_SSP_PREFIX = 2  /* prefixes: rank r reads once every rank <= r - 1 - delay has written and writes
                         * once every rank <= r - delay has read (the Write Protocol's slowest reader) */
} pdb_ssp_gates;

/* Launch and wait options; a zeroed struct (or NULL) selects the defaults. */
typedef struct {
    int32_t blocks_per_sm;     /* persistent grid = blocks_per_sm x #SM (at most the occupancy
                                  maximum); 0 = that maximum, for WINDOW 3, for READY 2 or 4;
                                  pdb_bsp_epoch: the most blocks of one launch, 0 = no limit */
    int32_t ticket_chunk;      /* READY: consecutive examples a warp takes per ticket; 0 = 1 or 2 by
                                  how often examples conflict, under pdb_ssp_epoch 2 */
    double wait_timeout_s;     /* limit of every device-side wait; 0 = 2 seconds; at most 10^6 seconds */
    uint64_t *trace;           /* optional (NULL = off), pdb_sgd_epoch and pdb_ssp_epoch: device array of
                                * n_epochs * n_rows * 2 words; per example (epoch-major) the %globaltimer
                                * value (ns) once all its reads are done, then once its update is computed
                                * and before any of its writes is issued, so a caller can check an
                                * execution against the Read and Write Constraints (Section 4.4) or the
                                * asynchronous ones (Section 7).  Costs two stores per example. */
    int32_t ssp_gates;         /* pdb_ssp_epoch: a pdb_ssp_gates value; 0 = PDB_SSP_COUNT */
} pdb_opts;

/* Sizes and timings; timings are CUDA-event milliseconds of the last call of
 * each kind on the given handles (0 when not run). */
typedef struct {
    int64_t n_rows, n_cols, nnz;
    int64_t n_levels;        /* LEVELS schedule: number of levels L; else -1 */
    int64_t max_level_width; /* LEVELS schedule: largest level; else -1 */
    int64_t max_chain;       /* most occurrences of one feature (longest per-feature chain) */
    double ms_build, ms_schedule, ms_sgd, ms_bsp;
    double ms_sgd_kernels;   /* pdb_sgd_epoch's update kernels alone (no record packing) */
    int64_t sched_mode;      /* mode the schedule runs (AUTO resolved); -1 without a schedule */
} pdb_stats;

typedef struct pdb_conflicts pdb_conflicts; /* opaque, library-owned device arrays */
typedef struct pdb_schedule pdb_schedule;   /* opaque, library-owned device arrays */
typedef struct pdb_bsp_plan pdb_bsp_plan;   /* opaque, library-owned device arrays */

/* ---------------------------------------------------------------- calls */

/* Conflict structure of D (Definitions 2-3; read protocol of Section 5).
 * Validates X on the device (row_ptr, id range, no repeated id in a row),
 * stable-sorts the (feature, position) pairs by feature and links
 * consecutive occurrences of each feature into a chain:
 *   csc_pos[nnz]    positions grouped by feature, data order inside a feature
 *   feat_ptr[F+1]   feature j occupies csc_pos[feat_ptr[j] .. feat_ptr[j+1])
 *   prev[p], next[p] previous / next position holding col[p], -1 if none
 *   rank[p]         number of earlier positions holding col[p]
 * It also marks, per position, whether the previous and the next
 * occurrence lie within a distance `near` (the WINDOW schedule's input; see
 * pdb_schedule_ready) and counts those pairs: near = 2^22 positions, or
 * k * 2^15 rounded up to a power of two for a mean example length k > 128,
 * or the value of the environment variable PDB_NEAR (>= 1) when set at
 * this call.  Any near >= 1 gives the same SGD result; it only decides which
 * positions wait on the watermark.
 * A feature occurring 2^29 times or more is reported as PDB_ETOOBIG.
 * Above 2^22 positions the position-order gate array is built on first use
 * (a READY, CHAIN or LEVELS schedule, or pdb_conflicts_arrays), enqueued on
 * that call's stream; the WINDOW schedule needs only the near pairs' words,
 * which the build writes directly.
 * *out receives a new handle (free with pdb_conflicts_free) even when the
 * device later reports a CSR error through pdb_status.  The handle keeps
 * referring to X's arrays (D is immutable, Definition 1): they must stay
 * valid and unchanged while the handle is in use.  Allocates its arrays
 * stream-ordered on `stream`. */
int pdb_build_conflicts(const pdb_csr *X, pdb_conflicts **out, void *stream);

/* Borrowed device pointers into the handle (valid until it is freed): the
 * per-feature occurrence chains of Section 5's read protocol.  Any output
 * pointer may be NULL.  prev/next/rank are derived from the CSC
 * order (rank = slot - feat_ptr[j], neighbours in the slot order) and are
 * materialized by a kernel enqueued on `stream` the first time one of them
 * is requested; read them after that work has completed. */
int pdb_conflicts_arrays(const pdb_conflicts *c, const int32_t **csc_pos, const int64_t **feat_ptr,
                         const int32_t **prev, const int32_t **next, const int32_t **rank, void *stream);

/* Schedule for pdb_sgd_epoch (each mode keeps the Read and Write
 * Constraints of Section 4.4 per feature, so every mode gives the sequential
 * result, Theorem 2).
 *   LEVELS (Theorem 3): level[t] = 1 + max over features j of t with an
 *     earlier occurrence of level[row of that occurrence], 0 if none
 *     (longest conflict path), computed by dataflow (examples in data order, each
 *     waiting, bounded, for its predecessors' levels) or, with the
 *     environment variable PDB_LEVELS=kahn, by a Kahn-style frontier sweep
 *     (one grid barrier per level); both give the same levels.  order[N]
 *     lists the examples by level, ascending id inside a level; level_ptr[L+1]
 *     delimits the levels.
 *   READY (Section 5, read protocol): one 64-bit record per feature,
 *     bits(w_j) | version_j << 32, filled from w by pdb_sgd_epoch; each
 *     position waits for the version equal to its occurrence rank (the
 *     conflicts' gate array).
 *   CHAIN (Algorithm 1 in data order on one SM): per position, whether an
 *     example among the 40 before it writes its feature last (its weight is
 *     then forwarded on chip) and where the next occurrence sits if within
 *     the 40 examples after; nothing when the
 *     longest example has more than 256 ids and the weights fit in shared
 *     memory (resident); PDB_ETOOBIG when they do not.
 *   WINDOW: per feature a 64-bit hand-off record for near pairs, one
 *     progress word per worker warp, a ticket and the completion watermark;
 *     the positions' near flags are in the gate.
 *   AUTO: CHAIN, WINDOW or READY (see pdb_sched_mode).
 * Allocates stream-ordered on `stream`. */
int pdb_schedule_build(const pdb_conflicts *c, pdb_sched_mode mode, pdb_schedule **out, void *stream);

/* LEVELS schedule arrays (borrowed device pointers, any may be NULL) and the
 * level count (Theorem 3's levels).  SYNCHRONIZES `stream` to read L from the device.
 * PDB_ESTATE for a READY schedule. */
int pdb_schedule_levels(const pdb_schedule *s, const int32_t **level, const int32_t **order,
                        const int64_t **level_ptr, int64_t *n_levels, void *stream);

/* READY and WINDOW schedule arrays (borrowed device pointers, any may be
 * NULL; Section 5's read protocol per feature): gate[nnz], per position bits
 * 0..28 the version it waits for (its occurrence rank), bit 29 set when the next occurrence of its feature lies
 * within the build's `near` distance, bit 30 when the previous one does,
 * bit 31 on the last occurrence of its feature (under WINDOW with more than
 * 2^22 positions: the WINDOW engine's copy, which holds only the words of
 * positions with a near pair and 0 elsewhere); and, READY only,
 * records[n_cols] (weight bits | version << 32; in epoch e the occurrence of
 * rank r waits for version e * n_rows + r, modulo 2^32;
 * meaningful while pdb_sgd_epoch runs; NULL under WINDOW).  PDB_ESTATE for LEVELS and CHAIN
 * schedules. */
int pdb_schedule_ready(const pdb_schedule *s, const uint32_t **gate, const uint64_t **records);

/* n_epochs passes of SGD over X in data order (Algorithm 1 with one
 * iteration per example), run concurrently under the schedule's constraint.
 * w (device, n_cols floats, caller-owned) is read and updated in place; y
 * (device, n_rows floats) are the labels.  For every example t:
 *   m = w . x_t         32 partial sums: element i of the row adds into
 *                       partial i mod 32 with a fused multiply-add, then
 *                       the partials combine pairwise (xor 16, 8, 4, 2, 1)
 *   g = dloss/dm (m, y) fp32; logistic uses exp by Cody-Waite reduction and
 *                       a degree-7 Taylor polynomial
 *   w_j = w_j - (eta*g) * x_tj  for the features of t
 * Each fp32 operation is rounded once, so the result is bitwise the same for
 * every schedule and equals the sequential run (Theorem 2).
 * X and c must be the same data the schedule was built from.  The host
 * waits for c's build to complete if it has not (the kernel variant depends
 * on the longest example, which the build records). */
int pdb_sgd_epoch(const pdb_csr *X, const float *y, const pdb_conflicts *c, const pdb_schedule *s, float *w,
                  pdb_loss loss, float eta, int n_epochs, const pdb_opts *opts, void *stream);

/* SGD with admissible delay (Section 7): like pdb_sgd_epoch under a READY
 * schedule, with the asynchronous Read and Write Constraints per feature
 * (iterations counted per feature: the occurrence of j with rank r is
 * iteration r of j), in the form opts->ssp_gates selects:
 *   PDB_SSP_COUNT   (default) rank r reads w_j once at least r - delay
 *                   writes of j are done, and writes once at least
 *                   r - delay + 1 occurrences of j have read;
 *   PDB_SSP_PREFIX  rank r reads once every rank <= r - 1 - delay of j has
 *                   written, and writes once every rank <= r - delay has
 *                   read (the paper's Write Protocol: a writer waits for
 *                   the slowest reader).  Keeps a done-bitmap per direction
 *                   over the CSC slots: nnz / 4 bytes in all, allocated on
 *                   first use and kept with the schedule.
 * Either way a write applies its step to the current w_j (an atomic fp32
 * add of -(eta*g)*x_j), so every example's update is applied exactly once;
 * w is updated in place.
 *   delay = 0    the sequential result, bitwise equal to pdb_sgd_epoch
 *                (both forms)
 *   delay > 0    the result depends on timing and is not deterministic.  A
 *                read of rank r sees at least r - delay writes of its
 *                feature.  Under PDB_SSP_PREFIX it sees every write of rank
 *                <= r - 1 - delay and none of rank >= r + delay; under
 *                PDB_SSP_COUNT a slow reader holds no writer back, so its
 *                read may also see writes of later occurrences
 *   delay >= the longest chain  no waits at all (Hogwild with atomic updates)
 *   coef         optional device array of n_epochs * n_rows floats (NULL for
 *                none): the step eta*g each example applied, epoch-major,
 *                for auditing a delayed run
 * s must be a READY schedule of c (PDB_ESTATE otherwise); delay < 0 or an
 * unknown opts->ssp_gates is PDB_EINVAL; under PDB_SSP_PREFIX a gate word
 * whose rank lies past its feature's occurrences is PDB_EFAULT (reported
 * through pdb_status).  Every wait is bounded (pdb_opts.wait_timeout_s). */
int pdb_ssp_epoch(const pdb_csr *X, const float *y, const pdb_conflicts *c, const pdb_schedule *s, float *w,
                  pdb_loss loss, float eta, int n_epochs, int64_t delay, float *coef, const pdb_opts *opts,
                  void *stream);

/* BSP comparison (Algorithm 2a with `batch` examples between barriers):
 * per batch [b*B, min((b+1)*B, N)) every example computes c_i = eta *
 * dloss/dm at the weights of the batch start (read barrier), then each
 * feature j takes delta_j = sum over the batch's examples, ascending, of
 * c_i * x_ij and w_j = w_j - delta_j (write barrier).  batch = 1 equals
 * sequential SGD (Theorem 1).  Two kernel launches per batch, of at most
 * opts->blocks_per_sm blocks per SM each when that is set (and then no launch
 * overlaps the one before it; 0 = each kernel's own grid).  No kernel waits for
 * another's memory, so opts->wait_timeout_s has nothing to limit.  Allocates
 * per-call scratch stream-ordered.  The host waits for the conflict build of c
 * to finish, and, as for any sequence of launches, while more of them are
 * pending than the launch queue holds (about a thousand): a call of 2 * batches *
 * n_epochs launches beyond that returns when all but the last ones have run. */
int pdb_bsp_epoch(const pdb_csr *X, const float *y, const pdb_conflicts *c, float *w, pdb_loss loss, float eta,
                  int64_t batch, int n_epochs, const pdb_opts *opts, void *stream);

/* Algorithm 2a split over data-parallel ranks.  Every rank holds the whole
 * data and a replica of w.  Per batch b (rows [b*B, min((b+1)*B, N))) each
 * rank computes the coefficients c_i = eta * dloss/dm of its slice of the
 * batch's rows at the batch-start weights (the reads), the ranks gather the
 * batch's coefficients in row order (a collective of the caller's choice),
 * and every rank applies delta_j = sum over the batch's examples, ascending,
 * of c_i * x_ij, w_j = w_j - delta_j (the writes).  The arithmetic and its
 * order are pdb_bsp_epoch's, so any split gives that call's result bit for
 * bit.
 *
 * pdb_bsp_plan_build: sorts c's pairs by (batch, feature, example) once for
 *   batch size `batch` (>= 1; above N it is N) into a plan handle (device
 *   arrays, library-owned; the plan borrows c, which must outlive it).
 *   SYNCHRONIZES `stream` (the batch bounds are copied to the host).
 *   PDB_EINVAL for a NULL argument or batch < 1.
 * pdb_bsp_plan_batches: number of batches, or -1 for NULL.
 * pdb_bsp_coef: coef[i - row_begin] = c_i for rows [row_begin, row_end),
 *   which must lie inside one batch (PDB_EINVAL otherwise); w = the batch's
 *   start weights (device, n_cols floats); coef device, caller-owned.
 *   X, y, loss as for pdb_sgd_epoch.  Asynchronous.
 * pdb_bsp_apply: the write half of batch `batch_index` with coef = all of
 *   the batch's coefficients in row order (device, rows of the batch
 *   floats); w updated in place.  Asynchronous.  An inconsistent plan is
 *   PDB_EFAULT in c's status word.
 * pdb_bsp_plan_free: waits for the work enqueued on the plan, frees its arrays. */
int pdb_bsp_plan_build(const pdb_conflicts *c, int64_t batch, pdb_bsp_plan **out, void *stream);
int64_t pdb_bsp_plan_batches(const pdb_bsp_plan *p);
int pdb_bsp_coef(const pdb_bsp_plan *p, const pdb_csr *X, const float *y, const float *w, pdb_loss loss, float eta,
                 int64_t row_begin, int64_t row_end, float *coef, void *stream);
int pdb_bsp_apply(const pdb_bsp_plan *p, float *w, int64_t batch_index, const float *coef, void *stream);
void pdb_bsp_plan_free(pdb_bsp_plan *p);

/* SYNCHRONIZES `stream` and returns the device status of handle c: PDB_OK
 * or the first error a kernel recorded (PDB_EINVAL, PDB_ERANGE, PDB_EDUP,
 * PDB_ETIMEOUT, PDB_EFAULT); PDB_ECUDA if the synchronization itself fails. */
int pdb_status(const pdb_conflicts *c, void *stream);

/* Sizes and timings; waits (host) for the work enqueued on c and s to read
 * the event timers and L, not for the device's other streams.  s may be
 * NULL. */
int pdb_get_stats(const pdb_conflicts *c, const pdb_schedule *s, pdb_stats *out);

/* Release a handle: waits for the work enqueued on this handle by earlier
 * calls (not for the rest of the device, whose other streams keep running),
 * then returns its arrays to the library's memory pool. */
void pdb_conflicts_free(pdb_conflicts *c);
void pdb_schedule_free(pdb_schedule *s);

/* Text of an error code. */
const char *pdb_strerror(int code);

/* Allocation-free variant of pdb_sgd_epoch with a READY schedule
 * (Algorithm 1 under Section 5's read protocol).  The paper has no
 * counterpart of the allocation-free form.  It is for callers that cannot
 * let a library allocate device memory while they train: a server that has
 * handed all device memory to its own pool and must not see it grow or
 * fragment, or a host runtime that accounts for every device allocation
 * itself.  It calls no cudaMalloc, cudaFree or allocating library routine:
 * its scratch (one 64-bit (weight, version) record per feature, a ticket
 * counter and a status word) is one fixed array inside the library of 2^20
 * records, about 8 MiB, that every GPU loading the library holds until the
 * process exits.
 *   X, y, w     as for pdb_sgd_epoch; X->n_cols must be <= 2^20, else
 *               PDB_ETOOBIG and nothing runs.
 *   gate[nnz]   per position, the gate word (occurrence rank of its feature
 *               in bits 0..28, bit 31 on the feature's last occurrence,
 *               bits 29-30 ignored here) -- the array that
 *               pdb_schedule_ready returns for a READY schedule of X (device,
 *               caller-owned here).
 * Same arithmetic and result as pdb_sgd_epoch.  Set-up: the first call on
 * each device (and again after that device's context is reset) looks up
 * the array's device address with cudaGetSymbolAddress.  The call cannot be
 * recorded into a CUDA graph (it synchronizes).  All calls on a device share the array,
 * which keeps the last call's contents (each call clears what must start at
 * zero): calls whose GPU work overlaps race, so order them on one stream.
 * SYNCHRONIZES `stream` (the status word is copied to the host) and returns
 * PDB_OK, a kernel-recorded error (PDB_ETIMEOUT, PDB_EFAULT), or a host
 * error. */
int pdb_sgd_epoch_ready_noalloc(const pdb_csr *X, const float *y, const uint32_t *gate, float *w, pdb_loss loss,
                                float eta, int n_epochs, void *stream);

/* ---------------------------------------------------------------- token models
 *
 * Operators of models over tokens: a chunk of the parameter database
 * (Definition 2) is a row of a table, a token's id names the row it reads and
 * updates (Definition 3), and an update sums an id's contributions in a fixed
 * order, as Algorithm 2a's write half does (pdb_bsp_apply: the data's; here the
 * data's in pieces, pdb_embed_grad), with vectors for scalars.  The softmax losses
 * take the place of pdb_loss.  The paper has no formulas for them; each declaration gives its own.
 *
 * Every call but pdb_clip's takes a pdb_tokens handle: the workspace of pdb_embed_grad, pdb_route and pdb_verify, and
 * the status word in which the kernels record an id out of range
 * or an expired wait (pdb_tokens_status).  A recorded error stops no later call: a bad id gives the
 * result its declaration states.  Calls that share a handle must be ordered on
 * one stream, and made while the device is current that was at pdb_tokens_create
 * (PDB_EINVAL otherwise).  Sums, softmax statistics and losses are held in fp32; a result
 * in 16 bits is rounded once.  No atomics add floating values: the same call on the same
 * inputs gives the same bits.  How a row of logits is split, and so the order of its sums, depends on
 * its length, its alignment and the number of rows of the call: the same row alone and among others may
 * differ in the last bits.  No call allocates but pdb_tokens_create (and pdb_embed_grad above
 * 65,536 ids: scratch of the radix sort, stream-ordered from the library's pool); all but
 * these and pdb_tokens_status, pdb_embed_grad up to 65,536 ids included, can be recorded into a CUDA graph (keep the
 * handle until the graph's last run has finished: pdb_tokens_free does not wait for it).
 * PDB_LOG prints nothing for these calls. */

/* Element types of a matrix: 32-bit, bfloat16, IEEE half. */
typedef enum { PDB_TYPE_FLOAT = 0, PDB_TYPE_BFLOAT = 1, PDB_TYPE_HALF = 2 } pdb_type;

/* rows x cols elements of one type in device memory; element (i, j) at
 * data[i * stride + j], stride >= cols (elements; any alignment of the element
 * type; stride is ignored for rows < 2).  Rows and columns may be 0. */
typedef struct {
    void *data;
    int64_t rows, cols, stride;
    int32_t type; /* a pdb_type value */
} pdb_mat;

/* n ids in device memory, 64 bits each when wide != 0, else 32: id i at
 * data[i * stride], stride >= 1 (ids; ignored for n < 2) */
typedef struct {
    const void *data;
    int64_t n, stride;
    int32_t wide;
} pdb_ids;

typedef struct pdb_tokens pdb_tokens; /* opaque, library-owned device arrays */

/* Handle for calls of at most max_tokens ids (below 2^31; in pdb_route, slots) and, in pdb_embed_grad, rows of at
 * most max_dim elements; holds 64 KB, and about 8 + max_dim / 4 bytes for each of
 * max_tokens (12 more above 65,536).  Allocates stream-ordered on `stream`.
 * pdb_tokens_free waits for the work enqueued on the handle, then releases it.
 * pdb_tokens_status SYNCHRONIZES `stream` and returns the first error that a
 * kernel recorded in the handle (PDB_OK when none). */
int pdb_tokens_create(int64_t max_tokens, int64_t max_dim, pdb_tokens **out, void *stream);
void pdb_tokens_free(pdb_tokens *t);
int pdb_tokens_status(const pdb_tokens *t, void *stream);

/* Tries of a device-side wait in later calls on the handle (pdb_distill with gradient is the one
 * that waits), each 20 ns to a microsecond, before PDB_ETIMEOUT: 2^22 unless set, and at most that.
 * With 0 no try is made and such calls end with PDB_ETIMEOUT and undefined results: for tests of
 * what a program does then. */
int pdb_tokens_set_wait_limit(pdb_tokens *t, int64_t tries);

/* out[i, :] = scale * table[ids[i], :]  (ids->n = out->rows, cols equal).
 * Reads of the chunks that the ids name (Definition 3).  An id equal to `pad`
 * gives a row of zeros, whatever its value; so does any other id outside [0, table->rows), which
 * is recorded as PDB_ERANGE.  The product is formed in fp32 and rounded once to
 * out's type.  out must not overlap the table. */
int pdb_embed(pdb_tokens *t, const pdb_mat *table, const pdb_ids *ids, float scale, int64_t pad, const pdb_mat *out,
              void *stream);

/* dtable[v, :] = scale * sum of dout[i, :] over the i with ids[i] = v, i
 * ascending (the ordered sums of Algorithm 2a's writes), 0 for an id that does not
 * occur; with accumulate != 0 the sum is added to dtable[v, :] and the other
 * rows are not touched, so that dtable = the table and scale = -eta * scale of
 * pdb_embed make the SGD step in place.  Ids equal to `pad` are left out; so are
 * other ids outside [0, dtable->rows), which are recorded as PDB_ERANGE.
 * The ids are sorted with a stable sort; an id's rows are summed in fp32 one after the other
 * in pieces of 32, and of an id with more the sums of every 8th piece together, then these (up to) eight in turn: an
 * order fixed by the id's number of rows.  The sum is multiplied by scale and rounded once to
 * dtable's type after the old value is added.  dout must not overlap dtable.
 * PDB_ETOOBIG beyond the handle's max_tokens or max_dim. */
int pdb_embed_grad(pdb_tokens *t, const pdb_ids *ids, const pdb_mat *dout, float scale, int64_t pad, int accumulate,
                   const pdb_mat *dtable, void *stream);

/* Per row of logits (z = scale * logits, scale > 0 the inverse temperature, at most 2.3e38,
 * p = softmax of z):
 *   lse[r]      log sum_j exp z_j
 *   logp[r]     z_t - lse, t = ids[r]
 *   entropy[r]  - sum_j p_j log p_j   (terms with p_j = 0 are 0)
 *   top_logp[r, 0..k), top_ids[r, 0..k)   the k largest logits, descending, ties
 *               by the lower id, as log probabilities, and their ids
 *               (row-major, k <= 64 and k <= cols; a NaN counts as largest)
 * Any output may be NULL (ids too, when logp is).  Where ids[r] = `ignore`,
 * logp[r] = 0; so also for any other id outside [0, cols), recorded as PDB_ERANGE.
 * A logit of -inf is a token that the mask leaves out.  A row with nothing left
 * has lse = logp = top_logp = -inf and entropy 0; a row that holds a NaN or
 * +inf has NaN for lse, logp, entropy and top_logp. */
int pdb_logprobs(pdb_tokens *t, const pdb_mat *logits, const pdb_ids *ids, float scale, int64_t ignore, float *logp,
                 float *lse, float *entropy, int64_t k, float *top_logp, int32_t *top_ids, void *stream);

/* Gradient of sum_r (dlogp[r] * logp[r] + dentropy[r] * entropy[r]) with
 * respect to the logits, lse and entropy as pdb_logprobs gave them:
 *   dlogits[r, j] = scale * (dlogp[r] * ([j = t] - p_j) - dentropy[r] * p_j * (log p_j + entropy[r]))
 * dlogp or dentropy may be NULL (zero); entropy is read with dentropy only,
 * ids with dlogp only.  p is formed from lse where |lse| < 256; above, where its rounding would show in p, the
 * row's maximum and sum are formed again.  A row whose two coefficients are 0 (dlogp counts as 0 where
 * pdb_logprobs leaves ids[r] out) or that has nothing left gets zeros, whatever it
 * holds.  dlogits may be the logits' own memory (same data, stride and type);
 * it must not overlap them otherwise. */
int pdb_logprobs_grad(pdb_tokens *t, const pdb_mat *logits, const pdb_ids *ids, float scale, int64_t ignore,
                      const float *lse, const float *entropy, const float *dlogp, const float *dentropy,
                      const pdb_mat *dlogits, void *stream);

/* Distillation from a teacher's top logits: row r of the student's logits
 * against K = top_logits->cols teacher logits (K <= 1024), slot k being token
 * top_ids->data[r * top_ids->stride + k]: here n = rows * K and stride, at least K,
 * is that of the rows.  With T = temperature > 0 (from 4.3e-39 to 1.8e19), p = softmax of logits[r] / T:
 *   teacher_lse == NULL   q_k = softmax of top_logits[r] / T over the row's slots
 *     loss[r] = T^2 * sum_k q_k (log q_k - log p_k)
 *   else   teacher_lse[r] = log sum exp of ALL the teacher's logits / T,
 *     q_k = exp(top_logits[r, k] / T - teacher_lse[r]), and what is left,
 *     q_t = 1 - sum_k q_k, stands in one bucket against the student's
 *     p_t = sum of p over the tokens in no slot: adds T^2 * q_t (log q_t - log p_t).
 *     q_t <= 1e-6 counts as 0 (the rounding of teacher_lse).
 * dlogits == NULL: the loss alone.  Else also the gradient of sum_r weight[r] * loss[r]
 * (weight == NULL: every weight 1), for tokens j:
 *   in a slot        weight * T * (p_j - sum of q_k over the slots of j)
 *   in none          weight * T * p_j * (1 - q_t / p_t)  (weight * T * p_j without the bucket)
 * loss may be NULL then.  A negative id is an empty slot; an id >= cols counts as one and is
 * recorded as PDB_ERANGE.  Slots of one token add up in q (a teacher that lists a token
 * twice).  A row without slots, or whose slots all hold -inf, has loss 0 and
 * gradient 0; a row of weight 0 has gradient 0, whatever it holds; a row of logits with
 * nothing but -inf has loss +inf and gradient 0 whatever its teacher logits hold.  Else a NaN in a row's logits or in its slots' teacher logits makes its
 * loss and all of its gradient NaN.
 * dlogits may be the logits' own memory (same data, stride and type); it must not overlap
 * them otherwise.  PDB_ETOOBIG above 1024 slots or 2^21 tokens.  Every wait of the kernel is bounded
 * (pdb_tokens_set_wait_limit): one that runs out is recorded as PDB_ETIMEOUT, ends the call's work on further rows of the
 * same blocks, and leaves loss and dlogits undefined. */
int pdb_distill(pdb_tokens *t, const pdb_mat *logits, const pdb_ids *top_ids, const pdb_mat *top_logits,
                const float *teacher_lse, float temperature, float *loss, const float *weight, const pdb_mat *dlogits,
                void *stream);

/* Drafted tokens verified (speculative sampling: Leviathan, Kalman, Matias 2023; Chen et al. 2023): a draft model, as pdb_distill trains
 * one, has proposed n_drafts tokens for each of n sequences; the tokens that come out are distributed as if drawn one by one from the
 * target.  Sequence s has the target's logits in rows s * (n_drafts + 1) + d, d = 0 .. n_drafts (n = target->rows /
 * (n_drafts + 1)), the draft's in rows s * n_drafts + d of `draft` (the target's type and columns), d < n_drafts, and the drafted
 * tokens t_d = draft_ids->data[s * draft_ids->stride + d] (n * n_drafts ids; the stride is that of the rows).  With
 * p_d = softmax(scale * target row), q_d = softmax(draft_scale * draft row), and u_d = accept_u[s * n_drafts + d], from d = 0 on:
 *   u_d q_d(t_d) < p_d(t_d)   t_d is accepted
 *   else                      a token is drawn from max(p_d - q_d, 0), and the sequence ends
 * draft == NULL: q_d is 1 at t_d (drafts that come from no model; draft_scale is not read).  A negative id ends the
 * sequence's drafts; so does an id >= cols, recorded as PDB_ERANGE, and a draft row that has nothing left or holds a NaN or +inf. Where
 * they end, and behind the last, a token is drawn from p_d.  Drawn is the smallest j whose running sum of weights passes draw_u[s]
 * times their sum.  n_drafts = 0: a token is drawn for each row (draft_ids and accept_u are not read).
 *   accepted[s]             a, the number of accepted drafts (may be NULL)
 *   tokens[s, 0..n_drafts]  row-major: the accepted drafts, the drawn token, then -1
 *   logp[s, 0..n_drafts]    log p_d of these tokens, 0 behind them (may be NULL)
 * A target row that has nothing left, or holds a NaN or +inf, accepts nothing, and -1 stands where the drawn token would.
 * The random numbers are the caller's, in [0, 1); others count as their nearest end in the draw.  What 32-bit statistics (of which logp is formed, as in
 * pdb_logprobs) or terms good to 2^-31 cannot tell apart is decided on terms good to 2^-40 of themselves, summed as whole numbers of 2^-92 of the rows'
 * sums (weights below 2^-90 of them may count as none), so that the tokens do not depend on how rows are split.
 * Rows behind the first refusal, and behind a sequence's last draft, change no result, but a call may read
 * them (with few sequences, whose rows are all read at once).  PDB_ETOOBIG above 64 drafts or
 * 2^21 tokens.  These are the draws a program makes with its models between the reads of Definition 3. */
int pdb_verify(pdb_tokens *t, const pdb_mat *target, const pdb_ids *draft_ids, int64_t n_drafts, const pdb_mat *draft,
               float scale, float draft_scale, const float *accept_u, const float *draw_u, int32_t *tokens, int32_t *accepted,
               float *logp, void *stream);

/* Tokens to experts and back: layers whose parameters are chunks (Definition 2) of which each token names a few.  Token i has k slots;
 * slot j names expert ids->data[i * ids->stride + j] (ids->n = n * k; the stride is that of the rows).  The experts' rows stand
 * one expert after the other, an expert's slots in ascending order of (i, j) (the data's order, as in Algorithm 2a's writes):
 *   place[i, j]   the slot's row (row-major, n * k), -1 for none
 *   source[r]     the slot i * k + j that has row r, -1 for none
 *   ends[e]       the row behind expert e's last
 * capacity == 0: the rows are packed, n * k of them; expert e starts at ends[e - 1].  Else expert e starts at row e * capacity
 * and has that many at most (n_experts * capacity rows); its slots behind them have none.  A negative id is a slot without an
 * expert; so is one >= n_experts, recorded as PDB_ERANGE.  PDB_ETOOBIG above 64 slots, 4096 experts, 2^31 - 1 rows, or n * k beyond
 * the handle's max_tokens. */
int pdb_route(pdb_tokens *t, const pdb_ids *ids, int64_t k, int64_t n_experts, int64_t capacity, int32_t *place,
              int32_t *source, int32_t *ends, void *stream);

/* rows[place[i, j], :] = x[i, :] (reads as in Definition 3), and zeros in rows with source[r] < 0; rows whose source is a slot that does not
 * name them are left as they were.  Rounded once to the rows' type.  place (x->rows * k) and source (rows->rows) as pdb_route
 * gives them; a place >= rows->rows counts as none and is recorded as PDB_ERANGE, here and below.  rows must not overlap x.
 * Its gradient is pdb_route_join without weights, of the rows' gradient. */
int pdb_route_rows(pdb_tokens *t, const pdb_mat *x, const int32_t *place, int64_t k, const int32_t *source,
                   const pdb_mat *rows, void *stream);

/* y[i, :] = sum over the slots j that have a row, ascending, of weight[i, j] * rows[place[i, j], :] (weight row-major, n * k;
 * NULL: every weight 1).  Sums in fp32 in that order (each row's writes in the data's order, Algorithm 2a), rounded once to y's type; a
 * token without rows gets zeros.  y must not overlap rows. */
int pdb_route_join(pdb_tokens *t, const pdb_mat *rows, const int32_t *place, int64_t k, const float *weight,
                   const pdb_mat *y, void *stream);

/* Gradients of pdb_route_join (read and written as Definition 3's chunks): for dy = the gradient of y,
 *   drows[place[i, j], :] = weight[i, j] * dy[i, :], zeros in rows with source[r] < 0
 *   dweight[i, j]         = sum over c of dy[i, c] * rows[place[i, j], c], 0 for a slot without a row
 * rows and dweight may be NULL together (drows alone).  Products and sums in fp32, in an order that depends on cols, types and
 * alignment only; drows, of rows' type and size, is rounded once and may be the rows' own memory (same data, stride and type); it must
 * not overlap them otherwise, nor dy. */
int pdb_route_join_grad(pdb_tokens *t, const pdb_mat *rows, const int32_t *place, int64_t k, const int32_t *source,
                        const float *weight, const pdb_mat *dy, const pdb_mat *drows, float *dweight, void *stream);

/* The norm over many gradients, and a step clipped to it: with N = sqrt(sum over all n matrices of g^2) and
 * f = max_norm / N where N > max_norm, else 1, for every matrix
 *   out = scale * f * g, or with accumulate != 0   out = out + scale * f * g
 * so that the gradients themselves as results and scale = 1 clip them in place, and the weights as results, accumulate and scale = -eta make
 * the SGD step (Section 6.3's, over all of a model's chunks).  norm, one float, holds N (may be NULL); max_norm >= 0, infinity for no
 * clipping; scale finite.  A gradient that holds a NaN or an infinity makes N one, and no result is written: the step is left
 * out.  N is formed from 32-bit sums of squares of at most a piece of a matrix, added up in 64 bits in a fixed order; squares that
 * leave fp32's range are formed in 64 bits.  The factor scale * f is rounded to fp32, as are its product with g and
 * the sum with out; out is rounded once to its type.
 *
 * A plan holds where the matrices lie and the sums' workspace: pdb_clip_plan_build takes n gradients and their results, of the same rows and
 * columns each, any types, and copies the descriptions (allocates, SYNCHRONIZES `stream`: 45 to 610 us for 3 to 59 matrices); the matrices must outlive the plan.  A result may be its
 * gradient's own memory (same data, stride and type); results must not overlap otherwise, one another or any gradient
 * (PDB_EINVAL).  PDB_ETOOBIG above 2^40 elements.  Calls on a plan must be ordered on one stream, and made while the device is current
 * that was at its building (PDB_EINVAL otherwise); they can be recorded into a CUDA graph (keep the plan until its last run has
 * finished).  pdb_clip_plan_free waits for the work enqueued on the plan. */
typedef struct pdb_clip_plan pdb_clip_plan; /* opaque, library-owned device arrays */
int pdb_clip_plan_build(const pdb_mat *grads, const pdb_mat *outs, int64_t n, pdb_clip_plan **out, void *stream);
int pdb_clip(const pdb_clip_plan *p, float max_norm, float scale, int accumulate, float *norm, void *stream);
void pdb_clip_plan_free(pdb_clip_plan *p);

/* ---------------------------------------------------------------- utilities */

/* cudaMemcpyAsync with the kind inferred from the pointers (for bindings that
 * need to read the borrowed arrays). */
int pdb_memcpy(void *dst, const void *src, size_t bytes, void *stream);

/* Number of CUDA kernels this library has launched in this process so far
 * (every launch site counts once per launch). */
int64_t pdb_launch_count(void);

/* out[i] = the library's device exp of x[i] (device arrays of n floats), the
 * same function the logistic gradient uses.  The paper fixes no exponential;
 * this one is Cody-Waite range reduction (Cody and Waite 1980) with a
 * degree-7 Taylor polynomial, within 2 ulp of exp on [-87, 88.5] and exact
 * at 0, so the oracle can restate it bit for bit.  n < 0, or a NULL array
 * with n > 0, is PDB_EINVAL. */
int pdb_eval_expf(const float *x, float *out, int64_t n, void *stream);

/* out[i] = eta-free loss derivative dloss/dm at margin m[i] and label y[i]
 * (device arrays of n floats), the same function every engine applies
 * (Section 6.3's SGD step, gradient of Eq. 2 without a regulariser):
 * logistic -y / (1 + exp(y m)) with the exp above, squared m - y, hinge
 * (y m < 1 ? -y : 0).  For the logistic loss with y = +1 or -1 and
 * 1 <= 1 + exp(y m) < 2^126 the quotient is formed as a reciprocal, equal
 * bit for bit to the IEEE division.  n < 0, an unknown loss, or a NULL array
 * with n > 0 is PDB_EINVAL. */
int pdb_eval_grad(const float *m, const float *y, float *out, int64_t n, pdb_loss loss, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PDB_H */
