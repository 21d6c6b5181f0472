/*
 * pgc.h — C ABI of libpgc, the GB300 (sm_103a) hot path of Pipelined
 * Gradient Coding (PGC).
 *
 * One GPU simulates an n-worker PGC training step that tolerates s
 * stragglers (c = s + 1 partitions per worker).  Every call is ordered on the
 * CUDA stream given to pgc_create.  A context is not thread-safe.
 *
 * Status codes: every int-returning call returns PGC_OK (0) or a negative
 * PGC_E* code; pgc_strerror turns a code into text.  On any error the
 * context's state (step counter, parameters, stores) is unchanged, except for
 * PGC_ECUDA / PGC_ETIMEOUT which leave the context unusable (destroy it).
 *
 * Layouts: features of partition D_k are row-major [m_k][d] (fp32 or bf16
 * bits); labels are float32 [m_k] (logistic: 0/1, least squares: real) or
 * int32 [m_k] class indices (softmax).  Parameters beta are float32 [K][d]
 * row-major (K = 1 for logistic and least squares).
 */
#ifndef PGC_H_
#define PGC_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ------------------------------------------------------ */
#define PGC_OK        0
#define PGC_EINVAL   (-1)  /* bad argument (sizes, enum, NULL pointer)       */
#define PGC_EMASK    (-2)  /* straggler mask is not exactly s ones, n-s zeros */
#define PGC_ESTATE   (-3)  /* call out of order (e.g. step before load)      */
#define PGC_ENOMEM   (-4)  /* device or pinned-host allocation failed        */
#define PGC_ECUDA    (-5)  /* a CUDA runtime call or kernel failed           */
#define PGC_ENOTSUP  (-6)  /* valid but unsupported combination             */
#define PGC_ETIMEOUT (-7)  /* a bounded device-side wait gave up            */
#define PGC_ESCRATCH (-8)  /* problem larger than pgc_gradient_noalloc's
                              fixed scratch, or than the workspace given    */
#define PGC_ESINGULAR (-9) /* GC-CR: the draws leave a worker's encoding
                              system singular, or the encoding cannot decode
                              the straggler set                             */

/* ---- enumerations (passed as int32) ------------------------------------ */
/* Dataset placement, §III: FR needs c | n; CR places cyclically.          */
#define PGC_FR 0
#define PGC_CR 1
/* Per-sample loss f: logistic cross-entropy (y in {0,1}), least squares
 * (1/2)(x.beta - y)^2, softmax cross-entropy over K classes.             */
#define PGC_LOGISTIC 0
#define PGC_LSQ      1
#define PGC_SOFTMAX  2
/* Storage type of the features.                                           */
#define PGC_F32  0
#define PGC_BF16 1

typedef struct pgc_ctx pgc_ctx;

/* Filled by pgc_step.  The arrays are owned by the caller and may be NULL. */
typedef struct pgc_step_info {
  int64_t  t;               /* index of the step just taken (0 = warm-up)    */
  int32_t  slot;            /* o_t = (t - 1) mod c written this step; -1 at t = 0 */
  int32_t  received;        /* n - s coded gradients decoded                 */
  int32_t *eval_partition;  /* [n]: partition W_i evaluated; -1 at t = 0     */
  int32_t *fr_rep;          /* [n/c] (FR only): worker that represents group j */
} pgc_step_info;

/*
 * pgc_create — allocate a PGC run (§III problem statement, §IV-A, §V-B).
 *   out      : receives the context (set to NULL on error).
 *   n, s     : workers and tolerated stragglers; 1 <= c = s + 1 <= n; FR
 *              additionally needs c | n.  n <= 1024.
 *   scheme   : PGC_FR or PGC_CR.   loss: PGC_LOGISTIC, PGC_LSQ, PGC_SOFTMAX.
 *   dtype    : storage of the features (PGC_F32 or PGC_BF16).
 *   d        : features per sample (>= 1).  K: classes (1 unless softmax;
 *              softmax needs 2 <= K <= 4096).
 *   rows     : host array [n], rows m_k >= 1 of partition D_k.
 *   lr       : learning rate eta of beta <- beta - eta * ghat (§III).
 *   w0       : host array [K*d] initial beta, or NULL for zeros.
 *   stream   : cudaStream_t every call is ordered on (NULL = legacy stream).
 * Allocates all device state (partitions, parameters, the per-owner gradient
 * stores, slot totals, scratch).  Errors: PGC_EINVAL, PGC_ENOTSUP,
 * PGC_ENOMEM, PGC_ECUDA.  Argument checks happen before any CUDA call.
 */
int pgc_create(pgc_ctx **out, int32_t n, int32_t s, int32_t scheme, int32_t loss,
               int32_t dtype, int64_t d, int64_t K, const int64_t *rows, float lr,
               const float *w0, void *stream);

/* Training schemes on the same kernels (§VI-A, the paper's baselines). */
#define PGC_MODE_PGC    0   /* pipelined gradient coding (default)                  */
#define PGC_MODE_IS_SGD 1   /* ignore stragglers: worker W_i evaluates D_i each step;
                               the master averages the n - s received gradients.
                               Needs scheme PGC_CR (the decode runs as CR with one
                               slot per worker, coefficient 1/(n - s)).             */
#define PGC_MODE_GC     2   /* gradient coding (GC, §VI-A): every worker evaluates
                               all c of its partitions each step.  PGC_FR: the
                               master decodes one coded gradient per group (1/n),
                               which recovers (1/n) sum_k g_k exactly.  PGC_CR:
                               GC-CR (§V-A), worker W_j uploads
                               sum_l c_{j,l} g_{(j+l) mod n} with the encoding of
                               pgc_set_gc_encoding and the master applies the
                               decode weights d_m(J) of the received set, times
                               1/n: exact as well.  PGC_CR needs n <= 64.        */
#define PGC_MODE_NAIVE_CR 3 /* the naive pipelined construction on cyclic
                               repetition (§V-A): PGC-CR's rotation and stores
                               (one partition evaluated per step), but W_j uploads
                               sum_l c_{j,l} (its latest gradient of
                               D_{(j+l) mod n}) and the master decodes with GC-CR's
                               weights d_m(J), times 1/n.  Stale copies enter with
                               the decoding coefficients alpha_{m,k} = d_m c_{j_m,l}
                               (pgc_get_gc_decode).  Needs PGC_CR and n <= 64.   */

/*
 * pgc_create_mode — pgc_create with a training scheme from PGC_MODE_*; the
 * other arguments and errors are pgc_create's (PGC_EINVAL also for an unknown
 * mode or a mode/scheme pair listed as unsupported above).  With s = 0 every
 * mode is plain distributed gradient descent (DGD, §III).
 */
int pgc_create_mode(pgc_ctx **out, int32_t mode, int32_t n, int32_t s, int32_t scheme, int32_t loss,
                    int32_t dtype, int64_t d, int64_t K, const int64_t *rows, float lr,
                    const float *w0, void *stream);

/*
 * pgc_set_gc_encoding — GC-CR's encoding coefficients c_{j,l} (§V-A), for the
 * modes that decode with them (PGC_MODE_NAIVE_CR; PGC_MODE_GC with PGC_CR).
 * §V-A takes them from gradient coding's cyclic-repetition construction,
 * which the device builds from the given random numbers: H = [draws |
 * -(row sums of draws)] is s x n with H 1 = 0; worker W_j's row of the
 * encoding matrix B is supported on partitions j..j+s (mod n), has
 * c_{j,0} = B[j][j] = 1, and its other s entries solve
 * H[:, {j+1..j+s}] x = -H[:, j] (fp64, partial pivoting).
 *   draws : host array [s][n-1], row-major (for instance standard normal
 *           draws); ignored when s = 0 (then B is the identity).
 * Must be called before the first pgc_step of those modes (PGC_ESTATE
 * otherwise); may be called again.  Not part of a checkpoint.  Errors:
 * PGC_EINVAL (other mode, NULL or non-finite draws), PGC_ESINGULAR (a
 * worker's system is singular; the context stays usable), PGC_ECUDA.
 */
int pgc_set_gc_encoding(pgc_ctx *ctx, const double *draws);

/*
 * pgc_get_gc_encoding — copy the encoding coefficients to host coeff[n][c]:
 * coeff[j*c + l] = c_{j,l}, W_j's weight on its gradient of D_{(j+l) mod n}.
 * Errors: PGC_EINVAL (other mode), PGC_ESTATE (not set), PGC_ECUDA.
 */
int pgc_get_gc_encoding(pgc_ctx *ctx, double *coeff);

/*
 * pgc_get_gc_decode — what the device derived at the last step of a GC-CR
 * mode (§V-A): d (host [n], or NULL) = the decode weights d_j(J) solving
 * sum_{j in J} d_j B[j] = 1 over the received set J (0 for stragglers), in
 * fp64; alpha_range (host [2], or NULL) = the maximum and the minimum of the
 * decoding coefficients alpha_{m,k} = d_m c_{j_m,l} over the received workers
 * and the partitions each holds.  The decoded gradient is
 * (1/n) sum_j d_j sum_l c_{j,l} store[j][l].  A straggler set the encoding
 * cannot decode (sum_j d_j B[j] misses 1 by more than 1e-8 relative, or a
 * pivot vanishes) leaves that step's beta unchanged and makes the call that
 * reads the device status (pgc_step with host outputs, pgc_sync) return
 * PGC_ESINGULAR; the context then takes no more steps.  Errors: PGC_EINVAL,
 * PGC_ESTATE (no step yet), PGC_ECUDA.
 */
int pgc_get_gc_decode(pgc_ctx *ctx, double *d, double *alpha_range);

/*
 * pgc_load_partitions — copy the n partitions into device memory (§III: the
 * partitions are placed before training).  X[k] points to [m_k][d] features
 * of the create-time dtype, y[k] to m_k labels (float32, or int32 for
 * softmax).  on_device != 0: the pointers are device pointers; otherwise host
 * pointers.  The library keeps its own copy; the caller may free its buffers
 * after the call returns.  May be called again to replace the data; it does
 * not reset the step counter.  Errors: PGC_EINVAL (NULL entry), PGC_ECUDA.
 */
int pgc_load_partitions(pgc_ctx *ctx, const void *const *X, const void *const *y,
                        int32_t on_device);

/*
 * pgc_step — one PGC training step t (§IV-A PGC-FR, §V-B PGC-CR).
 *   straggler_mask : host array [n]; 1 marks a straggler, 0 a worker whose
 *                    coded gradient reaches the master.  Exactly s ones.
 *   grad_out       : [K*d] float32, receives the decoded gradient ghat^(t)
 *                    (NULL: not returned).
 *   w_out          : [K*d] float32, receives beta^(t+1) (NULL: not returned).
 *   outputs_on_device : != 0: grad_out / w_out are device pointers and the
 *                    call returns without waiting for the GPU; 0: host
 *                    pointers, the call waits until they hold the results
 *                    (pinned host buffers mapped into the device's address
 *                    space are written by the decode kernel itself, unless
 *                    they are large and their rows of d floats do not all
 *                    start on 16 bytes; others are filled by copies after it).
 *   info           : may be NULL; receives t, o_t and the schedule indices.
 * Step 0 is the warm-up: every worker evaluates all c of its partitions at
 * beta^(0).  From step 1 on, worker W_i evaluates only the partition in its
 * slot o_t = (t-1) mod c; stragglers still evaluate and store.  FR workers of
 * one group evaluate the same partition at the same beta, so it is computed
 * once per group.  The decode uses the coded gradients of the n - s received
 * workers with the coefficients of §IV-A (FR: one per group, times 1/n) or
 * §V-B (CR: times 1/((n-s)c)), derived on the device from the mask, and is
 * fused with the SGD update.  Errors: PGC_ESTATE (no partitions loaded),
 * PGC_EMASK, PGC_EINVAL, PGC_ECUDA, PGC_ETIMEOUT.
 */
int pgc_step(pgc_ctx *ctx, const uint8_t *straggler_mask, float *grad_out, float *w_out,
             int32_t outputs_on_device, pgc_step_info *info);

/*
 * pgc_loss — F(beta^(t)) = (1 / sum_k m_k) sum over all samples of f, at the
 * current parameters (§III).  Untimed helper; waits for the GPU.
 * Errors: PGC_ESTATE, PGC_EINVAL, PGC_ECUDA.
 */
int pgc_loss(pgc_ctx *ctx, double *loss_out);

/*
 * pgc_sync — wait for every call issued on the context's stream and report
 * a device-side failure (PGC_ETIMEOUT if a bounded wait gave up, PGC_EMASK
 * if the decode kernel saw an invalid mask).  Steps with device outputs do
 * not wait; call this before trusting their results.
 */
int pgc_sync(pgc_ctx *ctx);

/* pgc_destroy — free everything; NULL is accepted.  Returns PGC_OK. */
int pgc_destroy(pgc_ctx *ctx);

/* pgc_strerror — static text for a status code. */
const char *pgc_strerror(int32_t code);

/* pgc_gradient_path — static name of the kernel path the context computes
 * per-partition gradients with (fixed at pgc_create): "grad_rows" (logistic,
 * least squares), "tc_fused" (softmax on the tensor cores, residual in the
 * logits GEMM), "tc" (tensor cores, separate residual kernel),
 * "softmax_rows" (few classes, whole rows per CTA pair), "softmax_cluster" (few
 * classes, 8-CTA clusters), "softmax_cc" (single precision: up to 128 classes
 * on the tensor cores with operands in three bf16 parts, else CUDA cores);
 * "" for NULL. */
const char *pgc_gradient_path(const pgc_ctx *ctx);

/* pgc_last_cuda_error — name of the CUDA runtime error behind the most
 * recent PGC_ECUDA / PGC_ENOMEM returned on the calling thread (for example
 * "cudaErrorLaunchOutOfResources"), or "" if there was none.  Static text. */
const char *pgc_last_cuda_error(void);

/* ---- host-only helpers: pure index arithmetic, no CUDA call ------------- */

/*
 * pgc_placement — the partitions each worker holds (§III; §IV-A for FR,
 * §V-B for CR), table[i*c + l] = partition in slot l of worker W_i.
 * table: host [n*c].  Errors: PGC_EINVAL.
 */
int pgc_placement(int32_t scheme, int32_t n, int32_t s, int32_t *table);

/*
 * pgc_schedule — partition each worker evaluates at step t (§IV-A, §V-B):
 * eval_partition[i] (host [n]) = the partition in slot (t-1) mod c of W_i,
 * or -1 for every worker at t = 0; *slot = (t-1) mod c or -1.
 * Errors: PGC_EINVAL.
 */
int pgc_schedule(int32_t scheme, int32_t n, int32_t s, int64_t t,
                 int32_t *eval_partition, int32_t *slot);

/* ---- inspection of device state (tests; each call waits for the GPU) ---- */

/*
 * pgc_get_store — copy worker W_i's stored gradient in slot l (the gradient
 * of the partition in slot l of its holdings, as last evaluated) to host
 * out[K*d].  FR workers of one group share one store.  Errors: PGC_EINVAL,
 * PGC_ESTATE, PGC_ECUDA.
 */
int pgc_get_store(pgc_ctx *ctx, int32_t worker, int32_t slot, float *out);

/*
 * pgc_get_store_cols — as pgc_get_store, for the parameters [col0, col0 +
 * ncols) of the flattened K*d vector only (host out[ncols]); reads a few
 * columns of every store without copying whole gradients.  Errors:
 * PGC_EINVAL (range outside [0, K*d)), PGC_ESTATE, PGC_ECUDA.
 */
int pgc_get_store_cols(pgc_ctx *ctx, int32_t worker, int32_t slot, int64_t col0, int64_t ncols, float *out);

/*
 * pgc_get_decode — the decoding coefficients the device derived from the
 * last step's mask: coeff[i] (host [n]) = weight a_i of W_i's coded gradient
 * (§IV-A: 1/n for each FR group's representative; §V-B: 1/((n-s)c) for each
 * received CR worker; GC-CR modes: d_i(J)/n; 0 otherwise).  Errors:
 * PGC_ESTATE, PGC_ECUDA.
 */
int pgc_get_decode(pgc_ctx *ctx, float *coeff);

/* pgc_get_weights — copy the current beta to host out[K*d]. */
int pgc_get_weights(pgc_ctx *ctx, float *out);

/* pgc_set_weights — overwrite beta with host w[K*d] (teacher forcing in
 * tests; also the checkpoint-restore path).  Errors: PGC_EINVAL, PGC_ECUDA. */
int pgc_set_weights(pgc_ctx *ctx, const float *w);

/*
 * Checkpoint and resume of a run: the step counter t, beta, every store
 * (owners x c gradients) and the slot totals U — everything a later step
 * reads.  The features and labels are not part of it: the resumed context
 * must be created with the same arguments and loaded with the same
 * partitions.
 *
 * pgc_checkpoint_bytes — *bytes = size of the checkpoint of this context:
 *   104 bytes of header (13 int64: magic 0x3154504B43434750 "PGCCKPT1",
 *   version 1, mode, scheme, loss, dtype, n, s, c, d, K, t, stepped) then fp32
 *   beta [K][d], stores [owners][c][K][d] and U [c][K][d], host byte order.
 * pgc_checkpoint_save — write it to host buf[bytes] (waits for the stream).
 * pgc_checkpoint_load — restore it from host buf[bytes] into a context with
 *   the same mode, scheme, loss, dtype, n, s, d and K; the next pgc_step is
 *   step t of the saved run.
 * Errors: PGC_EINVAL (NULL, wrong size, header of another configuration),
 * PGC_ESTATE (a failed context), PGC_ECUDA.
 */
int pgc_checkpoint_bytes(pgc_ctx *ctx, int64_t *bytes);
int pgc_checkpoint_save(pgc_ctx *ctx, void *buf, int64_t bytes);
int pgc_checkpoint_load(pgc_ctx *ctx, const void *buf, int64_t bytes);

/* pgc_step_count — number of steps taken so far (host-side counter). */
int64_t pgc_step_count(const pgc_ctx *ctx);

/* ---- measurement ---------------------------------------------------------- */

/* Kernel groups of one step, in launch order, as counted and timed below.
 * Paths without a group leave it empty (zero time, zero launches). */
#define PGC_KGRAD   0   /* gradient: streaming row kernel, few-class softmax
                           kernel, tensor-core logits GEMM, or the single-
                           precision softmax kernels                                    */
#define PGC_KRESID  1   /* tensor-core softmax: residual R = softmax(Z) - Y    */
#define PGC_KGRADB  2   /* tensor-core softmax: gradient GEMM R^T X            */
#define PGC_KCOMMIT 3   /* gradient-store commit                               */
#define PGC_KDECODE 4   /* decode coefficients + decode + SGD                  */
#define PGC_NKGROUPS 5

/*
 * pgc_timing — enable != 0 starts recording CUDA events on the context's
 * stream around each kernel group of every following step (and clears what
 * was recorded); 0 stops.  Errors: PGC_EINVAL, PGC_ECUDA.
 */
int pgc_timing(pgc_ctx *ctx, int32_t enable);

/*
 * pgc_timing_read — wait for the stream, then return for each kernel group
 * the summed device time in milliseconds (ms[PGC_NKGROUPS]) over the steps
 * recorded since timing was enabled, and the kernels launched by the library
 * in those steps (launches[PGC_NKGROUPS]).  Either array may be NULL.
 * *steps_out (nullable) receives the number of recorded steps.
 */
int pgc_timing_read(pgc_ctx *ctx, double *ms, int64_t *launches, int64_t *steps_out);

/* ---- allocation-free gradient --------------------------------------------- */

/*
 * pgc_gradient_noalloc — g_out = (1/m) sum over the m rows x of one partition
 * of r(x) * x, with r = sigmoid(x.w) - y (PGC_LOGISTIC) or x.w - y (PGC_LSQ):
 * the per-partition gradient pgc_step evaluates, computed without allocating
 * any device memory.  The paper has no counterpart; this exists for callers
 * that cannot call cudaMalloc / cudaFree when they need a gradient: a
 * framework whose caching pool already holds the free device memory, or a
 * loop that must not take cudaFree's implicit device synchronisation.
 *
 *   X     : device [m][d] features (PGC_F32, or PGC_BF16 bits), 16-byte aligned
 *   y     : device [m] float32 labels;  w: device [d] float32 parameters
 *           (both 4-byte aligned)
 *   g_out : device [d] float32, 16-byte aligned (written)
 *   stream: cudaStream_t to run on; the call waits for it before returning.
 *
 * Scratch: a fixed 16 MiB array inside the library (a __device__ global),
 * held on every GPU that loads the library until the process exits.  The
 * first call on a device looks up the array's device address (with that
 * device current) and keeps it for the life of the process; make that first
 * call before any stream capture.  cudaDeviceReset on a device unloads the
 * library's module there and makes the kept address stale: a process that
 * resets a device must not call this entry point on it afterwards.  All
 * calls share the array and it keeps the last call's contents; each call
 * rewrites what it reads, but calls that overlap on the GPU (other streams,
 * other threads) race on it.
 *
 * Limits: d must be a row length the gradient kernel takes without padding
 * (fp32: 32, 64, 128 * 2^k up to 16384; bf16: 64, 128, 256 * 2^k up to
 * 32768), else PGC_ENOTSUP.  The scratch holds a copy of the m labels (4 m
 * bytes) and one partial sum of 4 d bytes per SM; problems that do not fit
 * the 16 MiB return PGC_ESCRATCH (on a 152-SM GPU: about 1.7 million rows at
 * fp32 d = 16384, about 4 million at d = 1024).  Other errors: PGC_EINVAL,
 * PGC_ECUDA, PGC_ETIMEOUT.
 */
int pgc_gradient_noalloc(int32_t loss, int32_t dtype, int64_t m, int64_t d, const void *X,
                         const float *y, const float *w, float *g_out, void *stream);

/* ---- losses on rows of logits, with their gradients ------------------------ */

/*
 * The calls below take a caller's logits where a run's softmax loss forms its
 * own: rows of V logits in device memory, one row per token, and give a loss
 * and its gradient with respect to every logit.  The paper has no counterpart;
 * they serve models whose last product is made elsewhere.
 *
 * With the temperature tau, the row's largest logit m and
 * L = log sum_v exp((x_v - m) / tau), the target y of a row has
 *   logp = (x_y - m) / tau - L,   d logp / d x_v = ([v = y] - p_v) / tau,
 *   p_v = exp((x_v - m) / tau - L).
 *
 * Common to all of them:
 *  - They keep no state and allocate nothing.  All pointers but the structure
 *    itself are device pointers on the current device; the work is ordered on
 *    `stream` (cudaStream_t; NULL = legacy stream) and the call returns without
 *    waiting, so it can be captured into a CUDA graph.  Calls that may overlap
 *    (two streams, two graphs) need workspaces and outputs of their own.
 *  - workspace: 16-byte aligned device memory of the bytes that
 *    pgc_loss_workspace / pgc_balance_workspace return; its contents do not
 *    matter before a call and mean nothing after it.
 *  - Sums, maxima and probabilities are held in 32 bits (sums over tokens in two
 *    floats), a bf16 gradient is rounded once.  A call repeated on the same inputs gives the same bits.
 *  - A row whose target is negative takes no part (prompts, padding): its logits are
 *    not read, its log probability is 0 and its gradient row is zeros.  A
 *    target >= classes is not followed: log probability, gradient row and
 *    loss are NaN (zeros in a gradient row of no sequence, or of derivative 0).  A row
 *    all of whose logits are -inf has no distribution: NaN as well.  A target of logit
 *    -inf has log probability -inf.  Classes may be masked by -inf or by any large
 *    negative number, down to the type's lowest value.
 *  - offsets: int32, sequence i is rows offsets[i] .. offsets[i + 1] - 1 (so
 *    a padded batch is offsets of equal steps, its padding rows of negative
 *    target).  Rows of no sequence take no part.  Offsets that fall or leave [0, rows]
 *    are not followed: loss and gradients are NaN.  A sequence may be empty.
 *  - Errors: PGC_EINVAL before any CUDA call (sizes, enumerations, NULL, alignment: logits
 *    and gradient to their element, the rest to 4 bytes), PGC_ESCRATCH (workspace too small),
 *    PGC_ENOTSUP where listed, PGC_ECUDA.
 */
typedef struct pgc_logits {
  const void    *x;           /* logits: row t at x + t * ld elements              */
  const int32_t *target;      /* [rows] class of each row, negative: none           */
  void          *grad;        /* gradient, of the logits' type, row t at grad + t * grad_ld;
                                 NULL: only the loss.  May be x itself (with
                                 grad_ld = ld), otherwise it overlaps nothing       */
  int64_t rows, classes;      /* 0 <= rows < 2^31, 1 <= classes < 2^31              */
  int64_t ld, grad_ld;        /* row pitches in elements, classes <= ld <= 2^31     */
  int32_t dtype;              /* PGC_F32 or PGC_BF16                                */
  float   temperature;        /* tau > 0 (1: the logits as they are), log2(e) / tau finite */
} pgc_logits;

/* pgc_loss_workspace — bytes of workspace of a preference or policy loss over
 * `rows` rows and `sequences` sequences (two per pair; 0 without offsets).
 * Errors: PGC_EINVAL. */
int pgc_loss_workspace(int64_t rows, int64_t sequences, int64_t *bytes);

/*
 * pgc_token_logprob — logp[rows] = log probability of each row's target, and
 * stats[rows][2] (8-byte aligned) = (m, L) of the row, for the gradient call; (0, 0)
 * for a row without a target.  z->grad is not used.
 */
int pgc_token_logprob(const pgc_logits *z, float *logp, float *stats, void *stream);

/*
 * pgc_token_logprob_grad — z->grad[t][v] = dlogp[t] ([v = y_t] - p_tv) / tau:
 * the gradient of any loss whose derivative with respect to the rows' log
 * probabilities is dlogp[rows].  stats: as pgc_token_logprob returned them for the
 * same logits.  A row whose dlogp is 0 gets zeros.
 */
int pgc_token_logprob_grad(const pgc_logits *z, const float *stats, const float *dlogp, void *stream);

#define PGC_PREF_SIGMOID 0   /* (1-e) log(1 + exp(-h)) + e log(1 + exp(h))            */
#define PGC_PREF_HINGE   1   /* (1-e) max(0, 1 - h) + e max(0, 1 + h)                 */
#define PGC_PREF_SQUARED 2   /* (1-e) (h/beta - 1/(2 beta))^2 + e (h/beta + 1/(2 beta))^2 */

/*
 * pgc_preference_loss — paired log ratios.  Sequence 2 i is the chosen and
 * 2 i + 1 the rejected answer of pair i; the score s of a sequence is the sum of
 * its rows' log probabilities (average != 0: their mean; 0 for a sequence
 * without targets), and
 *   h_i = beta ((s_2i - r_2i) - (s_2i+1 - r_2i+1)) - margin
 * with the reference scores r.  loss = scale / pairs * sum_i f(h_i), f by `kind`
 * with e = smoothing (0 <= e <= 1).
 *   offsets  : [2 pairs + 1].   ref_logp: [pairs][2], or NULL for zeros.
 *   beta > 0, margin, scale finite.
 *   loss     : [1];  logp: [pairs][2] receives the scores s.
 * No pairs: the loss is 0.
 */
int pgc_preference_loss(const pgc_logits *z, int32_t kind, int64_t pairs, const int32_t *offsets, const float *ref_logp,
                        float beta, float margin, float smoothing, int32_t average, float scale, float *loss,
                        float *logp, void *workspace, int64_t workspace_bytes, void *stream);

#define PGC_MEAN_TOKENS    0   /* every row with a target weighs 1 / their number      */
#define PGC_MEAN_SEQUENCES 1   /* 1 / (its sequence's rows with a target x sequences that have one) */
#define PGC_SUM            2   /* 1                                                    */

/*
 * pgc_policy_loss — clipped policy loss with a KL term.  For each row with a
 * target, r = exp(logp - old_logp), A its advantage, q = r clamped to
 * [1 - clip_low, 1 + clip_high], u = ref_logp - logp:
 *   loss = scale * sum_t w_t (-min(r A, q A) + kl (exp(u) - u - 1)).
 * The derivative is that of r A where r A <= q A, and 0 of q A elsewhere.
 *   reduction: w_t, PGC_MEAN_* or PGC_SUM; offsets [sequences + 1] are read for
 *     PGC_MEAN_SEQUENCES only.
 *   old_logp, advantage: [rows].  ref_logp: [rows], or NULL (then kl must be 0).
 *   0 <= clip_low <= 1, clip_high >= 0; kl, scale finite.
 *   loss [1]; terms [3] = the weighted sums (without scale) of -min(r A, q A), of
 *     exp(u) - u - 1 (0 without ref_logp) and of the rows where q A < r A.
 *   logp [rows]: the rows' log probabilities.
 */
int pgc_policy_loss(const pgc_logits *z, int32_t reduction, int64_t sequences, const int32_t *offsets,
                    const float *old_logp, const float *advantage, const float *ref_logp, float clip_low,
                    float clip_high, float kl, float scale, float *loss, float *terms, float *logp, void *workspace,
                    int64_t workspace_bytes, void *stream);

/* pgc_balance_workspace — bytes of workspace of pgc_balance_loss. Errors: PGC_EINVAL. */
int pgc_balance_workspace(int64_t rows, int64_t experts, int64_t *bytes);

/*
 * pgc_balance_loss — a router's choice, its counts and its balance loss.  Rows
 * of `experts` logits (dtype, ld as in pgc_logits); n rows have mask[t] != 0 (all,
 * if mask is NULL).  With p = softmax of a row (temperature 1) and the counts c,
 *   loss = alpha experts / (k n^2) sum_e c_e sum_t p_te,
 * whose gradient takes the counts as constants.
 *   choice : [rows][k].  given = 0: receives the experts of each row's k largest
 *     logits, largest first, ties to the lower expert; -1 in a row that takes no
 *     part, and where fewer than k logits are above -inf.  given != 0: read; entries outside
 *     [0, experts) count for no expert, the same expert twice counts twice.
 *   counts : [experts] times each expert was chosen by rows that take part.
 *   grad   : as in pgc_logits (NULL: only the loss); zeros for rows that take
 *     no part.  A row all of whose logits are -inf adds nothing and gets zeros.
 *   loss   : [1], 0 if n = 0.
 * Errors: as above; PGC_ENOTSUP for more than 1024 experts or k > 64.
 */
int pgc_balance_loss(int32_t dtype, int64_t rows, int64_t experts, const void *logits, int64_t ld, const uint8_t *mask,
                     int32_t k, int32_t given, int32_t *choice, float alpha, float *loss, int32_t *counts, void *grad,
                     int64_t grad_ld, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * pgc_token_scores — what a row says of its classes beside its target.  With
 * q_v = (x_v - m) / tau - L the log probability of class v and p = exp(q):
 *   logp      [rows] q_y; NULL exactly if z->target is NULL, when every row takes part
 *   entropy   [rows] -sum_v p_v q_v (a class of p = 0 adds nothing)
 *   top       [rows][k] the classes of the k largest logits, largest first, ties to the lower class
 *   top_logp  [rows][k] their q.  Where fewer than k logits are above -inf: -1 and -inf
 *   stats     [rows][2] (8-byte aligned) = (m, L), as pgc_token_logprob returns it
 * A row of negative target: 0, 0, -1, -inf, (0, 0).  A target >= classes: logp alone is
 * NaN.  A row with NaN among its logits, or a logit of +inf, has logp, entropy and
 * top_logp NaN; NaN is no alternative.  z->grad is not used.  k may exceed the classes; 0 <= k <= 64,
 * PGC_ENOTSUP above.
 */
int pgc_token_scores(const pgc_logits *z, int32_t k, float *logp, float *entropy, int32_t *top, float *top_logp,
                     float *stats, void *stream);

/*
 * pgc_token_scores_grad — the gradient of any loss whose derivatives with respect to the rows' log
 * probabilities and entropies are dlogp[rows] and dentropy[rows] (either may be NULL, but not both):
 *   z->grad[t][v] = (dlogp[t] ([v = y_t] - p_tv) - dentropy[t] p_tv (q_tv + H_t)) / tau.
 * stats, entropy: as pgc_token_scores returned them for the same logits (entropy is read with
 * dentropy only).  dlogp needs z->target.  A row of negative target, or whose
 * derivatives are both 0, gets zeros; a target >= classes NaN unless its dlogp is 0; a row without a
 * distribution, or with a NaN derivative, NaN.
 */
int pgc_token_scores_grad(const pgc_logits *z, const float *stats, const float *entropy, const float *dlogp,
                          const float *dentropy, void *stream);

/* ---- tokens to their experts and back --------------------------------------- */

/*
 * A router chose k experts for each of `tokens` tokens (as pgc_balance_loss
 * does): slot s = t k + j holds an expert, or, outside [0, experts), nothing.
 * pgc_route sorts the slots by expert; the other calls move rows of d elements
 * (dtype) between the tokens' order and that one, so that the experts'
 * products are made over consecutive rows: those of expert e are
 * offsets[e] .. offsets[e + 1] - 1.
 *
 * Common to all of them: what is common to the losses on rows of logits.  Also:
 *  - place [tokens][k]: the row of each slot.  An entry outside [0, rows) has no row: it
 *    is not copied, adds nothing, and its weight's gradient is 0.  So `rows` may be less
 *    than the slots that hold an expert (rows behind it are cut off).  Entries that
 *    have a row differ from one another.
 *  - Rows of the experts' order that no slot has are left as they were.
 *  - Sums run over j in order, in 32 bits; a bf16 result is rounded once.
 *  - rows, tokens < 2^31 and tokens k < 2^31, 1 <= d <= 2^30, d <= pitch <= 2^31; k <= 64 and experts <= 1024,
 *    PGC_ENOTSUP above.  No output overlaps an input, but where it says so.
 */

/* pgc_route_workspace — bytes of workspace of pgc_route.  Errors: PGC_EINVAL, PGC_ENOTSUP. */
int pgc_route_workspace(int64_t tokens, int32_t k, int32_t experts, int64_t *bytes);

/*
 * pgc_route — sorts the slots by expert, in their order within one.
 *   choice  [tokens][k]
 *   place   [tokens][k] the row of each slot, -1 where it holds nothing
 *   slot    [tokens k]  the slot of each row (its token is slot / k), -1 behind the last one
 *   offsets [experts + 1] the first row of each expert, and their end
 * A token may hold the same expert twice: two rows.
 */
int pgc_route(int64_t tokens, int32_t k, int32_t experts, const int32_t *choice, int32_t *place, int32_t *slot,
              int32_t *offsets, void *workspace, int64_t workspace_bytes, void *stream);

/* pgc_spread — out[place[t][j]] = x[t].  x: tokens rows of pitch ld; out: `rows` rows of pitch out_ld. */
int pgc_spread(int32_t dtype, int64_t tokens, int32_t k, int64_t d, const void *x, int64_t ld, const int32_t *place,
               int64_t rows, void *out, int64_t out_ld, void *stream);

/*
 * pgc_join — out[t] = sum_j weight[t][j] rows_in[place[t][j]]; weight [tokens][k]
 * float32, or NULL for ones: the gradient of pgc_spread.  A token without rows gets zeros.
 */
int pgc_join(int32_t dtype, int64_t tokens, int32_t k, int64_t d, const void *rows_in, int64_t ld, int64_t rows,
             const int32_t *place, const float *weight, void *out, int64_t out_ld, void *stream);

/*
 * pgc_join_grad — the gradient of pgc_join for the derivative dy (tokens rows):
 *   drows[place[t][j]] = weight[t][j] dy[t],   dweight[t][j] = <dy[t], rows_in[place[t][j]]>.
 * drows may be rows_in itself (with drows_ld = ld).
 */
int pgc_join_grad(int32_t dtype, int64_t tokens, int32_t k, int64_t d, const void *dy, int64_t dy_ld, const void *rows_in,
                  int64_t ld, int64_t rows, const int32_t *place, const float *weight, void *drows, int64_t drows_ld,
                  float *dweight, void *stream);

/* ---- AdamW over many tensors ------------------------------------------------- */

/*
 * pgc_adamw_step — one AdamW step over any number of tensors, in launches of up to
 * 240 tensors.  With g = grad * grad_scale, every element:
 *   m' = beta1 m + (1 - beta1) g,   v' = beta2 v + (1 - beta2) g^2,
 *   p' = p (1 - lr weight_decay) - lr (m' / (1 - beta1^step)) / (sqrt(v' / (1 - beta2^step)) + eps),
 * in 32 bits; p' is rounded to the parameters' type once, and to bf16 for `copy`.
 *
 * bits = 32: m and v are float32.  bits = 8: they are one byte an element, and every 256
 * elements (a block; the last one of a tensor may be shorter) have two scales, powers of two:
 *   m : an 8-bit float of 4 bits of exponent (bias 7) and 3 of fraction, times m_scale
 *   v : code c: 0 for zero; from 127 on 2^(-3 + (c - 127) / 16), below it 2^(-3 + (c - 127) / 8), with
 *       the fractions of an exponent taken in equal steps (16 or 8 an octave), times v_scale
 * m_scale is 2^(e - 7) and v_scale 2^(e - 4), 2^e the largest power of two in the block's largest magnitude; a block
 * whose largest is below 2^-111 becomes zeros.  A value between two codes goes to the
 * upper one with the probability of its place between them (1 / 65536 steps; a positive v never to 0), by 32
 * bits drawn from (seed, step, the tensor's index in the list, the element's): the same call
 * gives the same bits.  The parameters of a step see m' and v' before that rounding.  A block that meets an
 * infinity or NaN in m' or v' is NaN from then on.  The rounding noise that this leaves in v, for gradients of normal
 * distribution, has a standard deviation of 6 % at beta2 = 0.95 and 14 % at 0.999, and where v is under 2^-8 of its
 * block's largest, of 13 % and 20 %.  A positive v below code 1 (under about 2^-23 of its block's largest: gradients
 * 3000 times smaller) is raised to it, so that its parameter moves less than with 32 bits.
 *
 * Tensors are contiguous and overlap nothing; a NULL grad leaves its tensor as it is.  Moments start as zeros
 * (all bytes and scales).  The structures are read before the call returns.
 * Nothing is allocated, the work is ordered on `stream`, and the call returns without waiting.
 * A captured graph replays the step and lr that it was captured with, but those on the device.
 * Errors: PGC_EINVAL before any CUDA call (types, bits, NULL, alignment to the element, n outside [0, 2^38],
 * step < 1, a rate that is not finite, eps < 0, a beta outside [0, 1)), PGC_ECUDA.
 */
typedef struct pgc_adamw_tensor {
  void       *param;          /* [n] param_dtype, updated                          */
  const void *grad;           /* [n] grad_dtype, or NULL                           */
  void       *copy;           /* [n] bf16, receives p'; or NULL                    */
  void       *m, *v;          /* [n] moments                                       */
  float      *m_scale, *v_scale;  /* bits = 8: [(n + 255) / 256]                   */
  int64_t     n;
} pgc_adamw_tensor;

typedef struct pgc_adamw {
  double lr, beta1, beta2, eps, weight_decay;
  int64_t step;               /* 1 for the first one                               */
  const int64_t *step_at;     /* device, at least 1: in place of step; or NULL     */
  const float *lr_at;         /* device: in place of lr; or NULL                   */
  const float *grad_scale;    /* device: factor of the gradients; or NULL for 1    */
  uint32_t seed;
  int32_t param_dtype, grad_dtype;   /* PGC_F32 or PGC_BF16                        */
  int32_t bits;               /* 32 or 8                                           */
} pgc_adamw;

int pgc_adamw_step(const pgc_adamw *s, const pgc_adamw_tensor *tensors, int64_t count, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PGC_H_ */
