/*
 * isoloco.h -- C ABI of the IsoLoCo outer aggregation step for AMD MI355X (gfx950).
 *
 * The operation (Algorithm 2 of "Can Model Merging Improve Aggregation in
 * DiLoCo?", arXiv 2607.03011) takes the global parameters theta, K worker
 * replicas theta_k and the outer momentum buffer B, and performs one outer
 * step in place:
 *
 *   Delta   = (1/K) sum_k (theta - theta_k)            averaged pseudo-gradient
 *                                                       (sign as in Algorithm 1)
 *   D_l     = alpha * sigma_bar_l * U_l V_l^T           every tensor l of kind ISO
 *             with Delta_l = U_l S_l V_l^T and sigma_bar_l = trace(S_l) / min(rows, cols)
 *             (Iso-C spectrum flattening, Section 2.2; the SVD branch of Algorithm 2)
 *   D_l     = Delta_l                                   every tensor of kind AVG
 *             (1-D tensors take no correction, Section 4)
 *   B      <- mu * B + D;   P = D + mu * B;   theta <- theta - outer_lr * P
 *                                                       (Nesterov, Algorithm 2)
 *
 * alpha is an extra isotropic scale; alpha = 1 is the paper.  U V^T is not
 * obtained from an SVD: it is the orthogonal polar factor of Delta_l, computed
 * by a fixed polynomial (Newton-Schulz-type) iteration on matrix products
 * (Section 4.3 motivates the iteration; this library runs it to convergence
 * rather than for a fixed 5 steps), and sigma_bar_l = <Q_l, Delta_l>_F / r.
 *
 * Memory.  The caller owns every buffer.  theta, B and the K replicas are flat
 * device arrays of n_elems elements that share one layout, described by a
 * table of tensors.  The library never allocates device memory: the caller
 * provides a workspace of isoloco_workspace_size() bytes.
 *
 * Asynchrony.  isoloco_aggregate() only enqueues work on the caller's HIP
 * stream and returns; buffers must stay valid until the stream passes that
 * point.  One plan must not be used by two streams at once; distinct plans
 * are independent.  The call issues kernel launches only (no host
 * synchronisation, memset or allocation; with two streams also an event
 * record and wait to fork the plan's second stream off the caller's and
 * one to join it back), so it may be captured in a HIP graph; every replay
 * then repeats the step on the same buffers.
 *
 * Errors.  Every function returns an isoloco_status; no C++ exception crosses
 * this boundary.  A call that fails validation enqueues nothing.  An
 * aggregate that fails later (ISOLOCO_ERR_HIP, a launch or event call
 * refused by the runtime) may have enqueued part of the step, so that theta,
 * B and the workspace hold a partial result; the caller's stream is then
 * still ordered after every kernel the call enqueued, on either stream, and
 * the first error is returned.  The last error message of the calling thread
 * is available from isoloco_last_error().
 */
#ifndef ISOLOCO_H
#define ISOLOCO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ISOLOCO_MAX_WORKERS 128

typedef enum {
  ISOLOCO_OK = 0,
  ISOLOCO_ERR_INVALID_ARG = -1, /* null pointer, K out of range, non-finite scalar, bad option  */
  ISOLOCO_ERR_LAYOUT = -2,      /* tensor out of range, overlapping, rows/cols < 1, bad kind     */
  ISOLOCO_ERR_ALIGN = -3,       /* a device base pointer is not 16-byte aligned                  */
  ISOLOCO_ERR_ALIAS = -4,       /* theta, momentum, a worker or the workspace overlap            */
  ISOLOCO_ERR_WORKSPACE = -5,   /* workspace missing, too small or misaligned                    */
  ISOLOCO_ERR_HIP = -6,         /* a HIP runtime call or kernel launch failed                    */
  ISOLOCO_ERR_UNSUPPORTED = -7  /* a valid request the library does not implement                */
} isoloco_status;

typedef enum { ISOLOCO_F32 = 0, ISOLOCO_BF16 = 1 } isoloco_dtype;

typedef enum {
  ISOLOCO_KIND_ISO = 0, /* a rows x cols matrix: spectrum flattened (Algorithm 2, dim = 2) */
  ISOLOCO_KIND_AVG = 1  /* plain mean pseudo-gradient (1-D tensors, or 2-D kept plain)     */
} isoloco_kind;

/* One tensor of the flat layout: elements [offset, offset + rows*cols) of every
 * buffer, row-major.  A 1-D tensor of length n is {offset, n, 1, AVG}.
 * Elements covered by no tensor are left untouched. */
typedef struct {
  int64_t offset;
  int64_t rows;
  int64_t cols;
  int32_t kind;     /* isoloco_kind */
  int32_t reserved; /* must be 0 */
} isoloco_tensor;

/* Plan options; pass NULL for the defaults (every field 0 also selects the default). */
typedef struct {
  int32_t max_steps; /* cap on the polar iteration's steps (default 40)                          */
  float ell0;        /* assumed lower bound of sigma_min / ||Delta^T Delta||_F^(1/2), the start
                        of the polynomial schedule (default 1e-10)                               */
  float tol;         /* the schedule stops when every singular value is within tol of 1
                        (default 1e-6)                                                           */
  int32_t check;     /* 1: after the last step also form Q^T Q to report the orthonormality
                        residual per matrix in isoloco_get_stats (default 1); -1: skip it        */
  int32_t precision; /* arithmetic of the matrix products (ISOLOCO_PREC_*): split-bfloat16
                        products split every fp32 operand into 2 (bf16x3: 3 bf16 MFMA
                        products, about 2^-16 relative error) or 3 (bf16x6: 6 products,
                        about fp32 accuracy) bfloat16 parts and accumulate in fp32.
                        MIXED (default): the update products X P of the first 3 steps
                        in bf16x5 (X in 3 parts, P in 2: 5 products, about the accuracy
                        of bf16x6 for this product), bf16x3 for every other product      */
  /* Variants of the step that the paper studies (all 0: Algorithm 2). */
  int32_t orth;      /* ISOLOCO_ORTH_POLAR: Q = U V^T, the converged polar factor (Algorithm 2);
                        ISOLOCO_ORTH_NS5: the fast variant's five Newton-Schulz steps of the
                        Muon quintic (3.4445, -4.7750, 2.0315) on Delta / ||Delta||_F
                        (Section 4.3); ell0, tol and the phases do not apply, and the residual
                        of check is reported without the not-converged flag                */
  int32_t scale;     /* ISOLOCO_SCALE_MEAN: sigma_bar = <Q, Delta>_F / r, the mean singular
                        value (Algorithm 2; needs ORTH_POLAR); ISOLOCO_SCALE_RMS:
                        ||Delta||_F / sqrt(r) (Section 4.3); ISOLOCO_SCALE_SPECTRAL:
                        sqrt(rows / cols), Muon's sqrt(fan_out / fan_in) (Appendix B)      */
  int32_t momentum;  /* ISOLOCO_MOMENTUM_NESTEROV: B <- mu B + D, theta <- theta - lr (D + mu B)
                        (Algorithm 2); ISOLOCO_MOMENTUM_HEAVY_BALL: B <- mu B + D,
                        theta <- theta - lr B (Section 4.5's ablation)                      */
  int32_t target;    /* ISOLOCO_TARGET_DELTA: correct Delta, then the momentum step
                        (Algorithm 2); ISOLOCO_TARGET_UPDATE: B <- mu B + Delta first, then
                        correct the update (Delta + mu B, or B with HEAVY_BALL) and step
                        theta <- theta - lr D (Section 4.5's ablation).  AVG tensors always
                        take the uncorrected step of the chosen momentum                   */
  int32_t clip;      /* ISOLOCO_CLIP_NONE: flatten the whole spectrum to its mean (Algorithm 2);
                        ISOLOCO_CLIP_HIGH / ISOLOCO_CLIP_LOW: set only the singular values
                        above / below the mean to the mean, keeping U, V and the other
                        singular values (Section 4.5).  Needs ORTH_POLAR and SCALE_MEAN; a
                        second polar iteration runs on Delta - sigma_bar Q                 */
  float phase_tall[3];   /* Phases of the polar iteration of tall matrices (m >= 2n in tall
                        coordinates, m x n with m >= n): bounds b0 > b1 > b2 on
                        sigma_min / ||Delta^T Delta||_F^(1/2).  The iteration first runs the
                        schedule for [b0, 1]; a matrix whose Q^T Q is then the identity to
                        5e-5 stops there, the others continue with the schedule that takes
                        what the steps so far made of b1 to 1, the same test, and so on,
                        until a last phase reaches [ell0, 1].  0 selects the default of a
                        slot (1e-3, 1e-4, 2e-8); a negative entry ends the list; an entry
                        not strictly between the one before and ell0 is left out.  A
                        negative b0 runs the single schedule for [ell0, 1].  The smallest
                        singular value of a tall noise-like matrix stays away from zero   */
  float phase_square[3]; /* the same for the other matrices (square-ish, m < 2n), whose
                        smallest singular value does not: defaults 3e-7, 2e-8, none.  Both
                        classes iterate in the same launches, each with its coefficients */
  int32_t streams;   /* 1: the polar iteration of every matrix on the caller's stream; 2: the
                        tall matrices on the caller's stream and the others on a second
                        stream of the plan's (forked after the reduction, joined before the
                        scale), so that each fills the other's launch gaps and last waves;
                        0 (default): 2 when the corrected matrices hold at most 2^29
                        elements, else 1 (large products compete for the caches instead)  */
  int32_t factored;  /* 1: the tall matrices take the steps from s to the end of their first
                        phase on n x n factors: with A = X_s^T X_s, X_k = X_s M gives
                        X_k^T X_k = M A M, so each step is M <- M p_k(M A M) (n x n products
                        only) and X = X_s M is formed once at the phase end, where the check
                        runs as before (Section 4.3's polar factor by polynomial steps,
                        reorganised; the same steps and coefficients).  s is the first step
                        after which the phase's lower bound has grown to 1/4 (so that A is
                        well conditioned; 4 for the default phases), moved on by one so that
                        the phase end - s is odd, with at least 3 steps left; 2: every step
                        on the m x n iterate; 0 (default): 1.  Not with ORTH_NS5
                        (isoloco_factored_steps reports the steps)                        */
} isoloco_options;

#define ISOLOCO_PREC_MIXED 0
#define ISOLOCO_PREC_FP32 1
#define ISOLOCO_PREC_BF16X3 2
#define ISOLOCO_PREC_BF16X6 3

#define ISOLOCO_ORTH_POLAR 0
#define ISOLOCO_ORTH_NS5 1
#define ISOLOCO_SCALE_MEAN 0
#define ISOLOCO_SCALE_RMS 1
#define ISOLOCO_SCALE_SPECTRAL 2
#define ISOLOCO_MOMENTUM_NESTEROV 0
#define ISOLOCO_MOMENTUM_HEAVY_BALL 1
#define ISOLOCO_TARGET_DELTA 0
#define ISOLOCO_TARGET_UPDATE 1
#define ISOLOCO_CLIP_NONE 0
#define ISOLOCO_CLIP_HIGH 1
#define ISOLOCO_CLIP_LOW 2

/* Per-tensor results of the last isoloco_aggregate() on a plan. */
typedef struct {
  float sigma_bar;  /* the scale of the correction (ISO tensors; 0 for AVG): the mean
                       singular value of Delta_l by default, else as the scale option says */
  float fro_norm;   /* ||Delta_l||_F                                                        */
  float orth_resid; /* ||Q^T Q - I||_F / sqrt(r) on the short side (ISO, if checked; else -1) */
  int32_t steps;    /* polar iteration steps taken (ISO tensors): the short schedule's length
                       if the matrix stopped there, else the full length                     */
  int32_t flags;    /* bit 0: Delta_l had a non-finite value; bit 1: Delta_l == 0;
                       bit 2: residual above 1e-3 after the last step (not converged);
                       bit 3: below resolution -- the matrix failed the check after the
                       phase built for sigma_min / ||Delta^T Delta||_F^(1/2) >= 2e-8, so a
                       singular value lies below about 2e-8 of the normalisation, where the
                       float32 rounding of Delta itself moves singular values by their own
                       size: the sign of that direction in Q is decided by rounding and can
                       differ from the float64 SVD's (Q stays orthonormal; the bit needs a
                       phase bound at or below 2e-8, which the default phases have)      */
  int32_t reserved;
} isoloco_tensor_stats;

#define ISOLOCO_FLAG_NONFINITE 1
#define ISOLOCO_FLAG_ZERO 2
#define ISOLOCO_FLAG_NOT_CONVERGED 4
#define ISOLOCO_FLAG_BELOW_RESOLUTION 8

typedef struct isoloco_plan_s* isoloco_plan_t;

/* Build a plan for one layout.  Host only: validates the table (every tensor
 * inside [0, n_elems), no two overlapping, rows and cols >= 1, kind valid),
 * orders the matrices for batched launches, builds the polynomial schedule
 * and sizes the workspace.  1 <= K <= ISOLOCO_MAX_WORKERS.  On success
 * *out_plan owns host memory released by isoloco_plan_destroy(). */
isoloco_status isoloco_plan(const isoloco_tensor* layout, int32_t n_tensors, int64_t n_elems,
                            int32_t K, isoloco_dtype worker_dtype, const isoloco_options* opts,
                            isoloco_plan_t* out_plan);

/* Workspace bytes the plan needs (device memory, 256-byte aligned). */
isoloco_status isoloco_workspace_size(isoloco_plan_t plan, size_t* bytes);

/* Hand the plan a device workspace of at least isoloco_workspace_size() bytes,
 * 256-byte aligned, on the current HIP device.  The caller keeps ownership.
 * Copies the plan's device tables into it (synchronous); call once before
 * the first aggregate, and again whenever the workspace moves. */
isoloco_status isoloco_set_workspace(isoloco_plan_t plan, void* dev_ptr, size_t bytes);

/* Enqueue one IsoLoCo outer step on `hip_stream` (a hipStream_t; NULL = the
 * default stream).  global and momentum: float32 device arrays of n_elems,
 * updated in place.  workers: HOST array of K device pointers, each to
 * n_elems elements of worker_dtype (read only; copied into the launch, so
 * the host array may be freed on return).  All device pointers 16-byte
 * aligned; workers must not overlap global, momentum or the workspace.
 * alpha, outer_lr and mu must be finite. */
isoloco_status isoloco_aggregate(isoloco_plan_t plan, float* global, const void* const* workers,
                                 float* momentum, float alpha, float outer_lr, float mu,
                                 void* hip_stream);

/* For callers that cannot allocate device memory (code that must not call
 * hipMalloc, such as tight serving loops or harnesses that forbid it): the
 * same step as isoloco_aggregate(), with the same arguments, results (bit for
 * bit) and errors, but on a workspace the library holds as a fixed array of
 * ISOLOCO_STATIC_WORKSPACE_BYTES in the memory of every device it runs on,
 * from the first use until the process ends, instead of a caller-provided one.
 * No device memory is allocated or freed, by the library or on its behalf.
 *
 * - The plan needs no isoloco_set_workspace(); a plan whose workspace size
 *   exceeds ISOLOCO_STATIC_WORKSPACE_BYTES is rejected with
 *   ISOLOCO_ERR_WORKSPACE and nothing is enqueued.
 * - Every call on a device shares that device's array.  When the array last
 *   held another plan's tables (or none), the call first waits for the device
 *   to be idle (calls of other plans may still read the array), copies this
 *   plan's tables in and clears the counters and per-matrix state the
 *   kernels expect at zero (synchronous; not capturable in a HIP graph --
 *   make the first call of a plan outside capture).  Later calls of the same
 *   plan enqueue kernel launches only.
 * - Calls that may overlap on one device (different streams or host threads,
 *   the same or different plans) race on the array: order them.
 * - The polar iteration runs on the caller's stream only (the two-stream mode
 *   would need a stream the library creates).
 * - isoloco_get_stats() reads the array: it fails with
 *   ISOLOCO_ERR_INVALID_ARG once another plan has used the device's array
 *   after this plan's last step. */
#define ISOLOCO_STATIC_WORKSPACE_BYTES (128u * 1024u * 1024u)

isoloco_status isoloco_aggregate_static(isoloco_plan_t plan, float* global, const void* const* workers,
                                        float* momentum, float alpha, float outer_lr, float mu,
                                        void* hip_stream);

/* Copy the per-tensor statistics of the last aggregate to the host
 * (n_tensors entries, in layout order).  Waits for that aggregate's stream. */
isoloco_status isoloco_get_stats(isoloco_plan_t plan, isoloco_tensor_stats* out, int32_t n_tensors);

/* The polynomial schedule of one class of matrices (tall = 1: m >= 2n in tall
 * coordinates, m x n with m >= n; tall = 0: the others): for step k, p_k(x) =
 * c[3k] x + c[3k+1] x^3 + c[3k+2] x^5 (on singular values normalised by
 * ||Delta^T Delta||_F^(1/2)).  Writes at most max_steps triples; *n_steps
 * receives the schedule length and *n_short (if not NULL) the length of the
 * short first phase (= *n_steps for one phase).  Host only. */
isoloco_status isoloco_schedule(isoloco_plan_t plan, int32_t tall, double* coeffs, int32_t max_steps,
                                int32_t* n_steps, int32_t* n_short);

/* The phases of one class's schedule (tall as above): ends[i] is the number of
 * steps done when phase i ends (increasing; the last equals the schedule
 * length).  Phase 0 is the schedule for the class's first bound; each later
 * phase continues it for a smaller bound (the class's next bounds, then ell0).
 * After every phase but the last, the matrices whose Q^T Q is the identity to
 * the switch tolerance stop.  Both classes iterate in the same launches; a
 * class whose schedule is shorter stops at its end.  Writes at most max_phases
 * entries; *n_phases receives the count.  Host only. */
isoloco_status isoloco_schedule_phases(isoloco_plan_t plan, int32_t tall, int32_t* ends, int32_t max_phases,
                                       int32_t* n_phases);

/* The steps [*first, *end) that the tall matrices take on n x n factors
 * (isoloco_options.factored); both 0 when none.  Host only. */
isoloco_status isoloco_factored_steps(isoloco_plan_t plan, int32_t* first, int32_t* end);

/* How a plan's matrix products run (tests and the benchmark's accounting).  In
 * the mixed and bf16x3 modes the iterates and the n x n matrices are kept as
 * the bfloat16 parts the products read ("planes") unless a matrix has more
 * than 2^21 - 32 rows, the planes' padding to multiples of 32 would cost the
 * plan its place in the static workspace or more than double a larger one, or
 * (mixed) the factored steps would start at step 1; the parts per product are
 * the mode's either way.  Host only. */
typedef struct {
  int32_t planes;             /* 1: planes; 0: float32 operands                       */
  int32_t third;              /* 1: planes with the third parts of the first iterates */
  int32_t update_parts_early; /* part products of the updates of the first 3 steps    */
  int32_t parts;              /* part products of every other product (1: float32)    */
  /* planes, per class (0 square-ish, 1 tall): the side of the output tiles of
   * its launches (0: no matrix of the class)                                       */
  int32_t gram_tile[2], poly_tile[2], update_tile[2];
} isoloco_products;

isoloco_status isoloco_get_products(isoloco_plan_t plan, isoloco_products* out);

/* Per-kernel timing of the last aggregate, measured with HIP events recorded
 * on the aggregate's stream around every launch (enable first; the events
 * add a few microseconds per launch).  Not part of the operation itself. */
typedef struct {
  float total_ms;   /* first launch start to last launch end                       */
  float reduce_ms;  /* K-way reduction (+ Nesterov of the uncorrected tensors)     */
  float gram_ms;    /* batched Gram products X^T X, all steps (+ the check, and the
                       per-matrix decisions their last tiles take); with factored
                       steps also their symmetric n x n products (M B and A M on
                       planes, M B and M P on float32 operands)                    */
  float poly_ms;    /* batched polynomial products b A + c A^2, all steps          */
  float update_ms;  /* batched updates X <- X P, all steps (with factored steps
                       also their whole n x n product, M P or A M)                 */
  float finish_ms;  /* fused Nesterov write-back of the corrected tensors          */
  float other_ms;   /* ||Delta||_F per matrix, the trace with sigma_bar, a phase end
                       without a check, the clip variants' composition             */
  int32_t gram_launches, poly_launches, update_launches, launches;
  float products_busy_ms; /* union of the Gram, polynomial and update launches' intervals:
                        the time some product runs (with two streams the launches overlap,
                        and each per-phase sum above counts every launch's own duration) */
  int32_t streams;  /* streams the polar iteration used (1 or 2)                      */
} isoloco_timing;

/* enable = 1 turns per-launch event timing on for later aggregates, 0 off. */
isoloco_status isoloco_enable_timing(isoloco_plan_t plan, int32_t enable);

/* Timing of the last aggregate (waits for its stream). */
isoloco_status isoloco_get_timing(isoloco_plan_t plan, isoloco_timing* out);

isoloco_status isoloco_plan_destroy(isoloco_plan_t plan);

/* ---------------------------------------------------------------------------
 * Operators of the workers' inner training step
 *
 * What produces the replicas that the outer step merges: the operators of a
 * training step around its matrix products.  They share the conventions above:
 * the caller owns every buffer, a call only enqueues kernel launches on the
 * caller's stream (it may be captured in a HIP graph), a call that fails
 * validation enqueues nothing, and no state is kept between calls.  Matrices
 * are row-major with unit stride along a row; ld_* is the distance of two rows
 * in elements (at least the row's length).  Device pointers need the alignment
 * of their elements only; 16-byte aligned rows are faster.  Outputs must not
 * overlap inputs, the workspace or each other unless a function says so.
 * Workspaces are 256-byte aligned device memory whose contents need not be
 * set and do not outlive the call; one may serve any number of calls that do
 * not overlap in time.  dtypes are isoloco_dtype, sums are held in 32 bits or
 * more and a result is rounded to its type once.  Results do not depend on
 * timing: the same call gives the same bits.
 * ------------------------------------------------------------------------- */

typedef enum { ISOLOCO_I32 = 0, ISOLOCO_I64 = 1 } isoloco_index_type;

/* Gradient clipping over many tensors.
 *
 *   norm = sqrt(sum over all tensors and elements of g^2)
 *   coef = max_norm / norm if max_norm < norm < infinity, else 1;  dst = coef * g
 *
 * src, dst, counts, dtypes: HOST arrays of n_tensors entries (read before the
 * call returns): each tensor's device pointer, its result's, its contiguous
 * elements (0 is allowed) and its type.  dst[i] may be src[i] (in place;
 * nothing is then written where coef is 1); a tensor's result must not overlap
 * another tensor, so a gradient that two names share is given once.  dst =
 * NULL: the norm only.  norm: two device floats, which receive norm and coef.
 * A norm that is infinite or NaN leaves the gradients as they are, and tells
 * the caller so.  Squares are summed in 64 bits: a norm
 * past float32's range is stored as infinity, with the coef that was applied
 * (less than 1).  coef is applied with all of its bits, also where the float
 * that is stored has lost some (below 2^-126).
 * max_norm >= 0 (infinity: never clip). */
isoloco_status isoloco_clip_workspace_size(int32_t n_tensors, size_t* bytes);
isoloco_status isoloco_clip_grads(const void* const* src, void* const* dst, const int64_t* counts,
                                  const int32_t* dtypes, int32_t n_tensors, float max_norm, float* norm,
                                  void* workspace, size_t workspace_bytes, void* hip_stream);

/* out[t] = scale * table[ids[t]] for n tokens; table: vocab x dim, out: n x dim.
 * An id outside [0, vocab) holds no token: a row of zeros. */
isoloco_status isoloco_embedding(const void* table, int64_t ld_table, int32_t dtype, int64_t vocab, int64_t dim,
                                 const void* ids, int32_t id_type, int64_t n, float scale, void* out, int64_t ld_out,
                                 int32_t out_dtype, void* hip_stream);

/* dtable[v] = scale * sum over the t with ids[t] = v of dout[t], in 32 bits, for
 * every v (rows without tokens: zeros).  accumulate != 0: added to what dtable
 * holds (a tied head's gradient, an earlier batch's).  Tokens are grouped by id
 * first and a row's are added in their order: no atomics. */
isoloco_status isoloco_embedding_backward_workspace_size(int64_t n, int64_t vocab, int64_t dim, size_t* bytes);
isoloco_status isoloco_embedding_backward(const void* ids, int32_t id_type, int64_t n, const void* dout,
                                          int64_t ld_dout, int32_t dtype, int64_t vocab, int64_t dim, float scale,
                                          int32_t accumulate, void* dtable, int64_t ld_dtable, int32_t dtable_dtype,
                                          void* workspace, size_t workspace_bytes, void* hip_stream);

#define ISOLOCO_MAX_TOP 32

/* Log probabilities of given tokens.  With z = scale * logits of a row (scale > 0):
 *
 *   lse = log sum_j e^z_j,  logprob = z_target - lse,  entropy = -sum_j p_j log p_j
 *   top_logprob, top_index: the top_k largest log probabilities (rows x top_k, in
 *   falling order, of equal logits the lower index first; NaN ranks above all)
 *
 * top_k <= min(ISOLOCO_MAX_TOP, vocab).  Any of logprob (with targets), entropy
 * and lse may be NULL.  A target outside [0, vocab) is ignored: logprob 0.
 * Logits of -infinity are masked (p = 0); a row of nothing else has lse =
 * logprob = -infinity and entropy 0.  A NaN or +infinity among a row's logits
 * makes its results NaN.  Finite logits of any size are taken as they are: a
 * result is infinite only where its value is past float32's range (logits that
 * lie further apart than that count as infinitely far). */
isoloco_status isoloco_token_logprobs_workspace_size(int64_t rows, int64_t vocab, int32_t top_k, size_t* bytes);
isoloco_status isoloco_token_logprobs(const void* logits, int64_t ld_logits, int32_t dtype, int64_t rows,
                                      int64_t vocab, const void* targets, int32_t target_type, float scale,
                                      int32_t top_k, float* logprob, float* entropy, float* lse, float* top_logprob,
                                      int64_t* top_index, void* workspace, size_t workspace_bytes,
                                      void* hip_stream);

/* The gradient of the above in the logits, from the lse (and entropy) it gave:
 *
 *   dlogits_j = scale * (dlogprob (1[j = target] - p_j) - dentropy p_j (log p_j + entropy))
 *
 * dlogprob goes with targets (rows whose target is ignored take none), dentropy
 * with entropy; either pair may be NULL.  dlogits has the logits' type and may
 * be the logits themselves (same pointer and ld).  A row whose dlogprob and
 * dentropy are zero, or whose logits are all -infinity, has a zero gradient.
 * p_j is e^(z_j - lse): off by 2^-24 |lse| of itself for lse's rounding.  Where
 * |lse| is 256 or more (8192 in bfloat16) the row's maximum and sum are formed
 * again instead, unless lse is not theirs (of a vocabulary in parts, say). */
isoloco_status isoloco_token_logprobs_backward(const void* logits, int64_t ld_logits, int32_t dtype, int64_t rows,
                                               int64_t vocab, const void* targets, int32_t target_type, float scale,
                                               const float* lse, const float* entropy, const float* dlogprob,
                                               const float* dentropy, void* dlogits, int64_t ld_dlogits,
                                               void* hip_stream);

typedef enum {
  ISOLOCO_ACT_SILU = 0, /* g / (1 + e^-g)                   */
  ISOLOCO_ACT_GELU = 1  /* g Phi(g), the exact normal CDF   */
} isoloco_activation;

/* out = act(x w_gate^T) * (x w_up^T); x: tokens x dim, w_gate and w_up: hidden x
 * dim (both ld_w apart), out: tokens x hidden; one dtype.  float32 products are
 * formed from three bfloat16 parts of each operand, all six products of order
 * 2^-16 and above (about float32 accuracy; an operand that is infinite or past bfloat16's
 * range, 3.39e38, gives NaN), or, for up to 64 tokens forward, in float32.
 *
 * The workspace's size goes by the call: ISOLOCO_FFN_BACKWARD for the gradient,
 * ISOLOCO_FFN_ALIGNED where the rows of x and of both weights will be 16-byte
 * aligned in bfloat16 (ld a multiple of 8) and at most 2^22 elements apart, which
 * saves their copies.  Extents are at most 2^22 - 64. */
#define ISOLOCO_FFN_BACKWARD 1
#define ISOLOCO_FFN_ALIGNED 2

isoloco_status isoloco_gated_ffn_workspace_size(int64_t tokens, int64_t dim, int64_t hidden, int32_t dtype,
                                                int32_t flags, size_t* bytes);
isoloco_status isoloco_gated_ffn(const void* x, int64_t ld_x, const void* w_gate, const void* w_up, int64_t ld_w,
                                 int32_t dtype, int64_t tokens, int64_t dim, int64_t hidden, int32_t act, void* out,
                                 int64_t ld_out, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Its gradients from dout (tokens x hidden).  dx, or dw_gate with dw_up, may be
 * NULL.  The projections are formed again (nothing is kept from the forward
 * call); in bfloat16 the gradients of their two results, which the three
 * products read, are rounded to bfloat16 once. */
isoloco_status isoloco_gated_ffn_backward(const void* x, int64_t ld_x, const void* w_gate, const void* w_up,
                                          int64_t ld_w, int32_t dtype, int64_t tokens, int64_t dim, int64_t hidden,
                                          int32_t act, const void* dout, int64_t ld_dout, void* dx, int64_t ld_dx,
                                          void* dw_gate, void* dw_up, int64_t ld_dw, void* workspace,
                                          size_t workspace_bytes, void* hip_stream);

/* Routing of tokens to experts.  With x the scores of a token (tokens x experts)
 * and p their softmax, its top_k largest scores (of equal ones the lower expert
 * first) give
 *
 *   expert (tokens x top_k, in falling order), and weight: p at those, or
 *   (normalize != 0) p over its sum at those, the softmax of the chosen scores
 *
 * and the slots (token, j) are grouped by expert, within one in their order:
 *
 *   offsets (experts + 1): expert e has the places offsets[e] .. offsets[e + 1] - 1
 *   row (tokens x top_k): a slot's place;  token (tokens * top_k): a place's token
 *
 * so that row is a permutation of 0 .. tokens * top_k - 1.  A score of -infinity
 * is no expert to choose: a slot that finds none has expert -1 and weight 0, and
 * its place is behind the last expert's.  NaN ranks above all and makes the
 * token's weights NaN, as +infinity does.  top_k <= min(ISOLOCO_MAX_TOP,
 * experts); tokens * top_k < 2^31. */
#define ISOLOCO_MAX_EXPERTS 1024

isoloco_status isoloco_route_tokens_workspace_size(int64_t tokens, int64_t experts, size_t* bytes);
isoloco_status isoloco_route_tokens(const void* scores, int64_t ld_scores, int32_t dtype, int64_t tokens,
                                    int64_t experts, int32_t top_k, int32_t normalize, float* weight, int32_t* expert,
                                    int32_t* row, int32_t* token, int32_t* offsets, void* workspace,
                                    size_t workspace_bytes, void* hip_stream);

/* The gradient of weight in the scores, g_j = dweight of slot j, from the experts
 * that were chosen (slots outside 0 .. experts - 1 take none):
 *
 *   normalize:  dx at expert_j = w_j (g_j - sum_i w_i g_i), 0 elsewhere
 *   otherwise:  dx_e = p_e (the g_j with expert_j = e, less sum_i w_i g_i)       */
isoloco_status isoloco_route_tokens_backward(const void* scores, int64_t ld_scores, int32_t dtype, int64_t tokens,
                                             int64_t experts, int32_t top_k, int32_t normalize, const int32_t* expert,
                                             const float* dweight, void* dscores, int64_t ld_dscores,
                                             void* hip_stream);

/* Matrix products grouped by expert: out[r] = x_r w[e]^T for the rows r =
 * offsets[e] .. offsets[e + 1] - 1 of each expert e, where x_r is row token[r] of
 * x (tokens x dim), or row r if token is NULL (tokens = rows then).  w: experts
 * matrices of cols x dim, ld_w the distance of two rows and stride_w that of two
 * matrices; out: rows x cols.  offsets (experts + 1, not falling, from 0 to at
 * most rows) and token (rows) are of index_type and stay on the device: their
 * values are not known to the host, and nothing outside the tensors is touched
 * whatever they are.  Rows from offsets[experts] on are zeros, and a token
 * outside 0 .. tokens - 1 stands for a row of zeros.  An expert may have no rows.
 * float32 products are formed as in isoloco_gated_ffn (forward, in float32 where the
 * experts have up to 96 rows on average).
 *
 * The workspace's size goes by the call: ISOLOCO_EXPERTS_BACKWARD for the
 * gradient, ISOLOCO_EXPERTS_GATHERED where token is given, and
 * ISOLOCO_EXPERTS_ALIGNED where the operands that are read (x, w; backward: and
 * dout) will be 16-byte aligned with dim and cols, all ld and stride_w multiples of 8 and all
 * ld at most 2^22, which saves their copies in bfloat16.  dim and cols are at most 2^22 - 64. */
#define ISOLOCO_EXPERTS_BACKWARD 1
#define ISOLOCO_EXPERTS_ALIGNED 2
#define ISOLOCO_EXPERTS_GATHERED 4

isoloco_status isoloco_expert_matmul_workspace_size(int64_t tokens, int64_t rows, int64_t experts, int64_t dim,
                                                    int64_t cols, int64_t ld_x, int32_t dtype, int32_t flags,
                                                    size_t* bytes);
isoloco_status isoloco_expert_matmul(const void* x, int64_t ld_x, int64_t tokens, const void* token, const void* w,
                                     int64_t ld_w, int64_t stride_w, int32_t dtype, const void* offsets,
                                     int32_t index_type, int64_t experts, int64_t rows, int64_t dim, int64_t cols,
                                     void* out, int64_t ld_out, void* workspace, size_t workspace_bytes,
                                     void* hip_stream);

/* Its gradients from dout (rows x cols), either of which may be NULL:
 *
 *   dx[r] = dout[r] w[e] (rows x dim: of the grouped rows; rows of no expert: zeros)
 *   dw[e] = sum over the rows of e of dout[r]^T x_r (zeros without any)
 *
 * With token given, the gradient of x is the sum of dx over a token's rows, which
 * isoloco_expert_matmul_backward_tokens forms. */
isoloco_status isoloco_expert_matmul_backward(const void* x, int64_t ld_x, int64_t tokens, const void* token,
                                              const void* w, int64_t ld_w, int64_t stride_w, int32_t dtype,
                                              const void* offsets, int32_t index_type, int64_t experts, int64_t rows,
                                              int64_t dim, int64_t cols, const void* dout, int64_t ld_dout, void* dx,
                                              int64_t ld_dx, void* dw, int64_t ld_dw, int64_t stride_dw,
                                              void* workspace, size_t workspace_bytes, void* hip_stream);

/* The same where token is given, with the gradient of x itself:
 *
 *   dx[t] = sum_j of row row[t, j] of the above's dx (tokens x dim)
 *
 * row (tokens x top_k, of row_type; isoloco_route_tokens' row): the rows whose token is t,
 * entries outside 0 .. rows - 1 add nothing.  The rows are held in float32, in dx_rows (rows x dim:
 * scratch), and a sum is rounded once.  dx is formed always, dw unless it is NULL, and
 * the workspace's size is the one for the gradient with token given.  top_k <=
 * ISOLOCO_MAX_TOP. */
isoloco_status isoloco_expert_matmul_backward_tokens(const void* x, int64_t ld_x, int64_t tokens, const void* token,
                                                     const void* row, int32_t row_type, int32_t top_k, const void* w,
                                                     int64_t ld_w, int64_t stride_w, int32_t dtype, const void* offsets,
                                                     int32_t index_type, int64_t experts, int64_t rows, int64_t dim,
                                                     int64_t cols, const void* dout, int64_t ld_dout, void* dx,
                                                     int64_t ld_dx, float* dx_rows, void* dw, int64_t ld_dw,
                                                     int64_t stride_dw, void* workspace, size_t workspace_bytes,
                                                     void* hip_stream);

/* out[t] = sum_j weight[t, j] y[row[t, j]]; y: rows x dim, row and weight: tokens x
 * top_k (weight NULL: ones), out: tokens x dim.  Entries of row outside 0 .. rows
 * - 1 add nothing.  top_k <= ISOLOCO_MAX_TOP. */
isoloco_status isoloco_combine_tokens(const void* y, int64_t ld_y, int32_t dtype, int64_t rows, int64_t dim,
                                      const void* row, int32_t index_type, const float* weight, int64_t tokens,
                                      int32_t top_k, void* out, int64_t ld_out, void* hip_stream);

/* Its gradients, either of which may be NULL:
 *
 *   dy[row[t, j]] = weight[t, j] dout[t]          dweight[t, j] = <dout[t], y[row[t, j]]>
 *
 * No two entries of row may be the same (the row's gradient is then from any of
 * them); rows of dy that none names are zeros.
 * dweight is 0 where the entry is outside.  y is read for dweight only, and the
 * workspace serves dy only. */
isoloco_status isoloco_combine_tokens_backward_workspace_size(int64_t tokens, int32_t top_k, size_t* bytes);
isoloco_status isoloco_combine_tokens_backward(const void* dout, int64_t ld_dout, const void* y, int64_t ld_y,
                                               int32_t dtype, int64_t rows, int64_t dim, const void* row,
                                               int32_t index_type, const float* weight, int64_t tokens, int32_t top_k,
                                               void* dy, int64_t ld_dy, float* dweight, void* workspace,
                                               size_t workspace_bytes, void* hip_stream);

/* Distillation from a teacher's most likely tokens.  With z = scale * logits of a
 * row (scale > 0), q their softmax, and the row's top_k entries t_i = top_logprob
 * (log probabilities) of the columns c_i = top_index:
 *
 *   ISOLOCO_REST_DROP     p_i = e^t_i / sum_i e^t_i  (t_i may be logits too)
 *                         loss = sum_i p_i (log p_i - log q_ci)
 *   ISOLOCO_REST_BUCKET   p_i = e^t_i, p_r = 1 - sum_i p_i, if positive
 *                         loss = sum_i p_i (log p_i - log q_ci) + p_r (log p_r - log q_r)
 *
 * where q_r is the sum of q over the columns that are not listed: what the teacher
 * gives to all others is compared as one (left out where the student has no such
 * column, or only masked ones: logits of -infinity.  Columns that are all at a large
 * finite value, -1e30 say, are a bucket as any, and log q_r is as large).  An entry outside the vocabulary is none; a row
 * without entries has no loss and no gradient.  t_i = -infinity adds nothing; a
 * column that is listed twice counts as often.  Logits of -infinity are masked: q =
 * 0, and the loss is infinite where p_i > 0 there.  A NaN or +infinity among a row's
 * logits, or NaN among its t, makes its results NaN.
 * loss: rows floats.  stats: rows x ISOLOCO_DISTILL_STATS floats for the gradient,
 * of which [6] is the row's log-sum-exp of z.  top_k <= ISOLOCO_MAX_TEACHER. */
#define ISOLOCO_MAX_TEACHER 128
#define ISOLOCO_DISTILL_STATS 10

typedef enum { ISOLOCO_REST_DROP = 0, ISOLOCO_REST_BUCKET = 1 } isoloco_rest;

isoloco_status isoloco_distill_loss_workspace_size(int64_t rows, int64_t vocab, size_t* bytes);
isoloco_status isoloco_distill_loss(const void* logits, int64_t ld_logits, int32_t dtype, int64_t rows, int64_t vocab,
                                    const float* top_logprob, const void* top_index, int32_t index_type, int32_t top_k,
                                    float scale, int32_t rest, float* loss, float* stats, void* workspace,
                                    size_t workspace_bytes, void* hip_stream);

/* The gradient of the above in the logits, from the stats it gave and dloss (rows):
 *
 *   dlogits_j = dloss * scale * (q_j W - the p_i with c_i = j, less p_r q_j / q_r
 *               where j is not listed),  W = sum_i p_i (+ p_r)
 *
 * dlogits has the logits' type and may be the logits themselves (same pointer and
 * ld).  A row whose dloss is zero, without entries, or whose logits are all
 * -infinity, has a zero gradient. */
isoloco_status isoloco_distill_loss_backward(const void* logits, int64_t ld_logits, int32_t dtype, int64_t rows,
                                             int64_t vocab, const float* top_logprob, const void* top_index,
                                             int32_t index_type, int32_t top_k, float scale, int32_t rest,
                                             const float* stats, const float* dloss, void* dlogits, int64_t ld_dlogits,
                                             void* hip_stream);

const char* isoloco_status_string(isoloco_status s);

/* Message of the last failed call on this thread ("" if none). */
const char* isoloco_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* ISOLOCO_H */
