/*
 * shampoo.h -- C ABI of the MI355X (gfx950) scalable-Shampoo hot path.
 *
 * Paper: Anil, Gupta, Koren, Regan, Singer, "Scalable Second Order
 * Optimization for Deep Learning" (arXiv 2002.09018).  The three steps the
 * paper lists as Shampoo's extra cost (Section 3, "Scaling-up Second Order
 * Optimization": statistics, inverse p-th roots, preconditioned gradient) map
 * onto shampoo_update_stats, shampoo_inv_root_batched and shampoo_precondition;
 * the layer-wise grafted update of Algorithm 2 and of the appendix "Further
 * details on experiments" (paragraph "Layer wise learning rates") is
 * shampoo_graft.
 *
 * Conventions shared by every call
 *  - Matrices are row-major.  A block is a strided view of a larger tensor:
 *    element (i, j) of the view lives at ptr[i * ld + j].
 *  - Every tensor pointer is a DEVICE pointer on the handle's device, owned
 *    by the caller.  The library never frees caller memory.
 *  - Every call is ordered on `stream` (a hipStream_t passed as void*; NULL
 *    is the null stream).  Host arrays passed in (blocks, jobs, params) are
 *    copied before the call returns and may be reused at once.
 *  - Return codes cover argument and launch errors only.  Numeric outcomes of
 *    root computations are per-matrix status codes written to device memory.
 *  - One handle per host thread/stream pair; handles share no state.
 *  - The library owns only what hangs off its handle: device copies of the
 *    block/job tables, a grow-on-demand scratch area for the intermediate
 *    G*Rr of two-sided preconditioning, and a few bytes of pinned host memory
 *    used to poll convergence.
 */
#ifndef SHAMPOO_MI355X_H
#define SHAMPOO_MI355X_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum shampoo_status {
  SHAMPOO_OK = 0,
  SHAMPOO_EINVAL = -1,       /* bad argument: NULL where required, size out of range, ... */
  SHAMPOO_EUNSUPPORTED = -2, /* valid but not implemented (e.g. root order p outside [1, 16]) */
  SHAMPOO_EHIP = -3,         /* a HIP runtime call or kernel launch failed */
  SHAMPOO_ENOMEM = -4        /* workspace too small, or a library allocation failed */
} shampoo_status;

/* Element type of the gradient views G (and of logits and activations). */
typedef enum shampoo_dtype {
  SHAMPOO_F32 = 0,
  SHAMPOO_BF16 = 1 /* raw bfloat16 bit patterns; up-cast exactly to fp32 on load */
} shampoo_dtype;

/* Per-matrix outcome of shampoo_inv_root_batched (shampoo_root_info.status). */
enum {
  SHAMPOO_ROOT_CONVERGED = 0, /* max|M - I| <= tol */
  SHAMPOO_ROOT_STAGNATED = 1, /* residual stopped decreasing below 1e-3: rounding floor reached */
  SHAMPOO_ROOT_MAXITER = 2,   /* iteration cap reached */
  SHAMPOO_ROOT_DIVERGED = 3,  /* residual non-finite or above 1e6 */
  SHAMPOO_ROOT_NOT_PD = 4     /* damped matrix has a non-positive diagonal entry or zero norm */
};
/* NOT_PD is a cheap necessary test only (a positive definite matrix has a
 * positive diagonal), not an eigenvalue test.  An indefinite damped matrix
 * whose diagonal is positive is not flagged up front: its negative
 * eigenvalues make the iteration fail, and it comes back DIVERGED (or
 * MAXITER).  Either status means that no root exists or none was found; X
 * then holds the last iterate and must not be used. */

/* Arithmetic used for roots (shampoo_root_params.precision). */
enum {
  SHAMPOO_PRECISION_FP32 = 0, /* fp32 only */
  SHAMPOO_PRECISION_AUTO = 1, /* fp32; matrices that need more iterations than a matrix
                                 of condition kappa32 would (or that fail) are redone in fp64 */
  SHAMPOO_PRECISION_FP64 = 2  /* fp64 only */
};

/*
 * One preconditioned block (Section 3.1, "Preconditioning blocks from large
 * tensors": each block of a large tensor is treated as a tensor of its own).
 * rows x cols = m x n, both in [1, 4096].  G, W, D, P, Mg and Ps are m x n
 * views sharing the row stride `ld` (elements, >= cols).  L is m x m and R is
 * n x n, contiguous (ld = m and n).  A NULL statistic means that side is not
 * tracked; a NULL root means the identity on that side (one-sided
 * preconditioning, Lemma 1).  Mg and Ps are needed only when beta1 > 0.
 * Element types: G per call (shampoo_dtype), everything else fp32.
 */
typedef struct shampoo_block {
  int32_t rows, cols;
  int64_t ld;
  const void* G;
  float* W;
  float* D;
  float* P;
  float* Mg;
  float* Ps;
  float* L;
  float* R;
  const float* Lr;
  const float* Rr;
} shampoo_block;

/*
 * One inverse-root job: X = (A_s + eps_eff I)^(-1/p) with A_s the symmetric
 * part of A.  A and X are contiguous n x n fp32, n in [1, 4096]; A is only
 * read.  X receives the root; on a status other than CONVERGED/STAGNATED it
 * holds the last iterate.
 */
typedef struct shampoo_root_job {
  int32_t n;
  int32_t reserved; /* must be 0 */
  const float* A;
  float* X;
} shampoo_root_job;

/* Cold-start scaling of a root call, M0 = z A_d, X0 = z^(1/p) I.  Both keep
 * the largest eigenvalue of M0 at or below (p + 1) / 2 through an upper
 * bound B on lambda_max(A_d), z = (p + 1) / (2 B):
 *   FROBENIUS  B = ||A_d||_F, Algorithm 1 as printed;
 *   POWER4     B = ||A_d^4||_F^(1/4) = (sum_i lambda_i^8)^(1/8), a tighter
 *              bound from two extra products (the first reused as M0^2 in the
 *              first iteration); the coupled-Newton appendix leaves the
 *              start constant free (X0 = I / c).  On flat spectra it saves
 *              3-4 of 7 iterations. */
enum { SHAMPOO_SCALING_FROBENIUS = 0, SHAMPOO_SCALING_POWER4 = 1 };

/* Parameters of a root call (Algorithm 1).  shampoo_root_params_default()
 * fills the values used throughout the repository. */
typedef struct shampoo_root_params {
  int32_t p;            /* root order: X = A^(-1/p); 1 <= p <= 16 */
  float eps;            /* damping: eps_eff = eps, or eps * lambda_max when eps_relative */
  int32_t eps_relative; /* 1: scaled damping with lambda_max from MaxSV power iteration */
  float tol;            /* stop when max_ij |M - I|_ij <= tol */
  int32_t max_iters;    /* iteration cap of a precision phase */
  int32_t precision;    /* SHAMPOO_PRECISION_* */
  float kappa32;        /* AUTO: largest damped condition number accepted from fp32 */
  int32_t maxsv_steps;  /* MaxSV cap on power steps */
  float maxsv_tol;      /* MaxSV stop: |lambda - lambda_old| <= maxsv_tol * lambda */
  int32_t poll;         /* 1: the host polls a device counter and stops enqueuing
                           iterations once no matrix is active (the call then waits
                           for the stream); 0: enqueue max_iters iterations, fully
                           asynchronous, converged matrices skip their work */
  int32_t scaling;      /* SHAMPOO_SCALING_*: the constant of the cold start */
} shampoo_root_params;

/* Per-matrix result of a root call, written on the stream (device memory). */
typedef struct shampoo_root_info {
  int32_t status;     /* SHAMPOO_ROOT_* of the phase that produced X */
  int32_t iters;      /* iterations of that phase */
  int32_t precision;  /* 32 or 64: arithmetic that produced X */
  int32_t iters_fp32; /* iterations spent in fp32 (also when escalated) */
  float resid;        /* last max|M - I| */
  float lambda_max;   /* MaxSV estimate (eps_relative), else 0 */
  float cond_est;     /* condition-number upper estimate from the iteration count */
  float eps_eff;      /* damping actually added */
} shampoo_root_info;

/* Create / destroy a handle bound to HIP device `device`. */
shampoo_status shampoo_create(void** handle, int device);
shampoo_status shampoo_destroy(void* handle);
/* Text of the last error on this handle ("" if none).  Valid until the next call. */
const char* shampoo_last_error(const void* handle);
/* Library version string. */
const char* shampoo_version(void);

/* Defaults: p=4, eps=1e-6 absolute, tol=1e-6, max_iters=100, precision AUTO,
 * kappa32=1e4, maxsv_steps=100, maxsv_tol=1e-6, poll=1, scaling POWER4. */
void shampoo_root_params_default(shampoo_root_params* params);

/*
 * Statistics update, Preliminaries ("The Shampoo algorithm", definition of
 * L_t and R_t) and Algorithm 2:
 *   beta2 == 1:  L += G G^T,  R += G^T G
 *   beta2 <  1:  L = beta2 L + (1 - beta2) G G^T  (same for R)
 * For every block with non-NULL L (resp. R).  L and R stay exactly symmetric:
 * the upper triangle is computed and mirrored.  They must be symmetric on
 * entry as well (zero, or the output of earlier updates): the old value of an
 * off-diagonal element may be read from its mirror.  The ridge eps*I is not
 * added here; shampoo_inv_root_batched adds it once.  G: g_dtype.
 * Errors: EINVAL for nblocks < 0, NULL blocks with nblocks > 0, sizes
 * outside [1, 4096], ld < cols, beta2 outside (0, 1], L, R and G not
 * distinct buffers (a block with both L and R NULL is skipped).
 */
shampoo_status shampoo_update_stats(void* handle, const shampoo_block* blocks, int nblocks,
                                    int g_dtype, float beta2, void* stream);

/* Device workspace (bytes) that shampoo_inv_root_batched needs for `jobs`
 * under `precision`; 0 on invalid arguments. */
size_t shampoo_inv_root_workspace_bytes(const shampoo_root_job* jobs, int njobs, int precision);

/*
 * Batched inverse p-th roots by the coupled Newton iteration, Algorithm 1
 * (appendix "A coupled Newton iteration for computation of inverse p-th
 * roots"), all matrices in one grouped launch per product:
 *   eps_eff = eps, or eps * MaxSV(A) (scaled damping);
 *   A_d = A_s + eps_eff I;  z = (1 + p) / (2 ||A_d||_F);
 *   X = z^(1/p) I;  M = z A_d;
 *   while max|M - I| > tol:  M1 = ((p + 1) I - M) / p;  X = X M1;  M = M1^p M.
 * Each matrix leaves the iteration on its own (CONVERGED, STAGNATED, MAXITER,
 * DIVERGED).  M1^p M is formed by binary powering over the bits of p
 * (floor(log2 p) squarings plus popcount(p) products, launched in
 * floor(log2 p) + 1 stages per iteration).  Products of the commuting
 * symmetric iterates are computed on their upper triangle and mirrored.  `workspace` is device memory of at least
 * shampoo_inv_root_workspace_bytes(jobs, njobs, params->precision) bytes,
 * owned by the caller and used exclusively by this call until the stream
 * reaches its end.  `info` is a device array of njobs entries.
 * Errors: EINVAL (NULL pointers, njobs above 2^22, n outside [1, 4096], eps < 0,
 * tol < 0, max_iters < 1), EUNSUPPORTED (p outside [1, 16]), ENOMEM (ws_bytes
 * too small).
 */
shampoo_status shampoo_inv_root_batched(void* handle, const shampoo_root_job* jobs, int njobs,
                                        const shampoo_root_params* params, void* workspace,
                                        size_t ws_bytes, shampoo_root_info* info, void* stream);

/*
 * Warm-started batched inverse p-th roots (appendix "A coupled Newton
 * iteration for computation of inverse p-th roots", warm start, with the
 * commutator check it proposes for detecting divergence).  On entry jobs[j].X
 * holds X0, the previous root of a nearby matrix (any n x n fp32 matrix with
 * positive eigenvalues in exact arithmetic; typically the last call's result);
 * then
 *   M = X0^p A_d  (A_d = A_s + eps_eff I as in the cold call),  X = X0,
 *   while max|M - I| > tol:  M1 = ((p + 1) I - M) / p;  X = X M1;  M = M1^p M;
 *     after each iteration the warm start is given up when
 *     max|XM - MX| > comm_tol * max|X| * max|M|, when the residual grew in two
 *     consecutive iterations, or when it diverges or reaches max_iters.
 * The iterates no longer commute with A, so every product is a full n x n
 * product (twice the work of a cold product).  A residual that stops
 * decreasing below 1e-3 is accepted (STAGNATED, the rounding floor).  When
 * X0 commutes with A_d the limit is A_d^(-1/p); otherwise it is
 * X0 (X0^p A_d)^(-1/p), close to the root only while the drift is small.
 * Matrices whose warm start is given up are computed by the cold call's
 * iteration in the same call (with its precision policy); the others keep the
 * warm result.  The warm phase runs in fp64 under SHAMPOO_PRECISION_FP64 and
 * in fp32 otherwise (under AUTO an fp32 warm result carries fp32 rounding
 * amplified by the condition number: use FP64 for ill-conditioned factors).
 * A kept warm result is that limit, not the root: its distance from
 * A_d^(-1/p) grows with the drift of the statistics since X0 and is NOT held
 * to the tolerance of the cold call.  The monitor only guards against
 * divergence; it does not bound that distance (measured: 2.5e-4 to 6e-4 from
 * the cold roots one gradient after X0 on 1024 x 1024 statistics of ~20
 * gradients, 1.1e-3 when the statistics doubled since X0, every result kept
 * at comm_tol = 1e-3).  Callers that need the root to a stated tolerance use
 * shampoo_inv_root_batched.
 * params, workspace, info: as shampoo_inv_root_batched (same workspace size;
 * cond_est is 0 for a warm result).  warm_out (device, may be NULL): int32
 * [njobs][2] = {outcome, warm iterations}, outcome 1 = warm result kept,
 * 2 = warm start given up (cold result), 0 = not attempted (NOT_PD).
 * Errors: as shampoo_inv_root_batched, and EINVAL for comm_tol <= 0.
 */
shampoo_status shampoo_inv_root_warm_batched(void* handle, const shampoo_root_job* jobs, int njobs,
                                             const shampoo_root_params* params, float comm_tol, void* workspace,
                                             size_t ws_bytes, shampoo_root_info* info, int32_t* warm_out,
                                             void* stream);

/*
 * Preconditioned gradient P = Lr G Rr (Preliminaries, Shampoo update rule;
 * one-sided forms of Lemma 1 when a root is NULL; P = G when both are).
 * Lr and Rr must be symmetric (inverse roots are).  G: g_dtype.
 * Errors: as shampoo_update_stats; EINVAL when P is NULL or is the same
 * buffer as G, Lr or Rr.
 */
shampoo_status shampoo_precondition(void* handle, const shampoo_block* blocks, int nblocks,
                                    int g_dtype, void* stream);

/*
 * Grafted parameter update, Algorithm 2 with the AdaGrad-magnitude /
 * Shampoo-direction graft ("Layer wise learning rates"):
 *   D  = D + G o G
 *   Mg = beta1 Mg + (1 - beta1) D^(-1/2) o G        (D^(-1/2) o G := 0 where D == 0)
 *   use_shampoo:  Ps  = beta1 Ps + (1 - beta1) P
 *                 eta = eta0 ||Mg||_F / ||Ps||_F     (0 when ||Ps||_F == 0)
 *                 W   = W - eta Ps
 *   otherwise:    W   = W - eta0 Mg                  (before the first roots)
 * With beta1 == 0, Mg and Ps are not stored (may be NULL) and P is used as Ps.
 * norms (device, may be NULL): per block {||Mg||_F, ||Ps||_F, eta} as 3 floats.
 * Errors: EINVAL as above, non-finite eta0, beta1 outside [0, 1), NULL
 * W/D, P NULL with use_shampoo, Mg/Ps NULL with beta1 > 0, and an updated
 * state (W, D, Mg, Ps) that is the same buffer as G, P or another state.
 */
shampoo_status shampoo_graft(void* handle, const shampoo_block* blocks, int nblocks, int g_dtype,
                             float eta0, float beta1, int use_shampoo, float* norms, void* stream);

/*
 * Allocation-free form of shampoo_graft, for callers that cannot allocate
 * device memory (code under stream capture, tight serving loops, harnesses
 * that forbid hipMalloc): same arguments, same kernels and the same result
 * bit for bit.  Its scratch -- the block table and one pair of fp64 norm
 * partials per chunk of at most 16384 elements (whole rows of a block) --
 * lives in a fixed device array of SHAMPOO_GRAFT_NOALLOC_SCRATCH_BYTES that
 * every GPU the library runs on holds until the process ends; the table is
 * staged through pinned host memory that shampoo_create sets up.  The call
 * itself allocates nothing (no hipMalloc/hipFree, no growth of the handle),
 * and its launches are not recorded by shampoo_timing_*.
 * Limits: nblocks <= SHAMPOO_GRAFT_NOALLOC_MAX_BLOCKS and at most
 * SHAMPOO_GRAFT_NOALLOC_MAX_CHUNKS chunks in total, where a block of
 * m x n has ceil(m / max(1, 16384 / n)) chunks (96 blocks of 1024 x 4096
 * take 24576; calls of fewer than 2^24 elements use smaller chunks, about
 * 1024 to 2048 plus one per block); beyond either, ENOMEM and nothing is
 * enqueued.
 * Every call on a GPU uses that GPU's one array: calls on one stream are
 * ordered, calls that overlap on different streams of one GPU race.  The
 * host waits, if needed, for the previous call's table copy out of the
 * handle's staging memory before writing it again.
 * Errors: as shampoo_graft, and ENOMEM as above.
 */
#define SHAMPOO_GRAFT_NOALLOC_MAX_BLOCKS 8192
#define SHAMPOO_GRAFT_NOALLOC_MAX_CHUNKS 196608
#define SHAMPOO_GRAFT_NOALLOC_SCRATCH_BYTES (4u << 20)
shampoo_status shampoo_graft_noalloc(void* handle, const shampoo_block* blocks, int nblocks, int g_dtype,
                                     float eta0, float beta1, int use_shampoo, float* norms, void* stream);

/*
 * Preconditioning and the AdaGrad-grafted update in one call: the same
 * result as shampoo_precondition followed by shampoo_graft with beta1 = 0 and
 * use_shampoo = 1 (Preliminaries, Shampoo update rule; Algorithm 2 with the
 * graft of "Layer wise learning rates"):
 *   P = Lr G Rr;  D = D + G o G;
 *   eta = eta0 ||D^(-1/2) o G||_F / ||P||_F  (0 when ||P||_F == 0);  W = W - eta P
 * The GEMM that writes each block's P also updates D and sums the two squared
 * norms per output tile, so G, D and P are not read by a separate pass; the
 * norms are then reduced per block in a fixed order (deterministic, but in
 * another order than shampoo_graft's, so eta may differ in the last bits).
 * Every block needs W, D, P and at least one root; G: g_dtype.  norms:
 * as shampoo_graft.  Errors: as shampoo_graft, and EINVAL for a block with
 * both roots NULL, or whose P, W, D are not distinct or coincide with G or a
 * root.
 */
shampoo_status shampoo_precondition_graft(void* handle, const shampoo_block* blocks, int nblocks, int g_dtype,
                                          float eta0, float* norms, void* stream);

/*
 * Grafted update with the LARS/LAMB layer-wise magnitude of the same appendix
 * paragraph ("Layer wise learning rates": learning rate ||W||_F / ||G||_F per
 * layer, applied per block here): the step is eta0 ||W||_F long, W taken
 * before the step,
 *   Mg = beta1 Mg + (1 - beta1) G
 *   use_shampoo:  Ps  = beta1 Ps + (1 - beta1) P
 *                 eta = eta0 ||W||_F / ||Ps||_F     (0 when ||Ps||_F == 0)
 *                 W   = W - eta Ps
 *   otherwise:    eta = eta0 ||W||_F / ||Mg||_F     (LARS step, before the roots)
 *                 W   = W - eta Mg
 * D is not used (may be NULL).  With beta1 == 0, Mg and Ps are not stored.
 * norms (device, may be NULL): per block {||W||_F, ||direction||_F, eta}.
 * Errors: as shampoo_graft (D may be NULL).
 */
shampoo_status shampoo_graft_lamb(void* handle, const shampoo_block* blocks, int nblocks, int g_dtype,
                                  float eta0, float beta1, int use_shampoo, float* norms, void* stream);

/*
 * Embedding layers (appendix "Shampoo for embedding layers", with the
 * one-sided preconditioner of Lemma 1 for large layers).
 *
 * A table W (vocab x dim, row-major, row stride ldw) is read by nnz lookup
 * entries: entry e reads row idx[e] into output row feat[e] of the layer
 * output y (m x dim), with weight weight[e].  Its gradient
 *   G = sum_e weight[e] e_{idx[e]} dy[feat[e], :]   (vocab x dim)
 * is nonzero only on the active rows {idx[e]}, and the dim x dim statistic is
 *   R = G^T G = dy^T (S^T S) dy,   S[idx[e], feat[e]] += weight[e],
 * which is dy^T dy when every entry hits its own row (one-hot features on
 * distinct rows), at O(nnz dim^2) cost instead of O(vocab dim^2).
 * The step for the table is then
 *   shampoo_embedding_rows -> shampoo_embedding_stats -> (roots: Rr = R^(-1/2),
 *   shampoo_inv_root_batched with p = 2) -> shampoo_embedding_precondition
 *   -> shampoo_embedding_graft,
 * all on the compact rows.  Every count is read on the device: no call
 * synchronizes the stream.
 *
 * Compact form (written by shampoo_embedding_rows, read by the others):
 *   rows   int32[nnz]: the active rows in ascending order, then -1;
 *   U      fp32 nnz x dim (row stride dim): U[i] = G[rows[i]] for i < u,
 *          summed over the entries of that row in entry order within fixed
 *          chunks of 64 sorted entries, the chunk sums then added in order
 *          (deterministic); rows i >= u are not written;
 *   count  int32[2]: count[0] = u (active rows), count[1] = entries dropped
 *          because idx is outside [0, vocab) or feat outside [0, m).
 */

/* Workspace (bytes) of shampoo_embedding_rows and shampoo_embedding_stats
 * for nnz entries of width dim; 0 on invalid arguments (nnz outside
 * [1, 2^26], dim outside [1, 4096]). */
size_t shampoo_embedding_workspace_bytes(int nnz, int dim);

/*
 * Compacts the lookup gradient.  idx: nnz rows; feat: nnz output rows, or
 * NULL for feat[e] = e (one entry per output row, m >= nnz); weight: nnz
 * weights, or NULL for 1 (one-hot); dy: m x dim, row stride ld_dy.  All
 * device pointers.  rows, U, count: outputs as above.  Sorting uses a stable
 * device radix sort whose temporary storage the handle allocates and keeps.
 * Errors: EINVAL (NULL pointers, nnz or dim out of range, vocab outside
 * [1, 2^31 - 1), m < 1, ld_dy < dim), ENOMEM (workspace too small).
 */
shampoo_status shampoo_embedding_rows(void* handle, const int32_t* idx, const int32_t* feat, const float* weight,
                                      int nnz, int64_t vocab, const float* dy, int m, int dim, int64_t ld_dy,
                                      int32_t* rows, float* U, int32_t* count, void* workspace, size_t ws_bytes,
                                      void* stream);

/*
 * R = beta2 R + c U^T U over the first count[0] rows of U (c = 1 if
 * beta2 == 1 else 1 - beta2): the statistic of the table, dim x dim, kept
 * exactly symmetric (and required symmetric on entry, as for
 * shampoo_update_stats).  The active rows are split into a fixed number of
 * equal parts (set from nnz and dim); their partial products are added in
 * part order (deterministic).
 * Errors: EINVAL (NULL pointers, sizes, beta2 outside (0, 1]), ENOMEM.
 */
shampoo_status shampoo_embedding_stats(void* handle, const float* U, const int32_t* count, int nnz, int dim,
                                       float* R, float beta2, void* workspace, size_t ws_bytes, void* stream);

/*
 * P = U Rr for the first count[0] rows (Rr symmetric, dim x dim): the
 * preconditioned compact gradient G R^(-1/2) of Lemma 1's one-sided form.
 * Rows of P at or past count[0] are not written.  Errors: EINVAL.
 */
shampoo_status shampoo_embedding_precondition(void* handle, const float* U, const int32_t* count, int nnz, int dim,
                                              const float* Rr, float* P, void* stream);

/*
 * Grafted update of the active rows (beta1 = 0 form of shampoo_graft): for
 * i < count[0] and r = rows[i],
 *   D[r] += U[i] o U[i];  eta = eta0 ||D^(-1/2) o G||_F / ||P||_F  (norms over
 *   the active rows, which are all of G's nonzeros);  W[r] -= eta P[i]
 * (use_shampoo = 0: W[r] -= eta0 D[r]^(-1/2) o U[i]).  Rows of W and D that
 * no entry touched are left exactly as they were.  norms (device, may be
 * NULL): {||D^(-1/2) o G||_F, ||P||_F, eta}.
 * Errors: EINVAL (NULL pointers, sizes, ldw < dim, non-finite eta0).
 */
shampoo_status shampoo_embedding_graft(void* handle, const int32_t* rows, const int32_t* count, int nnz, int dim,
                                       const float* U, const float* P, float* W, float* D, int64_t vocab,
                                       int64_t ldw, float eta0, int use_shampoo, float* norms, void* stream);

/*
 * From the loss to the gradient.  The calls below compute what a training
 * step has in hand before shampoo_update_stats: the loss at the output layer
 * and its gradient, 8-bit checkpoints of activations, and the weight gradient
 * G that the calls above take.  They use no handle scratch: two calls of one
 * handle may overlap on different streams if their buffers differ.
 */

/*
 * Log probabilities of given tokens.  z = row r of the logits (rows x vocab,
 * row stride ld >= vocab, element type dtype, SHAMPOO_F32 or SHAMPOO_BF16):
 *   lse[r]     = log sum_j exp(z_j)
 *   logp[r]    = z_t - lse[r], t = targets[r]; 0 when t is outside [0, vocab)
 *                (a token without loss)
 *   entropy[r] = -sum_j p_j log p_j,  p_j = exp(z_j - lse[r])
 *   top_ids, top_logp (rows x k, contiguous): the k largest logits in
 *                descending order, equal ones by ascending index, and
 *                z_j - lse[r]; -1 and -inf past the last entry above -inf
 * Sums are kept in fp32.  An entry of -inf is not allowed: it has probability
 * 0 and is never an alternative.  A row of -inf only has lse = -inf, logp =
 * -inf (0 without a target), entropy 0 and no alternatives; a row holding a
 * NaN or +inf has lse, entropy, top_logp and (with a target) logp NaN, and
 * top_ids -1.  logp and targets may both be NULL, entropy may be NULL, and
 * top_ids and top_logp are NULL when k == 0.
 * `workspace` is device memory of at least
 * shampoo_token_logprobs_workspace_bytes(rows, vocab, k) bytes (0 when the
 * call needs none), used exclusively by this call until the stream reaches
 * its end.  rows == 0 does nothing.
 * Errors: EINVAL (NULL pointers, rows outside [0, 2^31), vocab outside
 * [1, 2^30], ld < vocab, k outside [0, SHAMPOO_MAX_TOP], dtype, a workspace that
 * overlaps the logits), ENOMEM (workspace too small).
 */
#define SHAMPOO_MAX_TOP 64
size_t shampoo_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int k);
shampoo_status shampoo_token_logprobs(void* handle, const void* logits, int dtype, int64_t rows, int64_t vocab,
                                      int64_t ld, const int32_t* targets, float* logp, float* lse, float* entropy,
                                      int k, int32_t* top_ids, float* top_logp, void* workspace, size_t ws_bytes,
                                      void* stream);

/*
 * The gradient of shampoo_token_logprobs with respect to the logits.  Given
 * the gradients of its outputs (g_logp, g_lse, g_entropy: rows; g_top: rows x
 * k; each may be NULL for zero),
 *   dz_j = p_j (g_lse - g_logp - sum_i g_top_i - g_entropy (log p_j + H))
 *          + [j = t] g_logp + sum_i [j = top_ids_i] g_top_i,
 * with p_j = exp(z_j - lse[r]) and H = entropy[r] (needed with g_entropy).  A
 * target outside [0, vocab) has no g_logp, an alternative outside it no g_top.
 * Rows with lse = -inf have gradient 0.  dlogits has the logits' element type
 * (rounded once, to nearest even) and row stride ld_d >= vocab; it may be the
 * logits themselves (same pointer, ld_d == ld), else it shares no element with
 * them.  Deterministic.
 * Errors: EINVAL (NULL logits, lse or dlogits; targets NULL with g_logp,
 * entropy NULL with g_entropy, top_ids NULL with g_top; sizes and dtype as
 * above; dlogits == logits with ld_d != ld, or overlapping them otherwise).
 */
shampoo_status shampoo_token_logprobs_grad(void* handle, const void* logits, int dtype, int64_t rows, int64_t vocab,
                                           int64_t ld, const int32_t* targets, const float* lse,
                                           const float* entropy, int k, const int32_t* top_ids,
                                           const float* g_logp, const float* g_lse, const float* g_entropy,
                                           const float* g_top, void* dlogits, int64_t ld_d, void* stream);

/*
 * Activation checkpoints in 8 bits.  A checkpoint holds a rows x cols tensor
 * as signed 8-bit codes with one power-of-two scale for every 32 columns of a
 * row (the last group of a row may be shorter):
 *   x^ = q 2^e,  |q| <= 127,  e the smallest exponent in [-126, 121] for which
 *   the group's largest |x| 2^-e rounds to at most 127,  q = x 2^-e rounded to
 *   nearest even
 * (|x - x^| <= 2^(e-1): for e > -126 at most 1/127 of the group's largest |x|,
 * for e = -126 multiples of 2^-126, a group up to 2^-127 becoming 0; values from
 * 127.5 2^121 on, which would round to 2^128, are held as 127 2^121).  x^ is exact
 * in bfloat16.  A group that holds an infinity or NaN is NaN throughout.
 * Layout, one buffer of shampoo_act_checkpoint_bytes(rows, cols) bytes aligned
 * to 16: with ldq = cols rounded up to 32, rows x ldq codes (0 in the
 * columns at and past cols); then, at the next multiple of 256 bytes, rows x
 * (ldq / 32) bytes s = e + 127 (255 and codes 0 for a NaN group).
 * Sizes: rows in [0, 2^31), cols in [1, 2^20]; row strides >= cols.
 * rows == 0 does nothing (the weight gradient then is beta G).
 */
enum {
  SHAMPOO_ACT_NONE = 0,      /* y = x */
  SHAMPOO_ACT_RELU = 1,      /* y = max(x, 0); slope 0 at 0 */
  SHAMPOO_ACT_GELU = 2,      /* y = x (1 + erf(x / sqrt 2)) / 2 */
  SHAMPOO_ACT_GELU_TANH = 3, /* y = x (1 + tanh(sqrt(2 / pi) (x + 0.044715 x^3))) / 2 */
  SHAMPOO_ACT_SILU = 4       /* y = x / (1 + exp(-x)) */
};
size_t shampoo_act_checkpoint_bytes(int64_t rows, int64_t cols);

/*
 * One pass over X (rows x cols, row stride ld_x, dtype): Y = act(X) (same
 * type, row stride ld_y; NULL: not wanted), the checkpoint of X (ckpt_x) and
 * the checkpoint of Y as stored (ckpt_y); each may be NULL, not all three.
 * Y may be X itself (ld_y == ld_x); otherwise tensors and checkpoints of a call
 * share no memory (column ranges of one wider buffer do not).
 * Errors: EINVAL (NULL X, no output, sizes, strides, dtype, act, a checkpoint
 * not aligned to 16 bytes, overlapping buffers).
 */
shampoo_status shampoo_act_encode(void* handle, const void* X, int dtype, int64_t rows, int64_t cols, int64_t ld_x,
                                  int act, void* Y, int64_t ld_y, void* ckpt_x, void* ckpt_y, void* stream);

/* X = the values x^ of a checkpoint (dtype; exact).  Errors: as above. */
shampoo_status shampoo_act_decode(void* handle, const void* ckpt, int64_t rows, int64_t cols, void* X, int dtype,
                                  int64_t ld_x, void* stream);

/*
 * Activation gradient dX = dY o act'(x^) from the checkpoint of the
 * activation's input.  dY and dX: dtype, row strides ld_dy and ld_dx; dX may
 * be dY itself (ld_dx == ld_dy).  Errors: as above.
 */
shampoo_status shampoo_act_grad(void* handle, const void* ckpt, int64_t rows, int64_t cols, int act, const void* dY,
                                int dtype, int64_t ld_dy, void* dX, int64_t ld_dx, void* stream);

/*
 * Weight gradient of a linear layer Y = X W from the checkpoint of its input:
 *   G = beta G + X^^T dY     (cols x out, row stride ld_g; G is not read when
 *                             beta == 0)
 * dY: rows x out, row stride ld_dy, dtype; G: g_dtype (either type; rounded
 * once at the end).  Products of x^ with bfloat16 gradients are exact and
 * summed in fp32; fp32 gradients are split into three bfloat16 terms, exactly
 * from 2^-110 in size on (below, what lies under 2^-133 is cut off).
 * Long sums over few output tiles are cut into parts that are added in a fixed
 * order (deterministic).  `workspace`: at least
 * shampoo_act_weight_grad_workspace_bytes(rows, cols, out) bytes of device
 * memory (0: none needed), as for shampoo_token_logprobs.
 * Sizes: out in [1, 2^20].  Errors: as above, EINVAL for a non-finite beta or
 * G or the workspace overlapping another buffer, ENOMEM (workspace too small).
 */
size_t shampoo_act_weight_grad_workspace_bytes(int64_t rows, int64_t cols, int64_t out);
shampoo_status shampoo_act_weight_grad(void* handle, const void* ckpt, int64_t rows, int64_t cols, const void* dY,
                                       int dtype, int64_t out, int64_t ld_dy, void* G, int g_dtype, int64_t ld_g,
                                       float beta, void* workspace, size_t ws_bytes, void* stream);

/*
 * The layers around the step.  A model's output layer without its logits, a gated
 * feed-forward block, and dropout, with their gradients: the dW that these calls
 * write are the gradients that shampoo_update_stats and shampoo_precondition take.
 * They use no handle scratch: two calls of one handle may overlap on different
 * streams if their buffers differ.  `workspace`: at least the stated bytes of device
 * memory (0: none needed), aligned to 16, used exclusively by the call until the
 * stream reaches its end.  Matrices are row-major with any row stride of at least
 * their columns and any alignment to their element; bf16 ones whose address is a
 * multiple of 16 bytes and whose columns and stride are multiples of 8 are read as
 * they lie, others are copied into the workspace first (tables and weights of calls of
 * few rows are not: another kernel, with another order of the sums).  Products of bf16 values
 * are exact; fp32 values are split into three bf16 terms, exactly from 2^-110 in size on
 * (below, what lies under 2^-133 is cut off), of whose nine products the six largest
 * are formed.  Sums are kept in fp32, in a fixed order: results repeat to the bit.  A
 * NaN spreads as in the formulas; an infinity (in fp32 also a value from 2^128 - 2^119
 * on) gives an infinity or a NaN where its products reach.
 */

/*
 * Log probabilities of given tokens from the last activations: z = X W^T (X: rows x
 * dim, W: vocab x dim, both dtype), z not kept,
 *   lse[r]  = log sum_j exp(z_rj)
 *   logp[r] = z_rt - lse[r], t = targets[r]; 0 when t is outside [0, vocab) (a token
 *             without loss)
 * logp and targets may both be NULL.  z is not rounded to dtype.  logp is never above 0.
 * rows == 0 does nothing.
 * Errors: EINVAL (NULL pointers, rows outside [0, 2^31), dim outside [1, 2^20],
 * vocab outside [1, 2^30], strides, dtype, a workspace not aligned to 16, outputs or
 * workspace that overlap another buffer), ENOMEM (workspace too small), EUNSUPPORTED
 * (a product of 2^22 tiles or more).
 */
size_t shampoo_vocab_logprobs_workspace_bytes(int64_t rows, int64_t dim, int64_t vocab, int dtype);
shampoo_status shampoo_vocab_logprobs(void* handle, const void* X, const void* W, int dtype, int64_t rows, int64_t dim,
                                      int64_t vocab, int64_t ld_x, int64_t ld_w, const int32_t* targets, float* logp,
                                      float* lse, void* workspace, size_t ws_bytes, void* stream);

/*
 * Its gradient.  Given lse and the gradients of the outputs (g_logp with targets, g_lse;
 * fp32, rows; each may be NULL for zero),
 *   dz_rj = (g_lse - g_logp) exp(z_rj - lse) + [j = t] g_logp   (no g_logp without a target)
 *   dX = dz W             (rows x dim, dtype)
 *   dW = beta dW + dz^T X (vocab x dim, g_dtype; not read when beta == 0)
 * dX or dW may be NULL.  The logits are formed again, in pieces of the vocabulary.
 * dz is kept in three bf16 terms (24 bits) where dtype or g_dtype is fp32 (a bf16 dX
 * takes two of them, 16 bits), else of up to 32 rows in two, of more in one (8 bits, as a
 * stored bf16 gradient of logits).
 * g_dtype counts without dW too.  The order of dX's sums may differ between calls with dW
 * and without.  A row whose gradients are all 0 has dz = 0 whatever W and lse hold, and
 * adds nothing to dW if X is finite there.  rows == 0: dW = beta dW.
 * Errors: as above, EINVAL for a non-finite beta, g_logp without targets, or neither dX nor
 * dW.
 */
size_t shampoo_vocab_logprobs_grad_workspace_bytes(int64_t rows, int64_t dim, int64_t vocab, int dtype, int g_dtype);
shampoo_status shampoo_vocab_logprobs_grad(void* handle, const void* X, const void* W, int dtype, int64_t rows,
                                           int64_t dim, int64_t vocab, int64_t ld_x, int64_t ld_w,
                                           const int32_t* targets, const float* lse, const float* g_logp,
                                           const float* g_lse, void* dX, int64_t ld_dx, void* dW, int g_dtype,
                                           int64_t ld_dw, float beta, void* workspace, size_t ws_bytes, void* stream);

/*
 * Gated feed-forward block: G = X Wg, U = X Wu (X: rows x dim, Wg and Wu: dim x width),
 *   H = act(G) o U   (act: SHAMPOO_ACT_*, of the sums before they are rounded)
 * G and U are written too unless both are NULL.  X, weights and outputs: dtype.
 * rows == 0 does nothing.  Sizes: dim in [1, 2^20], width in [1, 2^19].
 * Errors: as above, EINVAL for a bad act or only one of G and U.
 */
size_t shampoo_gated_ffn_workspace_bytes(int64_t rows, int64_t dim, int64_t width, int dtype);
shampoo_status shampoo_gated_ffn(void* handle, const void* X, const void* Wg, const void* Wu, int dtype, int64_t rows,
                                 int64_t dim, int64_t width, int64_t ld_x, int64_t ld_wg, int64_t ld_wu, int act,
                                 void* H, int64_t ld_h, void* G, int64_t ld_g, void* U, int64_t ld_u, void* workspace,
                                 size_t ws_bytes, void* stream);

/*
 * Its gradients from dH (rows x width, dtype), with G and U as they were kept, or both
 * NULL: then the projections are formed again and not rounded.
 *   dG = dH o U o act'(G), dU = dH o act(G)
 *   dX = dG Wg^T + dU Wu^T          (rows x dim, dtype)
 *   dWg = beta dWg + X^T dG, dWu = beta dWu + X^T dU   (dim x width, g_dtype; not read
 *                                                       when beta == 0)
 * dX may be NULL, or dWg and dWu; what is said of dz and of the order of dX's sums above
 * holds here of dG and dU.
 * rows == 0: dWg = beta dWg, dWu = beta dWu.
 * Errors: as above, EINVAL for only one of G and U or of dWg and dWu, or no output.
 */
size_t shampoo_gated_ffn_grad_workspace_bytes(int64_t rows, int64_t dim, int64_t width, int dtype, int g_dtype);
shampoo_status shampoo_gated_ffn_grad(void* handle, const void* X, const void* Wg, const void* Wu, int dtype,
                                      int64_t rows, int64_t dim, int64_t width, int64_t ld_x, int64_t ld_wg,
                                      int64_t ld_wu, int act, const void* dH, int64_t ld_dh, const void* G,
                                      int64_t ld_g, const void* U, int64_t ld_u, void* dX, int64_t ld_dx, void* dWg,
                                      int64_t ld_dwg, void* dWu, int64_t ld_dwu, int g_dtype, float beta,
                                      void* workspace, size_t ws_bytes, void* stream);

/*
 * Dropout: Y = R + [kept] X 65536 / (65536 - n), n = rate 65536 rounded to nearest even; R
 * may be NULL (zero), Y may be X or R (same row stride).  n = 65536 keeps nothing.  The mask
 * is that of a counter-based generator, never stored: Philox 4x32 with 10 rounds (Salmon,
 * Moraes, Dror and Shaw 2011), key = seed (low word, high word), counter = (column / 8,
 * row, offset low, offset high); of the 128 bits, 16-bit half column % 8 (low halves of
 * the words first) decides: kept if it is at least n.  The gradient with respect to X is
 * the same call on dY with R NULL.  What is not kept leaves no trace, NaN included.
 * Calls whose masks must differ take another seed or offset (one offset covers any
 * tensor).  Sizes: rows in [0, 2^31), cols in [1, 2^20].
 * Errors: EINVAL (NULL X or Y, sizes, strides, dtype, rate outside [0, 1], Y overlapping X
 * or R without being the same).
 */
shampoo_status shampoo_dropout(void* handle, const void* X, const void* R, void* Y, int dtype, int64_t rows,
                               int64_t cols, int64_t ld_x, int64_t ld_r, int64_t ld_y, double rate, uint64_t seed,
                               uint64_t offset, void* stream);

/*
 * Measurement support.  While enabled, every launch of the timed kernel
 * classes below is bracketed by HIP events on its stream.
 * shampoo_timing_read synchronizes those events, returns the summed duration
 * (ms) and launch count of one class, and clears that class.
 */
enum {
  SHAMPOO_KCLASS_NEWTON_F32 = 0, /* grouped Newton products, fp32 */
  SHAMPOO_KCLASS_NEWTON_F64 = 1, /* grouped Newton products, fp64 */
  SHAMPOO_KCLASS_STATS = 2,      /* grouped statistics SYRK */
  SHAMPOO_KCLASS_PRECOND = 3,    /* grouped preconditioning GEMMs */
  SHAMPOO_KCLASS_GRAFT = 4,      /* graft reduction and update passes */
  SHAMPOO_KCLASS_ROOT_AUX = 5,   /* root prologue/epilogue/state kernels */
  SHAMPOO_KCLASS_EMB = 6,        /* embedding row compaction (sort, runs, segment sums) */
  SHAMPOO_KCLASS_NEWTON_WARM = 7, /* full products of warm-started roots (fp32 or fp64) */
  SHAMPOO_KCLASS_LOGPROBS = 8,   /* token log probabilities and their gradient */
  SHAMPOO_KCLASS_ACT = 9,        /* activation checkpoints: encode, decode, activation gradient */
  SHAMPOO_KCLASS_WGRAD = 10,     /* weight gradients from checkpoints */
  SHAMPOO_KCLASS_VOCAB = 11,     /* loss from the last activations and its gradient */
  SHAMPOO_KCLASS_FFN = 12,       /* gated feed-forward block and its gradient */
  SHAMPOO_KCLASS_DROPOUT = 13,   /* dropout */
  SHAMPOO_KCLASS_COUNT = 14
};
shampoo_status shampoo_timing_enable(void* handle, int enable);
shampoo_status shampoo_timing_read(void* handle, int kclass, double* total_ms, int64_t* launches);

#ifdef __cplusplus
}
#endif
#endif /* SHAMPOO_MI355X_H */
