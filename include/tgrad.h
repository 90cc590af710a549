/*
 * tgrad.h -- C ABI of the B200 (sm_100a) TensorGRaD optimizer-step library.
 *
 * One state object per complex weight tensor W in C^{I_1 x ... x I_N}.  A step
 * is Algorithm 1 of the paper ("Adam with Sparse and Low-Rank Gradient
 * Compression"): the gradient is split into an unstructured sparse part
 * (magnitude top-k index set Omega, Section 2.2 "Unstructured sparse gradient
 * tensor") and a low-rank Tucker part (factor matrices U^(n), Section 2.2
 * "Low-rank gradient tensor decomposition"); Adam runs on the k sparse values
 * and on the Tucker core; the core is expanded back through the U^(n), the
 * sparse update is scatter-added, and W is updated in place.
 *
 * Conventions
 *  - All tensors are dense, row-major (last index fastest).  TGRAD_C64 stores
 *    each entry as two fp32 (re, im); TGRAD_C32H as two IEEE fp16 (re, im) and
 *    TGRAD_C32B as two bfloat16 (the paper's mixed-precision recipe, Section 2.3:
 *    weights and gradients in half precision, every optimizer state in fp32; the
 *    paper does not name the 16-bit format).
 *  - The caller passes grad = d(phi)/dW.  Algorithm 1 is written for
 *    G = -grad and W <- W + eta*Gtilde(G); the library evaluates the same
 *    stages on grad and subtracts, which is bit-identical.
 *  - Pointers named d_* are DEVICE pointers, everything else is host memory.
 *  - The library never allocates or frees device memory and, but for the
 *    side streams of tgrad_step_batched and the one a refresh uses (below),
 *    never creates streams.  The caller owns: the weight, the gradient, one persistent
 *    block (Omega, U^(n), moments, status words, a split copy of U^(N-1)
 *    laid out for the compression kernel) and one workspace block
 *    (scratch; contents need not survive between calls, but the same
 *    workspace must not be used by two states concurrently).  Sizes come
 *    from tgrad_state_bytes().  Both blocks must be 256-byte aligned.
 *  - All device work is enqueued asynchronously on the given stream
 *    (a cudaStream_t passed as void*; NULL = the legacy default stream).
 *  - Argument errors are detected on the host before anything is enqueued and
 *    leave every buffer untouched.  Conditions found on the device (Jacobi
 *    sweep cap reached, non-finite gradient seen by the selection) set sticky
 *    bits that tgrad_query_status() reads.  Nothing aborts or traps.
 *  - A state is not thread-safe; distinct states may be used from distinct
 *    threads.
 */
#ifndef TGRAD_H_
#define TGRAD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tgrad_state tgrad_state;   /* opaque host handle; owns no device memory */

typedef enum {
  TGRAD_OK = 0,
  TGRAD_ERR_INVALID_ARG = 1,
  TGRAD_ERR_UNSUPPORTED = 2,
  TGRAD_ERR_BUFFER_TOO_SMALL = 3,
  TGRAD_ERR_CUDA = 4,
  TGRAD_ERR_NO_CONVERGE = 5,
  TGRAD_ERR_NONFINITE = 6,
  TGRAD_ERR_BAD_STATE = 7,
  TGRAD_ERR_TOO_LARGE = 8      /* tgrad_select_topk_noalloc: more entries than its built-in scratch covers */
} tgrad_status;

/* sticky device flags reported by tgrad_query_status() */
#define TGRAD_FLAG_NO_CONVERGE 1   /* the Jacobi eigensolver hit jacobi_max_sweeps */
#define TGRAD_FLAG_NONFINITE   2   /* a NaN/Inf magnitude was seen while selecting Omega */
#define TGRAD_FLAG_COPY_TIMEOUT 4  /* a streaming kernel gave up waiting for one of its own asynchronous copies
                                      (every device-side wait is bounded); the blocks that saw it returned early,
                                      so W and the moments of that step are undefined.  Not expected in normal
                                      operation; treat the state as lost */

typedef enum {
  TGRAD_C64 = 0,   /* interleaved 2 x fp32 */
  TGRAD_C32H = 1,  /* interleaved 2 x IEEE fp16 */
  TGRAD_C32B = 2,  /* interleaved 2 x bfloat16 (general kernels only: no fp16 tensor-core fast path) */
  TGRAD_R32 = 3,   /* fp32; the real types are for the dense tensors and logits of the calls at the end of this file, */
  TGRAD_R16H = 4,  /* IEEE fp16                                            not for the weight of a tgrad_state        */
  TGRAD_R16B = 5   /* bfloat16 */
} tgrad_dtype;

#define TGRAD_MAX_NDIM 8

/* Hyper-parameters of Algorithm 1 (its "Require" line) plus storage options. */
typedef struct {
  int32_t ndim;                     /* N, 2 <= ndim <= TGRAD_MAX_NDIM (N = 2: the matrix case,  */
                                    /* where the Tucker factors are the singular subspaces)     */
  int64_t dims[TGRAD_MAX_NDIM];     /* I_1..I_N, row-major; prod(dims) < 2^32                   */
  int32_t ranks[TGRAD_MAX_NDIM];    /* Tucker ranks, 1 <= r_n <= I_n                            */
  int64_t k;                        /* |Omega| = ceil(rho*I), computed exactly by the caller;   */
                                    /* k < 2^31                                                 */
  int32_t T;                        /* subspace change frequency, >= 1                          */
  float lr;                         /* eta                                                      */
  float alpha;                      /* scale of the reconstructed low-rank update               */
  float lambda;                     /* scale of the sparse update                               */
  float beta1, beta2, eps;          /* Adam decay rates and epsilon                             */
  float weight_decay;               /* decoupled decay W <- (1 - eta*wd) W before the update    */
  int32_t wg_dtype;                 /* tgrad_dtype of W and grad; all states are fp32           */
  int32_t auto_refresh;             /* 1: tgrad_step refreshes Omega and U^(n) when t % T == 0  */
  int32_t jacobi_max_sweeps;        /* sweep cap of the eigensolver (0 -> default 30)           */
  float jacobi_tol;                 /* off-diagonal tolerance relative to max diag (0 -> 1e-6)  */
  int32_t warm_refresh;             /* 1: a refresh starts its eigenvector iteration from the factor matrices
                                       the state holds (the paper's "warm restart" of the factors, appendix
                                       "Tensor Decomposition / Implementation") instead of a fixed pseudo-random
                                       start; if the subspace moved little this saves iterations, and the result
                                       is the same eigen-decomposition to the same tolerance.  Stored factors
                                       that are unusable (never set, not finite) are noticed on the device and
                                       that refresh starts cold.  0: every refresh starts cold               */
  int32_t hooi_iters;               /* refinement sweeps of TuckerFactors after the truncated-SVD factors (higher-
                                       order orthogonal iteration, the paper's appendix "Tensor Decomposition /
                                       Implementation"): per sweep and mode, the residual is compressed in every
                                       other mode with the current factors and U^(n) becomes the leading left
                                       singular vectors of the result.  0: none.  With warm_refresh = 1 and
                                       factors in the state, the sweeps start from those factors and the
                                       truncated-SVD stage is skipped (the warm restart of the decomposition).
                                       Needs extra workspace, and each trailing slab must still fit in shared
                                       memory with one of its two factors replaced by the identity            */
  int32_t composition;              /* order of the two parts (Section 2.2 "Residual and composition"):
                                       0: sparse part first, low-rank part on its residual (Algorithm 1);
                                       1: low-rank part first, the sparse part selected from and fed with
                                          G - P_U(G), P_U(G) the low-rank approximation of the gradient;
                                       2: both parts applied to the gradient itself and added                 */
  int32_t sparse_strategy;          /* how Omega is chosen at a refresh (Section 2.2 "Unstructured sparse gradient
                                       tensor"): 0 top-k magnitude; 1 uniform random k-subset; 2 sampling without
                                       replacement with probabilities proportional to |g|.  1 and 2 rank the
                                       entries by a key built from one Philox-4x32-10 word per entry (counter =
                                       flat index, refresh number t / T) and take the k largest                */
  uint64_t seed;                    /* key of that generator                                                   */
} tgrad_config;

/* Selectors for tgrad_export_state / tgrad_import_state.  FACTOR_BASE + n is
 * U^(n+1), an I_n x r_n row-major complex64 matrix. */
enum {
  TGRAD_WHAT_OMEGA = 1,        /* k x uint32, strictly ascending flat indices */
  TGRAD_WHAT_M_L = 2,          /* prod(r_n) x complex64, row-major core order */
  TGRAD_WHAT_V_L = 3,          /* prod(r_n) x fp32                            */
  TGRAD_WHAT_M_S = 4,          /* k x complex64, slot j <-> Omega[j]          */
  TGRAD_WHAT_V_S = 5,          /* k x fp32                                    */
  TGRAD_WHAT_CORE = 6,         /* last step's compressed gradient (export only; workspace) */
  TGRAD_WHAT_N_L = 7,          /* last step's normalised core update (export only)         */
  TGRAD_WHAT_N_S = 8,          /* last step's normalised sparse update (export only)       */
  TGRAD_WHAT_GRAM_BASE = 32,   /* + n: the Gram matrix the last refresh took U^(n+1) from, I_n x I_n complex64 (export
                                  only): A_n = R_(n) R_(n)^H, or with refinement sweeps that of the residual
                                  compressed in every other mode */
  TGRAD_WHAT_FACTOR_BASE = 64  /* + n */
};

/* Sizes of the two caller-owned device blocks for a configuration.
 * Counts follow the state inventory of Algorithm 1 (its initialisation
 * statements) and of the appendix "Parameter Complexity Analysis":
 * prod(r_n) core-shaped entries for each low-rank moment, sum I_n r_n factor
 * entries, k indices and k entries for each sparse moment.
 * The sizes do not depend on the device the state will run on.
 *
 * Limits of this implementation; a configuration outside them returns
 * TGRAD_ERR_UNSUPPORTED here and from tgrad_init_state:
 *   prod(dims) < 2^32 (flat indices are uint32) and k < 2^31;
 *   every I_n <= 1024 (size of the on-device eigensolver);
 *   r_N <= 32 (rank of the last mode);
 *   one trailing slab of I_{N-1} x I_N entries, with the operand tables of
 *   its two mode products, must fit in the 227 KB of shared memory of one SM
 *   (roughly I_{N-1} * (I_N + r_N) complex64 entries <= 28,000). */
tgrad_status tgrad_state_bytes(const tgrad_config* cfg, size_t* persistent_bytes, size_t* workspace_bytes);

/* Algorithm 1 initialisation: t <- 0, M_L, V_L, M_S, V_S <- 0 (enqueued on
 * the stream).  Omega and U^(n) are undefined until the first refresh.
 * Returns a host handle in *out that refers to, but does not own, the two
 * device blocks. */
tgrad_status tgrad_init_state(const tgrad_config* cfg, void* d_persistent, size_t persistent_bytes,
                              void* d_workspace, size_t workspace_bytes, void* cuda_stream, tgrad_state** out);

/* One pass of the loop body of Algorithm 1 for one tensor: (refresh if
 * auto_refresh and t mod T == 0), sparse gather, residual, Tucker compression
 * (chained mode-n products with U^(n)H, Section 2.2), AdamUpdate on the sparse
 * values and on the core, reconstruction scaled by alpha, scaled sparse add,
 * W <- W - eta*Gtilde, t <- t+1.
 * d_weight: in/out, prod(dims) entries of wg_dtype.  d_grad: input of the same
 * shape and dtype; it is restored to its input value before the call's work
 * completes, but is written temporarily during a refresh.
 * Returns TGRAD_ERR_BAD_STATE if no refresh has happened yet and auto_refresh
 * is 0. */
tgrad_status tgrad_step(tgrad_state* st, void* d_weight, void* d_grad, void* cuda_stream);

/* tgrad_step with the gradient multiplied by the device scalar *d_scale (NULL: 1), which the call's kernels read when
 * they run: a clipping coefficient that an earlier call on the stream computes (tgrad_grad_norm) is applied without a
 * pass over the gradient and without the host knowing it.  The compression is linear, so the factor is applied to the
 * Tucker core and to the sparse values where Adam reads them; the selection of Omega and the factor matrices do not
 * depend on a positive factor and are taken from the gradient as it is.  tgrad_export_state's CORE is that of the
 * gradient as it is. */
tgrad_status tgrad_step_scaled(tgrad_state* st, void* d_weight, void* d_grad, const float* d_scale, void* cuda_stream);

/* The `t mod T = 0` branch of Algorithm 1 on the supplied gradient:
 * Omega <- magnitude top-k of grad (key = fp32 re*re + im*im without fused
 * multiply-add, ties to the lower flat index, stored ascending);
 * R <- grad with Omega zeroed; U^(n) <- eigenvectors of the r_n largest
 * eigenvalues of R_(n) R_(n)^H (Jacobi), descending, each column scaled by the
 * unit phase that makes its largest-modulus component real positive.
 * Moments are not touched.  d_grad is modified while the call's work runs and
 * restored at its end.
 * Part of a refresh (the eigenvectors of the leading modes, while the Gram
 * matrices of the trailing modes are accumulated) runs on one side stream per
 * device, created at the first refresh on that device and kept for the life of
 * the process.  It is forked from and joined back into the caller's stream with
 * events: work enqueued on that stream before the call happens before all of
 * the refresh, work enqueued after it happens after all of it.  If the stream
 * cannot be created everything runs on the caller's stream.  The same holds
 * for a refresh that tgrad_step runs by itself. */
tgrad_status tgrad_refresh_subspace(tgrad_state* st, void* d_grad, void* cuda_stream);

/* Batched variants over a list of layers: semantically n independent calls
 * (the tensors of an FNO's spectral layers are independent).  Arrays are HOST
 * arrays of handles / device pointers.
 * tgrad_step_batched and tgrad_refresh_subspace_batched run the tensors' kernel chains side by side: they fork
 * them onto up to four streams that the library creates per device at the
 * first batched call (an exception to "creates no streams") and join
 * them back into the given stream, so for the caller the call orders like
 * any other work on that stream.  The states must have distinct workspaces,
 * and d_weights / d_grads must not overlap between tensors. */
tgrad_status tgrad_step_batched(tgrad_state* const* states, void* const* d_weights, void* const* d_grads,
                                int32_t n_tensors, void* cuda_stream);
/* the same with one scale for all gradients, as in tgrad_step_scaled */
tgrad_status tgrad_step_batched_scaled(tgrad_state* const* states, void* const* d_weights, void* const* d_grads,
                                       int32_t n_tensors, const float* d_scale, void* cuda_stream);
tgrad_status tgrad_refresh_subspace_batched(tgrad_state* const* states, void* const* d_grads, int32_t n_tensors,
                                            void* cuda_stream);

/* Synchronises the stream, then reports the sticky flags (TGRAD_FLAG_*), the
 * step counter t and the number of Jacobi sweeps the last refresh used per
 * mode (sweeps may be NULL; otherwise ndim int32). */
tgrad_status tgrad_query_status(tgrad_state* st, void* cuda_stream, int32_t* sticky_flags, int64_t* t,
                                int32_t* sweeps);

/* Checkpoint / inspection: copy one state component to or from HOST memory.
 * `bytes` must equal the component's size exactly.  Both calls synchronise the
 * stream.  tgrad_set_step sets the counter t (host side). */
tgrad_status tgrad_export_state(tgrad_state* st, int32_t what, void* host_dst, size_t bytes, void* cuda_stream);
tgrad_status tgrad_import_state(tgrad_state* st, int32_t what, const void* host_src, size_t bytes,
                                void* cuda_stream);
tgrad_status tgrad_set_step(tgrad_state* st, int64_t t);

/* Optional diagnostics of the last step, not part of the timed path (synchronises the stream).  d_grad must be the
 * gradient that step was given.  out[0] = ||G||_F;  out[1] = ||G_S||_F / ||G||_F, the share of the gradient the
 * sparse part took;  out[2] = || X - P_U X ||_F / ||G||_F, the part the low-rank compression lost, X being what the
 * low-rank part was given (the residual of the sparse part in Algorithm 1's order, the gradient otherwise) -- with
 * orthonormal factors this is sqrt(||X||^2 - ||core||^2), the reconstruction error Section 2.2 reports for its
 * decompositions;  out[3] = max over modes and entries of |U^(n)H U^(n) - I|.
 * TGRAD_ERR_BAD_STATE before the first step. */
tgrad_status tgrad_diagnostics(tgrad_state* st, const void* d_grad, void* cuda_stream, double* out);

/* Frees the host handle only. */
tgrad_status tgrad_destroy_state(tgrad_state* st);

const char* tgrad_status_string(tgrad_status s);

/* Magnitude top-k selection for callers that cannot allocate device memory.
 * (The paper has no counterpart of this call; it computes the same Omega as
 * the refresh, "Unstructured sparse gradient tensor" with the top-k strategy.)
 *
 * Who needs it: code that runs where cudaMalloc is off limits -- inside a
 * framework's allocator callback or memory-pool hook (allocating there
 * re-enters the allocator), in a process whose device memory was handed out
 * in full at start-up, or in a latency-critical loop that must not take the
 * driver's allocation lock.  The other entry points need a workspace block
 * that somebody allocated; this one needs none.
 *
 * The scratch of the selection (radix histograms, threshold state, per-block
 * counts) lives in a fixed array inside the library's device image, about
 * 290 KB, which every GPU that loads the library holds until the process
 * exits.  That fixes the largest input: numel <= TGRAD_NOALLOC_MAX_NUMEL,
 * otherwise TGRAD_ERR_TOO_LARGE and nothing is enqueued.
 *
 * d_grad, d_omega and d_values must be 16-byte aligned, like the pointers of
 * the other entry points (TGRAD_ERR_INVALID_ARG otherwise, nothing enqueued).
 * d_grad:   device, numel entries of wg_dtype (tgrad_dtype), read only.
 * d_omega:  device, out, k x uint32: the flat indices of the k entries of
 *           largest |g|^2 (fp32 re*re + im*im without fused multiply-add),
 *           ties to the lower index, ascending.
 * d_values: device, out, k x complex64: grad at those indices (widened to
 *           fp32 if stored as fp16), i.e. Sparse(G, Omega) as index-value pairs.
 * Work is enqueued on the stream; nothing is allocated or freed, on the
 * device or by any library, and the stream is not synchronised.
 *
 * First call on a device: the library looks up the device address of its
 * scratch array once per device (the device that is current at the call) and
 * remembers it.  Make that first call outside any stream capture.
 * Sharing: all calls on a device use the same scratch, which keeps what the
 * last call left there; each call clears what it needs zeroed on its own
 * stream first.  Two calls whose work overlaps on the GPU (different streams,
 * or different threads and streams) race on it -- keep them on one stream or
 * order them with events.  Non-finite inputs give an unspecified result. */
#define TGRAD_NOALLOC_MAX_NUMEL (1ll << 26)
tgrad_status tgrad_select_topk_noalloc(const void* d_grad, int64_t numel, int64_t k, int32_t wg_dtype,
                                       uint32_t* d_omega, void* d_values, void* cuda_stream);

/* Kernels launched by this library since it was loaded (host-side counter). */
int64_t tgrad_launch_count(void);

/* Optional per-stage device timing of tgrad_step (CUDA events recorded on the
 * caller's stream between the stages of a non-refresh step).  Stages, in
 * order: 0 trailing-mode compression fused with the sparse gather (streams
 * grad), 1 mode products of the compression except the first mode, 2 first-mode
 * compression + Adam on the core and on the sparse values + first-mode
 * reconstruction, 3 remaining mode products of the reconstruction, 4
 * trailing-mode reconstruction fused with the weight update and sparse add
 * (streams W).
 * tgrad_get_stage_times synchronises the stream and returns, for the steps
 * since the last call (at most the 64 most recent), the summed milliseconds
 * per stage in ms_sum[5] and the number of steps in *n_steps. */
#define TGRAD_NUM_STAGES 5
tgrad_status tgrad_set_stage_timing(tgrad_state* st, int32_t enable);
tgrad_status tgrad_get_stage_times(tgrad_state* st, void* cuda_stream, float* ms_sum, int32_t* n_steps);

/* ---------------------------------------------------------------------------
 * What a training loop computes between a model's logits and the step above.
 *
 * The calls below keep nothing between calls and hold no state: lists of
 * tensors are HOST arrays that travel with the launch, results and workspaces
 * are device memory of the caller (256-byte aligned workspaces, whose contents
 * need not survive and which two calls that may overlap must not share).
 * Everything is enqueued on the stream, nothing synchronises, every sum has a
 * fixed order (the same inputs give the same bits), and all arithmetic is in
 * fp32 or wider with one rounding to the storage type at the end.
 * Pointers need the alignment of their element type only.  Every wait of a kernel on its copies or on another warp's
 * progress is bounded; one that ran out, which nothing in normal operation leads to, leaves NaN in all results (loss,
 * log-probabilities, entropy, gradient) of the rows that were not finished. */

typedef struct {
  void* d_data;        /* numel entries, contiguous in memory (in any order of the dimensions) */
  int64_t numel;       /* entries (complex ones for the complex types); 0 is allowed            */
  int32_t dtype;       /* tgrad_dtype, complex or real                                          */
  int32_t reserved;
} tgrad_tensor;

/* Gradient norm over a list of tensors: d_out[2 + i] = n_i = sqrt(sum |g|^2) of tensor i, d_out[0] = sqrt(sum n_i^2),
 * d_out[1] = min(1, max_norm / (d_out[0] + 1e-6)), the coefficient that brings the global norm down to max_norm (1 for
 * max_norm = infinity).  d_out holds 2 + n floats.  Magnitudes far from 1 are summed without overflow or underflow.
 * A NaN or infinity in the list gives a norm of NaN or infinity and the coefficient that follows from the formula (NaN
 * or 0); the caller that wants to skip such a step reads d_out[0]. */
tgrad_status tgrad_grad_norm_bytes(int32_t n, size_t* workspace_bytes);
tgrad_status tgrad_grad_norm(const tgrad_tensor* grads, int32_t n, float max_norm, float* d_out, void* d_workspace,
                             size_t workspace_bytes, void* cuda_stream);
/* The same, and every gradient multiplied by d_out[1] in place.  Tensors of the list must not overlap. */
tgrad_status tgrad_clip_grads(const tgrad_tensor* grads, int32_t n, float max_norm, float* d_out, void* d_workspace,
                              size_t workspace_bytes, void* cuda_stream);

/* AdamW on a list of dense tensors (those without a Tucker structure: biases, norms, embeddings): with the gradient g
 * multiplied by *d_grad_scale first,
 *   m <- beta1 m + (1 - beta1) g,  v <- beta2 v + (1 - beta2) |g|^2,
 *   w <- (1 - lr weight_decay) w - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps).
 * dtype: TGRAD_R32, TGRAD_R16H, TGRAD_R16B or TGRAD_C64, of weight and gradient.  m is fp32 (complex64 for TGRAD_C64), v
 * fp32 with one entry per weight: for complex weights |g|^2 is the squared modulus, as in Algorithm 1.  16-bit weights
 * may have fp32 master weights, which are then what is updated; the 16-bit ones receive their rounded values. */
typedef struct {
  void* d_weight;
  const void* d_grad;
  void* d_exp_avg;       /* m */
  float* d_exp_avg_sq;   /* v */
  float* d_master;       /* fp32 weights, or NULL */
  int64_t numel;
  int32_t dtype;
  int32_t reserved;
} tgrad_adamw_tensor;
typedef struct {
  double lr, beta1, beta2, eps, weight_decay;
  int64_t step;               /* counts from 1 */
  const float* d_grad_scale;  /* device scalar, or NULL (1) */
} tgrad_adamw_config;
tgrad_status tgrad_adamw_step(const tgrad_adamw_tensor* list, int32_t n, const tgrad_adamw_config* config, void* cuda_stream);

/* Rows of logits with one target each.  With z = logits / temperature of a row, p = softmax(z):
 *   lse = log sum exp z,  logp = z[target] - lse,  entropy = -sum p log p.
 * A row whose target is negative is ignored: its logits are not read, its outputs and its gradient are 0.  A target
 * >= vocab gives NaN.  Logits of -infinity have p = 0 and gradient 0; a row of nothing else has no distribution (NaN).
 * rows < 2^28 and vocab <= 2^30. */
typedef struct {
  const void* d_logits;
  int64_t rows, vocab;
  int64_t row_stride;        /* entries from one row to the next, >= vocab */
  const int64_t* d_targets;  /* rows */
  int32_t dtype;             /* TGRAD_R32, TGRAD_R16H or TGRAD_R16B */
  double temperature;        /* > 0 (1e-30 to 1e30) */
} tgrad_logits;

/* Each output (rows fp32) may be NULL. */
tgrad_status tgrad_token_logprob(const tgrad_logits* logits, float* d_logp, float* d_lse, float* d_entropy, void* cuda_stream);
/* d_dlogits (dtype of the logits) = gradient of sum(grad_logp logp + grad_entropy entropy) with respect to the logits.
 * d_lse and d_entropy are those of the forward call; d_grad_entropy may be NULL (and d_entropy with it).  A row whose
 * coefficients are 0 has a gradient of 0 whatever its logits are.  Probabilities are as exact as d_lse, an fp32 number: off by
 * up to 2^-24 |lse|, 1 % at |lse| = 2 * 10^5 (a temperature of 10^-4, say); the two losses below do not go by it.
 * Here and below d_dlogits may be d_logits itself, with the same stride. */
tgrad_status tgrad_token_logprob_backward(const tgrad_logits* logits, const float* d_lse, const float* d_entropy,
                                          const float* d_grad_logp, const float* d_grad_entropy, void* d_dlogits,
                                          int64_t dlogits_stride, void* cuda_stream);

/* Clipped policy loss, forward and backward.  With r = exp(logp - old_logp) and A the advantage of a row's token,
 *   policy  = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)
 *   kl      = exp(ref_logp - logp) - (ref_logp - logp) - 1      (0 without ref_logp)
 *   loss    = sum over the rows of weight (policy + kl_coef kl - entropy_coef entropy).
 * The weights carry the mask and the normalisation (1 / tokens for a mean): a row of weight 0 adds nothing to the sums and
 * has a gradient of 0 whatever its logits, old_logp, ref_logp and advantage are.  Where the clipped term is the smaller one no gradient flows through the ratio; at a tie it does.
 * d_stats[5] = loss and the weighted sums of policy, kl, entropy and of the rows that were clipped.
 * d_dlogits = grad_scale * d loss / d logits; NULL: forward only.  d_logp and d_entropy (rows) may be NULL. */
typedef struct {
  const float* d_old_logp;
  const float* d_ref_logp;     /* or NULL */
  const float* d_advantages;
  const float* d_weights;
  float clip_low, clip_high, kl_coef, entropy_coef;
  float grad_scale;            /* factor of the gradient (loss scaling) */
  float reserved;
  float* d_stats;
  float* d_logp;
  float* d_entropy;
  void* d_dlogits;
  int64_t dlogits_stride;
} tgrad_policy_args;
tgrad_status tgrad_policy_loss_bytes(int64_t rows, size_t* workspace_bytes);
tgrad_status tgrad_policy_loss(const tgrad_logits* logits, const tgrad_policy_args* args, void* d_workspace,
                               size_t workspace_bytes, void* cuda_stream);

/* Loss on pairs of answers, forward and backward.  Answer s has the rows [starts[s], starts[s + 1]), answers 2 b and
 * 2 b + 1 are the chosen and the rejected one of pair b (rows of prompts have a negative target):
 *   rewards[s] = beta * sum over its rows of (logp - ref_logp),  h = rewards[2 b] - rewards[2 b + 1],
 *   loss = mean over the pairs of -(1 - label_smoothing) log sigma(h) - label_smoothing log sigma(-h).
 * starts is read on the device; rows outside every answer take no part (a gradient of 0 whatever their logits are).  An answer may be empty, and no pairs give a
 * loss of 0.  d_dlogits as above, NULL: forward only. */
typedef struct {
  const int32_t* d_starts;     /* 2 * pairs + 1, not decreasing */
  const float* d_ref_logp;     /* rows */
  int32_t pairs;
  float beta, label_smoothing;
  float grad_scale;
  float* d_loss;
  float* d_rewards;            /* 2 * pairs */
  float* d_logp;               /* rows */
  void* d_dlogits;
  int64_t dlogits_stride;
} tgrad_preference_args;
tgrad_status tgrad_preference_loss_bytes(int64_t rows, int32_t pairs, size_t* workspace_bytes);
tgrad_status tgrad_preference_loss(const tgrad_logits* logits, const tgrad_preference_args* args, void* d_workspace,
                                   size_t workspace_bytes, void* cuda_stream);

/* For tests of that reporting: the kernels that stream rows of logits through shared memory stop within the first row that takes
 * more than so many copies (0: before any row), and the waits for further ones run out, after half a second.  Negative: never,
 * the default.  For the whole process; the calls after this one take it. */
tgrad_status tgrad_set_copy_limit(int32_t copies);

#ifdef __cplusplus
}
#endif
#endif /* TGRAD_H_ */
