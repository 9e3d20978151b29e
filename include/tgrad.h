/*
 * tgrad.h - C ABI of the TensorGRaD optimizer hot path for AMD MI355X (gfx950).
 *
 * One context (`tgrad_ctx`) serves one complex weight tensor W of an FNO
 * spectral layer and holds the compressed optimizer state of the paper's
 * Algorithm 1 ("Adam with Sparse and Low-Rank Gradient Compression", arxiv
 * 2501.02379): the sparse support Omega, the Tucker factors U^(n), and the Adam
 * moments on the k sparse values and on the Tucker core.
 *
 * Conventions that hold for every call
 *  - Return value: TGRAD_OK (0) or a negative TGRAD_ERR_* code.  Nothing aborts
 *    or throws across this boundary.  `tgrad_strerror` names a code.
 *  - "device pointer" = address in the memory of the GPU that is current when
 *    `tgrad_init` is called; "host pointer" = ordinary process memory.
 *  - The library never allocates or frees device memory.  The caller allocates
 *    `state_dev` and `workspace_dev` with the sizes `tgrad_query_sizes` reports
 *    (256-byte aligned) and keeps both alive until `tgrad_destroy`.
 *  - All device work is enqueued on the one HIP stream given at init.  Neither
 *    `tgrad_step` nor `tgrad_refresh_factors` waits for the device; only
 *    `tgrad_get_state`, `tgrad_set_state` and `tgrad_get_kernel_times` do.
 *  - Every kernel launch is checked where it happens.  A HIP error that is already pending when
 *    `tgrad_step`, `tgrad_step_static` or `tgrad_refresh_factors` is entered belongs to the caller:
 *    the call returns TGRAD_ERR_HIP, launches nothing and leaves the error in place.
 *  - Which kernels serve a configuration is a function of the configuration and the entry point alone
 *    (no environment switches): matrix-core kernels for the shapes they cover (last-mode rank <= 32 and last extent
 *    >= 2; two modes per pass when the shape allows), one-thread-per-output kernels for the rest.
 *  - A context is used from one host thread at a time.
 *  - Tensors are dense, row-major (last mode fastest).  TGRAD_C64 elements are
 *    interleaved (re, im) float32 pairs (8 bytes); TGRAD_CBF16 elements are
 *    interleaved (re, im) bfloat16 pairs (4 bytes).
 *  - Most products of a step run on bf16 matrix instructions, every float32 number in three parts of 8 bits.  Finite numbers
 *    down to 2^-110 (8e-34) keep the accuracy of float32 sums; smaller ones lose their last bits (2e-4 of them at 2^-122).
 *  - The gradient argument is the ordinary gradient dphi/dW.  Algorithm 1 writes
 *    G = -grad and W <- W + eta * G~; every operation it applies to G is odd, so
 *    this library computes the same W as  W <- W (1 - lr wd) - lr * D(grad).
 */
#ifndef TGRAD_H
#define TGRAD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TGRAD_MAX_NDIM 6
#define TGRAD_MAX_HOOI_SWEEPS 64
#define TGRAD_MAX_EIG_SWEEPS 30       /* Jacobi sweeps an eigen-solve may take */
#define TGRAD_MAX_EXTENT 256          /* largest I_n the factor refresh accepts */
#define TGRAD_STATIC_WORKSPACE_BYTES (32u << 20)   /* scratch of tgrad_step_static, per GPU */

typedef struct tgrad_ctx tgrad_ctx;   /* opaque; host memory owned by the library */

enum { TGRAD_C64 = 0, TGRAD_CBF16 = 1 };
enum { TGRAD_SELECT_TOPK_MAG = 0, TGRAD_SELECT_RANDOM = 1 };
enum { TGRAD_ORDER_US_LR = 0, TGRAD_ORDER_LR_US = 1, TGRAD_ORDER_SUM = 2 };

enum {
  TGRAD_OK = 0,
  TGRAD_ERR_INVALID_ARG = -1,   /* null pointer, bad shape/rank/k, misaligned buffer, bad selector */
  TGRAD_ERR_UNSUPPORTED = -2,   /* valid in the paper's terms, but not built (see field comments) */
  TGRAD_ERR_NOT_READY = -3,     /* step or state read before any refresh / factor injection */
  TGRAD_ERR_HIP = -4,           /* a HIP runtime call or kernel launch failed */
  TGRAD_ERR_TOO_SMALL = -5,     /* host buffer smaller than the requested item */
  TGRAD_ERR_NOT_CONVERGED = -6  /* tgrad_get_state of a factor whose eigen-solve stopped at its sweep limit
                                   with rotations still to do (the factor is delivered all the same) */
};

/* Items of `tgrad_get_state` / `tgrad_set_state` (host-side formats in the comments). */
enum {
  TGRAD_STATE_STEP = 0,         /* int64: t, the number of completed steps */
  TGRAD_STATE_INDICES = 1,      /* int64[k]: Omega, ascending row-major linear indices */
  TGRAD_STATE_CORE_M = 2,       /* float32[2*C]: M_L, interleaved complex, C = prod r_n, row-major */
  TGRAD_STATE_CORE_V = 3,       /* float32[C]:   V_L */
  TGRAD_STATE_SPARSE_M = 4,     /* float32[2*k]: M_S, aligned with Omega */
  TGRAD_STATE_SPARSE_V = 5,     /* float32[k]:   V_S */
  TGRAD_STATE_SPARSE_G = 6,     /* float32[2*k]: values gathered at Omega by the last step (read-only) */
  TGRAD_STATE_CORE_G = 7,       /* float32[2*C]: compressed gradient of the last step (read-only) */
  TGRAD_STATE_GRAM0 = 32,       /* + n: float64[2*I_n*I_n] mode-n Gram of the last refresh (read-only) */
  TGRAD_STATE_FACTOR0 = 64,     /* + n: float32[2*I_n*r_n]: U^(n), row-major I_n x r_n, interleaved complex */
  TGRAD_STATE_EIG_INFO0 = 96    /* + n: int32[3] of mode n's last eigen-solve: {1 if it stopped at the sweep limit
                                   else 0, Jacobi sweeps run, 1 if the Jacobi solver ran because the tridiagonal
                                   one declined (close eigenvalues) else 0} (read-only; compressed modes only) */
};

/*
 * Problem statement = the `Require` line of Algorithm 1 (W, eta, alpha, beta1,
 * beta2, rank r, sparsity rho, sparse scale lambda, refresh period T) plus what
 * an implementation must fix (eps, decoupled weight decay, storage types).
 */
typedef struct {
  int32_t ndim;                       /* N, 2..TGRAD_MAX_NDIM */
  int64_t shape[TGRAD_MAX_NDIM];      /* I_n >= 1; I = prod I_n < 2^31; I_n <= TGRAD_MAX_EXTENT */
  int32_t rank[TGRAD_MAX_NDIM];       /* Tucker rank r_n, 1..I_n.  r_n == I_n: the mode is not
                                         compressed (identity factor) */
  int64_t k_sparse;                   /* k = ceil(rho * I), 0..I, computed by the caller exactly */
  int32_t grad_dtype;                 /* TGRAD_C64 or TGRAD_CBF16 */
  int32_t weight_dtype;               /* TGRAD_C64, or TGRAD_CBF16: weights kept in half precision
                                         (section "Mixed precision training"; optimizer states stay
                                         float32): bf16 (re, im) pairs, 4 bytes per element, widened
                                         exactly, updated in float32, rounded once to nearest even */
  float lr;                           /* eta */
  float beta1, beta2, eps;            /* Adam decay rates and epsilon */
  float alpha;                        /* scale of the reconstructed update */
  float lambda;                       /* scale of the sparse part inside it */
  float weight_decay;                 /* decoupled (AdamW) decay; 0 disables */
  int32_t refresh_every;              /* T >= 1: tgrad_step refreshes first when t % T == 0.
                                         0: only tgrad_refresh_factors refreshes */
  int32_t hooi_sweeps;                /* 0 = HOSVD factors (appendix "Implementation": truncated SVD of
                                         each unfolding).  1..TGRAD_MAX_HOOI_SWEEPS: that many HOOI
                                         sweeps after it; a sweep re-solves mode 1, 2, .., N in turn,
                                         each on the residual compressed in every other mode with the
                                         factors as they stand (an updated factor is used at once) */
  int32_t select_rule;                /* how SparseIndices picks Omega (section "Unstructured sparse
                                         gradient tensor"): TGRAD_SELECT_TOPK_MAG = the k entries of
                                         largest |g|^2 (float32), ties to the lower linear index;
                                         TGRAD_SELECT_RANDOM = a uniform random k-subset that depends
                                         only on (select_seed, t at the refresh): the k largest of the
                                         keys fmix32(fmix32(i ^ s0) + s1), fmix32 = MurmurHash3's
                                         32-bit finalizer, s0 = lo32(seed) ^ (t32 * 0x9E3779B9),
                                         s1 = hi32(seed) + t32 + 0x7F4A7C15, t32 = t mod 2^32 */
  uint64_t select_seed;               /* TGRAD_SELECT_RANDOM only */
  int32_t order;                      /* how the two components are composed (paragraph "Residual and
                                         composition"; ablation on sparse / low-rank combinations):
                                         TGRAD_ORDER_US_LR = Algorithm 1: support from G, low rank on G
                                         with the support removed; TGRAD_ORDER_LR_US = low rank on the
                                         full G, the sparse part works on R = G - G~_L (support = top-k
                                         of R at refresh, values = R of the current gradient at the
                                         support every step; the refresh needs one more G-sized
                                         float32 buffer in the workspace); TGRAD_ORDER_SUM = both on
                                         the full G */
  int32_t warm_restart;               /* 0 or 1; 1 needs hooi_sweeps >= 1 (else INVALID_ARG): a refresh
                                         that finds every factor present (from an earlier refresh or
                                         tgrad_set_state) starts its sweeps from those factors instead
                                         of from HOSVD (the warm restart of the same appendix) */
  int32_t eig_max_sweeps;             /* which eigen-solver the refresh uses for extents up to 128:
                                         0 = Householder tridiagonalisation + bisection + inverse iteration,
                                         and cyclic Jacobi (up to TGRAD_MAX_EIG_SWEEPS sweeps) only for a matrix
                                         whose leading eigenvalues are too close for inverse iteration;
                                         1..TGRAD_MAX_EIG_SWEEPS = cyclic Jacobi with that many sweeps at most
                                         for every solve (extents above 128 always use Jacobi).  A Jacobi solve
                                         that uses its sweeps up is reported by tgrad_get_state (NOT_CONVERGED) */
} tgrad_config;

/*
 * Bytes of device memory a context needs.  Host-only, touches no GPU.
 *  cfg             host pointer, read only.
 *  state_bytes     host pointer, out: persistent optimizer state (Omega as int32, M_S, V_S, M_L,
 *                  V_L, U^(n); the quantity the paper's memory model counts).
 *  workspace_bytes host pointer, out: scratch that carries nothing from one step to the next
 *                  except the support's bitmask and offsets and kernel-ready copies of the factors
 *                  (a refresh writes all of them anew), what tgrad_get_state and tgrad_check report
 *                  of the last call, and, for orders other than TGRAD_ORDER_US_LR, a table of zeros
 *                  that tgrad_init writes.
 * Errors: INVALID_ARG, UNSUPPORTED.
 */
int tgrad_query_sizes(const tgrad_config* cfg, size_t* state_bytes, size_t* workspace_bytes);

/*
 * Create a context (Algorithm 1, the initialisation lines: t <- 0, all moments <- 0).
 *  out            host pointer, receives the context.
 *  cfg            host pointer, copied.
 *  state_dev      device pointer, >= state_bytes, 256-byte aligned; zeroed asynchronously here.
 *  workspace_dev  device pointer, >= workspace_bytes, 256-byte aligned.
 *  hip_stream     a hipStream_t (NULL = the default stream); every later call enqueues on it.
 * Errors: INVALID_ARG, UNSUPPORTED, HIP.
 */
int tgrad_init(tgrad_ctx** out, const tgrad_config* cfg, void* state_dev, void* workspace_dev,
               void* hip_stream);

/*
 * Algorithm 1, the `t mod T = 0` branch, for cfg.order == TGRAD_ORDER_US_LR:
 * Omega <- SparseIndices(G, rho, cfg.select_rule); R_L <- G - Sparse(G, Omega);
 * {U^(n)} <- TuckerFactors(R_L, r): HOSVD (eigenvectors of the r_n largest eigenvalues of each mode-n
 * Gram matrix R_L(n) R_L(n)^H, descending, every column multiplied by the unit phase that makes its
 * largest-modulus entry real and positive), then cfg.hooi_sweeps HOOI sweeps (from the factors in
 * place instead of from HOSVD when cfg.warm_restart applies).  The two other composition orders
 * take the factors from the full G and (TGRAD_ORDER_LR_US) the support from G - G~_L; see cfg.order.
 * Top-k order: (|g|^2 descending, linear index ascending), |g|^2 evaluated in float32 as
 * fl(fl(re*re) + fl(im*im)).  Touches neither the moments nor t.
 *  grad_dev   device pointer to G (cfg.grad_dtype), read only.
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_refresh_factors(tgrad_ctx* ctx, const void* grad_dev);

/*
 * One pass of Algorithm 1's loop body on (W, G): refresh first if cfg.refresh_every > 0 and
 * t % refresh_every == 0; g_S <- G[Omega]; g_L <- (G with Omega zeroed) x_1 U1^H ... x_N UN^H;
 * AdamUpdate on g_S with (M_S, V_S) and on g_L with (M_L, V_L), tau = t + 1 in the bias
 * correction, N = (M / (1 - beta1^tau)) / (sqrt(V / (1 - beta2^tau)) + eps), V from |x|^2;
 * D <- alpha * (N_L x_1 U1 ... x_N UN); D[Omega] += lambda * N_S;
 * W <- W (1 - lr wd) - lr D; t <- t + 1.
 *  weight_dev  device pointer to W (layout per cfg.weight_dtype), updated in place.
 *  grad_dev    device pointer to G (cfg.grad_dtype), read only, must not alias W.
 * Errors: INVALID_ARG, NOT_READY (refresh_every == 0 and no refresh yet), HIP.
 */
int tgrad_step(tgrad_ctx* ctx, void* weight_dev, const void* grad_dev);

/*
 * Multiply the gradient of every later `tgrad_step` of this context by a number that lies on the device when the step runs: the
 * factor that clips a global norm (tgrad_norm.coef below), an inverse loss scale.  The gradient itself is neither rewritten nor read
 * once more: its compressed parts, which are linear in it, are scaled before AdamUpdate.  The support and the factors of a refresh
 * come from the gradient as it is; a positive factor changes neither, up to rounding.  SPARSE_G and CORE_G report scaled values.
 * There is no skip here as tgrad_group_adamw has it (skip_nonfinite): a NaN factor, or an infinite entry under the factor 0 that an
 * infinite norm gives, makes moments and weight NaN, and a refresh on such a gradient leaves a support and factors of no use to the
 * steps behind it.  A program whose gradients may overflow (float16 under a loss scale) reads tgrad_norm.norm on the host in front of
 * tgrad_step, and leaves the step out where it is not finite.
 * tgrad_step_static takes no factor: give it a scaled gradient (tgrad_group_scale).
 *  scale_dev  device pointer to one float32, read by every step, or NULL: no scaling (as after tgrad_init).
 * Errors: INVALID_ARG.
 */
int tgrad_set_grad_scale(tgrad_ctx* ctx, const float* scale_dev);

/*
 * tgrad_step for callers that cannot allocate device memory and cannot hold a context: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  It does what
 * `tgrad_step` does for a context at step count t (refresh first when t % cfg.refresh_every == 0,
 * then the loop body), but allocates nothing, neither on the device nor on the host: there is no
 * context, and the scratch that `workspace_dev` provides elsewhere is a fixed array inside the
 * library, TGRAD_STATIC_WORKSPACE_BYTES per GPU, which every GPU that runs the library holds until
 * the process ends.  A configuration whose `tgrad_query_sizes` workspace exceeds that size is
 * rejected with TGRAD_ERR_UNSUPPORTED and nothing is launched, unless (leading extents of 8192 and
 * more in front of few rows; sizes within 1 % of the limit) other kernels of this library, slower there, do with that size.
 *  cfg         host pointer; refresh_every must be >= 1 (INVALID_ARG otherwise).
 *  state_dev   device pointer, >= state_bytes of `tgrad_query_sizes`, 256-byte aligned: the optimizer
 *              state (Omega, M_S, V_S, M_L, V_L, U^(n)).  The caller zero-fills it before the call
 *              with t = 0 and passes the same buffer, untouched, to the calls with t = 1, 2, ...; a
 *              call with t % refresh_every != 0 on a state that no earlier call has refreshed is
 *              not detected.
 *  t           the number of steps this state has taken so far.
 *  weight_dev, grad_dev  as for `tgrad_step`.
 *  hip_stream  stream to enqueue on (NULL = the default stream).  Does not wait.
 * All calls on one GPU share that GPU's array, which keeps the last call's contents: every call
 * rebuilds what it reads from there, and calls that overlap in time on one GPU (two streams, two
 * threads) race.  The device must be the current one.
 * Errors: INVALID_ARG, UNSUPPORTED, HIP.
 */
int tgrad_step_static(const tgrad_config* cfg, void* state_dev, int64_t t, void* weight_dev,
                      const void* grad_dev, void* hip_stream);

/*
 * Copy one state item to the host (waits for the stream first).
 *  what      a TGRAD_STATE_* selector (FACTOR0 + n / GRAM0 + n for mode n).
 *  host_out  host pointer, receives the item in the format listed at the selector.
 *  cap       bytes available at host_out.
 * Errors: INVALID_ARG, TOO_SMALL, NOT_READY (indices/factors before any refresh), HIP.
 */
int tgrad_get_state(tgrad_ctx* ctx, int what, void* host_out, size_t cap);

/*
 * Non-finite gradient entries seen by the last refresh (waits for the stream).  The top-k selection
 * already builds a histogram of the leading bits of |g|^2 for every refresh; the entries whose
 * |g|^2 is inf or NaN (a non-finite part, or a magnitude above 1.8e19) are its top bins, so this
 * costs no extra pass over the gradient.  Algorithm 1 is undefined on such a gradient.
 *  nonfinite  host pointer, out: their number.
 * Errors: INVALID_ARG; UNSUPPORTED (rand-k selection or k_sparse == 0: no such histogram exists);
 *         NOT_READY (no refresh yet); HIP.
 */
int tgrad_check(tgrad_ctx* ctx, int64_t* nonfinite);

/*
 * Overwrite one state item from the host (checkpoint restore, or injecting externally computed
 * factors / support).  Read-only selectors are rejected.  INDICES must be strictly ascending and
 * within [0, I); setting INDICES and every FACTOR marks the context ready.  Waits for the stream.
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_set_state(tgrad_ctx* ctx, int what, const void* host_in, size_t bytes);

/*
 * Per-kernel timing with HIP events on the context's stream (for roofline reports).
 * `tgrad_set_profiling(ctx, 1)` makes later calls bracket every kernel launch with events;
 * `tgrad_get_kernel_times` waits for the stream and returns, for up to `cap` kernels, the name
 * (pointer to a static string), the summed duration in milliseconds and the launch count since
 * profiling was last switched on.  Returns the number of kernels written (>= 0) or an error.
 */
int tgrad_set_profiling(tgrad_ctx* ctx, int enabled);
int tgrad_get_kernel_times(tgrad_ctx* ctx, const char** names, double* total_ms, int64_t* launches,
                           int cap);

/*
 * Plain device-to-device copy kernel of a known size, for calibrating hardware counters: a
 * profiler's HBM read / write counters for this launch correspond to exactly `bytes` read and
 * `bytes` written, which fixes the scale of the same counters on the optimizer's kernels.
 *  dst_dev, src_dev  device pointers, 16-byte aligned, non-overlapping, `bytes` long each.
 *  bytes             a multiple of 16.
 *  hip_stream        stream to enqueue on (NULL = the default stream).  Does not wait.
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_calibration_copy(void* dst_dev, const void* src_dev, size_t bytes, void* hip_stream);

/*
 * The memory access pattern of the weight-update kernel without its arithmetic, for calibrating that kernel's
 * bandwidth fraction: every wavefront owns a tile of `tile_bytes`, loads all of it and then stores it back in
 * place unchanged; wavefronts take slabs of `tiles_per_slab` consecutive tiles.  (The plain copy above moves
 * the same bytes with fewer concurrent streams and reaches a higher rate; this is the ceiling of the pattern
 * that a kernel with one tile per wavefront has.)
 *  buf_dev         device pointer, 16-byte aligned, `bytes` long; its contents are rewritten with themselves.
 *  bytes           at least tile_bytes * tiles_per_slab; whole slabs are moved, a remainder is left alone.
 *  tile_bytes      a multiple of 16, at most 17408 (the update kernel's tile: 32 rows of the last mode).
 *  tiles_per_slab  >= 1 (the update kernel: extent of mode N-1 / 32).
 *  hip_stream      stream to enqueue on (NULL = the default stream).  Does not wait.
 *  bytes_read      host pointer: receives the bytes the launch reads (it writes as many).
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_calibration_tile_stream(void* buf_dev, size_t bytes, int tile_bytes, int tiles_per_slab, void* hip_stream,
                                  int64_t* bytes_read);

/*
 * Register-resident matrix-core loop over the whole chip, for calibrating the matrix-core fractions that
 * are reported for the projection and Gram kernels: what the hardware delivers with no memory traffic at all.
 *  kind        0 = the float32 instruction of the projection kernels (32 x 32 x 2), 1 = the float64
 *              instruction of the Gram kernels (16 x 16 x 4).
 *  iterations  loop length per wavefront, >= 1 (each iteration issues four matrix instructions).
 *  sink_dev    device pointer to at least 4 writable bytes, 4-byte aligned (never written in practice: it
 *              keeps the loop from being optimised away).
 *  hip_stream  stream to enqueue on (NULL = the default stream).  Does not wait.
 *  flops       host pointer: receives the floating-point operations of the launch (2 per multiply-add);
 *              divide by the launch's duration, measured by the caller on that stream.
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_calibration_mfma(int kind, int64_t iterations, void* sink_dev, void* hip_stream, double* flops);

/* Release the context (host memory only; device buffers stay the caller's). */
int tgrad_destroy(tgrad_ctx* ctx);

/*
 * ---- Around tgrad_step: what a training step does before and behind it --------------------------------------------------
 *
 * The loss at its head (token log-probabilities, a clipped policy loss with a KL term, a preference loss; value and gradient
 * with respect to the logits), the global norm of all gradients, clipping, and AdamW for the parameters that have no
 * low-rank part.  The clip factor stays on the device: tgrad_group_adamw and, after tgrad_set_grad_scale, tgrad_step apply it to
 * what they read, so that clipping needs no pass over the gradients.
 *
 * Real element types, beside TGRAD_C64 and TGRAD_CBF16.
 */
enum { TGRAD_F32 = 2, TGRAD_BF16 = 3, TGRAD_F16 = 4 };

typedef struct tgrad_group tgrad_group;   /* opaque; host memory owned by the library */

/* One tensor of a group: dense, any shape.  Pointers need the alignment of their element type only. */
typedef struct {
  int64_t numel;        /* elements, >= 0 (a complex number counts once) */
  void* grad;           /* gradient, grad_dtype; read by tgrad_group_grad_norm and tgrad_group_adamw */
  void* out;            /* tgrad_group_scale / _clip: where the scaled gradient goes, grad_dtype; NULL = in place */
  void* param;          /* tgrad_group_adamw: parameter, param_dtype, updated in place; NULL in a group that takes no steps */
  void* exp_avg;        /* ... first moments: float32, (re, im) pairs of it for complex tensors */
  void* exp_avg_sq;     /* ... second moments: float32, one per element (of |g|^2 for complex tensors, as in tgrad_step) */
  int32_t grad_dtype;   /* any of the five types */
  int32_t param_dtype;  /* real if grad_dtype is, complex if it is; ignored where param is NULL */
  float lr_scale;       /* the tensor's learning rate is lr * lr_scale */
  float weight_decay;   /* its decoupled (AdamW) decay */
} tgrad_tensor;

/* What tgrad_group_grad_norm leaves on the device. */
typedef struct {
  double sumsq;         /* sum of |g|^2 over all tensors, added up in float64, plus *add_sumsq */
  float norm;           /* its root */
  float coef;           /* min(1, max_norm / (norm + 1e-6)); 0 for an infinite norm, NaN for a NaN */
} tgrad_norm;

/*
 * Bytes of device memory a group of n tensors needs.  Host-only, touches no GPU.  Errors: INVALID_ARG, UNSUPPORTED (more
 * than 2^20 tensors, 2^40 elements in one, 2^43 in all).
 */
int tgrad_group_query_size(const tgrad_tensor* tensors, int64_t n, size_t* workspace_bytes);

/*
 * Create a group of n >= 1 tensors.
 *  tensors        host pointer, n entries, copied.
 *  workspace_dev  device pointer, >= workspace_bytes, 256-byte aligned; keeps the list of tensors until tgrad_group_destroy.
 *  hip_stream     a hipStream_t (NULL = the default stream); every later call enqueues on it.  Does not wait.
 * Tensors that are written (out, param, moments) must not overlap one another or, but for out == grad, anything that is read.
 * Errors: INVALID_ARG (a null or misaligned pointer, a bad type, param without moments), UNSUPPORTED, HIP.
 */
int tgrad_group_init(tgrad_group** out, const tgrad_tensor* tensors, int64_t n, void* workspace_dev, void* hip_stream);

/*
 * New addresses, rates and decays for a group's tensors (gradients that are allocated anew in every step); numel, types and
 * which pointers are NULL stay as at init.  Enqueued behind the calls before it.  Errors: INVALID_ARG, HIP.
 */
int tgrad_group_bind(tgrad_group* group, const tgrad_tensor* tensors);

/*
 * Global 2-norm of all gradients of the group and the factor that clips it.
 *  max_norm       >= 0.
 *  add_sumsq_dev  device pointer, 8-byte aligned, or NULL: sum of squares of gradients that lie elsewhere (another group's
 *                 tgrad_norm.sumsq, other ranks'), added before the root.
 *  norm_dev       device pointer, 8-byte aligned: receives the result.  May hold *add_sumsq_dev.
 * The order of the sum depends on the sizes alone, never on timing.  Errors: INVALID_ARG, HIP.
 */
int tgrad_group_grad_norm(tgrad_group* group, float max_norm, const double* add_sumsq_dev, tgrad_norm* norm_dev);

/*
 * out = grad * norm_dev->coef for every tensor, in float32, rounded once to the type (nearest even).  In place, a factor of 1
 * leaves everything as it is and reads nothing.  Errors: INVALID_ARG, HIP.
 */
int tgrad_group_scale(tgrad_group* group, const tgrad_norm* norm_dev);

/* tgrad_group_grad_norm, then tgrad_group_scale with its result. */
int tgrad_group_clip(tgrad_group* group, float max_norm, const double* add_sumsq_dev, tgrad_norm* norm_dev);

typedef struct {
  double lr, beta1, beta2, eps;   /* lr >= 0, 0 <= beta < 1, eps >= 0 */
  int32_t skip_nonfinite;         /* 1: where norm_dev holds an infinite or NaN norm, nothing is written (tgrad_step has no such skip) */
} tgrad_adamw;

/*
 * One AdamW step of every tensor, tau = t + 1:  g' = coef g;  M <- beta1 M + (1 - beta1) g';
 * V <- beta2 V + (1 - beta2) |g'|^2;  p <- p (1 - lr wd) - lr (M / (1 - beta1^tau)) / (sqrt(V / (1 - beta2^tau)) + eps).
 * In float32; a bf16 or float16 parameter is widened exactly and rounded once to nearest even.
 *  t         steps taken before this one, >= 0.
 *  norm_dev  device pointer: the clip factor.  NULL = 1 (skip_nonfinite then has to be 0).
 * Errors: INVALID_ARG (also for a group with a NULL param), HIP.
 */
int tgrad_group_adamw(tgrad_group* group, const tgrad_adamw* hyper, int64_t t, const tgrad_norm* norm_dev);

/* Release the group (host memory only). */
int tgrad_group_destroy(tgrad_group* group);

/*
 * Logits and the token of every row.  z = data / temperature.  A row whose target lies outside 0..vocab-1 (-100, say) is
 * ignored: nothing of it is read, its log-probability is 0 and its gradient 0.
 */
typedef struct {
  const void* data;         /* device pointer: TGRAD_F32, TGRAD_BF16 or TGRAD_F16, rows of `vocab` consecutive elements */
  int64_t rows;             /* 0..2^31-1 */
  int64_t vocab;            /* 1..2^30-1 */
  int64_t row_stride;       /* elements from one row to the next, >= vocab */
  const int64_t* targets;   /* device pointer, int64[rows] */
  int32_t dtype;
  float temperature;        /* > 0 */
} tgrad_logits;

/*
 * logp[n] = z[n, y_n] - lse[n],  lse[n] = log sum_v exp z[n, v], in float32.  Entries of -inf have probability 0; a row of
 * nothing else, or with a NaN or +inf in it, has a NaN.  Reads the logits once.
 *  logp, lse   device pointers, float32[rows]; either may be NULL.
 *  hip_stream  stream to enqueue on (NULL = the default stream).  Does not wait.  The same holds for the calls below.
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_token_logprobs(const tgrad_logits* logits, float* logp, float* lse, void* hip_stream);

/*
 * dlogits[n, v] = dlogp[n] / temperature * ([v = y_n] - exp(z[n, v] - lse[n])), rounded once to the logits' type.
 *  lse, dlogp      device pointers, float32[rows].  A row with dlogp = 0 is not read.  From |lse| = 7e5 on, where lse's rounding
 *                  alone moves exp(z - lse) by several percent, exponents above 0 count as 0.
 *  dlogits         device pointer, the logits' type, rows `dlogits_stride` >= vocab elements apart; what lies between them is
 *                  left alone.  May be logits->data, with the same stride.
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_token_logprobs_backward(const tgrad_logits* logits, const float* lse, const float* dlogp, void* dlogits,
                                  int64_t dlogits_stride, void* hip_stream);

typedef struct {
  float clip_low, clip_high;   /* the ratio is clipped to 1 - clip_low .. 1 + clip_high; clip_low 0..1, clip_high >= 0 */
  float kl_beta;               /* weight of the KL term; 0: it is only reported */
} tgrad_policy;

/* Bytes of scratch of tgrad_policy_loss and tgrad_preference_loss.  Host-only.  Errors: INVALID_ARG. */
int tgrad_loss_query_size(int64_t rows, int64_t pairs, size_t* workspace_bytes);

/*
 * Clipped policy loss with a KL term towards a reference, and its gradient:
 *   r = exp(logp - old);  pg = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A);  d = ref - logp;  kl = exp(d) - d - 1
 *   loss = sum_n w_n (pg + kl_beta kl);  dlogits = dloss d loss / d logits.
 * Where both arguments of the minimum are equal the gradient is that of the unclipped one.  A = 0: both are 0, whatever r, one beyond
 * float32 among them.
 *  weight, advantage, old_logp  device pointers, float32[rows].  weight carries the mask and the normalisation (1 / number of
 *                tokens, say); a row of weight 0 is ignored like one without a target: none of its entries anywhere is read.
 *  ref_logp      the same, or NULL: kl = 0.
 *  dloss         device pointer to one float32 (a loss scale), or NULL: 1.
 *  workspace_dev device pointer, >= tgrad_loss_query_size(rows, 0), 256-byte aligned.
 *  stats         device pointer, float32[4]: sums over n of w (pg + kl_beta kl), w pg, w kl, w [clipped].
 *  logp          device pointer, float32[rows], or NULL.
 *  dlogits       as for tgrad_token_logprobs_backward, or NULL: no gradient.
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_policy_loss(const tgrad_logits* logits, const tgrad_policy* policy, const float* weight, const float* advantage,
                      const float* old_logp, const float* ref_logp, const float* dloss, void* workspace_dev, float* stats,
                      float* logp, void* dlogits, int64_t dlogits_stride, void* hip_stream);

typedef struct {
  float beta;              /* > 0 */
  float label_smoothing;   /* 0 .. 0.5: share of pairs that are labelled the wrong way round */
} tgrad_preference;

/*
 * Preference loss on paired log ratios, and its gradient.  Sequence i is rows seq_start[i] .. seq_start[i + 1] - 1 of the logits; the first
 * `pairs` sequences are the chosen answers, the next `pairs` the rejected ones, in the same order.
 *   R_i = beta sum_n w_n (logp_n - ref_n);  h = R_chosen - R_rejected
 *   loss = mean over pairs of -(1 - s) log sigma(h) - s log sigma(-h);  dlogits = dloss d loss / d logits.
 * A sequence without rows, or whose weights are all 0, has R = 0.
 *  seq_start  device pointer, int64[2 pairs + 1], ascending; bounds outside 0 .. rows are taken as the nearest inside.
 *             Rows in no sequence have no gradient.  1 <= pairs < 2^22.
 *  weight, ref_logp  device pointers, float32[rows]; rows of weight 0 are ignored.
 *  dloss, workspace_dev (tgrad_loss_query_size(rows, pairs)), logp, dlogits  as for tgrad_policy_loss.
 *  loss       device pointer, one float32.
 *  rewards    device pointer, float32[2 pairs]: R.
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_preference_loss(const tgrad_logits* logits, const tgrad_preference* preference, int64_t pairs,
                          const int64_t* seq_start, const float* weight, const float* ref_logp, const float* dloss,
                          void* workspace_dev, float* loss, float* rewards, float* logp, void* dlogits,
                          int64_t dlogits_stride, void* hip_stream);

/*
 * ---- A block of the model in 8 bits: its products, what it keeps for the backward pass, the norms around it ----------------
 *
 * With the optimizer's moments compressed, a training step's memory is its activations.  These calls keep them as 8-bit codes that
 * the forward products are taken of and that the backward pass reads as they are.  Each takes the stream to enqueue on
 * (NULL = the default stream), waits for nothing and allocates nothing; outputs overlap neither each other nor inputs unless it is said.
 */

/* rows x cols numbers.  Rows of consecutive elements, any alignment of the element type. */
typedef struct {
  void* data;           /* device pointer; may be NULL where rows is 0 */
  int64_t rows;         /* 0..2^31-1 */
  int64_t cols;         /* 1..2^30 */
  int64_t row_stride;   /* elements from one row to the next, >= cols; what lies between rows is neither read nor written */
  int32_t dtype;        /* TGRAD_F32, TGRAD_BF16 or TGRAD_F16 */
} tgrad_matrix;

/*
 * rows x cols numbers in 8 bits: value = code * scale (in float32).  With a the largest magnitude of a group, scale = a / 127 and code =
 * 127 v / a, the exact quotient rounded to nearest even: -127..127.  (Scales end where 127 times one is finite.)  A group whose largest magnitude is below 2^-119 is all
 * zeros, with scale 0; one with an infinity or NaN in it has scale NaN and codes 0, so that all its values are NaN.
 */
typedef struct {
  void* codes;          /* device pointer, int8; rows that start at multiples of 16 bytes are read fastest */
  float* scale;         /* device pointer, float32[rows][ceil(cols / group)], dense */
  int64_t rows, cols;   /* as above */
  int64_t row_stride;   /* bytes from one row to the next, >= cols */
  int32_t group;        /* columns that share a scale, counted from a row's first: 32, 64, 128, 256, 512; 0: the whole row */
} tgrad_codes;

/* Codes and scales of x.  x and out have the same rows and cols.  Errors: INVALID_ARG, HIP. */
int tgrad_quantize(const tgrad_matrix* x, const tgrad_codes* out, void* hip_stream);

/* The values that codes stand for, rounded once to out's type.  Errors: INVALID_ARG, HIP. */
int tgrad_dequantize(const tgrad_codes* codes, const tgrad_matrix* out, void* hip_stream);

enum { TGRAD_CODES_MATMUL = 0, TGRAD_CODES_LINEAR = 1, TGRAD_CODES_GRAD_INPUT = 2, TGRAD_CODES_GRAD_WEIGHT = 3 };
/* added to a gradient's op: dy's rows do not start at multiples of 16 bytes, are no multiple of 8 long, or lie more than 2^21 elements apart */
#define TGRAD_CODES_UNALIGNED 4
#define TGRAD_CODES_UNROUNDED 8        /* added to a gradient's op: values of codes are not rounded to dy's type (tgrad_codes_gradient) */
#define TGRAD_CODES_MAX_INNER 131072   /* longest sum of products of codes that int32 holds: 127^2 2^17 < 2^31 */

/*
 * Bytes of scratch of the calls below, for tokens x inner times inner x outer.  Two-byte dy that is not aligned is copied there first, which
 * needs TGRAD_CODES_UNALIGNED; but for up to 16 tokens of codes with a scale a row and for unrounded values with a float32 result, which copy none,
 * as float32 dy does not.  0: none, and the call's workspace_dev may be NULL.  Host-only.  Errors: INVALID_ARG.
 */
int tgrad_codes_query_size(int op, int64_t tokens, int64_t inner, int64_t outer, size_t* workspace_bytes);

/*
 * y[t, n] = x.scale[t] w.scale[n] sum_k x.code[t, k] w.code[n, k].  The sum is exact (int32); it is converted and multiplied in float32
 * and rounded once to y's type.
 *  x              tokens x inner, group 0; inner <= TGRAD_CODES_MAX_INNER.  Codes are -127..127, as tgrad_quantize writes them.
 *  w              outer x inner, group 0: the weight, a row for each output.
 *  y              tokens x outer.
 *  workspace_dev  device pointer, >= tgrad_codes_query_size, 256-byte aligned.
 * Errors: INVALID_ARG, UNSUPPORTED (inner; 2^33 results), HIP.
 */
int tgrad_codes_matmul(const tgrad_codes* x, const tgrad_codes* w, const tgrad_matrix* y, void* workspace_dev, void* hip_stream);

/*
 * tgrad_quantize of x into `keep` (group 0), then tgrad_codes_matmul of it, with the same results; for a few tokens in one launch.
 *  keep   receives the codes of x, for the backward pass.  NULL: not kept, and they lie in scratch.
 *  workspace_dev  as above; with `keep` the size for TGRAD_CODES_MATMUL is enough.
 */
int tgrad_codes_linear(const tgrad_matrix* x, const tgrad_codes* w, const tgrad_codes* keep, const tgrad_matrix* y,
                      void* workspace_dev, void* hip_stream);

/*
 * The product's gradients, with the gradient of a code's value taken as that of the number it was made from:
 *   dx[t, k] = sum_n dy[t, n] w[n, k]     dw[n, k] = sum_t dy[t, n] x[t, k]
 * w and x are the values of codes, in groups of any size.  bf16 and float16: values are rounded to as many bits as dy's type has, whatever its
 * exponents reach (float16: 11 bits down to 2^-28 of the largest value, fewer below), products are exact and added up in float32.  float32, and up to 16 tokens of codes with a scale a row: dy times that scale is
 * rounded to float32 and split into three bf16 parts, which keep 24 bits (below 2^-110 the last ones are lost), codes are exact.
 *  dx, dw  dy's type, or TGRAD_F32; rounded once.  The order of the sums depends on sizes and alignment alone.
 *  workspace_dev  as above.
 * Errors: INVALID_ARG, UNSUPPORTED (2^33 results, more than 2^30 tokens, two-byte rows of more than 2^21), HIP.
 */
int tgrad_codes_grad_input(const tgrad_matrix* dy, const tgrad_codes* w, const tgrad_matrix* dx, void* workspace_dev, void* hip_stream);
int tgrad_codes_grad_weight(const tgrad_matrix* dy, const tgrad_codes* x, const tgrad_matrix* dw, void* workspace_dev, void* hip_stream);

/*
 * The same two, by op: TGRAD_CODES_GRAD_INPUT or _WEIGHT, with what is added to it for tgrad_codes_query_size.  With TGRAD_CODES_UNROUNDED the error that
 * rounded values bring into a two-byte gradient is gone, for twice the matrix operations: values are taken in two parts of dy's type (off by 2^-14 of
 * themselves in bf16; in float16 by 2^-20, down to 2^-28 of the largest value), and with a float32 result dy and values as in float32.
 * Errors: as above; INVALID_ARG for another op.
 */
int tgrad_codes_gradient(int op, const tgrad_matrix* dy, const tgrad_codes* codes, const tgrad_matrix* out, void* workspace_dev, void* hip_stream);

enum { TGRAD_ACT_SILU = 0, TGRAD_ACT_GELU = 1 };   /* x / (1 + exp(-x)); x (1 + erf(x / sqrt(2))) / 2 */

/*
 * y = act(x), or act(x) * gate, in float32, and the checkpoint that its backward pass needs.
 *  gate       the same size and type as x, or NULL.
 *  y, y8      one of them: the result in x's type, or as codes for the next product (group 0).
 *  x8, gate8  receive the codes of x and gate, in groups of 32..512 columns.  Both NULL: no checkpoint; gate8 goes with gate.
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_activation(const tgrad_matrix* x, const tgrad_matrix* gate, int act, const tgrad_matrix* y, const tgrad_codes* y8,
                     const tgrad_codes* x8, const tgrad_codes* gate8, void* hip_stream);

/*
 * dx = dy act'(x) [* gate] and dgate = dy act(x), of the values that the checkpoint stands for.
 *  gate8, dgate  both or neither.  dx and dgate have dy's size and type.
 * Errors: INVALID_ARG, HIP.
 */
int tgrad_activation_backward(const tgrad_matrix* dy, const tgrad_codes* x8, const tgrad_codes* gate8, int act, const tgrad_matrix* dx,
                              const tgrad_matrix* dgate, void* hip_stream);

/* The norms after and before a block and what joins them.  norm(v) = (v - m) / sqrt(mean((v - m)^2) + eps), m = mean(v) or 0. */
typedef struct {
  const void* post_weight;   /* device pointer, [cols]: norm of the block's output; NULL: the output goes in as it is */
  const void* pre_weight;    /* device pointer, [cols]: norm of the sum, for the next block; NULL: none */
  const void* gate;          /* device pointer, [ceil(rows / rows_per_gate)][cols], the block's type; NULL: 1 */
  int64_t gate_stride;       /* elements from one row of the gate to the next, >= cols */
  int64_t rows_per_gate;     /* >= 1: rows 0 .. rows_per_gate - 1 take the gate's first row, and so on */
  int32_t weight_dtype;      /* type of both weights */
  float scale;               /* of the residual branch; finite */
  float eps;                 /* > 0 */
  int32_t centered;          /* 1: m is the mean; 0: m = 0 */
} tgrad_block;
#define TGRAD_NORM_MAX_COLS 32768

/*
 * x_out = x + scale * gate * (norm(block) * post_weight), rounded to the stream's type;  h = norm(x_out) * pre_weight.
 *  x, x_out  the residual stream before and after: float32, or the block's type.
 *  block     the block's output.  NULL: h = norm(x) * pre_weight alone; x_out, post_weight and gate are NULL then.
 *  h, h8     one of them where there is a pre_weight: the next block's input in the block's type, or as codes (group 0).
 *  stats     device pointer, float32[rows][4]: mean and factor 1 / sqrt(...) of the block's norm and of the sum's, for the
 *            backward pass; NULL: not kept.
 * Statistics are float32.  Errors: INVALID_ARG, UNSUPPORTED (cols > TGRAD_NORM_MAX_COLS), HIP.
 */
int tgrad_block_norm(const tgrad_block* desc, const tgrad_matrix* x, const tgrad_matrix* block, const tgrad_matrix* x_out,
                     const tgrad_matrix* h, const tgrad_codes* h8, float* stats, void* hip_stream);

/* Bytes of scratch of tgrad_block_norm_backward; rows_per_gate: 1 without a gate.  Host-only.  Errors: INVALID_ARG, UNSUPPORTED. */
int tgrad_block_norm_query_size(int64_t rows, int64_t cols, int64_t rows_per_gate, size_t* workspace_bytes);

/*
 * Gradients of tgrad_block_norm, for d = its gradient with respect to x_out (all of it, h's share among it):
 *   dx = d = dx_out + norm'(dh * pre_weight),  dblock = norm'(scale * d * gate * post_weight),
 *   dgate = sum over its rows of scale * d * norm(block) * post_weight,  dpost = sum of scale * d * gate * norm(block),
 *   dpre = sum of dh * norm(x_out).
 *  dx_out  gradient with respect to x_out from elsewhere, the stream's type; NULL: none.
 *  dh      gradient with respect to h; NULL where there is no pre_weight.
 *  x_out   as the forward call left it (its x, where there was no block).
 *  stats   as the forward call left them.
 *  dx, dblock  the stream's and the block's type; dblock NULL without a block.  dx may be dx_out, with the same stride.
 *  dgate   the gate's size and type, rows of cols elements, dense; NULL without a gate.
 *  dpost, dpre   device pointers, float32[cols]; NULL without their weights.
 *  workspace_dev  device pointer, >= tgrad_block_norm_query_size, 256-byte aligned.
 * The order of the sums depends on the sizes alone.  Errors: INVALID_ARG, UNSUPPORTED, HIP.
 */
int tgrad_block_norm_backward(const tgrad_block* desc, const tgrad_matrix* dx_out, const tgrad_matrix* dh, const tgrad_matrix* x_out,
                              const tgrad_matrix* block, const float* stats, const tgrad_matrix* dx, const tgrad_matrix* dblock,
                              void* dgate, float* dpost, float* dpre, void* workspace_dev, void* hip_stream);

/* Static description of a status code. */
const char* tgrad_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* TGRAD_H */
