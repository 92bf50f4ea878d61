/*
 * fw.h -- C ABI of the feature-whitening-by-gradient-transformation hot path
 * for NVIDIA B200 (sm_100a).
 *
 * Method: "Feature Whitening via Gradient Transformation for Improved
 * Convergence" (arXiv 2010.01546).  Per layer and per batch the library
 *   (a) folds a block of layer inputs into the running mean, covariance and
 *       feature power                                   (Sec. 2, Eqs. 2-5; Eqs. 37-38),
 *   (b) runs the recursive condition-number reduction that builds the
 *       whitening transform T and Q = T^T T             (Sec. 4, Eqs. 36-50),
 *   (c) multiplies the weight gradient by the smoothed Q and applies the SGD
 *       step                                            (Sec. 3.1, Eqs. 27-30; Eq. 35).
 *
 * Notation (im2col form): a layer input is a patch vector of length M, the
 * layer is z = W (x - mu) + b with W of shape N x M (the paper's S is N here).
 * X holds one patch per row: rows = B*H*W, leading dimension ldx >= M.
 *
 * Conventions
 *  - Every pointer except fw_layer*, fw_layer_desc* and the arrays of a
 *    grouped call (layer handles, pointer tables, row counts: HOST arrays of
 *    DEVICE pointers) is a DEVICE pointer owned by the caller.  Matrices are
 *    dense row-major fp32 unless stated; X may be bf16.
 *  - The library never allocates or frees device memory.  All per-layer state
 *    and scratch live in the caller-supplied workspace, which must outlive the
 *    layer and be 256-byte aligned.
 *  - Compute calls validate their arguments on the host, return an error code
 *    synchronously and launch nothing on error; otherwise they enqueue work on
 *    the layer's CUDA stream and return without waiting.  Conditions found on
 *    the device (non-finite input, a step with no usable subspace, a bounded
 *    wait that gave up) are kept in a per-layer status word in the layer's own
 *    workspace, read by fw_layer_sync_status; no kernel reports through
 *    process-wide state.
 *  - Compute calls may be captured into a CUDA graph once a call of the same
 *    kind has run outside of it.  A replay repeats the choices that were made at
 *    capture (first block or not, Phi_y stale or not, T still the identity or
 *    not), so a pass is captured after the first block and the first reduction.
 *  - A layer is not thread-safe.  Calls on different layers are independent;
 *    a grouped call requires all its layers to share one stream.
 *  - There is no CPU fallback: without a CUDA device every compute call
 *    returns FW_ERR_CUDA.
 */
#ifndef FW_H_
#define FW_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct fw_layer fw_layer; /* opaque host object owned by the library */

typedef enum {
  FW_OK = 0,
  FW_ERR_INVALID_ARG = 1, /* null pointer, negative count, bad enum            */
  FW_ERR_SHAPE = 2,       /* M, N, rows, ld outside the supported range        */
  FW_ERR_STATE = 3,       /* call order: e.g. reduction before any covariance  */
  FW_ERR_WORKSPACE = 4,   /* workspace too small or misaligned                 */
  FW_ERR_CUDA = 5,        /* a CUDA runtime call failed                        */
  FW_ERR_TIMEOUT = 6,     /* a bounded device-side wait gave up                */
  FW_ERR_UNSUPPORTED = 7, /* valid request this build has no kernel for        */
  FW_WARN_NO_SUBSPACE = 64, /* some step found no coherent column set: a_e = 0 */
  FW_WARN_NONFINITE = 65    /* NaN/Inf seen in X, G or the state               */
} fw_status;

/* Element types.  The X of a layer is fp32 or bf16; e4m3 (8-bit floats, with a
 * scale beside them) is a type of the norm's output and of the gated block. */
typedef enum { FW_F32 = 0, FW_BF16 = 1, FW_E4M3 = 2 } fw_dtype;

/* Engine of the two dense contractions (X^T X and G Q) and of the re-sync
 * products.  FP32: FFMA, matches an fp64 reference to ~1e-6.  TF32 / BF16:
 * tcgen05 tensor cores with fp32 accumulation (TF32 for fp32 X, BF16 for bf16
 * X), matches to ~1e-3.  The recursion itself is always fp32. */
typedef enum { FW_PREC_FP32 = 0, FW_PREC_TF32 = 1, FW_PREC_BF16 = 2 } fw_prec;

/* Start vector of the power iterations: the column-alignment estimate of
 * Sec. 4.2 (Eqs. 45-50), or simply the largest-norm column normalised. */
typedef enum { FW_INIT_ALIGN = 0, FW_INIT_MAXCOL = 1 } fw_init;

typedef struct {
  int32_t M, N;      /* input features (patch length), output features          */
  int32_t x_dtype;   /* fw_dtype                                                 */
  int32_t prec;      /* fw_prec                                                  */
  int32_t init;      /* fw_init                                                  */
  float alpha;       /* inter-block averaging of the moments, Eqs. 2-3, 37      */
  float beta;        /* smoothing of Q, Eq. 35                                   */
  float gamma;       /* leakage of the transform, Eq. 42 (0 < gamma <= 1)       */
  float delta;       /* power-reduction target, Eq. 40                           */
  float eps;         /* floor of the denominator in Eq. 40                       */
  float c_rel;       /* relative coherence threshold, Eq. 48                     */
  float c_abs;       /* absolute coherence threshold, Eq. 48                     */
} fw_layer_desc;

/* Fills *d with the recursive method's hyper-parameters of Sec. 6
 * (alpha 0.1, beta 0.1, gamma 0.99, delta 0.25, c_rel 0.025, c_abs 1e-6,
 * eps 1e-5), fp32 X, FP32 engine, alignment start vector. */
void fw_layer_desc_default(fw_layer_desc* d, int32_t M, int32_t N);

/* Device bytes a layer of this description needs (state + scratch); 0 if the
 * description is invalid.  Supported: 1 <= M <= 8192, 1 <= N <= 8192. */
size_t fw_layer_workspace_bytes(const fw_layer_desc* d);

/* Creates a layer in the given workspace and enqueues its initialisation on
 * `cuda_stream` (a cudaStream_t, may be 0): T = Q = Qs = I, mu = 0, no block
 * seen yet (Eqs. 12-13; Qs(-1) = I of Sec. 3.2).  The handle is host memory
 * owned by the library until fw_layer_destroy. */
fw_status fw_layer_create(const fw_layer_desc* d, void* dev_workspace, size_t bytes,
                          void* cuda_stream, fw_layer** out);

/* Frees the host object only; the workspace stays the caller's. */
fw_status fw_layer_destroy(fw_layer* L);

/* Puts the layer back into the state fw_layer_create leaves it in (T = Q = Qs
 * = I, mu = 0, no block seen, no open block, status cleared), in the same
 * workspace, on the layer's stream.  Attached parameters stay attached. */
fw_status fw_layer_reset(fw_layer* L);

/* Optional.  Attaches the layer's parameters (W: N x M, b: N, device fp32) so
 * that fw_cov_update can compensate the bias for the change of the running
 * mean (Eq. 31: b += W (mu_new - mu_old), the sign that leaves
 * z = W (x - mu) + b unchanged).  Pass NULLs to detach. */
fw_status fw_layer_attach_params(fw_layer* L, float* W, float* b);

/* (a) Moments of one block of patch rows (Eqs. 2-5, 37-38).
 * X: rows x M, row-major, leading dimension ldx (elements), fp32 or bf16 per
 * the description.  Computes X^T X and the column sums in one pass over X,
 * then mu, Phi_x (centred on the updated running mean, normalised by the
 * block's rows), phi and lam_bar; the first block sets them, later blocks
 * average with alpha.  Marks the whitened covariance Phi_y = T Phi_x T^T stale.
 *
 * flags: a block may span several calls (Sec. 2: the moments are computed "in
 * blocks of L batches").  FW_COV_ACCUMULATE adds this call's X^T X, column
 * sums and row count to the open block and changes no moment; FW_COV_COMMIT
 * (the default, 0) adds this call's rows and closes the block: mu, Phi_x, phi
 * and the bias compensation then see all rows accumulated since the last
 * commit, exactly as if they had been passed in one call.  The pilot shift
 * that centres short fp32 blocks inside the Gram pass is fixed by the block's
 * first call.
 * rows must be >= 1; ldx >= M; for the tensor-core engines X must be 16-byte
 * aligned and ldx * sizeof(element) a multiple of 16. */
#define FW_COV_COMMIT 0u
#define FW_COV_ACCUMULATE 1u
fw_status fw_cov_update(fw_layer* L, const void* X, int64_t rows, int64_t ldx, uint32_t flags);

/* (a) from the activation itself.  The layer input of a convolution is "any
 * spatial dimension vectorised" (Sec. 2): patch rows of length M = C k k cut
 * from an NHWC activation A[B][H][W][C] (stride 1, zero padding (k - 1) / 2,
 * columns ordered (ky, kx, c)).  These calls take A and never materialise the
 * patch matrix, which for k = 3 is nine times the activation: the Gram kernel
 * reads shifted windows of a zero-padded copy of A.  Semantics, flags and
 * results are those of fw_cov_update on the patch matrix of rows = B H W.
 *   k = 1: A is the patch matrix; no scratch is needed.
 *   k = 3: scratch (device, caller-owned, 256-byte aligned, at least
 *          fw_nhwc_scratch_bytes bytes, free again when the call's work on the
 *          stream is done) holds the padded copy.  Needs a tensor-core layer
 *          with fp32 X (FW_PREC_TF32), C a multiple of 4, and H divisible by
 *          the image rows a pipeline stage covers (any power-of-two H; 14 and
 *          28 also); otherwise FW_ERR_UNSUPPORTED and the caller falls back to
 *          fw_cov_update on a patch matrix of its own. */
size_t fw_nhwc_scratch_bytes(int32_t B, int32_t H, int32_t W, int32_t C, int32_t k);
fw_status fw_cov_update_nhwc(fw_layer* L, const float* A, int32_t B, int32_t H, int32_t W, int32_t C, int32_t k,
                             void* scratch, size_t scratch_bytes, uint32_t flags);
/* HOST arrays of length n, as in the other grouped calls. */
fw_status fw_group_cov_update_nhwc(fw_layer* const* L, int32_t n, const float* const* A, const int32_t* B,
                                   const int32_t* H, const int32_t* W, const int32_t* C, const int32_t* k,
                                   void* const* scratch, const size_t* scratch_bytes, uint32_t flags);

/* (b) K steps of the recursion of Sec. 4 on the current moments, each with P
 * power iterations refining the subspace estimate (P = 0: the estimate of
 * Sec. 4.2 as it is), then one smoothing update of Qs (Eq. 35).  Per step:
 * xi, m' (Eqs. 45-46); c (Eq. 47); coherent set and aligned average
 * (Eqs. 48-50); v <- Phi_y v / ||Phi_y v||, P times; lambda_e = v^T Phi_y v
 * (Eq. 36); g_e, a_e (Eqs. 40-41); t = T^T v; rank-one updates of Q (Eq. 44),
 * T (Eq. 42) and Phi_y, with the leakage gamma of the description (gamma < 1
 * additionally tracks T Phi_x so that Phi_y stays T Phi_x T^T at O(M^2) per
 * step).  Runs entirely on the device.
 * trace_or_null: K x 4 device floats (lambda_e, g_e, |set|, m') per step.
 * K = 0 takes no step and leaves T, Q, Qs alone; it only brings Phi_y =
 * T Phi_x T^T up to date when the moments changed since the last call.
 * Requires a covariance (FW_ERR_STATE otherwise). */
fw_status fw_cond_reduce(fw_layer* L, int32_t K, int32_t P, float* trace_or_null);

/* (c) G_out = G Qs (Eq. 29 with the smoothed Q of Eq. 35).  G, G_out: N x M.
 * G_out may be G itself (in place: the product is formed in the layer's
 * workspace and copied over G); any other overlap of the two arrays is
 * rejected with FW_ERR_INVALID_ARG. */
fw_status fw_grad_transform(fw_layer* L, const float* G, float* G_out);

/* The direct method the gradient transformation replaces (Sec. 2), for
 * comparison: every sample is whitened on the way forward and its gradient is
 * sent back through the transform, two rows x M x M products per batch where
 * fw_grad_transform does one N x M x M product.  Same engine as fw_grad_transform.
 *   fw_whiten_forward   Y  = (X - 1 mu^T) T^T      (Eq. 11), X, Y: rows x M fp32
 *   fw_whiten_backward  dX = dY T                   (Eq. 14), dY, dX: rows x M fp32
 * with the layer's current mu and T.  Outputs may not overlap inputs.
 * fw_whiten_backward builds T (the library keeps T^T) in the Gram scratch of
 * the layer's workspace. */
fw_status fw_whiten_forward(fw_layer* L, const float* X, int64_t rows, float* Y);
fw_status fw_whiten_backward(fw_layer* L, const float* dY, int64_t rows, float* dX);

/* SGD step W <- W - lr G_t, b <- b - lr g_b (Eqs. 27-28; the bias gradient is
 * not transformed).  g_b and b may both be NULL to skip the bias. */
fw_status fw_step(fw_layer* L, float* W, float* b, const float* G_t, const float* g_b, float lr);

/* SGD with momentum and weight decay, the optimiser of the paper's experiments
 * (Sec. 6: momentum 0.9, weight decay 5e-4 / 1e-4), applied to the transformed
 * gradient:  v <- momentum v + (G_t + weight_decay W),  W <- W - lr v, and the
 * same for the bias with its untransformed gradient (no decay on the bias).
 * vW (N x M) and vb (N) are the caller's velocity buffers, zero before the
 * first step; b, g_b, vb may all be NULL.  momentum = weight_decay = 0 is fw_step. */
fw_status fw_step_momentum(fw_layer* L, float* W, float* b, const float* G_t, const float* g_b, float* vW,
                           float* vb, float lr, float momentum, float weight_decay);

/* Whitening from the eigenvalue decomposition (Sec. 2, Eqs. 7-10; Sec. 3.2,
 * Eqs. 32, 34, 35): the direct construction the recursion of Sec. 4 replaces.
 * Phi_x = V Lambda V^T is computed on the device (one-sided block Jacobi rotations
 * in fp64, all layers of a group in one cooperative launch) and the layer's state is
 * set to  T = V diag(sqrt g) V^T (the symmetric, "ZCA" whitening matrix, Eq. 9),
 * Q = T^T T, Phi_y = T Phi_x T^T, Qs <- beta Qs + (1 - beta) Q (Eq. 35), with gains
 *   g_max <= 0:  g_m = 1 / max(lambda_m, eps)                            (Eq. 10)
 *   g_max  > 0:  g_m = min(1 / (M lbar_m), g_max) for the Ms_hat largest
 *                eigenvalues, 1 for the others, lbar = lambda / sum lambda,
 *                Ms_hat = round(exp(-sum lbar log lbar)) in [1, M]      (Eqs. 32, 34;
 *                Eq. 32 in the reading that gives M for equal eigenvalues and 1
 *                for a single dominant one, as the text states).
 * Eigenvalues of at most 1e-13 of the largest are not told from zero (the fp32
 * Phi_x carries rounding far above that): they have no direction of their own
 * and share, on the subspace the other eigenvectors leave, the gain of lambda = 0.
 * With Eq. 10 that gain is 1 / eps, also where eps is smaller than they are.
 * The gradient transform, the step and a later fw_cond_reduce continue from this
 * state.  scratch: caller-owned device memory, 256-byte aligned, at least
 * fw_evd_scratch_bytes(M) bytes per layer, used only during the call's kernels.
 * Cost: about 5 M^3 fp64 operations per sweep and 6-14 sweeps (10 for M = 576, fewer
 * for graded matrices; up to 40 where Phi_x is not safely positive definite: then
 * its Cholesky factor is no start); M / 16 - 1
 * barriers of the layer's CTAs per sweep (bounded waits; a time-out is reported
 * by fw_layer_sync_status as FW_ERR_TIMEOUT).  Errors: FW_ERR_STATE without a
 * covariance or inside an open block, FW_ERR_WORKSPACE for a short scratch. */
size_t fw_evd_scratch_bytes(int32_t M);
fw_status fw_evd_whiten(fw_layer* L, void* scratch, size_t scratch_bytes, float g_max);
fw_status fw_group_evd_whiten(fw_layer* const* L, int32_t n, void* const* scratch, const size_t* scratch_bytes,
                              float g_max);

/* Eigenvalues of Phi_x (which = 0) or Phi_y (which = 1) in decreasing order to
 * lam_out (M device floats, may be NULL) and the normalised rank of Sec. 6,
 * kappa = exp(-sum lbar log lbar) / M, to kappa_out (one device float, may be
 * NULL).  Same decomposition and scratch as fw_evd_whiten; the layer's state is
 * not changed (Phi_y is brought up to date first when it is stale). */
fw_status fw_spectrum(fw_layer* L, int32_t which, void* scratch, size_t scratch_bytes, float* lam_out,
                      float* kappa_out);

/* Whiteness of the transformed input (Sec. 6, Eq. 51):
 * rho = M / sum_{m,m'} Phi_y[m][m']^2 / (Phi_y[m][m] Phi_y[m'][m']), the sum over
 * all pairs (1 for a diagonal Phi_y, 1/M for fully correlated features).
 * Writes one float to rho_out (device).  Requires a covariance. */
fw_status fw_whiteness(fw_layer* L, float* rho_out);

/* Grouped forms: the same operations over n layers in one launch sequence.
 * All arrays are HOST arrays of length n; the pointers inside are device
 * pointers.  n <= FW_MAX_GROUP; all layers must share a stream. */
#define FW_MAX_GROUP 64
fw_status fw_group_cov_update(fw_layer* const* L, int32_t n, const void* const* X,
                              const int64_t* rows, const int64_t* ldx, uint32_t flags);
fw_status fw_group_cond_reduce(fw_layer* const* L, int32_t n, int32_t K, int32_t P,
                               float* const* traces_or_null);
/* Fused (c): W <- W - lr (G Qs), b <- b - lr g_b for every layer.  b / g_b
 * tables may be NULL. */
fw_status fw_group_grad_transform_step(fw_layer* const* L, int32_t n, const float* const* G,
                                       float* const* W, float* const* b,
                                       const float* const* g_b, float lr);

/* First-block mean and covariance of `rows` patch rows without any workspace:
 * mu_out[M] = column means, phix_out[M x M] = (1/rows) sum (x - mu)(x - mu)^T,
 * i.e. what fw_cov_update leaves in FW_F_MU / FW_F_PHIX on a fresh layer.
 * (The paper has no counterpart for this entry point; it exists for callers
 * that cannot allocate.)  X: rows x M fp32, row-major, leading dimension ldx;
 * mu_out, phix_out: device fp32; cuda_stream: a cudaStream_t, may be 0.
 *
 * For callers that may not allocate device memory and therefore cannot give a
 * layer its workspace -- e.g. a hook running inside a framework whose caching
 * allocator owns the whole device, where a raw cudaMalloc would synchronise the
 * device and may fail.  The call allocates nothing, neither on the device nor
 * through any library: its split partial sums go to a fixed 8 MiB array inside
 * the library image, which every GPU that loads the library holds until the
 * process exits.
 *  - M <= FW_STATIC_MAX_M; a larger M returns FW_ERR_SHAPE with a message.
 *  - The first call on each device resolves the array's device address (with
 *    that device current); make that first call before any stream capture.
 *  - All calls share the one array, and it keeps the previous call's contents.
 *    Every slot a call reads it has written first, so nothing needs clearing,
 *    but two calls that overlap on the GPU (different streams, or different
 *    host threads) race on it: serialise them. */
#define FW_STATIC_MAX_M 256
fw_status fw_cov_block_static(const float* X, int64_t rows, int64_t ldx, int32_t M, float* mu_out,
                              float* phix_out, void* cuda_stream);

/* ---- Operators around the layers: what makes a layer's input and its gradient.
 * They keep no state.  rows >= 1; ld* are leading dimensions in elements, at most
 * 2^30.  Any alignment to whole elements is taken; where every matrix starts on 16
 * bytes and its rows are a multiple of 16 bytes apart, 16 bytes move at a time.  Of
 * inputs the aligned word or 16 bytes that hold an element may be read whole: up to
 * 15 bytes before a matrix and 2 behind it are read, never used.
 * Sums are fp32 in a fixed order: the same call gives the same bits. ---- */

/* Residual addition and root-mean-square norm, a transform of layer inputs like
 * fw_whiten_forward / _backward that needs no statistics across rows:
 *   s = x + res, rounded to `dtype` (s = x without res)
 *   rstd = 1 / sqrt(mean(s^2) + eps),  y = s rstd w
 * y is of `dtype`, or e4m3 with a scale for each row: y_scale = max|y| / 448 (at
 * least 2^-120; 1 for a row of zeros), y held as e4m3(y / y_scale).
 * x, res, sum: rows x M of `dtype`; w: M fp32; rstd, y_scale: rows fp32.
 *   res      NULL: no addition          sum   NULL: s is not kept; needs res
 *   y_scale  only, and always, with e4m3  rstd  NULL: not kept
 * sum and y may be x or res themselves (same address, type and ld); any other overlap
 * of outputs with inputs or with each other is FW_ERR_INVALID_ARG.
 * 1 <= M <= 16384.  A NaN or infinity in a row makes that row's y, rstd and
 * scale what the formulas give, and no other's.  The squares are added in fp32: where they pass
 * 3.4e38 (an |s| of 1.8e19, or of 2.9e17 in each of 4096 places) the sum is infinite and rstd and y are 0.
 * An e4m3 row is made from s w: where |s w| passes 3.4e38 its scale is infinite. */
typedef struct {
  int32_t M;         /* features                                                 */
  int32_t dtype;     /* fw_dtype of x, res, sum: FW_F32 or FW_BF16                */
  int32_t y_dtype;   /* dtype, or FW_E4M3 (forward)                              */
  float eps;         /* > 0                                                      */
} fw_norm_desc;
/* bf16 in and out, eps 1e-6 */
void fw_norm_desc_default(fw_norm_desc* d, int32_t M);
fw_status fw_rmsnorm_forward(const fw_norm_desc* d, int64_t rows, const void* x, int64_t ldx, const void* res,
                             int64_t ldr, const float* w, void* sum, int64_t lds, void* y, int64_t ldy,
                             float* y_scale, float* rstd, void* cuda_stream);
/* From dy (the gradient of y), s and rstd of the forward call:
 *   u = dy w,  n = s rstd,  dx = rstd (u - n mean(u n)) + dsum,  dw = sum over rows of dy n
 * dx is the gradient of x and of res alike; dsum (NULL: none) is the gradient that
 * reaches s by itself.  dy, s, dsum, dx: rows x M of `dtype` (y_dtype is not looked
 * at: the gradient passes an e4m3 rounding unchanged).  dw: M fp32, overwritten;
 * NULL: not wanted, and scratch may be NULL.  scratch: caller-owned, 256-byte aligned, at
 * least fw_rmsnorm_scratch_bytes(d) bytes, free again when the call's work is done.
 * dx may be dy, s or dsum itself. */
size_t fw_rmsnorm_scratch_bytes(const fw_norm_desc* d);
fw_status fw_rmsnorm_backward(const fw_norm_desc* d, int64_t rows, const void* dy, int64_t lddy, const void* s,
                              int64_t lds, const void* dsum, int64_t ldds, const float* w, const float* rstd, void* dx,
                              int64_t lddx, float* dw, void* scratch, size_t scratch_bytes, void* cuda_stream);

/* Gated feed-forward block: two layers of the same input, one gating the other,
 *   Zg = X Wg^T + bg,  Zu = X Wu^T + bu,  H = act(Zg) Zu (element by element)
 * Both projections, the activation and the product are one kernel on the tensor
 * cores (tcgen05, fp32 accumulation).  The backward call gives what fw_cov_update's companions take:
 * dWg, dWu are the gradients G of the layers (Wg, bg) and (Wu, bu), dbg, dbu their g_b.
 * X: rows x M, Wg, Wu: N x M, H, Zg, Zu: rows x N.
 *   FW_BF16  X, weights, outputs bf16
 *   FW_E4M3  X and weights e4m3 with a scale for each row of X (x_scale) and each row of
 *            Wg, Wu (wg_scale, wu_scale); H, Zg, Zu bf16; forward only
 * Scales and biases are fp32.  1 <= M, N <= 32768, 1 <= rows <= 2^26.  Every matrix but dWg, dWu starts on 16 bytes
 * and has rows a multiple of 16 bytes apart (M and N may be any).
 * Like a layer the block is a host object over caller-supplied device memory with a
 * stream of its own: calls on one block are not for several threads at once, and its
 * workspace belongs to the work in flight on its stream (two graphs that may run at
 * the same time take two blocks). */
typedef struct fw_gated fw_gated;
typedef enum {
  FW_ACT_SILU = 0,      /* a / (1 + exp(-a))                                      */
  FW_ACT_GELU = 1,      /* a (1 + erf(a / sqrt 2)) / 2                            */
  FW_ACT_GELU_TANH = 2, /* a (1 + tanh(sqrt(2 / pi) (a + 0.044715 a^3))) / 2      */
  FW_ACT_RELU = 3       /* max(a, 0); derivative 0 at 0                           */
} fw_act;
typedef struct {
  int32_t M, N;
  int32_t x_dtype;      /* FW_BF16 or FW_E4M3                                     */
  int32_t act;          /* fw_act                                                 */
  int32_t grad;         /* 1: the workspace has room for backward calls (bf16)    */
  int64_t max_rows;     /* grad: largest rows of a backward call                  */
} fw_gated_desc;
/* bf16, SiLU, no backward calls */
void fw_gated_desc_default(fw_gated_desc* d, int32_t M, int32_t N);
/* 0 if the description is invalid */
size_t fw_gated_workspace_bytes(const fw_gated_desc* d);
/* The workspace (256-byte aligned) outlives the block; on the current device. */
fw_status fw_gated_create(const fw_gated_desc* d, void* dev_workspace, size_t bytes, void* cuda_stream, fw_gated** out);
fw_status fw_gated_destroy(fw_gated* g);
/* Zg, Zu: both or (where no backward call follows) neither.  bg, bu: both or neither.
 * x_scale, wg_scale, wu_scale: with e4m3, and only then.  Outputs overlap nothing. */
fw_status fw_gated_forward(fw_gated* g, const void* X, int64_t rows, int64_t ldx, const float* x_scale, const void* Wg,
                           const void* Wu, int64_t ldw, const float* wg_scale, const float* wu_scale, const float* bg,
                           const float* bu, void* H, int64_t ldh, void* Zg, void* Zu, int64_t ldz);
/* From dH, the forward call's inputs and its Zg, Zu:
 *   da = dH Zu act'(Zg), db = dH act(Zg) (both rounded to bf16 for the products)
 *   dX = da Wg + db Wu (bf16; NULL: not wanted, and Wg, Wu may be NULL)
 *   dWg = da^T X, dWu = db^T X (both or neither; dense N x M of dw_dtype, FW_F32 as the layers'
 *   calls take them, or FW_BF16; X may be NULL without them)
 *   dbg, dbu = sums of da, db over the rows before they are rounded (both or neither)
 * Outputs are overwritten.  FW_ERR_WORKSPACE for a block made without grad, FW_ERR_SHAPE for more
 * than max_rows. */
fw_status fw_gated_backward(fw_gated* g, const void* dH, int64_t rows, int64_t lddh, const void* X, int64_t ldx,
                            const void* Wg, const void* Wu, int64_t ldw, const void* Zg, const void* Zu, int64_t ldz,
                            void* dX, int64_t lddx, void* dWg, void* dWu, int32_t dw_dtype, float* dbg, float* dbu);
/* Waits for the block's stream; FW_ERR_TIMEOUT if a bounded device-side wait gave up since the last
 * call (what the calls since then wrote is not to be used). */
fw_status fw_gated_sync_status(fw_gated* g);

/* Distillation loss against a teacher's top logits, and its gradient (what the weight
 * gradient of a network's last layer is formed from).  With q = softmax(Z / tau) of a
 * row and the K classes i_k that the teacher names, with its logits t_k:
 *   t_lse NULL: p = softmax(t / tau) over the named classes, p_t = 0
 *   t_lse     : p_k = exp(t_k / tau - t_lse), t_lse = the teacher's log sum exp(t / tau) over
 *               all V classes; p_t = max(0, 1 - sum p) for all classes it does not name
 *   loss = weight [sum_k p_k (log p_k - log q_ik) + p_t (log p_t - log q_t)]
 * where q_t is the student's mass on the classes that are not named, and dZ = d loss / dZ.
 * (Where a factor tau^2 is wanted it goes into weight, like the mean over rows.)
 *   Z, dZ   rows x V, z_dtype; dZ may be Z (same address and ld), no other overlap
 *   T, I    rows x K, dense: the teacher's logits (t_dtype), their classes (index_bits 32 or 64
 *           bits, signed).  A class outside [0, V) marks an absent entry; a class named twice counts
 *           once, with its first logit.
 *   weight  rows; NULL: 1.  A row of weight 0 is not read: loss, stat and dZ are 0.
 *   loss    rows;   stat  rows x 2: log sum exp(Z / tau) over all classes and over those not
 *           named (-inf for none); NULL in the forward call: not kept
 * forward: dZ NULL gives the loss alone; with dZ the gradient too, from the same pass over Z.
 * backward: the gradient from the forward call's stat (weight may be another, but a row that the
 * forward call left out has no stat to be read).  fp32 holds a stat beyond 1024 too coarsely for exponentials, and of
 * one at -3e38 nothing: such a row's sums are formed again from Z, without speed.
 * Logits of -inf have no mass (a mask): gradient 0, infinite loss where p_k > 0.  A row in which no
 * class has mass gives loss and gradient 0, and so does a row whose entries are all absent (t_lse
 * NULL).  The lowest finite value is a logit like any other: a row of it alone is flat.  A NaN in a
 * row, or +inf, makes that row's loss and gradient NaN.
 * Nothing keeps a status: where a bounded device-side wait gave up, rows that may not
 * be finished have NaN in their loss and among the elements of their gradient.
 * 1 <= K <= 1024, K <= V <= 2^20, rows < 2^28. */
typedef struct {
  int32_t V, K;
  int32_t z_dtype, t_dtype;   /* FW_F32 or FW_BF16                               */
  int32_t index_bits;         /* 32 or 64                                        */
  float tau;                  /* 1e-6 to 1e6                                     */
} fw_distill_desc;
/* bf16 logits, 32-bit classes, tau 1 */
void fw_distill_desc_default(fw_distill_desc* d, int32_t V, int32_t K);
fw_status fw_distill_forward(const fw_distill_desc* d, const void* Z, int64_t rows, int64_t ldz, const void* T,
                             const void* I, const float* t_lse, const float* weight, float* loss, float* stat,
                             void* dZ, int64_t lddz, void* cuda_stream);
fw_status fw_distill_backward(const fw_distill_desc* d, const void* Z, int64_t rows, int64_t ldz, const void* T,
                              const void* I, const float* t_lse, const float* weight, const float* stat, void* dZ,
                              int64_t lddz, void* cuda_stream);

/* State access (checkpointing, injecting a covariance, parity checks).
 * Matrices are M x M fp32 row-major, vectors M fp32, FW_F_LAMBDA_BAR one fp32.
 * Copies run on the layer's stream.  Setting FW_F_PHIX marks Phi_y stale, sets
 * lam_bar = trace(Phi_x)/M and counts as a first block having been seen;
 * setting FW_F_T also recomputes Q = T^T T and marks Phi_y stale. */
typedef enum {
  FW_F_MU = 0, FW_F_PHIX = 1, FW_F_PHI_DIAG = 2, FW_F_LAMBDA_BAR = 3,
  FW_F_T = 4, FW_F_Q = 5, FW_F_QS = 6, FW_F_PHIY = 7,
  FW_F_ALIGN_W = 8 /* get only: alignment weights of the last step, 1/c_m on the coherent set, else 0 */
} fw_field;
fw_status fw_layer_get(fw_layer* L, fw_field f, void* dev_dst, size_t bytes);
fw_status fw_layer_set(fw_layer* L, fw_field f, const void* dev_src, size_t bytes);

/* Waits for the layer's stream, then returns (and clears) the first
 * device-side condition recorded since the last call, or FW_OK. */
fw_status fw_layer_sync_status(fw_layer* L);

const char* fw_status_string(fw_status s);

/* Test aid for the time-out path (the paper has no counterpart).  Enqueues on
 * the layer's stream a one-warp kernel that waits on a barrier nothing arrives
 * on, with the same bounded wait the tensor-core pipelines use but a limit of
 * `polls` polls (1 .. 65536, microseconds in all).  The wait gives up, the
 * kernel records it in the layer's status word and returns normally, so the
 * next fw_layer_sync_status returns FW_ERR_TIMEOUT and the layer stays usable.
 * Nothing traps and nothing hangs. */
fw_status fw_debug_wait_probe(fw_layer* L, uint32_t polls);

/* Per-kernel-class device timing (a tracing aid; the paper has no counterpart).
 * Between fw_profile_begin and fw_profile_end every kernel launch of the
 * library is bracketed by CUDA events on its stream.  fw_profile_end waits for
 * them and writes, per class, the summed device time in milliseconds and the
 * number of launches into HOST arrays of length FW_PROF_CLASSES (either may be
 * NULL).  Off by default; event recording perturbs back-to-back launches a
 * little, so whole-step timings are taken with profiling off. */
typedef enum {
  FW_PROF_PILOT = 0,    /* pilot column means                         */
  FW_PROF_GRAM = 1,     /* X^T X + column sums                        */
  FW_PROF_MOMENTS = 2,  /* split reduction, centring, running average */
  FW_PROF_RESYNC = 3,   /* T Phi_x T^T products                       */
  FW_PROF_RECUR_MV = 4, /* matrix-vector passes of the recursion      */
  FW_PROF_RECUR_UPD = 5,/* rank-update pass over Q, T, Phi_y          */
  FW_PROF_SMOOTH = 6,   /* Qs update                                  */
  FW_PROF_GQ = 7,       /* G Qs (+ SGD epilogue)                      */
  FW_PROF_MISC = 8,
  FW_PROF_RECUR_CHIP = 9, /* whole K-step recursion of small layers, on chip */
  FW_PROF_CLASSES = 10
} fw_prof_class;
fw_status fw_profile_begin(void);
fw_status fw_profile_end(float* ms_per_class, int64_t* launches_per_class);

/* Tuning aids: environment variables read once, when the first call needs them.
 * None changes results; they exist for measurements.
 *   FW_PAIR_MIN_M   smallest M the CTA-pair Gram / re-sync kernels take (default 289)
 *   FW_PAIR_SPLITS  row slabs per problem of the CTA-pair kernels (default: chosen by the scheduler)
 *   FW_PAIR_DEBUG   print the chosen slabs to stderr
 *   FW_PASS_SHAPE   42 / 24 / 18 / 41: shape of the streaming recursion passes (default: by row-block count)
 *   FW_GRAM_WAVES_PCT  CTAs of a single-CTA Gram launch in percent of the SM count (default 200: two waves) */

/* 1 when fw_cond_reduce keeps this layer's Phi_y in distributed shared memory
 * for all K steps of a call (M <= 624, gamma = 1); 0 when a team of CTAs keeps it
 * in shared memory as far as it fits and exchanges results through L2 (larger M,
 * gamma = 1) or every pass is a launch that reads it from HBM (gamma < 1).
 * Reporting aid: the paths are bound by different things. */
int32_t fw_recursion_on_chip(const fw_layer_desc* d);

/* Number of kernels this library has launched since it was loaded. */
int64_t fw_launch_count(void);

/* Library version (major * 100 + minor). */
int32_t fw_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FW_H_ */
