/*
 * scalify.h - C ABI of the B200 (sm_100a) scaled-array kernels.
 *
 * The operations are the scaled primitives of "Scalify: scale propagation for
 * efficient low-precision LLM training" (arxiv 2407.17353).  A ScaledArray is
 * a pair (data, scale) whose value is data * scale (Section 2).  Here `data`
 * is a device buffer in a low-precision format and `scale` is ONE fp32 power
 * of two kept in DEVICE memory (Section 2: E8M0 scale simulated in float32;
 * Section 3.1: scalar scale per tensor).  Every scale this library writes is a
 * power of two obtained by rounding DOWN (Section 3.2, last paragraph).
 *
 * General contract
 *   - All `scalify_array.data`, `.scale`, workspace, statistic, mean/rinv
 *     pointers are DEVICE pointers owned by the caller.  The library
 *     allocates no device memory and frees nothing.  Descriptor structs and
 *     the arrays of descriptors passed to the Adam call are HOST memory and
 *     are read before the call returns.
 *   - `stream` is a cudaStream_t passed as void* (NULL = default stream).
 *     Calls only enqueue work; they never synchronise, except
 *     scalify_check_status.
 *   - A NULL `scale` pointer on an INPUT means "unscaled array", scale 1
 *     (Section 3.1, get_data_and_scale).  A NULL `scale` on an OUTPUT means
 *     the propagated scale is not stored.
 *   - Input scale words must be finite positive powers of two within
 *     [2^-126, 2^126]; a violation detected on the device sets
 *     SCALIFY_DEV_BAD_SCALE in the workspace status word where a workspace
 *     is available.
 *   - Layout: row-major, `shape[0..ndim-1]` outermost first, `stride[]` in
 *     elements, innermost stride 1, data pointer 16-byte aligned and every
 *     outer stride a multiple of 16 bytes.
 *   - An output scale word must not alias an input scale word of the same
 *     call unless a function says otherwise (SCALIFY_ERR_ALIAS).
 *   - Return value: 0 on success, a negative scalify_error otherwise.  A call
 *     that fails validation enqueues nothing.  No call aborts, throws, or
 *     traps on the device; every device-side wait is bounded and reports
 *     SCALIFY_DEV_TIMEOUT in the status word when it expires.
 *   - Rounding: data are converted round-to-nearest-even; FP8 conversions
 *     saturate to the largest finite value; subnormals are kept.
 */
#ifndef SCALIFY_H_
#define SCALIFY_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SCALIFY_E4M3 = 0, /* OCP FP8 E4M3 (finite only, max 448)  - forward operands (Section 1, Appendix A) */
  SCALIFY_E5M2 = 1, /* OCP FP8 E5M2 (max 57344)             - backward gradients (Section 1, Appendix A) */
  SCALIFY_F16 = 2,  /* IEEE binary16 */
  SCALIFY_BF16 = 3, /* bfloat16 */
  SCALIFY_F32 = 4   /* IEEE binary32 */
} scalify_dtype;

typedef enum {
  SCALIFY_STAT_NONE = 0,
  SCALIFY_STAT_AMAX = 1, /* max |data| */
  SCALIFY_STAT_L2 = 2    /* sqrt(mean(data^2)), the "L2 moment" of Section 3.3 */
} scalify_stat;

typedef enum {
  SCALIFY_OK = 0,
  SCALIFY_ERR_NULL = -1,        /* a required pointer is NULL */
  SCALIFY_ERR_DTYPE = -2,       /* dtype not valid for this argument */
  SCALIFY_ERR_SHAPE = -3,       /* shapes inconsistent or out of range */
  SCALIFY_ERR_ALIGNMENT = -4,   /* pointer or stride not 16-byte aligned, innermost stride not 1 */
  SCALIFY_ERR_WORKSPACE = -5,   /* workspace missing or too small */
  SCALIFY_ERR_UNSUPPORTED = -6, /* valid but not implemented combination */
  SCALIFY_ERR_CUDA = -7,        /* a CUDA runtime/driver call failed (see scalify_last_cuda_error) */
  SCALIFY_ERR_ALIAS = -8,       /* forbidden aliasing of scale words or buffers */
  SCALIFY_ERR_VALUE = -9        /* scalar argument out of range */
} scalify_error;

/* Bits of the device status word (first 4 bytes of any workspace). */
enum {
  SCALIFY_DEV_TIMEOUT = 1u,        /* a bounded device-side wait expired; results of that call are invalid */
  SCALIFY_DEV_BAD_SCALE = 2u,      /* an input scale word was not a finite positive power of two */
  SCALIFY_DEV_NONFINITE_STAT = 4u, /* a statistic was NaN or Inf; the rescale used factor 1 */
  SCALIFY_DEV_BAD_INDEX = 8u       /* a token id or target was out of range (treated as 0) */
};

typedef struct scalify_array {
  void* data;        /* device pointer, 16-byte aligned */
  int32_t dtype;     /* scalify_dtype */
  int32_t ndim;      /* 1..4 (4: only the attention calls, [batch, heads, T, hd]) */
  int64_t shape[4];  /* outermost first; unused entries ignored */
  int64_t stride[4]; /* in elements; stride[ndim-1] must be 1 */
  float* scale;      /* device pointer to one fp32 power of two, or NULL */
} scalify_array;

/* Operation codes for scalify_workspace_bytes. */
enum {
  SCALIFY_OP_MATMUL = 0,        /* d0 = batch*M, d1 = N */
  SCALIFY_OP_RESCALE = 1,       /* d0 = number of elements, d1 unused */
  SCALIFY_OP_LAYERNORM_BWD = 2, /* d0 = rows, d1 = row length */
  SCALIFY_OP_ADAM = 3,          /* d0 = number of tensors, d1 unused */
  SCALIFY_OP_STATISTIC = 4,     /* d0 = number of elements */
  SCALIFY_OP_CROSS_ENTROPY = 5, /* d0 = number of rows */
  SCALIFY_OP_COLSUM = 6,        /* d0 = rows, d1 = columns */
  SCALIFY_OP_MATMUL_SPLITK = 7, /* d0 = M, d1 = N: room for the partial products of a split contraction */
  SCALIFY_OP_RMSNORM_BWD = 8,   /* d0 = rows, d1 = row length */
  SCALIFY_OP_EMBEDDING_GRAD = 9 /* d0 = number of tokens, d1 = row length */
};

/* Bytes of workspace the given call needs (an upper bound; always >= 4096).
 * The first 256 bytes of a workspace form a header (status word, statistic
 * word, reduction tickets); scalify_workspace_init must have zeroed it once
 * before first use.  One workspace may serve successive calls on one stream;
 * two calls that may overlap on the GPU need separate workspaces.
 * For SCALIFY_OP_RESCALE and SCALIFY_OP_STATISTIC the figure grows with d0
 * (one fp64 partial per block of the statistic pass, at most 512 KiB); those
 * two calls also accept any smaller workspace of at least 4096 bytes and
 * then run the statistic pass with fewer, longer blocks (same result for
 * AMAX; for L2 the fp64 partial sums are combined in a different grouping). */
size_t scalify_workspace_bytes(int op, int64_t d0, int64_t d1);

/* Zero the workspace header (asynchronously, on `stream`). */
int scalify_workspace_init(void* workspace, size_t workspace_bytes, void* stream);

/* Synchronise `stream`, read and clear the status word of `workspace`.
 * Returns the SCALIFY_DEV_* bits (>= 0) or a negative scalify_error. */
int scalify_check_status(void* workspace, void* stream);

const char* scalify_status_string(int code);
/* The cudaError_t value recorded by the last call that returned SCALIFY_ERR_CUDA (per host thread). */
int scalify_last_cuda_error(void);
int scalify_version(void);

/*
 * Scaled matrix multiply (Section 3.2, the matmul rule of Algorithm 3; the
 * mixed-format FP8 operands and higher-precision output of Appendix A).
 *
 *   Y_s = A_s * B_s * kf(K),   Y_d = (op(A)_d . op(B)_d) / kf(K)
 *
 * with kf(K) = sqrt(K) rounded down to a power of two: under the paper's
 * assumption of independent unit-variance operands the contraction has
 * variance K, so dividing the data by kf(K) restores unit scale, and the
 * output scale depends only on the operand scales and the shape.
 *
 *   A : FP8 (E4M3 or E5M2), [M,K] (or [K,M] when transA != 0), ndim 2, or
 *       ndim 3 with a leading batch dimension.
 *   B : FP8 (E4M3 or E5M2, may differ from A), [K,N] (or [N,K] when transB).
 *       A 2-D B with a 3-D A is shared by all batches.
 *   Y : BF16, F16 or F32, [M,N] (or [batch,M,N]); receives the fp32
 *       accumulator times 1/kf(K), rounded once.  Y->scale receives Y_s.
 *   stat: statistic of the STORED Y data gathered in the epilogue (Section
 *       3.3).  SCALIFY_STAT_NONE: none.  Otherwise the statistic is left, as
 *       one fp32, at byte offset 16 of the workspace.
 *   Yq: optional (may be NULL; requires stat != NONE).  Receives the dynamic
 *       rescale of Y: r = statistic rounded down to a power of two,
 *       Yq_d = cast(Y_d / r), Yq_s = Y_s * r.  Any dtype; same shape as Y.
 *
 * Predicted rescale (Section 3.3: statistic and rebalancing are separate
 * primitives).  With stat = AMAX, a BF16/F16 Y, an FP8 Yq of its own and rows
 * of a multiple of 16 elements, the GEMM's epilogue already writes Yq with
 * the power of two of the statistic this workspace saw last (fp32 word at
 * byte offset 56 of the workspace), and the launch that follows rebuilds Yq
 * from Y only if this call's statistic has another power of two.  Y, Yq, both
 * scale words and the statistic word are the same bits either way and for any
 * content of that word; the call leaves its own statistic there.  Keep one
 * workspace per matmul of a training step for the prediction to hold.
 *
 * Y == NULL (FP8 output only): allowed with stat = AMAX and an FP8, contiguous
 * Yq with its own scale word and rows of a multiple of 16 elements.  The
 * values are still rounded to BF16 first and the statistic is still that of
 * the BF16 values, so Yq, Yq_s and the statistic word equal those of the call
 * with a BF16 Y bit for bit, but the intermediate is not stored: the epilogue
 * writes Yq with the predicted power of two, and a second launch of the same
 * kernel, whose thread blocks return at once when the prediction held,
 * computes the product again otherwise.  Never splits the contraction.
 *
 * Accumulation is fp32 on the tensor cores (tcgen05, kind::f8f6f4).  Row
 * strides must be multiples of 16 bytes.  Errors: see scalify_error.
  *
 * Split contraction: when the output has few tiles and K >= 2048 (a weight
 * gradient), and the workspace is at least scalify_workspace_bytes(
 * SCALIFY_OP_MATMUL_SPLITK, M, N), the K range is cut into up to 16 parts that
 * run as one batched launch writing fp32 partial products into the workspace; a
 * second launch adds them in a fixed order, rounds once and takes the statistic.
 * With the smaller SCALIFY_OP_MATMUL workspace the call never splits.  Results
 * of the two forms agree within the accumulation bar, not bit for bit.
 */
int scalify_scaled_matmul(const scalify_array* A, int transA, const scalify_array* B, int transB,
                          scalify_array* Y, int stat, scalify_array* Yq,
                          void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same product with a bias vector added in the kernel's epilogue (a linear
 * layer): the add rule applied to the product and the bias, rounded ONCE:
 *   Y_s = max(A_s B_s kf(K), bias_s)
 *   Y_d = (A_d B_d) / kf(K) * (A_s B_s kf(K) / Y_s)  +  bias_d[j] * (bias_s / Y_s)
 * (both factors are exact powers of two).  bias: [N], F16, BF16 or F32, contiguous.
 * Y may be F16, BF16, F32 or, as a static cast of the sum, E4M3 / E5M2.  stat, Yq,
 * workspace as for scalify_scaled_matmul; the contraction is never split.  The
 * unfused sequence (matmul, then scalify_scaled_add with the bias) rounds twice;
 * this call is its value with one rounding.
 * Errors: as scalify_scaled_matmul; NULL (no bias), DTYPE (bias not wide), SHAPE.
 */
int scalify_scaled_matmul_bias(const scalify_array* A, int transA, const scalify_array* B, int transB,
                               const scalify_array* bias, scalify_array* Y, int stat, scalify_array* Yq,
                               void* workspace, size_t workspace_bytes, void* stream);

/*
 * scalify_scaled_matmul with stat = AMAX and a rebalanced FP8 output, made cheaper by a PREDICTION of the
 * statistic (Section 3.3 observes that statistics change slowly, which is what delayed rescaling exploits;
 * here the result stays that of the exact dynamic rescale).  *stat_hint (DEVICE) holds a predicted
 * statistic, typically the one this call produced last step.  The GEMM writes the 16-bit intermediate Y
 * and, in the same epilogue, Yq = fp8(stored Y / r_pred) with r_pred = the hint rounded down to a power of
 * two (1 if the hint cannot define a scale).  A second, small launch compares r_pred with the power of two
 * of the TRUE statistic of Y: if they agree (the common case) Yq is already the exact result and only its
 * scale word is written; if not, Yq is rebuilt from Y as scalify_scaled_matmul would.  Either way Y, Yq,
 * both scale words and the statistic word are bit-identical to scalify_scaled_matmul(..., AMAX, Yq), and
 * *stat_hint is overwritten with this call's statistic.  In the common case the separate pass over Y
 * (2 bytes read + 1 written per element) is replaced by 1 extra written byte per element in the GEMM.
 *   Y: F16 or BF16, contiguous; Yq: E4M3 or E5M2, contiguous, same shape; other arguments and errors as
 *   scalify_scaled_matmul; SCALIFY_ERR_NULL if stat_hint or Yq is NULL.
 */
int scalify_scaled_matmul_speculative(const scalify_array* A, int transA, const scalify_array* B, int transB,
                                      scalify_array* Y, scalify_array* Yq, float* stat_hint, void* workspace,
                                      size_t workspace_bytes, void* stream);

/*
 * Scaled matrix multiply with DELAYED rescaling (Section 3.3: "Delayed rescaling can be
 * similarly implemented by decoupling the compute of statistics and rebalancing ..., keeping
 * track of the first one in the model state").  One kernel, no intermediate, no second pass:
 *
 *   r   = *stat_in rounded down to a power of two (1 if *stat_in is zero, below 2^-126 or
 *         non-finite): the statistic of an EARLIER step, kept by the caller on the device;
 *   Y_d = cast((op(A)_d . op(B)_d) / kf(K) / r),   Y_s = A_s * B_s * kf(K) * r;
 *   *stat_out (and workspace offset 16) = statistic `stat` of THIS step's un-rebalanced fp32
 *         values (op(A)_d . op(B)_d)/kf(K), for the next step.
 *
 * Y may be FP8 (E4M3 / E5M2) as well as BF16 / F16 / F32.  stat_out may be NULL, and may be the
 * same word as stat_in (it is written after the kernel has finished).  stat = SCALIFY_STAT_NONE
 * gathers nothing (stat_out must then be NULL).  Other arguments as scalify_scaled_matmul.
 */
int scalify_scaled_matmul_delayed(const scalify_array* A, int transA, const scalify_array* B, int transB,
                                  const float* stat_in, scalify_array* Y, int stat, float* stat_out,
                                  void* workspace, size_t workspace_bytes, void* stream);

/*
 * Statistic of the data component of X (Section 3.3: "L2 moment (or any other
 * statistic)"), written as one fp32 to `out_stat` (device) and to byte offset
 * 16 of the workspace.  X may be any dtype, contiguous.
 */
int scalify_statistic(const scalify_array* X, int stat, float* out_stat,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * Rescaling family (Sections 3.1 and 3.3; Algorithm 4).  Y has the same shape
 * as X, any dtype; both contiguous.  Y may alias X (same buffer) only when the
 * two dtypes have the same size.
 *
 *   stat == AMAX or L2, new_scale == NULL, stat_in == NULL:
 *       dynamic_rescale: s = statistic(X_d); r = s rounded down to a power of
 *       two (r = 1 when s is zero, non-finite or below 2^-126);
 *       Y_d = cast(X_d / r); Y_s = X_s * r.  Needs a workspace.
 *   stat == AMAX or L2, stat_in != NULL (device fp32):
 *       delayed rescale: as above with s read from *stat_in instead of being
 *       computed (Section 3.3: statistic gathered elsewhere, kept in state).
 *   stat == NONE, new_scale != NULL (device fp32):
 *       set_scaling: s' = *new_scale rounded down to a power of two;
 *       Y_d = cast(X_d * X_s / s'); Y_s = s'.  With X->scale == NULL this is
 *       as_scaled_array of an unscaled input.  Y->scale must not alias X->scale.
 *   stat == NONE, new_scale == NULL:
 *       plain cast (cast_on_forward / cast_on_backward of Appendix A):
 *       Y_d = cast(X_d); Y_s = X_s.
 *
 * Y->scale may alias X->scale for the dynamic and delayed forms (in-place
 * rebalance of a state tensor).
 *
 * The dynamic form with an output buffer of its own reads X once when the power
 * of two can be predicted: while the statistic is gathered, Y is already written
 * with the power of two of the statistic this workspace saw last (fp32 word at
 * byte offset 56 of the workspace, any content), and X is read a second time
 * only if this call's statistic has another power of two.  Y, Y_s and the
 * statistic word do not depend on that word; the call leaves its statistic there.
 */
int scalify_rescale(const scalify_array* X, int stat, const float* new_scale, const float* stat_in,
                    scalify_array* Y, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Scaled add / subtract (Section 3.2, the add rule of Algorithm 3):
 *   Y_s = sqrt(A_s^2 + B_s^2) rounded down to a power of two (= max(A_s,B_s)),
 *   Y_d = cast(A_d*(A_s/Y_s) +- B_d*(B_s/Y_s)).
 * A: [M,N] (or any contiguous shape); B: same shape as A, or a vector [N]
 * broadcast over the rows of A (bias).  A and B: F16, BF16 or F32, same
 * dtype; Y any dtype.  Y may alias A's buffer when sizes match.
 */
int scalify_scaled_add(const scalify_array* A, const scalify_array* B, int subtract,
                       scalify_array* Y, void* stream);

/*
 * Scaled LayerNorm forward (Section 3.2.1 and Appendix C.2): the data
 * component is normalised and the result carries scale 1, whatever X_s is:
 *   n = (x_d - mean) / (sqrt(var) + eps)        (eps_inside_sqrt == 0, as printed)
 *   n = (x_d - mean) / sqrt(var + eps)          (eps_inside_sqrt != 0, textbook)
 * followed by the affine part through the ordinary mul and add rules:
 *   Y_s = max(gamma_s, beta_s),  Y_d = cast(n*gamma_d*(gamma_s/Y_s) + beta_d*(beta_s/Y_s)).
 * X: [R,d] F16/BF16/F32, d*elem_size a multiple of 16 bytes, d <= 16384.
 * gamma, beta: [d], same dtype as each other (F16/BF16/F32), or both NULL
 * (then Y_d = n, Y_s = 1).  Y: [R,d], any dtype.  mean, rinv: optional device
 * fp32 [R] outputs (row mean and 1/(sigma+eps) or 1/sqrt(var+eps)), needed by
 * the backward call.
 */
int scalify_scaled_layernorm(const scalify_array* X, const scalify_array* gamma, const scalify_array* beta,
                             float eps, int eps_inside_sqrt, scalify_array* Y,
                             float* mean, float* rinv, void* stream);

/*
 * Scaled LayerNorm backward with dynamic rescale of the input gradient
 * (Section 4 and Algorithm 5: one dynamic rescale per residual branch, placed
 * on the gradient that leaves the LayerNorm).
 *   ghat = G_d*gamma_d;  dx = LayerNorm'(ghat; x_d)  (exact derivative of the
 *   forward above);  dX_s = G_s*gamma_s / X_s;
 *   dgamma_d = sum_rows(G_d*n)/kf(R), dbeta_d = sum_rows(G_d)/kf(R), both with
 *   scale G_s*kf(R) (reduction over R rows treated like a contraction of size R).
 * G, X: [R,d], F16/BF16/F32 (same dtype); mean, rinv: from the forward call.
 * dX: [R,d] BF16/F16/F32: the un-rebalanced gradient (always written).
 * stat_dx: statistic of the stored dX data, left at workspace offset 16.
 * dXq: optional rescaled gradient (any dtype), as Yq of the matmul.
 * dgamma, dbeta: optional [d] outputs, F32/BF16/F16 (both or neither).
 *
 * dX == NULL (one pass, the un-rebalanced gradient is not stored): allowed with
 * stat_dx != NONE and a contiguous FP8 dXq.  The values are still rounded to
 * the dtype of X first and the statistic is still that of those rounded values,
 * so dXq, dXq_s, the statistic word, dgamma and dbeta equal those of the call
 * with a dX of X's dtype bit for bit; the gradient is written with the power
 * of two of the statistic this workspace saw last (fp32 word at byte offset 56
 * of the workspace, any content) and a second launch of the same kernel, whose
 * thread blocks return at once when that prediction held, writes it again
 * otherwise.  The call leaves its own statistic in that word: keep one
 * workspace per LayerNorm of a training step for the prediction to hold.
 * (Section 3.3: statistic and rebalancing are separate primitives.)
 */
int scalify_scaled_layernorm_bwd(const scalify_array* G, const scalify_array* X, const scalify_array* gamma,
                                 const float* mean, const float* rinv, float eps, int eps_inside_sqrt,
                                 int stat_dx, scalify_array* dX, scalify_array* dXq,
                                 scalify_array* dgamma, scalify_array* dbeta,
                                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same backward pass with DELAYED rescaling of the input gradient (Section
 * 3.3: statistic and rebalancing decoupled, the statistic of an earlier step
 * kept in the caller's state), in ONE pass over G and X:
 *   r = the power of two at or below *stat_in (1 if *stat_in is zero,
 *   subnormal, Inf or NaN);  dX_d = cast(dx / r), rounded once from fp32;
 *   dX_s = G_s*gamma_s / X_s * r.
 * dX: [R,d] of ANY dtype (E5M2 for the gradient operand of the next matmul).
 * stat_dx (AMAX or L2; NONE: nothing gathered) is taken on this step's
 * un-rebalanced, unrounded dx and left at workspace offset 16 for the next
 * step; stat_in (device, fp32, not NULL) may be that same word.  Everything
 * else as scalify_scaled_layernorm_bwd.
 */
int scalify_scaled_layernorm_bwd_delayed(const scalify_array* G, const scalify_array* X, const scalify_array* gamma,
                                         const float* mean, const float* rinv, float eps, int eps_inside_sqrt,
                                         const float* stat_in, int stat_dx, scalify_array* dX,
                                         scalify_array* dgamma, scalify_array* dbeta,
                                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * Residual addition and root-mean-square norm in one pass, with an 8-bit output (a norm without mean and bias; the add
 * rule of Section 3.2 and the normalisation rule of Section 3.2.1 / Appendix C.2):
 *   H_s = max(X_s, R_s),   H_d = cast(X_d*(X_s/H_s) + R_d*(R_s/H_s))          (bit for bit scalify_scaled_add)
 *   n = H_d * rinv,   rinv = 1 / sqrt(mean(H_d^2) + eps)                        (of H as stored; scale 1)
 *   Y_s = gamma_s (1 without gamma),   Y_d = cast(n * gamma_d)
 * and, with Ymx instead of Y, the same values quantised with one exponent per 32 elements as scalify_mx_quantize does
 * (Ymx_s = gamma_s), ready for scalify_mx_matmul.
 * X: [rows,d], F16/BF16/F32: the branch that is added.  R: the residual stream, of X's dtype or F32; H: the new
 * residual stream, of R's dtype, which may be R's or X's own buffer (same row stride).  With R == NULL there is no
 * addition: H must be NULL and X is the stream that is normalised.  Y: any dtype.  Exactly one of Y and Ymx is given;
 * Ymx: rows of d = K elements, not transposed.  gamma: [d], F16/BF16/F32, or NULL.  rinv: optional fp32 [rows]
 * (device), needed by the backward call.  d <= 16384, any; rows may be strided.  A row of zeros gives zeros if
 * eps > 0; with no rows at all the output scale words alone are written.  The squares of H_d are fp32 (|H_d| up to
 * 2^56, and with eps = 0 a row's largest not below 2^-60; an infinity or NaN reaches its own row only).
 * status: optional DEVICE word (SCALIFY_DEV_BAD_SCALE).
 * Errors: NULL, DTYPE, SHAPE, ALIGNMENT, UNSUPPORTED (both Y and Ymx, transposed Ymx), VALUE (eps < 0), ALIAS (an
 * output, rinv and the exponents among them, overlapping another array of the call other than as above, or a scale word
 * shared with another array of the call).
 */
struct scalify_mx_array;
int scalify_scaled_add_rmsnorm(const scalify_array* X, const scalify_array* R, const scalify_array* gamma, float eps,
                               scalify_array* H, scalify_array* Y, struct scalify_mx_array* Ymx, float* rinv,
                               uint32_t* status, void* stream);

/*
 * Its gradient (the exact derivative at H as stored; the block exponents and the 8-bit rounding of the forward output
 * are passed straight through):
 *   g = G_d*gamma_d,  dh = rinv*(g - n*mean(g*n)),  scale G_s*gamma_s/H_s
 *   dX_s = max(G_s*gamma_s/H_s, Gr_s),   dX_d = cast(dh + Gr by the add rule)      (gradient of X and of R alike)
 *   dXq_d = cast(dX_d / r), dXq_s = dX_s*r:   the 8-bit copy of the STORED dX that the next matmuls read; r is the
 *       power of two at or below *stat_in, the statistic of an earlier step (delayed rescaling, Section 3.3), or 1
 *       with stat_in == NULL or a statistic that defines no scale
 *   dgamma_d = sum_rows(G_d*n)/kf(rows), scale G_s*kf(rows)
 * G: [rows,d], F16/BF16/F32, gradient of Y.  H, rinv: from the forward call (with R == NULL, H is its X).  Gr: gradient
 * of H from the residual path, of H's dtype, or NULL.  dX: H's dtype; may be Gr's or G's own buffer (same dtype and
 * row stride).  H's dtype is G's or F32.  dXq: E4M3/E5M2 or NULL.  dgamma: [d] F16/BF16/F32 or NULL.  stat_dx: statistic
 * of the stored dX data, left at workspace offset 16 (stat_in may be that word's copy, not the word itself).
 * Sums over rows are fp32 per block and fp64 over the blocks, in a fixed order: results do not depend on scheduling.
 * Workspace: SCALIFY_OP_RMSNORM_BWD (rows, d); may be NULL without dgamma and stat_dx.
 * Errors: NULL, DTYPE, SHAPE, ALIGNMENT, VALUE, ALIAS, WORKSPACE.
 */
int scalify_scaled_add_rmsnorm_bwd(const scalify_array* G, const scalify_array* Gr, const scalify_array* H,
                                   const scalify_array* gamma, const float* rinv, scalify_array* dX, scalify_array* dXq,
                                   const float* stat_in, int stat_dx, scalify_array* dgamma, void* workspace,
                                   size_t workspace_bytes, void* stream);

/*
 * Scaled GELU forward / backward (Section 3.2.1 and Appendix C.1):
 *   forward  (X_d * g(X_d*X_s), X_s);   backward  dX_d = G_d * f'(X_d*X_s), dX_s = G_s.
 * exact_erf == 0: tanh form; != 0: Gaussian-CDF form.  X, G: F16/BF16/F32
 * (same dtype), Y/dX any dtype, contiguous, same shape.
 */
int scalify_scaled_gelu(const scalify_array* X, int exact_erf, scalify_array* Y, void* stream);
int scalify_scaled_gelu_bwd(const scalify_array* G, const scalify_array* X, int exact_erf,
                            scalify_array* dX, void* stream);

/*
 * Diagnostic for the bounded device-side waits (no counterpart in the paper).  Enqueues a one-thread
 * kernel that waits, with the same routine and status path as the matmul pipeline, on a barrier that
 * nothing signals; after `limit_us` microseconds (1..1e6) the wait gives up, sets
 * SCALIFY_DEV_TIMEOUT in the workspace status word and the kernel ends normally.  `waited_us`
 * (optional device word) receives the time actually spent.  Nothing faults and the context stays
 * usable: this is how a lost copy or a lost MMA completion would surface.
 */
int scalify_debug_expire_wait(void* workspace, size_t workspace_bytes, uint32_t limit_us, uint32_t* waited_us,
                              void* stream);

/*
 * Diagnostic (no counterpart in the paper): y[i] = x[i] rounded to the nearest BF16 value (ties to even), as
 * fp32, computed by the routine the fused attention kernels use for the scores' BF16 intermediate (three fp32
 * operations instead of a conversion).  x, y: device fp32 arrays of n elements.  two_wide = 0: the scalar
 * form; 1: the form on two-wide fp32 instructions, which takes the elements in pairs (x[0], x[1]), ...
 * Lets a test compare both with the definition over any set of bit patterns.
 */
int scalify_debug_bf16_round(const float* x, float* y, int64_t n, int two_wide, void* stream);

/*
 * Diagnostics of the library's host-side state (no counterpart in the paper; host only, no GPU needed).
 * The library keeps two things between calls: the one-time set-up of each kernel PER DEVICE (dynamic
 * shared-memory limit, co-resident cluster count) and a cache of encoded TMA tensor maps keyed by pointer,
 * extents, strides and box.  scalify_debug_host_state_selftest drives both with made-up device numbers and a
 * stand-in encoder and returns 0 if each device was set up exactly once and the cache returned the right map
 * for every key; scalify_debug_tensor_map_cache reports how many encodes the real cache has saved (hits) and
 * made (misses) so far in this process.
 */
int scalify_debug_host_state_selftest(void);

/*
 * Bounds-checking build (no counterpart in the paper).  The library built with -DSCALIFY_DEBUG
 * (`libscalify_debug.so`) checks every global access of its memory-bound kernels that goes through their vector,
 * row-copy and scalar-tail helpers (the element-wise, LayerNorm, Adam, block-scale quantisation and support
 * kernels, and the split-K reduction; the tensor-core kernels move their tiles with TMA, which the hardware
 * bounds by the tensor map) against the byte spans of the arrays and workspaces its entry points have validated
 * so far.  An access outside all of them is counted, its address kept, and skipped (a load yields zeros), so
 * nothing faults.  Registration copies a table to the device synchronously: this build is for tests, not for
 * timing or stream capture.  Spans that touch are merged, and spans are never forgotten until reset.
 *
 * scalify_debug_bounds_report: synchronises the device; out[0] = accesses refused since the last report, out[1]
 * = address of the first, out[2] = its width in bytes; clears the counters.  reset_ranges != 0 also forgets every
 * registered span.  range_limit >= 0 caps the length of every span registered from now on (a self-test: accesses
 * past the cap, still inside the caller's buffers, are then refused and reported); -1 lifts the cap.
 * Returns SCALIFY_ERR_UNSUPPORTED in the ordinary build.
 */
int scalify_debug_bounds_report(uint64_t out[3], int reset_ranges, int64_t range_limit);
int scalify_debug_tensor_map_cache(uint64_t* hits, uint64_t* misses);

/*
 * Diagnostic (no counterpart in the paper): the launch shape the LayerNorm kernels would use for an
 * [R,d] input of dtype x_dtype on the current device, so that a test can state which code path it
 * exercised.  Host only, launches nothing.  plan[0] = thread blocks; plan[1] = rows every team of
 * warps walks one after another (forward: consecutive rows of its block's run; backward: the
 * persistent grid's stride loop); plan[2] = warps per row; plan[3] = rows kept in flight through
 * shared memory (0: the backward kernel prefetches one row in registers instead).
 */
int scalify_debug_layernorm_plan(int64_t R, int64_t d, int x_dtype, int backward, int32_t plan[4]);

/*
 * Multiply a ScaledArray by a scalar constant c that is a positive power of two (Section 3.4: a
 * broadcast scalar contributes the scale "c rounded down to a power of two" and its mantissa stays
 * in the data; for a power of two the mantissa is 1, so only the scale word changes: X_s *= c).
 * Other constants return SCALIFY_ERR_UNSUPPORTED.  Used for the 1/sqrt(head_dim) of attention.
 */
int scalify_scalar_mul_pow2(scalify_array* X, float c, void* stream);

/*
 * Support operations of a GPT-style training step.  The paper states no scale rule for these
 * (Section 3.2.1 only says that custom rules suit attention layers); the rules below are this
 * library's readings, chosen so that values follow the unscaled network exactly (model invariance,
 * Section 1) and bounded quantities carry scale 1 (as the gate of an activation, Appendix C.1).
 *
 * Embedding lookup through the add rule:  Y[i] = wte[ids[i]] + wpe[i mod seq_len],
 *   Y_s = max(wte_s, wpe_s).  ids: DEVICE int64 [n]; wte [vocab,d], wpe [>=seq_len,d] or NULL, same
 *   16/32-bit dtype; Y [n,d] any dtype; d*elem_size a multiple of 16 bytes.  An id outside
 *   [0,vocab) sets SCALIFY_DEV_BAD_INDEX in *status (optional device word) and reads row 0.
 * Backward: dwte[v] = sum of the rows of dY whose id is v, scale dY_s (the number of addends is data
 *   dependent, so no static factor; fp32 atomics, order not fixed); dwpe[p] = sum over the
 *   n/seq_len sequences divided by kf(n/seq_len), scale dY_s*kf(n/seq_len).  dwte [vocab,d] and
 *   dwpe [seq_len,d] (or NULL) are F32 and fully overwritten.
 */
int scalify_scaled_embedding(const int64_t* ids, int64_t n, int64_t seq_len, const scalify_array* wte,
                             const scalify_array* wpe, scalify_array* Y, uint32_t* status, void* stream);
int scalify_scaled_embedding_bwd(const int64_t* ids, int64_t n, int64_t seq_len, const scalify_array* dY,
                                 scalify_array* dwte, scalify_array* dwpe, void* stream);

/*
 * Embedding lookup with a constant factor c > 0 (a scalar constant, Section 3.4: its power of two goes into the scale,
 * the rest, in [1, 2), into the data):
 *   Y_s = wte_s * p2(c),   Y_d[i] = cast(wte_d[ids[i]] * (c / p2(c)))
 * ids: DEVICE int64 [n].  A token equal to padding_id gives a row of zeros (INT64_MIN: no padding); any other token
 * outside [0, vocab) does too, and sets SCALIFY_DEV_BAD_INDEX in *status (optional DEVICE word).  wte: [vocab,d] of any
 * dtype; Y: [n,d] of any dtype; any d; rows may be strided.  n may be 0: Y's scale word alone is written.
 * Errors: NULL, DTYPE, SHAPE, ALIGNMENT, VALUE (c not a positive normal number), ALIAS.
 */
int scalify_scaled_embedding_lookup(const int64_t* ids, int64_t n, int64_t padding_id, const scalify_array* wte, float c,
                                    scalify_array* Y, uint32_t* status, void* stream);

/*
 * Its gradient, summed over SORTED tokens (scalify_scaled_embedding_bwd uses atomics, whose order changes the last bits;
 * here the token ids alone fix the order of every sum, and the same call gives the same bits every time):
 *   dwte_d[v] = (c / p2(c)) * sum of the rows of dY_d whose token is v,   scale dY_s * p2(c)
 * (no static factor: the number of addends depends on the data), sums in fp32.  With `addend` (the gradient of a tied
 * output layer) the result is addend + that by the add rule, rounded once: dwte_s = max(dY_s * p2(c), addend_s).
 * Every row of dwte is written: a token that does not occur, and the padding token, get zeros (or the addend).
 * ids, padding_id, c as for the lookup (an unknown token sets SCALIFY_DEV_BAD_INDEX in the workspace status word and is
 * left out).  dY: [n,d] of any dtype; dwte: [vocab,d], F16/BF16/F32; addend: dwte's dtype and shape, or NULL, and may be
 * dwte's own buffer (same row stride: the gradient is then accumulated in place).  n may be 0.  n < 2^31 - 1,
 * vocab <= 2^24, d <= 256 * 65535, (n/8 + 1) * ceil(d/256) < 2^34.
 * Workspace: SCALIFY_OP_EMBEDDING_GRAD (n, d); one for n tokens serves every batch of at most n (2 MB of it whatever n is).
 * Errors: NULL, DTYPE, SHAPE, ALIGNMENT, VALUE, ALIAS, WORKSPACE.
 */
int scalify_scaled_embedding_grad(const int64_t* ids, int64_t n, int64_t padding_id, const scalify_array* dY, float c,
                                  const scalify_array* addend, scalify_array* dwte, void* workspace,
                                  size_t workspace_bytes, void* stream);

/*
 * Row softmax of the VALUES S_d*S_s over the last dimension, optionally causal (row i of each
 * [Tq,Tk] matrix attends to columns j <= i + Tk - Tq; requires Tk >= Tq); P_d in [0,1], P_s = 1,
 * masked entries exactly 0.  S: [Tq,Tk] or [batch,Tq,Tk], F16/BF16/F32, contiguous, Tk*elem_size a
 * multiple of 16 bytes and at most 4096 bytes; P: same shape, any dtype.
 * Backward: dS_d = P_d*(dP_d - sum_j dP_d[j] P_d[j]), dS_s = dP_s*P_s (the Jacobian is bounded by 1,
 * so the gradient scale passes through).  dP: F16/BF16/F32; P: E4M3/F16/BF16/F32; dS any dtype.
 */
int scalify_scaled_softmax(const scalify_array* S, int causal, scalify_array* P, void* stream);
int scalify_scaled_softmax_bwd(const scalify_array* dP, const scalify_array* P, scalify_array* dS, void* stream);

/*
 * Mean cross-entropy of the values z = logits_d*logits_s through logsumexp (Appendix B) over the
 * first n_classes columns of logits [n, ld>=n_classes] (padding columns ignored), and its gradient
 * w.r.t. the values: dlogits_d = (softmax(z) - onehot(target)) * rem, dlogits_s = 1/n rounded down
 * to a power of two, rem = (1/n)/dlogits_s in [1,2); padding columns receive 0.
 * logits: F16/BF16/F32 (row stride = shape[1]); targets: DEVICE int64 [n]; loss: DEVICE fp32;
 * dlogits: same shape as logits, any dtype, or NULL.  A target outside [0,n_classes) sets
 * SCALIFY_DEV_BAD_INDEX in the workspace status word.  Workspace: SCALIFY_OP_CROSS_ENTROPY, n.
 */
int scalify_scaled_cross_entropy(const scalify_array* logits, int64_t n_classes, const int64_t* targets, float* loss,
                                 scalify_array* dlogits, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Losses of the output layer z = H W^T WITHOUT its logits in memory, beside scalify_scaled_cross_entropy, which takes them
 * (8192 tokens of a vocabulary of 50257: 823 MB in BF16, and as much again for their gradient).  The rules are the
 * composition of the calls they replace: the matmul, the loss through logsumexp (Appendix B), two more matmuls.
 *
 *   z[t,v] = H_s W_s sum_k H_d[t,k] W_d[v,k]                                       (values; tensor cores, fp32)
 *   lse[t] = log sum_v exp(z[t,v] / T),   p[t,v] = exp(z[t,v] / T - lse[t])        (T: temperature; cross entropy 1)
 * Cross entropy:  loss[t] = lse[t] - z[t,target] + z_loss lse[t]^2.
 * Distillation, from a teacher's k logits t_i = T_s T_d[t,i] at places ids[t,i]:
 *   q_i = exp(t_i / T - teacher_lse[t]);  without teacher_lse: normalised over the row's entries (a softmax of them)
 *   loss[t] = sum_i q_i (log q_i - log p[t,ids_i])
 * With teacher_lse (of the teacher's WHOLE row, at this temperature: scalify_scaled_top_logits gives it) q are the teacher's
 * own probabilities, and the mass outside the k entries takes no part.  No factor T^2 is applied.
 *
 *   H: [n, d], W: [vocab, d] (a tied embedding's layout): both F16, both BF16, or each E4M3 or E5M2.  Rows may be strided, but
 *   do not overlap (no broadcast).
 *   ids: DEVICE int64, [n] or [n, k] contiguous.  An entry equal to padding_id (INT64_MIN: none) is left out; so is any
 *   other outside [0, vocab), which also sets SCALIFY_DEV_BAD_INDEX; so is a teacher's logit of -inf.  The same place twice
 *   counts twice.  A row without entries has loss 0 and no gradient.
 *   T: [n, k], F16, BF16 or F32 (rows may be strided), 1 <= k <= 256.  teacher_lse: DEVICE fp32 [n] or NULL.
 *   loss, lse: DEVICE fp32 [n] (lse of every row; the gradient needs it).  mean: optional DEVICE word, the sum of the losses
 *   (fp64, fixed order) over the number of rows that have entries; 0 if none has.
 *   0 <= n <= 2^24, 1 <= vocab <= 2^24, 1 <= d <= 65536; z_loss >= 0 finite; temperature and its reciprocal normal numbers.
 * The same call gives the same bits every time.  Infinities and NaN in H or W go through as the formulas have them: lse of a row
 * whose logits hold +inf is +inf, of -inf throughout -inf, with a NaN NaN; an entry with q = 0 adds nothing to the loss.  (A row
 * of H without entries, too, has to be finite: its gradient 0 is multiplied with it for dW.)
 * Accuracy: all sums are fp32.  The tensor cores that form the long ones drop, of every product, what lies below 2^-25 of the sum
 * so far: N products of one sign lose about N 2^-27 of their sum (8-bit operands' products have fewer digits and lose less).  So
 * one accumulator takes at most 1536 products of a logit here and 4096 in the gradients (8-bit operands: twice as many), and 16384
 * of the gradients' own sums over rows or vocabulary; those parts are added in fp32 (loss and lse, in the norm, d up to
 * 4096: operands of either sign 2.6e-7 of their size, 8-bit ones 7e-8; of one sign 1.1e-6 and 2e-7; d = 65536: 9e-7).
 *
 * Gradients of sum_t g[t] loss[t] with respect to the VALUES of H and W:
 *   D[t,v] = g[t] / T ((Q[t] + 2 z_loss lse[t]) p[t,v] - q[t,v]),  Q = sum q;      dH = D W,  dW = D^T H
 *   D_s  = g_s p2(1/T)                                 (a scalar constant carries its power of two, Section 3.4)
 *   dH_s = D_s W_s kf(vocab),   dW_s = D_s H_s kf(n)   (matmul rule)
 *   grad: [n] F32, contiguous, or NULL: the gradient of `mean`, g = 1 / rows with entries, g_s = 1/n rounded down to a power
 *   of two (as scalify_scaled_cross_entropy).  lse: of the forward call on the same arguments.
 *   dH: [n, d], dW: [vocab, d], F16 or BF16 each; either may be NULL (a frozen layer).  Every row is written.
 * The logits are computed again in pieces of the vocabulary (the workspace holds D of two pieces, each at most 128 MiB or 256
 * columns, the fp32 sums of dH, and FP16 copies of FP8 operands).  D is rounded to BF16 (BF16 operands) or to FP16 (the others;
 * FP8 operands are widened to FP16 exactly), half a step of relative error each, at a scale that brings the largest row
 * coefficient to 2^14: about as much error as rounding the results once (BF16 2.4e-3 of the norm instead of 1.7e-3, FP16
 * 2.5e-4 instead of 2.1e-4), and FP16 entries below 2^-38 of the largest coefficient count as zero.  For at most 16 rows a second
 * half keeps what that rounding leaves out.  Sums are fp32 (as above).
 * Errors: NULL, DTYPE, SHAPE, ALIGNMENT, VALUE, ALIAS (an output over an input or another output), WORKSPACE.
 */
/* Workspace of these calls (shapes and dtypes of H and W only; k = 0: cross entropy; >= 4096; 0 for arguments that the calls
 * refuse).  Enough for every batch of at most H's rows (it never falls as the rows grow), so that one for the longest batch
 * serves all.  backward != 0: enough for the forward call too, so that a step's calls on one stream share one workspace;
 * nothing is kept in it between calls. */
size_t scalify_linear_loss_workspace_bytes(const scalify_array* H, const scalify_array* W, int k, int backward);
int scalify_scaled_linear_cross_entropy(const scalify_array* H, const scalify_array* W, const int64_t* ids, int64_t padding_id,
                                        float z_loss, float* loss, float* lse, float* mean, void* workspace,
                                        size_t workspace_bytes, void* stream);
int scalify_scaled_linear_cross_entropy_bwd(const scalify_array* H, const scalify_array* W, const int64_t* ids,
                                            int64_t padding_id, float z_loss, const float* lse, const scalify_array* grad,
                                            scalify_array* dH, scalify_array* dW, void* workspace, size_t workspace_bytes,
                                            void* stream);
int scalify_scaled_linear_distill(const scalify_array* H, const scalify_array* W, const scalify_array* T, const int64_t* ids,
                                  int64_t padding_id, const float* teacher_lse, float temperature, float* loss, float* lse,
                                  float* mean, void* workspace, size_t workspace_bytes, void* stream);
int scalify_scaled_linear_distill_bwd(const scalify_array* H, const scalify_array* W, const scalify_array* T, const int64_t* ids,
                                      int64_t padding_id, const float* teacher_lse, float temperature, const float* lse,
                                      const scalify_array* grad, scalify_array* dH, scalify_array* dW, void* workspace,
                                      size_t workspace_bytes, void* stream);

/*
 * The k largest logits of every row, what a teacher hands to scalify_scaled_linear_distill:
 *   V_d[r] = the k largest of X_d[r], in descending order, equal ones (0 and -0 are) by column;  V_s = X_s
 *   ids[r] = their columns;   lse[r] = log sum_j exp(X_s X_d[r,j] / temperature)        (optional)
 * A NaN counts as larger than everything (and makes lse NaN; without one, +inf makes it +inf).
 * X: [n, vocab], F16, BF16 or F32; V: [n, k] of X's dtype; rows of
 * both may be strided; ids: DEVICE int64 [n, k] contiguous; lse: DEVICE fp32 [n] or NULL.  1 <= k <= min(256, vocab),
 * 0 <= n <= 2^24, vocab <= 2^24.  No workspace.  Errors: NULL, DTYPE, SHAPE, ALIGNMENT, VALUE (temperature), ALIAS.
 */
int scalify_scaled_top_logits(const scalify_array* X, float temperature, scalify_array* V, int64_t* ids, float* lse, void* stream);

/*
 * Scaled Adam step over a list of tensors (Sections 1, 3 and 4; Table 3 row 4:
 * FP8 gradients, FP16 scaled optimizer state and master weights).  In value
 * space this is textbook Adam with bias correction:
 *   m' = b1*m + (1-b1)*g;  v' = b2*v + (1-b2)*g^2;
 *   w' = w - lr * (m'/(1-b1^t)) / (sqrt(v'/(1-b2^t)) + eps)
 * and the new scales follow from tracing that expression with the static
 * rules (mul: product; add: max; div: ratio; sqrt: sqrt rounded down; a scalar
 * constant c carries the scale "|c| rounded down to a power of two",
 * Section 3.4):
 *   m'_s = max(p2(b1)*m_s, p2(1-b1)*g_s)
 *   v'_s = max(p2(b2)*v_s, p2(1-b2)*g_s^2)
 *   u_s  = p2(lr) * (m'_s/p2(1-b1^t)) / max(p2(sqrt(v'_s/p2(1-b2^t))), p2(eps))
 *   w'_s = max(w_s, u_s)
 * Each of m', v', w' is rounded once from fp32 arithmetic.
 *   grads[i]: any dtype (E5M2 typical); m[i], v[i]: F16 or F32 (same);
 *   w[i]: F16, BF16 or F32.  All four have the same element count, are
 *   contiguous, and m, v, w (data and scale words) are updated in place.
 *   Every m, v and w scale word of the whole list must be a word of its own
 *   (the kernels read the old scales while the new ones are written) and none
 *   of them a gradient's scale word; gradients may share one.  A repeated word
 *   returns SCALIFY_ERR_ALIAS and enqueues nothing.
 *   step >= 1 is t.  Needs a workspace (SCALIFY_OP_ADAM, n_tensors).
 */
int scalify_scaled_adam_step(int n_tensors, const scalify_array* grads, scalify_array* m, scalify_array* v,
                             scalify_array* w, float lr, float beta1, float beta2, float eps, int64_t step,
                             void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same step, which also writes the low-precision compute copy of every
 * updated weight that the next forward pass multiplies with (the static cast
 * on the forward path, Appendix A; Section 4: FP8 matmul operands, wider master
 * weights): w_cast[i]_d = cast(stored w'[i]_d), w_cast[i]_s = w'[i]_s.  The
 * cast starts from the value as stored in w[i] (already rounded to its dtype),
 * so the copy is bit-identical to a separate scalify_rescale(STAT_NONE) of
 * w[i], at one extra written byte per parameter instead of a 3-byte pass.
 *   w_cast[i]: E4M3, E5M2, F16 or BF16 (all the same, narrower than w[i]),
 *   contiguous, same element count as w[i], own scale word (no aliasing with
 *   g, m, v, w scale words; data must not alias w[i]).
 * Errors as scalify_scaled_adam_step; SCALIFY_ERR_NULL when w_cast is NULL.
 */
int scalify_scaled_adam_step_cast(int n_tensors, const scalify_array* grads, scalify_array* m, scalify_array* v,
                                  scalify_array* w, scalify_array* w_cast, float lr, float beta1, float beta2,
                                  float eps, int64_t step, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Orthogonalisation of matrices by Newton-Schulz products (the update of the Muon optimiser; no counterpart in the
 * paper, whose optimiser is Adam).  Per matrix U [rows, cols] (its data component: the result does not depend on scale):
 *   Z = U / (|U|_F + eps);   `steps` times:  A = Z Z^T,  Z = a Z + (b A + c A^2) Z    (on the shorter side, so that A is
 *   min(rows, cols) square);   O = Z
 * With (a, b, c) = (3.4445, -4.7750, 2.0315), used when coef is NULL, five steps bring the singular values to about
 * 1 +- 0.3, which is what the optimiser wants.  coef: HOST array of three floats, whose products have to fit FP16 whatever the
 * matrix is: with m = 33/32 at first and m = 33/32 max |a x + b x^3 + c x^5| over x <= m after each step,
 *   m <= 3.875  and  max |a + b x^2 + c x^4| over x <= m  <= 15.5      at the beginning of every step (else VALUE).
 * The products run on the tensor cores with FP16 operands at a power-of-two scale and fp32 accumulation, and the iterates
 * are held in FP16 (11 bits).  O is therefore a 16-bit array, and its error is ABSOLUTE where the matrix has directions with
 * little or nothing in them: what a rounding leaves there every step multiplies by a.  In the Frobenius norm, for |a| >= 1 and
 * results whose singular values are about 1,
 *   |O - definition| <= 2^-11 |a|^steps + 3e-3 |O|         (0.24 + 3e-3 |O| for the default; measured: half the first term;
 *                                                          the rounding of O to its own type comes on top)
 * so 1e-3 to 4e-3 of the norm for a full-rank matrix of some hundred rows, but a seventh of it for a matrix of rank one
 * (the gradient of one token).  The error is spread over all directions: with some hundred of them none gets more than 0.03
 * of the 1 that the occupied ones have.
 *   X: [rows, cols] or [batch, rows, cols], any dtype; rows may be strided.  O: the same shape, F16 or BF16.
 *   O_s = 1 / kf(max(rows, cols)) (a matrix with singular values 1 has entries of about 1/sqrt(longer side)).
 *   A matrix of zeros gives zeros; one with an infinity or NaN gives NaN (and SCALIFY_DEV_NONFINITE_STAT).  A norm
 *   (of the data component, whose squares are fp32) below 2^-60 counts as zero, one above 2^63 as infinite.
 *   1 <= rows, cols <= 32768; 1 <= steps <= 16.
 * Errors: NULL, DTYPE, SHAPE, ALIGNMENT, VALUE (eps < 0, coefficients, steps), ALIAS, WORKSPACE.
 */
int scalify_orthogonalize(const scalify_array* X, int steps, const float* coef, float eps, scalify_array* O,
                          void* workspace, size_t workspace_bytes, void* stream);
/* Bytes of workspace that the two calls need for this list of matrices (shapes only; >= 4096; 0 for a bad shape). */
size_t scalify_muon_workspace_bytes(int n_tensors, const scalify_array* w);

/* How a step's length goes with the matrix: factor =
 *   UNIT             1
 *   SPECTRAL         sqrt(max(1, rows/cols)), for a weight stored [outputs, inputs] (a transposed B operand of the matmul)
 *   SPECTRAL_IN_OUT  sqrt(max(1, cols/rows)), for a weight stored [inputs, outputs] (a plain B operand: Y = X W)
 *   RMS              0.2 sqrt(max(rows, cols)), the root mean square of an Adam step
 * The spectral ones are sqrt(max(1, outputs/inputs)): a layer with at least as many outputs as inputs then changes the root
 * mean square of its output by at most about lr times that of its input.  They need to know which side is which, so weights
 * of the two layouts go into calls of their own. */
enum { SCALIFY_MUON_UNIT = 0, SCALIFY_MUON_SPECTRAL = 1, SCALIFY_MUON_RMS = 2, SCALIFY_MUON_SPECTRAL_IN_OUT = 4 };

/*
 * Scaled Muon step over a list of matrices, beside scalify_scaled_adam_step for the other parameters.  In value space
 *   m' = mu*m + (1-mu)*g;   u = nesterov ? mu*m' + (1-mu)*g : m';   O = orthogonalised u (of u / m'_s)
 *   w' = w - lr*weight_decay*w - lr*factor*O
 * and the scales follow the static rules as for Adam (a scalar constant c carries "c rounded down to a power of two"):
 *   m'_s = max(p2(mu)*m_s, p2(1-mu)*g_s)  (without the first term for mu = 0);
 *   w'_s = max(w_s, p2(lr*factor) / kf(max(rows, cols)))
 * m' and w' are rounded once from fp32 arithmetic (u is not rounded before its norm).
 *   grads[i]: [rows, cols], any dtype; m[i]: F16 or F32; w[i]: F16, BF16 or F32; w_cast[i] (or w_cast == NULL): E4M3, E5M2,
 *   F16 or BF16, receives cast(stored w') with w'_s, as for scalify_scaled_adam_step_cast.  Row strides are free; one
 *   dtype per list.  m and w (data and scale words) are updated in place; all their scale words are required and
 *   distinct, and none is a gradient's; their data do not overlap each other or a gradient (gradients may share memory).
 *   0 <= momentum < 1;  lr >= 0;  0 <= lr*weight_decay < 1.  Matrices of one shape (or transposed) run as one batch.
 * Errors: NULL, DTYPE, SHAPE, ALIGNMENT, VALUE, ALIAS, WORKSPACE (scalify_muon_workspace_bytes of w).
 */
int scalify_scaled_muon_step(int n_tensors, const scalify_array* grads, scalify_array* m, scalify_array* w,
                             scalify_array* w_cast, float lr, float momentum, int nesterov, float weight_decay, int steps,
                             const float* coef, float eps, int factor, void* workspace, size_t workspace_bytes,
                             void* stream);

/*
 * Block scales (Section 2: the scale component may be any array that broadcasts
 * against the data; the paper names the E8M0 exponent byte and the OCP
 * micro-scaling formats as the standard it follows, and works with one scalar
 * scale per tensor; this is the block form of the same representation).
 *
 * A block-scaled array is FP8 data [rows, K] (row-major, dense, K innermost),
 * one E8M0 exponent per 32 consecutive elements of a row, and the usual
 * tensor-wide fp32 power-of-two scale:
 *   value[i,k] = data[i,k] * 2^(exponent[i, k/32] - 127) * scale.
 * Only the tensor-wide scale takes part in the static scale rules; the
 * exponents belong to the data component.
 * K must be a multiple of 128.  `sf` holds the exponents in the order the
 * block-scaled tensor-core instruction consumes: tiles of 128 rows x 4 blocks
 * (512 bytes), tile (r, k) at byte ((r * (K/128)) + k) * 512, and inside a tile
 * row `row`, block `blk` at byte (row % 32) * 16 + (row / 32) * 4 + blk.  The
 * row count is padded up to a multiple of 256: scalify_mx_sf_bytes(rows, K)
 * bytes, 16-byte aligned; the exponents of the padding rows must be valid
 * (scalify_mx_quantize writes 127 there).  All pointers are DEVICE pointers
 * owned by the caller.
 */
typedef struct scalify_mx_array {
  void* data;     /* FP8 elements [rows, K], 16-byte aligned */
  int32_t dtype;  /* SCALIFY_E4M3 or SCALIFY_E5M2 */
  int64_t rows;
  int64_t K;
  uint8_t* sf;    /* E8M0 exponents, tiled as described above */
  float* scale;   /* one fp32 power of two, or NULL (scale 1) */
  int32_t transposed; /* 0: data [rows, K].  1: data stored [K, rows] (row-major, `rows` contiguous, rows a
                         multiple of 16): the form of an operand whose contraction dimension is the slow one
                         of the forward tensor (weight and activation gradients); a block is then 32
                         consecutive ROWS of the storage at one column.  The exponent tiles are the same. */
} scalify_mx_array;

size_t scalify_mx_sf_bytes(int64_t rows, int64_t K);

/*
 * Quantises the data component of X [rows, K] (F16, BF16 or F32; row stride
 * stride[0]) into Y: per block of 32 elements, exponent e = floor(log2(max|x|))
 * - emax (emax = 8 for E4M3, 15 for E5M2: the OCP MX rule, i.e. a dynamic
 * rescale with the AMAX statistic per block, Section 3.3, the power of two
 * rounded down), clamped to [-127, 127]; data = round-to-nearest-even of
 * x * 2^-e, saturating.  A block whose maximum is zero, infinite or NaN gets
 * e = 0.  Y_s = X_s.  `status`: optional DEVICE word that receives
 * SCALIFY_DEV_BAD_SCALE.  Errors: NULL, DTYPE, SHAPE (K % 128), ALIGNMENT.
 * With Y->transposed, X is [K, rows] like the data it is quantised into, and
 * the blocks run down the columns; the values and exponents are those of the
 * plain form applied to the transposed matrix.
 */
int scalify_mx_quantize(const scalify_array* X, scalify_mx_array* Y, uint32_t* status, void* stream);

/*
 * Block-scaled matmul with the static matmul rule (Section 3.2) on the
 * tensor-wide scales:  Y_s = A_s * B_s * kf(K),
 *   Y_d[i,j] = (sum_k A_d[i,k] 2^(Ea[i,k/32]-127) * B_d[j,k] 2^(Eb[j,k/32]-127)) / kf(K)
 * with fp32 accumulation on the tensor cores (tcgen05 kind::mxf8f6f4 with the
 * exponents in tensor memory).  A is [M,K], B is [N,K] (either may be stored
 * transposed, see scalify_mx_array: the tensor cores then read it MN-major and
 * no transposed copy is made); Y [M,N] is F16, BF16
 * or F32 (row stride stride[0]).  stat: NONE, AMAX or L2 of the stored Y, left
 * in the workspace's statistic word as by scalify_scaled_matmul.  Workspace:
 * SCALIFY_OP_MATMUL (M, N).
 */
int scalify_mx_matmul(const scalify_mx_array* A, const scalify_mx_array* B, scalify_array* Y, int stat,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * Column sums of a scaled matrix: Y[j] = sum over the R rows of X[r, j], by the
 * rule for a sum of R independent terms (Section 3.2; the same rule as a matmul
 * with a ones operand and K = R, and as the dbeta of the LayerNorm backward):
 *   Y_s = X_s kf(R),   Y_d[j] = (sum_r X_d[r, j]) / kf(R)
 * This is the bias gradient of a linear layer.  X: any dtype, [R, N] (row stride
 * stride[0]); Y: F16, BF16 or F32, [N] contiguous.  Partial sums are fp32 per slab
 * of rows, the slabs are added in fp64 in a fixed order (results do not depend on
 * scheduling).  Workspace: SCALIFY_OP_COLSUM (R, N).
 * Errors: NULL, DTYPE, SHAPE, ALIGNMENT, WORKSPACE, ALIAS.
 */
int scalify_scaled_colsum(const scalify_array* X, scalify_array* Y, void* workspace, size_t workspace_bytes,
                          void* stream);

/*
 * The static cast of a gradient to FP8 (Appendix A: cast_on_backward) fused with the column sums of the cast
 * values: C = cast(X) with C_s = X_s, and Y = the column sums of C by the rule above, in one pass over X.  C, its
 * scale and Y are the bits scalify_rescale (plain cast) followed by scalify_scaled_colsum of its output give.
 * This is what the backward of a linear layer needs of the output gradient: its E5M2 copy for the two gradient
 * matmuls and the bias gradient.  X: BF16 or F16 [R, N]; C: E4M3 or E5M2 [R, N] (row stride a multiple of 16
 * bytes); Y: F16, BF16 or F32 [N].  Workspace: SCALIFY_OP_COLSUM (R, N).
 * Errors: NULL, DTYPE, SHAPE, ALIGNMENT, WORKSPACE, ALIAS.
 */
int scalify_scaled_cast_colsum(const scalify_array* X, scalify_array* C, scalify_array* Y, void* workspace,
                               size_t workspace_bytes, void* stream);

/*
 * Fused scaled attention forward: S = Q K^T, P = softmax(S c), O = P V in one
 * kernel per (head, 128 queries); the scores and the probabilities stay on chip.
 * The paper names attention as a place for a custom scale rule (Section 3.2.1)
 * and gives none; the rule here is the composition of the calls it replaces:
 *   S_s = Q_s K_s kf(hd),  S_d = (Q_d K_d^T) / kf(hd) rounded to BF16      (matmul rule)
 *   P   = softmax over the keys of the VALUES S_d S_s c, optionally causal
 *         (query i sees keys j <= i + Tk - Tq); bounded in [0,1], scale 1, rounded to E4M3
 *   O_s = V_s kf(Tk),      O_d = (P_d V_d) / kf(Tk)                          (matmul rule)
 * i.e. scalify_scaled_matmul, scalify_scalar_mul_pow2, scalify_scaled_softmax,
 * scalify_scaled_matmul.  The softmax is the exact two-sweep form (row maximum
 * and sum first, then the normalised probabilities), not an online rescaling.
 *   Q [heads, Tq, hd], K, V [heads, Tk, hd]: E4M3 or E5M2, hd = 64 or 128, 3-D views
 *   (row and head strides in stride[1], stride[0]; 2-D arrays are one head; 4-D
 *   arrays [batch, heads, T, hd] add a batch stride in front, so that the token-major
 *   buffers [batch * T, heads * hd] of a transformer are covered by ONE call);
 *   O [heads, Tq, hd]: F16, BF16 or F32, same kind of view; c: any finite
 *   scalar (a power of two only shifts the exponent; otherwise its mantissa is
 *   applied in fp32).  causal needs Tk >= Tq.
 *   S_dump (BF16) and P_dump (E4M3): optional dense [heads, Tq, Tk] DEVICE
 *   copies of S_d and P for checking (Tk % 32 == 0), normally NULL; with 4-D
 *   operands the leading dimension counts batch * heads (or is given as two).
 *   status: optional DEVICE word (SCALIFY_DEV_TIMEOUT, SCALIFY_DEV_BAD_SCALE).
 * Errors: NULL, DTYPE, SHAPE, ALIGNMENT, UNSUPPORTED (hd != 64, causal with
 * Tk < Tq), ALIAS (O_s aliasing an input scale word).
 */
int scalify_scaled_attention(const scalify_array* Q, const scalify_array* K, const scalify_array* V, float sm_scale,
                             int causal, scalify_array* O, scalify_array* S_dump, scalify_array* P_dump,
                             uint32_t* status, void* stream);

/*
 * Fused scaled attention backward: the gradients of scalify_scaled_attention with
 * respect to Q, K and V, from the gradient dO of its output and the probabilities
 * P it used (its P_dump).  Same custom rule (Section 3.2.1), i.e. the composition
 * of the calls it replaces:
 *   dP_s = dO_s V_s kf(hd),   dP_d = (dO_d V_d^T) / kf(hd) rounded to BF16       (matmul rule)
 *   dS_d = P_d (dP_d - sum_j dP_d[i,j] P_d[i,j]) rounded to E5M2,
 *   dS_s = dP_s P_s c                                  (softmax backward, scalar c)
 *   dQ_s = dS_s K_s kf(Tk),   dQ_d = (dS_d K_d) / kf(Tk)                          (matmul rule)
 *   dK_s = dS_s Q_s kf(Tq),   dK_d = (dS_d^T Q_d) / kf(Tq)
 *   dV_s = P_s dO_s kf(Tq),   dV_d = (P_d^T dO_d) / kf(Tq)
 * i.e. scalify_scaled_matmul, scalify_scaled_softmax_bwd, scalify_scalar_mul_pow2
 * and three more scalify_scaled_matmul.  Two launches: one CTA per (head, 128
 * queries) forms dP (twice, it never reaches memory), dS and dQ; one CTA per
 * (head, 128 keys) contracts P and dS over the queries into dV and dK.
 *   Q, dO [heads, Tq, hd], K, V [heads, Tk, hd]: E4M3 or E5M2, hd = 64 or 128, 3-D views
 *   as for the forward call.  P: E4M3, dense [heads, Tq, Tk], non-negative (the
 *   sign bit is ignored), exact zeros where the mask hides a key.  dS (output): E5M2, dense [heads, Tq, Tk], scale word
 *   required; with causal != 0 the 128 x 128 blocks wholly above the diagonal are
 *   not written.  dQ [heads, Tq, hd], dK, dV [heads, Tk, hd]: F16, BF16 or F32
 *   (one dtype), same kind of view.  c: the forward's scalar, a power of two.
 *   Tk % 32 == 0.  dP_dump (BF16, dense [heads, Tq, Tk]): optional copy of dP_d
 *   for checking, normally NULL.  status: optional DEVICE word.
 * Errors: NULL (also: dS without a scale word), DTYPE, SHAPE, ALIGNMENT,
 * UNSUPPORTED (hd != 64, causal with Tk < Tq, c not a power of two), ALIAS (an
 * output scale word aliasing another scale word of the call).
 */
int scalify_scaled_attention_bwd(const scalify_array* Q, const scalify_array* K, const scalify_array* V,
                                 const scalify_array* P, const scalify_array* dO, float sm_scale, int causal,
                                 scalify_array* dS, scalify_array* dQ, scalify_array* dK, scalify_array* dV,
                                 scalify_array* dP_dump, uint32_t* status, void* stream);

/*
 * Scaled Adam step without a workspace.  (No counterpart in the paper: this entry point exists
 * for the integration, not for the method.)
 *
 * Same operation, arguments and results as scalify_scaled_adam_step, for callers that cannot
 * allocate the workspace that call needs: code running after the application's own memory
 * pool has taken all device memory (a further cudaMalloc would fail), code on a path where
 * the device-wide synchronisation of cudaMalloc is not acceptable, and integrations that are
 * handed nothing but the tensors.  The scratch (old scale words and new reciprocals per
 * tensor, and the status word) is a fixed 33 KB array inside the library image; every GPU
 * that loads the library holds it until the process exits.  The call allocates nothing and
 * frees nothing.
 *
 *   n_tensors   at most 1024; more returns SCALIFY_ERR_WORKSPACE and enqueues nothing.
 *   status_out  optional DEVICE pointer to one uint32: receives the SCALIFY_DEV_* bits of this
 *               call (0 if none), written in stream order.  May be NULL.
 *
 * The first call on each device looks up the array's device address (with that device
 * current); make that first call before starting any stream capture.  All calls on a device
 * share the one array, which keeps the previous call's contents (the call clears what it
 * needs to start from zero): two calls that may overlap on the GPU - different streams
 * without an ordering between them - race on it; order them or use
 * scalify_scaled_adam_step with separate workspaces.
 */
int scalify_scaled_adam_step_static(int n_tensors, const scalify_array* grads, scalify_array* m, scalify_array* v,
                                    scalify_array* w, float lr, float beta1, float beta2, float eps, int64_t step,
                                    uint32_t* status_out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SCALIFY_H_ */
