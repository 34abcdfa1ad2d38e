/*
 * loract.h - C ABI of the LoRAct activation-compression library for AMD MI355X (gfx950).
 *
 * The library implements the data path of "LoRAct: low-rank activation compression"
 * (arXiv 2509.23472): the online compression of one saved activation matrix in the forward
 * pass (Section 3.1, Eqs. 2-3, by the sampling-based orthogonal decomposition of
 * Section 3.2, Algorithm 1) and the backward-side consumers of the factors (Section 3.1,
 * Eqs. 4-5), plus the randomized-SVD method the paper compares with (Section 3.2).
 *
 * Conventions shared by every entry point
 *   - Matrices are dense and row-major.  "dev" pointers are device (HBM) pointers owned by
 *     the caller; "host" pointers are ordinary host memory.  The library never allocates,
 *     frees or retains caller memory; scratch space is a caller-provided workspace.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All device
 *     work is enqueued on it in order; no entry point synchronises the device, except the
 *     loract_profile_* readers which wait for their own events.
 *   - Return value: LORACT_OK (0) or a negative loract_status.  Argument errors are detected
 *     on the host before anything is enqueued.  Numerical events on the device (a
 *     rank-deficient sketch) never abort; they are reported through the optional device
 *     status word.
 *   - Same inputs, parameters and seed give bit-identical outputs: all split reductions are
 *     combined in a fixed order, no floating-point atomics are used.
 *   - Element types: LORACT_BF16 is the 16-bit brain float (upper half of an IEEE binary32),
 *     LORACT_F32 is IEEE binary32.
 */
#ifndef LORACT_H
#define LORACT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LORACT_OK = 0,
  LORACT_ERR_INVALID_ARG = -1,        /* null pointer, non-positive size, k out of range, ... */
  LORACT_ERR_WORKSPACE_TOO_SMALL = -2,
  LORACT_ERR_UNSUPPORTED = -3,        /* dtype combination, rank above LORACT_MAX_RANK, ... */
  LORACT_ERR_NOT_IMPLEMENTED = -4,
  LORACT_ERR_HIP = -5                 /* a HIP runtime call failed; see loract_last_hip_error */
} loract_status;

typedef enum { LORACT_F32 = 0, LORACT_BF16 = 1 } loract_dtype;

/* Largest number of sketch columns (k, or k + oversampling for RSVD) the kernels accept. */
#define LORACT_MAX_RANK 320
#define LORACT_STATIC_SCRATCH_BYTES (16u << 20)   /* scratch built into the library, see loract_lora_grad_static */

/* Bits of the device status word written by loract_compress / loract_rsvd. */
#define LORACT_STATUS_RANK_DEFICIENT 1   /* a direction of the sketch was numerically dependent on
                                            the others and was dropped: U has a zero column */
#define LORACT_STATUS_INTERNAL 2         /* a workgroup's bounded wait for another workgroup of the
                                            same launch ran out: the outputs are not valid */

/* Problem statement of Algorithm 1: A in R^{m x n}, expected rank k, iterations t. */
typedef struct {
  int64_t m;             /* rows of X (tokens) */
  int64_t n;             /* columns of X (hidden size) */
  int64_t ldx;           /* leading dimension of X in elements, >= n */
  int32_t k;             /* target rank, 1 <= k <= min(m, n) */
  int32_t l;             /* sketch columns, k <= l <= min(m, n, LORACT_MAX_RANK); 0 = k.
                            loract_compress: sampled rows (Algorithm 1 takes l = k; l > k is the
                            sample of Theorem 4.3).  loract_rsvd: k + oversampling.  With l > k the
                            l x n factor Q^T X is cut to its k leading singular triplets */
  int32_t t;             /* power iterations (the power rounds of Algorithm 1); 0 on the hot path */
  int32_t x_dtype;       /* loract_dtype of X */
  int32_t factor_dtype;  /* loract_dtype of U and V; F32 input requires F32 factors */
  uint64_t seed;         /* seed of the row sample (compress) or of the Gaussian test matrix (rsvd) */
} loract_params;

const char* loract_version(void);
const char* loract_strerror(int code);
/* Text of the most recent HIP error seen by this thread's calls ("" if none). Host. */
const char* loract_last_hip_error(void);

/*
 * Algorithm 1, row sampling: the l distinct row indices sampled uniformly without replacement from
 * [0, m), in ascending order.  Pure host function; this is the definition the device path
 * uses when no explicit indices are given: splitmix64 started at `seed` drives Floyd's subset
 * sampling (for i = m-l .. m-1: j = next() mod (i+1); take j, or i if j was already taken).
 * idx_host: out, l int32 values.  Errors: INVALID_ARG if l < 0, l > m, m > 2^31-1 or null.
 */
int loract_sample_indices(int64_t m, int32_t l, uint64_t seed, int32_t* idx_host);

/*
 * Bytes of device workspace loract_compress / loract_rsvd need for these parameters
 * (256-byte aligned base expected).  Host.  Errors as for the call itself.
 */
int loract_workspace_bytes(const loract_params* p, size_t* bytes);

/*
 * Forward pass, Section 3.1 Eqs. (2)-(3) by Algorithm 1 (Section 3.2):
 *   A_k = X[S, :] (k sampled rows), Y = X A_k^T, t x [Y = QR; Y = X (X^T Q)], Y = QR,
 *   U = Q (m x k, orthonormal columns), V = Q^T X (k x n).
 * With l > k sampled rows (Theorem 4.3) Q has l columns and the factors are those of the k
 * leading singular triplets of B = Q^T X: U = Q W_k, V = W_k^T B (W_k: k leading eigenvectors
 * of B B^T), still m x k and k x n with orthonormal U.
 * X_dev        in,  m x n (ld = ldx), dtype x_dtype.
 * idx_host     in,  l ascending distinct row ids in host memory, or NULL to derive them from
 *              p->seed with loract_sample_indices.  Read before the call returns.
 * U_dev, V_dev out, m x k and k x n, contiguous, dtype factor_dtype.
 * ws_dev       scratch of at least loract_workspace_bytes(p) bytes; contents undefined after.
 * status_dev   optional int32 in device memory; set to 0 or an OR of LORACT_STATUS_* bits.
 * If Y is rank deficient (X holds duplicate or all-zero rows and they were sampled) U V
 * remains the projection of X onto range(Y) to working accuracy and U stays finite: a
 * dependent direction is either replaced by an arbitrary orthonormal completion, or, when it
 * vanishes to within float32 resolution, dropped: then that column of U (and row of V) is
 * zero and the status bit is raised.
 */
int loract_compress(const void* X_dev, const loract_params* p, const int32_t* idx_host,
                    void* U_dev, void* V_dev, void* ws_dev, size_t ws_bytes,
                    void* stream, int32_t* status_dev);

/*
 * Algorithm 1 with the rank chosen from the data.  The paper fixes k by hand and leaves adaptive
 * rank selection to future work (Conclusion); the rule used here is the measure of Section 2: the
 * number of kept dimensions when `energy` (0 < energy <= 1, Section 2 uses 0.9) of the energy --
 * the sum of the singular values -- is retained.  It is evaluated inside the sketch: with Q an
 * orthonormal basis of the l-column sketch (l = p->l sampled rows, 0 = p->k) and s_1 >= ... >= s_l the
 * singular values of B = Q^T X, k_eff is the smallest count with s_1 + ... + s_k_eff >= energy *
 * (s_1 + ... + s_l), at most p->k, and the factors are the k_eff leading singular triplets of B as
 * in loract_compress with l > k.
 * U_dev, V_dev  out, m x p->k and p->k x n as for loract_compress: columns of U and rows of V from
 *               k_eff on are zero, so U V is the rank-k_eff product whatever slice the caller keeps.
 * k_out_dev     out, int32 in device memory: k_eff.
 * Workspace, indices, stream, status and errors as for loract_compress.
 */
int loract_compress_adaptive(const void* X_dev, const loract_params* p, const int32_t* idx_host,
                             double energy, void* U_dev, void* V_dev, int32_t* k_out_dev,
                             void* ws_dev, size_t ws_bytes, void* stream, int32_t* status_dev);

/*
 * Backward pass, Section 3.1 Eq. (4): Xhat = U V.
 * U_dev m x k, V_dev k x n (contiguous, dtype factor_dtype); Xhat_dev out, m x n with leading
 * dimension ldxh >= n, dtype out_dtype.  No workspace.
 */
int loract_reconstruct(const void* U_dev, const void* V_dev, int64_t m, int64_t n, int32_t k,
                       int32_t factor_dtype, void* Xhat_dev, int64_t ldxh, int32_t out_dtype,
                       void* stream);

/*
 * Backward pass, Section 3.1 Eqs. (4)-(5) specialised to a LoRA down-projection whose input
 * was compressed: dA = Xhat^T (dY B_lora^T) * scale  (n x r_lora, float32), evaluated as
 * V^T (U^T (dY B_lora^T)) without forming Xhat.
 * dY_dev m x n_out and Blora_dev r_lora x n_out have dtype grad_dtype (contiguous);
 * 1 <= r_lora <= 64.  Workspace: loract_lora_grad_workspace_bytes.
 */
int loract_lora_grad_workspace_bytes(int64_t m, int64_t n, int32_t k, int64_t n_out,
                                     int32_t r_lora, size_t* bytes);
int loract_lora_grad(const void* U_dev, const void* V_dev, int64_t m, int64_t n, int32_t k,
                     int32_t factor_dtype, const void* dY_dev, int64_t n_out,
                     const void* Blora_dev, int32_t r_lora, int32_t grad_dtype, float scale,
                     float* dA_dev, void* ws_dev, size_t ws_bytes, void* stream);

/*
 * loract_lora_grad for callers that cannot allocate or hand over device memory: code under HIP
 * graph capture, tight serving or training loops, harnesses that forbid hipMalloc.  Same
 * arguments, kernels and result (bit for bit) as loract_lora_grad, without the workspace: the
 * scratch is a buffer of LORACT_STATIC_SCRATCH_BYTES (16 MiB) built into the library's device
 * image, one copy per GPU, held until the process ends.  The call allocates nothing: no hipMalloc,
 * hipFree or allocating library routine is reached.
 * Limit: shapes whose loract_lora_grad_workspace_bytes exceeds LORACT_STATIC_SCRATCH_BYTES are
 * rejected with LORACT_ERR_WORKSPACE_TOO_SMALL (loract_last_hip_error names both sizes) before
 * anything is enqueued; 8192 x 4096, rank 128, LoRA rank 16 needs 8 MiB.
 * All calls on one GPU share that GPU's buffer, which keeps the previous call's contents (no kernel
 * of the gradient relies on them): calls that overlap on one GPU -- from two streams or two
 * threads -- race; serialise them on one stream.  The first call on a device looks up the
 * buffer's address (no allocation, but not a stream operation: make one call before capturing).
 * loract_static_scratch_bytes returns the built-in size.
 */
size_t loract_static_scratch_bytes(void);
int loract_lora_grad_static(const void* U_dev, const void* V_dev, int64_t m, int64_t n, int32_t k,
                            int32_t factor_dtype, const void* dY_dev, int64_t n_out,
                            const void* Blora_dev, int32_t r_lora, int32_t grad_dtype, float scale,
                            float* dA_dev, void* stream);

/*
 * The comparator of Section 3.2: randomized SVD with a Gaussian test matrix Omega (n x l),
 * the same procedure as Algorithm 1 with Omega in place of the sampled rows: Y = X Omega,
 * t x [QR; Y = X (X^T Q)], QR, B = Q^T X (l x n); for l > k the result is truncated to the k leading singular triplets
 * of B, so that U (m x k) and V (k x n) have the same shapes as loract_compress returns.
 * omegaT_dev   optional, Omega stored transposed (l x n, contiguous, dtype x_dtype); NULL =
 *              generate it on the device from p->seed (see loract_gaussian_omega_t).
 */
int loract_rsvd(const void* X_dev, const loract_params* p, const void* omegaT_dev,
                void* U_dev, void* V_dev, void* ws_dev, size_t ws_bytes,
                void* stream, int32_t* status_dev);

/*
 * Fills omegaT_dev (l x n, dtype) with the counter-based standard normal deviates the
 * comparator uses: element e = j*n + c takes h = the (e+1)-th splitmix64 output of `seed`,
 * u1 = (high32(h) + 1) / 2^32, u2 = low32(h) / 2^32, value sqrt(-2 ln u1) cos(2 pi u2).
 */
int loract_gaussian_omega_t(void* omegaT_dev, int32_t l, int64_t n, int32_t dtype,
                            uint64_t seed, void* stream);

/*
 * Pre-norm unit, Section 3.3.  The activation that is stored (and handed to loract_compress) is
 * the OUTPUT of the RMS normalisation, A = Norm(X) = X / RMS(X) * gamma (Eqs. 6-7), shared by
 * Norm and the sub-layer; only the RMS vector (m floats) is kept beside the factors.
 *
 * forward:  rms_i = sqrt(mean_j X_ij^2 + eps), A_ij = X_ij / rms_i * gamma_j.
 *   X_dev m x n (ld ldx), A_dev m x n out (ld lda), both of dtype; gamma_dev n floats;
 *   rms_dev m floats out.
 * backward (Eqs. 8-10): from the reconstructed A (= U V), the stored RMS vector and dA = dL/dA:
 *   Xbar = A / gamma, dXbar = dA * gamma,
 *   dX_ij = (dXbar_ij - Xbar_ij * mean_j(dXbar_ij Xbar_ij)) / rms_i.
 *   A_dev, dA_dev, dX_dev m x n of dtype (leading dimensions lda, ldda, lddx); gamma must be
 *   nonzero.  No workspace; enqueued on `stream`.
 */
int loract_prenorm_forward(const void* X_dev, int64_t m, int64_t n, int64_t ldx, int32_t dtype,
                           const float* gamma_dev, float eps, void* A_dev, int64_t lda,
                           float* rms_dev, void* stream);
int loract_prenorm_backward(const void* A_dev, int64_t m, int64_t n, int64_t lda, int32_t dtype,
                            const float* rms_dev, const float* gamma_dev, const void* dA_dev,
                            int64_t ldda, void* dX_dev, int64_t lddx, void* stream);

/*
 * The sub-layer around a compressed activation (Section 3.3: Z = F(Norm(X)) + X): the linear maps with what
 * follows them, their backward pass, dropout, and the norm and rotation of queries and keys.
 * Outputs that share memory with each other, with the workspace or with what the call reads are refused (LORACT_ERR_INVALID_ARG), but
 * where an output may be an input: the same address and strides, so that every element is written by whoever has read it.
 */

/* Activations of loract_linear: none, max(z, 0), z Phi(z) (by erf), z / (1 + exp(-z)). */
typedef enum { LORACT_ACT_NONE = 0, LORACT_ACT_RELU = 1, LORACT_ACT_GELU = 2, LORACT_ACT_SILU = 3 } loract_act;
/* Layouts of loract_linear's weights. */
typedef enum { LORACT_W_OUT_IN = 0, LORACT_W_IN_OUT = 1 } loract_w_layout;
#define LORACT_MAX_LORA_RANK 64
#define LORACT_MAX_HEAD 1024     /* largest head size of loract_qknorm_rope_* */

/*
 * Dropout from a counter.  Element (i, j) of an m x n matrix is kept where the 16-bit field
 *   bits 16 (j mod 4) .. 16 (j mod 4) + 15  of  splitmix64 output number  i ceil(n/4) + floor(j/4) + 1  of `seed`
 * is at least thr = floor(65536 p + 1/2) (65535 at most), and then multiplied by 65536 / (65536 - thr); all others
 * become 0 whatever they hold.  The mask is a function of seed, i and j alone: it is never stored, and the gradient
 * is the same call on the output's gradient.
 *   Y = D(X) + R
 * X_dev, R_dev (optional), Y_dev: m x n of dtype (leading dimensions ldx, ldr, ldy); Y may be X or R.  0 <= p < 1.
 */
int loract_dropout(const void* X_dev, int64_t ldx, const void* R_dev, int64_t ldr, int64_t m, int64_t n, int32_t dtype,
                   double p, uint64_t seed, void* Y_dev, int64_t ldy, void* stream);

typedef struct {
  int64_t m;             /* tokens */
  int64_t n_in, n_out;   /* sizes of the map */
  int64_t ldx;           /* leading dimensions in elements: X (backward: unused) */
  int64_t ldw;           /* W (backward: unused) */
  int64_t ldr;           /* residual (backward: unused) */
  int64_t ldy;           /* Y (backward: dY) */
  int64_t ldz;           /* Z */
  int64_t ldp;           /* backward: dP (forward: unused) */
  int32_t dtype;         /* loract_dtype of X, W, T, B_lora, R, Z (backward: of dY, Z, T, dP) */
  int32_t out_dtype;     /* loract_dtype of Y; float32 inputs require float32 (backward: unused) */
  int32_t w_layout;      /* loract_w_layout */
  int32_t act;           /* loract_act */
  int32_t r_lora;        /* columns of T, 0 = no low-rank term, at most LORACT_MAX_LORA_RANK */
  float lora_scale;
  double p_drop;         /* 0 <= p_drop < 1 */
  uint64_t seed;         /* of the dropout mask */
} loract_linear_params;

/*
 * Linear map of a sub-layer with everything that follows it:
 *   P = X W^T + lora_scale T B_lora + bias,   Y = R + D(act(P))
 * X_dev     m x n_in.   W_dev  n_out x n_in (LORACT_W_OUT_IN) or n_in x n_out (LORACT_W_IN_OUT): with the other layout's name
 *           the same weights give the input gradient dP W of the backward pass.
 * bias_dev  n_out floats, or NULL.   T_dev m x r_lora and Blora_dev r_lora x n_out, contiguous: the low-rank update with
 *           T = X A (itself a call with W = A), as B_lora of loract_lora_grad; not read if r_lora is 0.
 * R_dev     m x n_out, or NULL.   Y_dev out, m x n_out of out_dtype; Y may be R where their types and ld are the same.
 * Z_dev     out, m x n_out of dtype, or NULL: P rounded to dtype, what the backward pass reads.
 * m, n_in, n_out up to 2^30 (n_in below 8, or n_out below 8 with LORACT_W_IN_OUT: m up to 2^30 - 64), else LORACT_ERR_UNSUPPORTED, from
 * the workspace query too.
 * Sums are float32.  Workspace: loract_linear_workspace_bytes.  NaN and infinities of X and W reach the outputs they belong to.
 */
int loract_linear_workspace_bytes(const loract_linear_params* p, size_t* bytes);
int loract_linear(const void* X_dev, const void* W_dev, const float* bias_dev, const void* T_dev, const void* Blora_dev,
                  const void* R_dev, const loract_linear_params* p, void* Y_dev, void* Z_dev, void* ws_dev,
                  size_t ws_bytes, void* stream);

/*
 * Backward of loract_linear up to the products, one pass over dY and Z:
 *   dP = act'(Z) D(dY),   dbias_j = sum_i dP_ij,   dB_lora = lora_scale T^T dP
 * Z_dev     what the forward call kept; not read (may be NULL) without an activation.
 * dP_dev    out, m x n_out of dtype; may be dY or Z with the same ld.   dbias_dev out, n_out floats, or NULL.
 * dB_dev    out, r_lora x n_out floats, or NULL (then T_dev is not read).  The sums are of the unrounded float32 dP.
 * The rest of the backward pass are calls on dP: dT = lora_scale dP B_lora^T and dX = dP W + dT A^T by loract_linear,
 * dA by loract_lora_grad.  Workspace: loract_linear_backward_workspace_bytes.
 */
int loract_linear_backward_workspace_bytes(const loract_linear_params* p, size_t* bytes);
int loract_linear_backward(const void* dY_dev, const void* Z_dev, const void* T_dev, const loract_linear_params* p,
                           void* dP_dev, float* dbias_dev, float* dB_dev, void* ws_dev, size_t ws_bytes, void* stream);

/* table_dev (n_pos x rot floats): for position first + p the rot / 2 cosines, then the rot / 2 sines, of
 * (first + p) theta^(-2 i / rot); the angle is formed in float64.  rot even, theta > 0. */
int loract_rope_table(float* table_dev, int64_t n_pos, int32_t rot, double theta, int64_t first, void* stream);

typedef struct {
  int64_t m;             /* tokens */
  int32_t heads_q, heads_k;      /* heads_k may be 0 */
  int32_t d;             /* head size, at most LORACT_MAX_HEAD */
  int32_t rot;           /* leading elements of a head that are rotated: even, 0 <= rot <= d */
  int32_t interleaved;   /* pairs are (i, i + rot/2), or (2i, 2i + 1) if nonzero */
  int32_t dtype;         /* loract_dtype of queries, keys and their gradients */
  int64_t n_pos;         /* rows of the table */
  float eps;             /* >= 0 */
  /* strides in elements, token then head, the elements of a head are contiguous: inputs, outputs (backward: dq, dk),
   * and the gradients of the forward's outputs (backward only) */
  int64_t q_token, q_head, k_token, k_head;
  int64_t qo_token, qo_head, ko_token, ko_head;
  int64_t dq_token, dq_head, dk_token, dk_head;
} loract_qk_params;

/*
 * RMS norm of every head of the queries and keys and the rotation by position in one pass:
 *   y = Rot_pos(x / sqrt(mean_d x_d^2 + eps) * gamma)
 * gamma_q_dev, gamma_k_dev: d floats, or NULL (ones).  table_dev: n_pos x rot floats of loract_rope_table (unread if rot is 0).
 * pos_dev: m int32 positions, or NULL: token t stands at t.  A token with a negative position is padding: its outputs (and
 * gradients) are zero and it adds nothing to gamma's gradients; a position of n_pos or more gives NaN.
 * forward   q_out may be q, k_out may be k (with the same strides).
 * backward  from the inputs and the gradients of the outputs: dq, dk and, where not NULL, dgamma_q, dgamma_k (d floats).
 *           dq may be dq_out or q, dk dk_out or k (with the same strides).
 * The heads of an output lie apart: its larger stride is at least what all heads (or tokens) of the smaller one span.
 * No workspace in the forward direction; loract_qknorm_rope_workspace_bytes in the backward one.
 */
int loract_qknorm_rope_workspace_bytes(const loract_qk_params* p, size_t* bytes);
int loract_qknorm_rope_forward(const void* q_dev, const void* k_dev, const loract_qk_params* p, const float* gamma_q_dev,
                               const float* gamma_k_dev, const float* table_dev, const int32_t* pos_dev, void* q_out_dev,
                               void* k_out_dev, void* stream);
int loract_qknorm_rope_backward(const void* q_dev, const void* k_dev, const loract_qk_params* p, const float* gamma_q_dev,
                                const float* gamma_k_dev, const float* table_dev, const int32_t* pos_dev,
                                const void* dq_out_dev, const void* dk_out_dev, void* dq_dev, void* dk_dev,
                                float* dgamma_q_dev, float* dgamma_k_dev, void* ws_dev, size_t ws_bytes, void* stream);

/*
 * What a step ends with and what its adapters are for: their update, the loss, and the adapters of many requests.
 * Outputs that share memory with each other, with the workspace or with what the call reads are refused as above.
 */

#define LORACT_ADAMW_BLOCK 256   /* elements of a state in 8 bits that share an exponent; tensors begin at multiples of it */

typedef struct {
  double lr, beta1, beta2, eps, weight_decay;   /* lr, weight_decay >= 0; eps 0, or 2^-126 or more; 0 <= beta < 1 */
  int64_t step;          /* t, from 1 on */
  uint64_t seed;         /* of the random roundings */
  int32_t p_dtype, g_dtype;      /* loract_dtype of the parameters and of the gradients */
  int32_t state_bits;    /* 32 or 8 */
} loract_adamw_params;

/*
 * One step of AdamW over `count` tensors at once; every operation in float32 and in this order:
 *   g = grad_scale g,  m' = beta1 m + (1 - beta1) g,  v' = beta2 v + (1 - beta2) (g g),  r' = sqrt(v')
 *   p' = (1 - lr weight_decay) p - (lr / (1 - beta1^t)) (m' / (r' (1 / sqrt(1 - beta2^t)) + eps))
 * the factors of t and of the rates rounded once from 64 bits, the last quotient formed with the hardware's reciprocal (an ulp; the states do
 * not depend on it).
 * p, g, copy, n    arrays of `count` in host memory, read before the call returns: the tensors' device pointers (contiguous; p of
 *                  p_dtype, updated in place; g of g_dtype) and their sizes (0: a tensor without elements).  copy, or any entry of it, may be
 *                  NULL: else p' rounded to bf16 is written there too (float32 parameters only).
 * m_dev, v_dev     the states of all tensors one after the other, each tensor padded to a multiple of LORACT_ADAMW_BLOCK elements, 16-byte
 *                  aligned; all zero before the first step.  state_bits 32: m and v, floats; exps_dev is not read.
 *                  state_bits 8: bytes, e4m3 numbers that stand for m and r = sqrt(v) in units of 2^(exps[block][0] - 127)
 *                  and 2^(exps[block][1] - 127), the unit that takes a block's largest finite magnitude to 320/3 or more and below
 *                  640/3, but exponents of 1 at least.  What is not finite is NaN from then on; a root that is not zero stays above zero.
 * Roundings to fewer bits than 32 are random (nearest ones would hold a moment or a weight where a step's change is less than half a
 * spacing), from a counter: element e of the state takes the lower (e even) or upper half of output floor(e / 2) + 1 of the splitmix64
 * stream that starts at output t of `seed`: bits 0-9 for m, 10-19 for r, 20-31 for a bf16 parameter.  A magnitude goes up to its upper
 * neighbour where its place between the two plus (bits + 1/2) / 2^10 (2^12) is at least 1.
 * lr_dev, step_dev, grad_scale_dev   a float, an int64 and a float in device memory, read when the step runs, or NULL: p->lr, p->step, 1.  A
 *                  captured step that is replayed takes what changes from these.  A step below 1 there gives NaN or infinities.
 * n up to 2^33 each, 2^39 together.  No workspace.
 */
int loract_adamw(void* const* p, const void* const* g, void* const* copy, const int64_t* n, int64_t count,
                 const loract_adamw_params* params, void* m_dev, void* v_dev, uint8_t* exps_dev, const float* lr_dev,
                 const int64_t* step_dev, const float* grad_scale_dev, void* stream);

#define LORACT_MAX_TOP 64        /* most alternatives of loract_token_logprobs */

typedef struct {
  int64_t m, n;          /* tokens, size of the vocabulary */
  int64_t ld, ldg;       /* leading dimensions in elements of the logits and of the gradient (ldg unused without one) */
  int32_t dtype;         /* loract_dtype of logits and gradient */
  int32_t target_bits;   /* of the targets: 32 or 64 */
  int32_t top;           /* alternatives, 0 to LORACT_MAX_TOP and at most n (only loract_token_logprobs reads it) */
  int32_t reserved;      /* 0 */
  double temperature;    /* T > 0 */
} loract_logprob_params;

/*
 * Log probabilities of given tokens under p = softmax(x / T), rows of an m x n matrix of logits; statistics and sums in float32.
 * x_dev          m x n (leading dimension ld).   targets_dev: m integers, or NULL.  A negative one is none (padding); one of n or more
 *                gives NaN.
 * logp_dev       out, m floats, or NULL: log p of the target, 0 without one.  Without targets_dev it must be NULL.
 * stats_dev      out, 3 x m floats: the row's maximum M, log2 of the sum of exp((x - M) / T), the entropy -sum p log p.
 * top_logp_dev, top_ids_dev    out, m x top floats and int32 (NULL if top is 0): the log probabilities and indices of the largest logits, ties
 *                in the order of their indices.  What is no number counts as -inf here.
 * A row of nothing but -inf (a mask that leaves nothing) has the log probabilities -inf, the entropy 0 and the statistics -inf, 0, 0;
 * one with NaN or +inf has NaN for all of them but, perhaps, the maximum.  m and n up to 2^30.
 */
int loract_token_logprobs_workspace_bytes(const loract_logprob_params* p, size_t* bytes);
int loract_token_logprobs(const void* x_dev, const void* targets_dev, const loract_logprob_params* p, float* logp_dev,
                          float* stats_dev, float* top_logp_dev, int32_t* top_ids_dev, void* ws_dev, size_t ws_bytes, void* stream);

/*
 * Its gradient, from the logits and stats_dev as the forward call (of the same x, temperature) left them:
 *   grad_ij = (1 / T) [ d_logp_i (delta_j,target - p_ij) - d_entropy_i p_ij (log p_ij + H_i) ]
 * d_logp_dev, d_entropy_dev: m floats each, or NULL (zeros; at least one is given); d_logp of a token without a target does not count, and a row
 * whose two gradients are zero is zero whatever it holds, as is a row of nothing but -inf.  A target of n or more gives a row of NaN.
 * grad_dev       out, m x n of dtype (ldg); may be x_dev with the same ld.  No workspace.
 */
int loract_token_logprobs_backward(const void* x_dev, const void* targets_dev, const loract_logprob_params* p, const float* stats_dev,
                                   const float* d_logp_dev, const float* d_entropy_dev, void* grad_dev, void* stream);

/*
 * Both in one call, where the gradients of the outputs are known before them (a mean over tokens): rows that fit a workgroup's registers
 * are read once.  grad_dev may be x_dev with the same ld.  Workspace: loract_token_logprobs_workspace_bytes with top = 0.
 */
int loract_token_logprobs_grad(const void* x_dev, const void* targets_dev, const loract_logprob_params* p, const float* d_logp_dev,
                               const float* d_entropy_dev, float* logp_dev, float* stats_dev, void* grad_dev, void* ws_dev, size_t ws_bytes,
                               void* stream);

typedef struct {
  int64_t m;             /* tokens */
  int64_t n_in, n_out;   /* sizes of the shared projection */
  int64_t adapters;
  int64_t ldx, ldr, ldy; /* leading dimensions in elements: X, R, Y */
  int32_t dtype;         /* loract_dtype of X, A and B */
  int32_t out_dtype;     /* of R and Y; float32 inputs require float32 */
  int32_t r;             /* rank of all adapters, 1 to LORACT_MAX_LORA_RANK (smaller ones have columns of A or rows of B that are zero) */
  int32_t reserved;      /* 0 */
} loract_requests_params;

/*
 * The adapters of many requests beside a projection that they share (serving):
 *   Y_i = R_i + scale_a (X_i A_a) B_a   with a = ids_i
 * X_dev      m x n_in.   A_dev adapters x n_in x r and B_dev adapters x r x n_out, contiguous: each pair as in loract_linear's low-rank term.
 * ids_dev    m int32: the token's adapter, in any order (neighbours that share one cost least); a negative one is none, Y_i = R_i; one that
 *            is not there (adapters or more) gives a row of NaN.
 * scales_dev adapters floats, or NULL (ones).   R_dev m x n_out, or NULL (zeros).
 * Y_dev      out, m x n_out; may be R with the same ld: then rows without an adapter are left as they are.
 * Sums are float32, and X A keeps all 24 digits between the products.  What an adapter or a token holds reaches the tokens with that
 * adapter and that token alone, be it infinite: an infinite element of B gives infinity by the sign of X A (of a magnitude of 2^-100 or more; 0 gives NaN).  adapters, n_in up to 2^30; m up to 2^27, n_out up to 2^24, and less together where a launch could not
 * hold them (LORACT_ERR_UNSUPPORTED, from the workspace query too).
 */
int loract_lora_requests_workspace_bytes(const loract_requests_params* p, size_t* bytes);
int loract_lora_requests(const void* X_dev, const void* A_dev, const void* B_dev, const int32_t* ids_dev, const float* scales_dev,
                         const void* R_dev, const loract_requests_params* p, void* Y_dev, void* ws_dev, size_t ws_bytes, void* stream);

/*
 * Per-kernel timing with HIP events on the stream the kernels are launched on.
 * begin: start bracketing every kernel launch of this library with event records.
 * end:   stop, wait for the recorded events, and aggregate by kernel name.
 * count/get: read the aggregate (name, total milliseconds, number of launches).
 * Recording adds two event records per launch; leave it off when measuring end-to-end time.
 */
int loract_profile_begin(void);
int loract_profile_end(void);
int loract_profile_count(void);
int loract_profile_get(int i, char* name_buf, int name_buf_len, double* total_ms,
                       int64_t* launches);

#ifdef __cplusplus
}
#endif
#endif /* LORACT_H */
