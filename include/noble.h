/*
 * noble.h -- C ABI of the NOBLE linear layer with the CosNet branch on GB300.
 *
 * The layer (NOBLE, arXiv 2603.06492, Eq. 1 in Section 3.1) is
 *
 *     y = x W^T + bias + sigma(x W_down^T) W_up^T
 *
 * written here with nn.Linear-style "out x in" weight storage, where the paper
 * writes the same thing with row vectors as x W + b + sigma(x W_down) W_up.
 * sigma is CosNet (Eq. 2 in Section 3.2; Eqs. 5-7 in Appendix A), applied per
 * token to h = x W_down^T in R^r:
 *
 *     a = cos(omega1 * h + phi1)           elementwise, learnable omega1, phi1
 *     b = a M          b_j = sum_i a_i M[i][j]
 *     c = cos(omega2 * b + phi2)           elementwise, learnable omega2, phi2
 *     sigma(h) = c
 *
 * Eq. 2 writes M . cos(...) for a column vector; this library reads it with
 * row vectors as b = a M, i.e. M[i][j] couples input channel i to output
 * channel j.  The backward pass is the chain rule through these definitions
 * (the paper trains with autograd and does not write it out).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Every pointer argument is a DEVICE pointer on the current CUDA device,
 *    except `desc`, which is a host pointer read during the call only.
 *  - The caller owns and allocates every buffer; no entry point allocates or
 *    frees device memory.  Cached TMA descriptors live in host memory.
 *  - All tensors are dense, row-major and contiguous:
 *        x [T][d_in]      y, dy [T][d_out]      dx [T][d_in]
 *        W [d_out][d_in]  W_down [r][d_in]      W_up [d_out][r]
 *        M [r][r]         omega1, phi1, omega2, phi2 [r]   bias [d_out]
 *  - Operand dtype (x, W, W_down, W_up, y, dy, dx) is desc->dtype: bf16 or
 *    fp32.  omega, phi, M, bias and every parameter gradient are always fp32.
 *    bf16 operands use tensor cores with fp32 accumulation; fp32 operands use
 *    exact fp32 FMA (no TF32), a validation mode.
 *  - Calls are asynchronous on `stream` (a cudaStream_t; NULL = legacy
 *    default stream).  Outputs are overwritten, never accumulated into.
 *  - Arguments are checked on the host before anything is enqueued.  On an
 *    argument error the call returns a status other than NOBLE_OK, enqueues
 *    nothing and leaves every output untouched; noble_last_error() then
 *    describes it.  NOBLE_ERR_CUDA from a failed launch part-way leaves the
 *    outputs undefined.
 *  - Requirements: T >= 0; d_in, d_out >= 8 and multiples of 8;
 *    r in {0, 16, 32, 64, 128, 256} (r = 0 is the plain layer, and the branch
 *    pointers may then be NULL); every pointer 16-byte aligned.  With T == 0
 *    the per-token pointers (x, y, dy, dx) and `saved` may be NULL; the
 *    forward pass then does nothing and the backward pass writes zero
 *    gradients.
 *  - Kernels never wait without a bound.  A wait that runs out records
 *    NOBLE_ERR_TIMEOUT in a device status word, which
 *    noble_get_device_status() reports.
 */
#ifndef NOBLE_H
#define NOBLE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st *noble_stream; /* same type as cudaStream_t */

typedef enum {
    NOBLE_OK = 0,
    NOBLE_ERR_INVALID_ARG = 1,     /* NULL pointer, negative or bad size      */
    NOBLE_ERR_MISALIGNED = 2,      /* a pointer is not 16-byte aligned         */
    NOBLE_ERR_UNSUPPORTED = 3,     /* r, d_in, d_out or dtype not supported    */
    NOBLE_ERR_BUFFER_TOO_SMALL = 4,/* saved / workspace size below the query   */
    NOBLE_ERR_CUDA = 5,            /* a CUDA runtime or driver call failed     */
    NOBLE_ERR_TIMEOUT = 6,         /* a device-side bounded wait expired       */
    NOBLE_ERR_NO_DEVICE = 7        /* no usable sm_103 device is current       */
} noble_status;

typedef enum { NOBLE_BF16 = 0, NOBLE_FP32 = 1 } noble_dtype;

/* desc->flags bits */
#define NOBLE_FLAG_SIMT_ONLY 1u /* bf16: run every step on CUDA cores (fp32
                                   FMA), not tensor cores; a second path for
                                   cross-checking the tensor-core kernels */
#define NOBLE_FLAG_INFERENCE 2u /* forward only, for inference (the branch
                                   stays in the model at inference, the
                                   Limitations section): on the
                                   tensor-core path h and b are not written
                                   and `saved` holds only c, the second K
                                   segment of the output GEMM (and the ready
                                   flags of a fused launch).  The backward
                                   entry points reject such a descriptor
                                   (NOBLE_ERR_INVALID_ARG).  The CUDA-core
                                   paths (fp32, SIMT_ONLY) use the full saved
                                   layout as scratch. */
#define NOBLE_FLAG_SIGMA_COS1 4u /* bottleneck sigma(h) = cos(omega1 h + phi1),
                                    the single-cosine activation of the
                                    ablation (Section 4.4, Table 5); M,
                                    omega2, phi2 are not used (may be NULL)
                                    and dM, domega2, dphi2 are written as 0 */
#define NOBLE_FLAG_SIGMA_IDENTITY 8u /* bottleneck sigma(h) = h, the linear
                                    collapse to x (W + W_down W_up)
                                    (Sections 1 and 3.1); omega, phi and M are
                                    not used (may be NULL) and their
                                    gradients are written as 0.  Not together
                                    with NOBLE_FLAG_SIGMA_COS1. */
/* The other activations f of the ablation (Section 4.4, Table 5), a 2-bit
 * field: sigma(h) = f(f(h) M) (two layers around the mixing matrix), or with
 * NOBLE_FLAG_SIGMA_SINGLE sigma(h) = f(h).  tanh; LeakyReLU f(u) = u for
 * u > 0, 0.01 u otherwise (the paper gives no slope; 0.01 is the common
 * default); GELU in its exact form u/2 (1 + erf(u / sqrt 2)).  The paper
 * gives frequencies and phases to the cosine only: omega1, phi1, omega2, phi2
 * are not used (may be NULL) and their gradients are written as 0; dM is
 * written as 0 for one layer.  Not together with NOBLE_FLAG_SIGMA_IDENTITY. */
#define NOBLE_FLAG_ACT_TANH 32u
#define NOBLE_FLAG_ACT_LEAKYRELU 64u
#define NOBLE_FLAG_ACT_GELU 96u
#define NOBLE_FLAG_ACT_MASK 96u
/* one activation layer, no mixing matrix: with the cosine (no ACT bits) the
 * same as NOBLE_FLAG_SIGMA_COS1 */
#define NOBLE_FLAG_SIGMA_SINGLE NOBLE_FLAG_SIGMA_COS1
/* The three-layer cosine of the ablation (Section 4.4, Table 5): CosNet with a
 * second mixing matrix and a third cosine,
 *     a2 = cos(omega2 b + phi2), b2 = a2 M2, c = cos(omega3 b2 + phi3),
 * b2_j = sum_i a2_i M2[i][j].  It has parameters the other variants lack, so
 * only noble_linear_fwd_cos3 / noble_linear_bwd_cos3 accept it (and they
 * accept nothing else); saved holds h, b, b2 (fp32) and c.  Not together with
 * another NOBLE_FLAG_SIGMA_* or NOBLE_FLAG_ACT_* bit. */
#define NOBLE_FLAG_SIGMA_COS3 128u
#define NOBLE_FLAG_FUSED_BRANCH 16u /* tensor-core path, CosNet bottleneck,
                                    r in {64, 128}: run the r-wide GEMM and
                                    the CosNet (forward h = x W_down^T and
                                    Eq. 2; backward dc = dy W_up and its chain
                                    rule) as tiles of the output GEMM launch
                                    (y, dx) instead of kernels of their own.
                                    Same results up to summation order.  Off by default:
                                    slower than the separate kernels at the
                                    measured shapes.  Other shapes and
                                    variants always run separately. */

typedef struct {
    int64_t T;      /* tokens (rows of x)                          */
    int64_t d_in;   /* input features                              */
    int64_t d_out;  /* output features                             */
    int64_t r;      /* bottleneck rank; 0 = plain linear layer     */
    int32_t dtype;  /* noble_dtype of the operands                 */
    uint32_t flags; /* NOBLE_FLAG_* bits; 0 = default              */
} noble_linear_desc;

/*
 * Bytes of the saved-activation buffer that noble_linear_fwd writes and
 * noble_linear_bwd reads (per token: h and b in fp32, c in the operand dtype;
 * only c with NOBLE_FLAG_INFERENCE on the tensor-core path), plus, when the
 * forward runs the bottleneck inside the output GEMM (NOBLE_FLAG_FUSED_BRANCH
 * on the tensor-core path, CosNet, r in {64, 128}), one 32-bit ready flag per
 * 128 tokens that the forward resets itself.  0 when r == 0.
 * Returns 0 for an invalid descriptor as well; the entry points then report
 * why.
 */
size_t noble_linear_saved_bytes(const noble_linear_desc *desc);

/*
 * Bytes of scratch memory noble_linear_bwd needs (dh in the operand dtype,
 * dc and db in fp32, and fixed-size per-block partial sums for dM, domega
 * and dphi).  Nonzero for every valid descriptor.
 */
size_t noble_linear_bwd_workspace_bytes(const noble_linear_desc *desc);

/*
 * Forward pass, Eq. 1 with sigma = CosNet (Eq. 2; Eqs. 5-7).
 *   In : x, W, bias (NULL = no bias), W_down, omega1, phi1, M, omega2,
 *        phi2, W_up.
 *   Out: y [T][d_out] (operand dtype);
 *        saved: `saved_bytes` >= noble_linear_saved_bytes(desc) bytes,
 *        opaque, to be passed unchanged to noble_linear_bwd (may be NULL
 *        when r == 0).  A smaller size returns NOBLE_ERR_BUFFER_TOO_SMALL.
 */
noble_status noble_linear_fwd(const noble_linear_desc *desc,
                              const void *x, const void *W, const float *bias,
                              const void *W_down, const float *omega1,
                              const float *phi1, const float *M,
                              const float *omega2, const float *phi2,
                              const void *W_up, void *y, void *saved,
                              size_t saved_bytes, noble_stream stream);

/*
 * Backward pass: gradients of L = sum(y * dy) by the chain rule through Eq. 1
 * and Eq. 2.
 *   In : dy [T][d_out] (operand dtype), the forward inputs, and `saved` as
 *        written by noble_linear_fwd with the same desc and parameters.
 *   Out: dx [T][d_in] (operand dtype);
 *        dW [d_out][d_in], dbias [d_out] (NULL = skip), dW_down [r][d_in],
 *        dM [r][r], domega1, dphi1, domega2, dphi2 [r], dW_up [d_out][r],
 *        all fp32 (branch gradients may be NULL when r == 0).
 *   workspace: `workspace_bytes` >= noble_linear_bwd_workspace_bytes(desc)
 *        bytes of device scratch, contents undefined on entry and exit.
 *        Smaller saved or workspace sizes return NOBLE_ERR_BUFFER_TOO_SMALL.
 * The fp32 reductions over tokens (dM, domega, dphi, dbias) run in a fixed
 * order, so repeated calls give bit-identical results.
 */
noble_status noble_linear_bwd(const noble_linear_desc *desc, const void *dy,
                              const void *x, const void *W,
                              const void *W_down, const float *omega1,
                              const float *phi1, const float *M,
                              const float *omega2, const float *phi2,
                              const void *W_up, const void *saved,
                              size_t saved_bytes, void *dx,
                              float *dW, float *dbias, float *dW_down,
                              float *dM, float *domega1, float *dphi1,
                              float *domega2, float *dphi2, float *dW_up,
                              void *workspace, size_t workspace_bytes,
                              noble_stream stream);

/*
 * Optimizer step: AdamW with decoupled weight decay (the optimizer of the
 * paper's training runs, Section 4.1: beta1 0.9, beta2 0.98, weight decay
 * 0.01) over a batch of parameter tensors, each with its own learning rate,
 * in one fused pass per 16 tensors.  For step t >= 1, elementwise with the
 * tensor's learning rate a = lr * lr_mult:
 *     p <- p - a * weight_decay * p             (only if `decay`)
 *     m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2
 *     p <- p - a / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * All arrays are device memory, fp32, `n` elements, updated in place (g is
 * read only).  `param_bf16` (optional) receives the new values rounded to
 * bf16, e.g. the operand copy of W, W_down or W_up the layer's kernels read.
 * Pointers must be 16-byte aligned (param_bf16 8-byte aligned).
 * Errors: NOBLE_ERR_INVALID_ARG for NULL pointers, n < 0, t < 1 or bad
 * hyperparameters; NOBLE_ERR_MISALIGNED.  Nothing is enqueued on error.
 */
typedef struct {
    float *param;
    void *param_bf16; /* optional */
    const float *grad;
    float *exp_avg;
    float *exp_avg_sq;
    int64_t n;
    float lr_mult;
    int32_t decay; /* 1: apply weight decay to this tensor */
} noble_adamw_tensor;

typedef struct {
    float lr, beta1, beta2, eps, weight_decay;
    int64_t step; /* t, counted from 1 */
} noble_adamw_hparams;

noble_status noble_adamw_step(const noble_adamw_tensor *tensors, int n_tensors,
                              const noble_adamw_hparams *hp, noble_stream stream);

/*
 * NOBLE's per-group learning-rate multipliers (Section 3.3 and the defaults of
 * Appendix A), with rho = min(d_in, d_out) / r:
 *   out[0] W, bias, W_down: 1      out[1] W_up: rho^(2 gamma)
 *   out[2] M: rho^gamma_M          out[3] omega1, omega2: omega_mult
 *   out[4] phi1, phi2: phi_mult
 * Paper defaults: gamma 0.3, gamma_M 0.45, omega_mult 3, phi_mult 5.
 * Host only.  NOBLE_ERR_INVALID_ARG for r == 0 or a NULL pointer.
 */
noble_status noble_linear_lr_multipliers(const noble_linear_desc *desc, float gamma, float gamma_M,
                                         float omega_mult, float phi_mult, float out[5]);

/*
 * Gradient bucket for data-parallel training (the paper trains on 8 GPUs
 * with data parallelism, Section 4.1.1).  Tokens are split across ranks; the
 * forward needs no exchange, and every parameter gradient is a sum over
 * tokens, so the one exchange of a step is an all-reduce (sum) of the
 * parameter gradients.  This describes one flat fp32 buffer holding all of a
 * layer's parameter gradients, so that noble_linear_bwd writes straight into
 * it (pass bucket + offset[i] as the i-th gradient pointer) and one
 * collective per layer reduces them.
 *
 * Order of the slots (index: gradient, element count):
 *   0 dW [d_out][d_in]   1 dbias [d_out]    2 dW_down [r][d_in]
 *   3 dW_up [d_out][r]   4 dM [r][r]        5 domega1 [r]   6 dphi1 [r]
 *   7 domega2 [r]        8 dphi2 [r]
 *   9 dM2 [r][r]  10 domega3 [r]  11 dphi3 [r]  (NOBLE_FLAG_SIGMA_COS3 only)
 * offset[i] is the byte offset of slot i from the start of the bucket, a
 * multiple of NOBLE_GRAD_ALIGN; count[i] its element count (0 for a slot the
 * descriptor does not have: the branch slots when r == 0, the three-layer
 * slots without NOBLE_FLAG_SIGMA_COS3).  total_bytes is the bucket size, a
 * multiple of NOBLE_GRAD_ALIGN.  Padding between slots is never written.
 * Host only; no CUDA call.  NOBLE_ERR_INVALID_ARG for NULL pointers or an
 * invalid descriptor.
 */
#define NOBLE_GRAD_COUNT 12
#define NOBLE_GRAD_ALIGN 256u
typedef struct {
    size_t offset[NOBLE_GRAD_COUNT];
    size_t count[NOBLE_GRAD_COUNT];
    size_t total_bytes;
} noble_grad_bucket;

noble_status noble_linear_grad_bucket(const noble_linear_desc *desc, noble_grad_bucket *out);

/*
 * Backward pass without a caller workspace, for callers that cannot allocate
 * device memory: code that runs inside a host framework or plugin which owns
 * every device allocation and hands its extensions no allocator, or a
 * real-time loop that forbids allocation once it has started.  The paper has
 * no counterpart; this is an interface convenience.
 *
 * Same arguments, results and errors as noble_linear_bwd, minus `workspace`
 * and `workspace_bytes`: the scratch is a static device array inside the
 * library, NOBLE_NOALLOC_SCRATCH_BYTES (64 MiB and 256 bytes) long, which every GPU that
 * loads the library holds until the process exits.  No cudaMalloc, cudaFree
 * or other allocating call is made.
 *  - A shape whose noble_linear_bwd_workspace_bytes() exceeds that size is
 *    rejected with NOBLE_ERR_BUFFER_TOO_SMALL before anything is enqueued.
 *  - The first call in a CUDA context looks up the array's device address
 *    (with that device current) and caches it for that context, so a device
 *    reset, which gives a new context, is followed by a new lookup; make the
 *    first call in a context before any stream capture.
 *  - Every call on a device shares the one array, and it keeps the last
 *    call's contents.  Nothing in it needs to start at zero: what a call reads
 *    there it has written itself.  Calls whose work overlaps on the
 *    GPU (other streams, other host threads) race on the array and give wrong
 *    results; the caller must order them, e.g. on a single stream.
 */
#define NOBLE_NOALLOC_SCRATCH_BYTES ((64u << 20) + 256u)
/*
 * Three-layer cosine bottleneck (NOBLE_FLAG_SIGMA_COS3): the extra parameters
 * M2 [r][r], omega3, phi3 [r] (fp32, device) and their gradients.  All are
 * required (not NULL) when r > 0.
 */
typedef struct {
    const float *M2;
    const float *omega3;
    const float *phi3;
} noble_cos3_params;
typedef struct {
    float *dM2;
    float *domega3;
    float *dphi3;
} noble_cos3_grads;

/* noble_linear_fwd for a NOBLE_FLAG_SIGMA_COS3 descriptor; the other
 * arguments as there.  Errors as noble_linear_fwd, and NOBLE_ERR_INVALID_ARG
 * for a descriptor without the flag. */
noble_status noble_linear_fwd_cos3(const noble_linear_desc *desc, const void *x,
                                   const void *W, const float *bias,
                                   const void *W_down, const float *omega1,
                                   const float *phi1, const float *M,
                                   const float *omega2, const float *phi2,
                                   const noble_cos3_params *p3, const void *W_up,
                                   void *y, void *saved, size_t saved_bytes,
                                   noble_stream stream);

/* noble_linear_bwd for a NOBLE_FLAG_SIGMA_COS3 descriptor, also writing
 * g3->dM2 = sum_t a2^T db2, g3->domega3, g3->dphi3 (overwritten).  The
 * workspace size is noble_linear_bwd_workspace_bytes of the same descriptor. */
noble_status noble_linear_bwd_cos3(const noble_linear_desc *desc, const void *dy,
                                   const void *x, const void *W,
                                   const void *W_down, const float *omega1,
                                   const float *phi1, const float *M,
                                   const float *omega2, const float *phi2,
                                   const noble_cos3_params *p3, const void *W_up,
                                   const void *saved, size_t saved_bytes, void *dx,
                                   float *dW, float *dbias, float *dW_down,
                                   float *dM, float *domega1, float *dphi1,
                                   float *domega2, float *dphi2,
                                   const noble_cos3_grads *g3, float *dW_up,
                                   void *workspace, size_t workspace_bytes,
                                   noble_stream stream);

noble_status noble_linear_bwd_noalloc(const noble_linear_desc *desc,
                                      const void *dy, const void *x,
                                      const void *W, const void *W_down,
                                      const float *omega1, const float *phi1,
                                      const float *M, const float *omega2,
                                      const float *phi2, const void *W_up,
                                      const void *saved, size_t saved_bytes,
                                      void *dx, float *dW, float *dbias,
                                      float *dW_down, float *dM,
                                      float *domega1, float *dphi1,
                                      float *domega2, float *dphi2,
                                      float *dW_up, noble_stream stream);

/*
 * Attention between a QKV and an output projection
 * ------------------------------------------------
 * The paper's models are transformers: what stands between two of their NOBLE
 * layers is attention over the heads of the QKV projection's output, with
 * rotary positions (Section 4.1.1).  In training noble_rope_fwd and
 * noble_attn_fwd run between the two projections and their _bwd counterparts
 * on the way back; in generation noble_kv_append and noble_attn_paged do.
 * The conventions above hold, except that tensors of heads have strides:
 */
typedef struct {
    void *p;           /* first feature of head 0 of token 0                   */
    int64_t row, head; /* elements from one token / one head to the next       */
} noble_heads;
/* Token t of head h is the d contiguous elements at p + t * row + h * head, in
 * the descriptor's dtype.  p and both strides are multiples of 16 bytes; a
 * stride may be 0 or negative for tensors that are only read.  The elements of
 * a tensor that is written must not overlap each other.  p may be NULL when
 * the tensor has no elements. */

/*
 * Rotary positions with per-head norms.  Each head x of the queries and keys is
 * first normalised by its root mean square (NOBLE_ROPE_NORM), then its first
 * `rot` features are rotated in pairs by the angles of its token's position:
 *     n = gain * x / sqrt(mean(x^2) + eps)          over all d features
 *     y_a = n_a cos - n_b sin,  y_b = n_b cos + n_a sin   for the pairs (a, b)
 * Pair i is the features (i, i + rot/2), or (2i, 2i + 1) with
 * NOBLE_ROPE_INTERLEAVED.  Features from `rot` on keep n.  Row p of `table`
 * holds position p's rot/2 cosines, then its rot/2 sines (noble_rope_table, or
 * the caller's own).
 */
#define NOBLE_ROPE_INTERLEAVED 1u
#define NOBLE_ROPE_NORM 2u
typedef struct {
    int64_t T;         /* tokens                                               */
    int64_t n_q, n_kv; /* heads of the queries, and of the keys (and values)   */
    int64_t d;         /* head size: a multiple of 8, 8 to 256                 */
    int64_t rot;       /* leading features that rotate: even, 0 to d           */
    int64_t positions; /* rows of the table                                    */
    float eps;         /* >= 0                                                 */
    int32_t dtype;     /* noble_dtype of the heads                             */
    uint32_t flags;    /* NOBLE_ROPE_* bits                                    */
} noble_rope_desc;

/*
 * Fills table[positions][rot] (fp32, device) for position p and pair i with
 * amplitude * cos / sin of p * f_i, f_i = base^(-2i/rot), each angle computed
 * in fp64.  For contexts longer than a model was trained on, frequencies are
 * scaled down by parts: with turns t_i = original * f_i / (2 pi) over the
 * original context, f_i is kept where t_i >= high_turns, divided by `factor`
 * where t_i <= low_turns, and in between
 *     f_i (g + (1 - g) / factor),  g = (t_i - low_turns) / (high_turns - low_turns).
 * factor 1 keeps every frequency; low_turns = high_turns = infinity divides
 * all of them.  `scaling` may be NULL: base 10000, factor 1, amplitude 1.
 */
typedef struct {
    double base;       /* > 0                                                  */
    double factor;     /* > 0                                                  */
    double original;   /* positions of the original context, > 0               */
    double low_turns, high_turns; /* low_turns <= high_turns                   */
    double amplitude;  /* finite                                               */
} noble_rope_scaling;
noble_status noble_rope_table(int64_t positions, int64_t rot, const noble_rope_scaling *scaling,
                              float *table, noble_stream stream);

/*
 * Forward: q_out, k_out from q, k (which they may be, with the same strides).
 *   pos     [T]: each token's position.  One outside [0, positions) is a
 *           caller's error: its outputs are written as 0 and
 *           noble_get_device_status() reports it (NOBLE_ERR_CUDA).
 *   gain_q, gain_k [d] fp32 (NULL: all ones); not read without NOBLE_ROPE_NORM.
 */
noble_status noble_rope_fwd(const noble_rope_desc *desc, const noble_heads *q, const noble_heads *k,
                            const int32_t *pos, const float *table, const float *gain_q, const float *gain_k,
                            const noble_heads *q_out, const noble_heads *k_out, noble_stream stream);

/*
 * Backward: with w the rotation of dy by the negative angle and xn = x / rms,
 *     dgain = sum over tokens and heads of w * xn
 *     dx    = (gain * w - xn * mean(gain * w * xn)) / rms
 * (dx = w without NOBLE_ROPE_NORM).  A token whose position is outside the table
 * has dx = 0 and no part in dgain, whatever its inputs are, and is reported as above.  q and k are the forward's inputs (NULL
 * descriptors allowed without NOBLE_ROPE_NORM); dq_in, dk_in may be dq, dk with
 * the same strides.  dgain_q, dgain_k [d] fp32, NULL to skip; they are added up
 * in a fixed order, and not written without NOBLE_ROPE_NORM.
 */
size_t noble_rope_bwd_workspace_bytes(const noble_rope_desc *desc);
noble_status noble_rope_bwd(const noble_rope_desc *desc, const noble_heads *dq, const noble_heads *dk,
                            const noble_heads *q, const noble_heads *k, const int32_t *pos, const float *table,
                            const float *gain_q, const float *gain_k, const noble_heads *dq_in,
                            const noble_heads *dk_in, float *dgain_q, float *dgain_k, void *workspace,
                            size_t workspace_bytes, noble_stream stream);

/*
 * A cache of keys and values in pages.  Token `t` of page `n` and head `h` is
 * the d contiguous elements at n * page + t * row + h * head, in k and in v;
 * all three strides are multiples of 16 bytes, and 64-bit throughout.
 */
typedef struct {
    void *k, *v;
    int64_t pages, page_size; /* page_size: tokens of a page, 1 to 2^20        */
    int64_t page, row, head;  /* strides in elements                           */
} noble_kv_cache;

/*
 * noble_rope_fwd on new tokens, with the keys, and the values as they are,
 * written into the cache: token t goes to slots[t] = page * page_size + place.
 * A negative slot is not stored (a padding token).  A slot beyond the cache is
 * a caller's error: it is not stored, and noble_get_device_status() reports
 * it.  Two tokens of a call must not share a slot.
 */
noble_status noble_kv_append(const noble_rope_desc *desc, const noble_heads *q, const noble_heads *k,
                             const noble_heads *v, const int32_t *pos, const int64_t *slots, const float *table,
                             const float *gain_q, const float *gain_k, const noble_heads *q_out,
                             const noble_kv_cache *cache, noble_stream stream);

/*
 * Attention over packed documents.  The T tokens are documents one behind the
 * other, document n being the tokens doc_start[n] <= t < doc_start[n + 1].
 * Query i of head h sees the keys j of its document with
 *     j <= i, or j < doc_start + prefix[n]    (NOBLE_ATTN_CAUSAL; prefix optional)
 *     i - j < window, and without NOBLE_ATTN_CAUSAL j - i < window  (window > 0)
 * of head h / (n_q / n_kv), and
 *     s_ij = scale q_i.k_j;  s_ij = softcap tanh(s_ij / softcap)    (softcap > 0)
 *     s_ij = s_ij - slope[h] |i - j|                                (slope optional)
 *     o_i  = sum_j exp(s_ij - lse_i) v_j,  lse_i = log sum_j exp(s_ij).
 * A query that sees nothing (a token of no document) has o = 0, lse = -inf and
 * takes no part in any gradient.
 * doc_start [n_docs + 1] must ascend within [0, T]; if it does not, results are
 * undefined, but no access leaves the tensors.
 * What a query does not see does not change its results, whatever values are
 * there, infinities and NaN too.  Of padding, the tokens behind the last document,
 * that holds to the bit.  Other infinities and NaN make the rows that share
 * a block of 128 tokens with them, and do not see them, be computed again one by
 * one: in fp32 throughout, so that their last digits may differ, and slowly, about
 * 1 us per query and key on one warp (64 such keys under 8 query heads of a
 * 32768-token document take the backward 3.8 s).
 *
 * bf16 runs on the tensor cores, with fp32 scores, softmax and sums; the
 * probabilities and the scores' gradients are rounded to bf16 for their
 * products.  fp32 operands run in fp32 FMA, as does bf16 with
 * NOBLE_ATTN_SIMT_ONLY or with a stride of 0, below 0 or from 2^38 on (in
 * elements).  Outputs must not overlap inputs.  Results do not depend on the
 * order in which a GPU runs the blocks: repeated calls agree bit by bit.
 */
#define NOBLE_ATTN_CAUSAL 1u
#define NOBLE_ATTN_SIMT_ONLY 2u
typedef struct {
    int64_t T;         /* tokens, up to 2^24                                   */
    int64_t n_docs;    /* documents, up to 2^24                                */
    int64_t n_q, n_kv; /* heads: n_q a multiple of n_kv                        */
    int64_t d;         /* head size: a multiple of 8, 8 to 128                 */
    int64_t window;    /* 0: none                                              */
    float scale;       /* of the products, usually 1 / sqrt(d)                 */
    float softcap;     /* 0: none                                              */
    int32_t dtype;     /* noble_dtype of q, k, v, o and their gradients        */
    uint32_t flags;    /* NOBLE_ATTN_* bits                                    */
} noble_attn_desc;

/* lse: fp32 [n_q][T]; prefix [n_docs] and slope [n_q] may be NULL. */
noble_status noble_attn_fwd(const noble_attn_desc *desc, const noble_heads *q, const noble_heads *k,
                            const noble_heads *v, const int32_t *doc_start, const int32_t *prefix,
                            const float *slope, const noble_heads *o, float *lse, noble_stream stream);

/*
 * Backward: dq, dk, dv of L = sum(o * do), from the forward's inputs and its o
 * and lse.  The gradients of a key head are summed over the query heads that
 * share it.  workspace as for noble_linear_bwd.
 */
size_t noble_attn_bwd_workspace_bytes(const noble_attn_desc *desc);
noble_status noble_attn_bwd(const noble_attn_desc *desc, const noble_heads *d_o, const noble_heads *q,
                            const noble_heads *k, const noble_heads *v, const int32_t *doc_start,
                            const int32_t *prefix, const float *slope, const noble_heads *o, const float *lse,
                            const noble_heads *dq, const noble_heads *dk, const noble_heads *dv, void *workspace,
                            size_t workspace_bytes, noble_stream stream);

/*
 * Attention of the newest q_len tokens of each sequence over a cache.  Token t
 * of sequence n (row n * q_len + t of q and o) is at position kv_len[n] - q_len
 * + t and sees the keys of the positions up to its own, with `window`, scale,
 * softcap and slope as in noble_attn_fwd.  Position j of sequence n lies in
 * page page_table[n][j / page_size] of the cache, at place j % page_size.  A
 * token at a negative position sees nothing: o = 0, lse = -inf.
 * Only what some new token of the sequence sees is read from the cache.  A page
 * number outside the cache, or a kv_len beyond max_pages * page_size or max_len,
 * is a caller's error: the keys concerned are left out, and
 * noble_get_device_status() reports it.
 * Scores, softmax and sums are fp32; of bf16 operands the probabilities are
 * rounded to bf16 for their product with the values.  fp32 runs in fp32 FMA.
 */
typedef struct {
    int64_t n_seq;     /* sequences, up to 65535                               */
    int64_t q_len;     /* new tokens of each, 1 to 64                          */
    int64_t n_q, n_kv, d; /* as in noble_attn_desc                             */
    int64_t max_pages; /* entries of a row of page_table                       */
    int64_t max_len;   /* no kv_len is longer; it sets how the work is split.  More
                          than 2^31 - 65536, up to 2^31 - 1, counts as that     */
    int64_t window;
    float scale, softcap;
    int32_t dtype;
    uint32_t flags;    /* 0                                                    */
} noble_paged_desc;
size_t noble_attn_paged_workspace_bytes(const noble_paged_desc *desc);
noble_status noble_attn_paged(const noble_paged_desc *desc, const noble_heads *q, const noble_kv_cache *cache,
                              const int32_t *page_table, const int32_t *kv_len, const float *slope,
                              const noble_heads *o, float *lse /* [n_seq * q_len][n_q], NULL to skip */,
                              void *workspace, size_t workspace_bytes, noble_stream stream);

/*
 * Around the projections of a training step
 * -----------------------------------------
 * What a model of NOBLE layers and attention takes besides them: the table that turns
 * tokens into rows, the norm in front of each projection, and, beside noble_adamw_step, the
 * optimizer step for matrices by orthogonalised momentum.  The conventions above hold.
 * Results repeat bit for bit.  A workspace belongs to one call at a time: calls that share
 * one, captured graphs included, must be ordered by the caller.
 */

/*
 * Layer norm of rows, with the residual stream in front of it.
 *     s = x + res, rounded to the operand type    (res optional: s = x)
 *     y = (s - mean(s)) rstd gain + bias,  rstd = 1 / sqrt(var(s) + eps)
 * with mean and variance (the mean square of s - mean(s)) over the d elements of a row, in
 * fp32.  gain, bias [d] fp32 (NULL: ones, zeros).  `sum` receives s where res is given and
 * is not written otherwise.  stats [T][2] fp32 receives mean and rstd, which the backward
 * pass reads (NULL to skip: inference).  sum may be x or res, and y may be x or res, but
 * sum and y differ; otherwise outputs do not overlap inputs.
 */
typedef struct {
    int64_t T;      /* rows, up to 2^31 - 1                                    */
    int64_t d;      /* elements of a row: a multiple of 8, 8 to 16384          */
    float eps;      /* >= 0                                                    */
    int32_t dtype;  /* noble_dtype of x, res, s, y and their gradients         */
    uint32_t flags; /* 0                                                       */
} noble_norm_desc;
noble_status noble_norm_fwd(const noble_norm_desc *desc, const void *x, const void *res, const float *gain,
                            const float *bias, void *sum, void *y, float *stats, noble_stream stream);

/*
 * Backward: with n = (s - mean) rstd and w = dy gain,
 *     dx = rstd (w - mean(w) - n mean(w n)) + dstream
 *     dgain = sum over rows of dy n,  dbias = sum over rows of dy
 * s is what the forward normed (its `sum`, or x), stats what it wrote.  dstream [T][d]
 * (NULL: zero) is the gradient that reaches s by the residual stream; dx is then the gradient
 * of x and of res alike.  dx may be dy or dstream.  dgain, dbias [d] fp32, NULL to skip; they
 * are added up in a fixed order.
 */
size_t noble_norm_bwd_workspace_bytes(const noble_norm_desc *desc);
noble_status noble_norm_bwd(const noble_norm_desc *desc, const void *dy, const void *s, const float *stats,
                            const float *gain, const void *dstream, void *dx, float *dgain, float *dbias,
                            void *workspace, size_t workspace_bytes, noble_stream stream);

/*
 * Embedding: y[t] = scale table[ids[t]], rounded once.  A negative token is padding: its row
 * of y is 0, and it has no part in the gradient.  A token from vocab on is a caller's
 * error: treated as padding, and noble_get_device_status() reports it (NOBLE_ERR_CUDA).
 */
typedef struct {
    int64_t T;      /* tokens, up to 2^24                                      */
    int64_t vocab;  /* rows of the table, 1 to 2^28                            */
    int64_t d;      /* elements of a row: a multiple of 8, 8 to 65536          */
    float scale;    /* finite                                                  */
    int32_t dtype;  /* noble_dtype of table, y and dy                          */
    uint32_t flags; /* 0                                                       */
} noble_embed_desc;
noble_status noble_embed_fwd(const noble_embed_desc *desc, const int32_t *ids /* [T] */,
                             const void *table /* [vocab][d] */, void *y /* [T][d] */, noble_stream stream);

/*
 * The table's gradient, dtable[v] = scale * (sum of dy[t] over the tokens t with ids[t] = v), fp32
 * throughout and in an order that only the tokens set.  Every row of dtable [vocab][d] is
 * written, rows without tokens as 0.
 */
size_t noble_embed_bwd_workspace_bytes(const noble_embed_desc *desc);
noble_status noble_embed_bwd(const noble_embed_desc *desc, const int32_t *ids, const void *dy, float *dtable,
                             void *workspace, size_t workspace_bytes, noble_stream stream);

/*
 * Optimizer step by orthogonalised momentum (Muon), for matrices, beside noble_adamw_step
 * for everything else.  For each tensor [rows][cols], with a = lr * lr_mult:
 *     m <- momentum m + g
 *     u = g + momentum m  (NOBLE_MUON_NESTEROV), else u = m
 *     X = u / (|u|_F + eps)
 *     `steps` times:  A = X X^T,  X <- 3.4445 X + (-4.7750 A + 2.0315 A A) X
 *     p <- p - a weight_decay p                             (only if `decay`)
 *     p <- p - a sqrt(max(1, rows / cols)) X
 * (with more rows than columns, the same on the transpose).  Five steps bring the singular values
 * of u, but for those that are next to nothing beside |u|_F, near 1.
 *
 * Products take fp16 operands, scaled, with fp32 sums: X is off by about 1e-3 of its norm
 * when u's singular values are of one order, more when they decay fast (1e-2 over six orders).
 * With NOBLE_MUON_PRECISE operands have 22 bits, in pairs of fp16: three times the
 * products, and up to 4e-5 of the norm in place of 1e-3.  Matrices of up to 256 rows or columns
 * always have them.  Everything else is fp32, the norm fp64.
 *
 * `param_bf16` (optional) receives the new parameters and `update` (optional) X, in bf16.  With
 * `update` alone (param NULL) a data-parallel job whose ranks share out the matrices exchanges
 * X and applies it itself.  A tensor whose u is 0 gets X = 0; one whose u is not finite gets
 * NaN, and no other does.  No memory that is written may belong to two tensors, or to a grad.
 * Which tensors share a call may change the last bits of the results.
 */
#define NOBLE_MUON_NESTEROV 1u
#define NOBLE_MUON_PRECISE 2u
typedef struct {
    float *param;      /* fp32, updated in place; NULL: only `update` is wanted */
    void *param_bf16;  /* optional                                              */
    const float *grad; /* fp32                                                  */
    float *momentum;   /* fp32, updated in place                                */
    void *update;      /* optional, bf16                                        */
    int64_t rows, cols; /* 0 to 65536; empty tensors are skipped                */
    float lr_mult;
    int32_t decay;     /* 1: apply weight decay to this tensor                  */
} noble_muon_tensor;

typedef struct {
    float lr, momentum, weight_decay, eps; /* momentum in [0, 1), the others >= 0 */
    int32_t steps;                         /* 0 to 16, usually 5                  */
    uint32_t flags;                        /* NOBLE_MUON_* bits                   */
} noble_muon_hparams;

size_t noble_muon_workspace_bytes(const noble_muon_tensor *tensors, int n_tensors, uint32_t flags);
noble_status noble_muon_step(const noble_muon_tensor *tensors, int n_tensors, const noble_muon_hparams *hp,
                             void *workspace, size_t workspace_bytes, noble_stream stream);

/*
 * Synchronises `stream`, then reads and clears the device status word of the
 * current device.  NOBLE_ERR_TIMEOUT if any kernel gave up a bounded wait
 * since the last call, NOBLE_ERR_CUDA if the stream reported an error or a
 * kernel skipped work, NOBLE_OK otherwise.
 */
noble_status noble_get_device_status(noble_stream stream);

/* Static description of a status code. */
const char *noble_status_string(noble_status s);

/* Description of the last error returned on the calling thread ("" if none). */
const char *noble_last_error(void);

/* Number of kernels this library has launched in the process so far. */
uint64_t noble_kernel_launch_count(void);

/*
 * Test hook: ORs `bits` into the current device's status word (synchronous),
 * so that the reporting path of a device-side timeout can be exercised
 * without making any kernel wait.
 */
noble_status noble_debug_raise_device_status(uint32_t bits);

/*
 * Test hook (no paper counterpart): launches on `stream` one small kernel that
 * waits, through the bounded mbarrier wait every pipeline kernel of this
 * library uses, on an mbarrier that nothing arrives at, for `limit_ns`
 * nanoseconds (0 < limit_ns <= 100 ms).  Nothing else is outstanding in that
 * kernel (no copy, no MMA), so the wait expires: the kernel ORs the timeout
 * flag into the device status word, writes 2 to the device word `*result`
 * (1 if the wait had completed) and exits.  A following
 * noble_get_device_status() then returns NOBLE_ERR_TIMEOUT, and the context
 * stays usable.  NOBLE_ERR_INVALID_ARG for a NULL `result` or a limit out of
 * range.
 */
noble_status noble_debug_wait_expiry(uint64_t limit_ns, uint32_t *result, noble_stream stream);

/*
 * Testing hook (no paper counterpart): synchronises `stream`, then reads and
 * clears the number of rows (of o, dq, dk, dv, or of o over a cache) that the
 * attention kernels of the current device have computed again because they came
 * out not finite.  Zero for inputs that are finite throughout.
 */
noble_status noble_debug_rows_again(uint64_t *count, noble_stream stream);

/*
 * Testing hook (no paper counterpart): the library's tensor-core GEMM alone,
 *     C[z][m][n] = sum_k A0(m,k) B0(n,k) + sum_k A1(m,k) B1(n,k) (+ bias[n])
 * with bf16 operands and fp32 accumulation.  A_s is row-major [M][K_s]
 * (a_mn = 0) or [K_s][M] (a_mn = 1); B_s is [N][K_s] (b_mn = 0) or [K_s][N]
 * (b_mn = 1).  bn selects the N tile (16..256; only the combinations the
 * layer uses exist).  C is fp32 (c_fp32 = 1) or bf16, row-major [M][N] per
 * split; with nsplit > 1 split z sums k-blocks [z*kb_per_split,
 * (z+1)*kb_per_split) of 64 and writes C + z*M*N.  M, N, K_s multiples of 8.
 */
noble_status noble_test_gemm_bf16(int64_t M, int64_t N, int64_t K0, int64_t K1,
                                  int a_mn, int b_mn, int bn, const void *A0,
                                  const void *B0, const void *A1,
                                  const void *B1, const float *bias, void *C,
                                  int c_fp32, int kb_per_split, int nsplit,
                                  noble_stream stream);

/*
 * Testing hook (no paper counterpart): the backward's grouped launch, alone,
 * after a kernel that lets it start at once and publishes its tile counter
 * `delay_ns` nanoseconds later (at most 10 ms); until then its pairs find
 * whatever the 16-byte aligned 64-bit device word `word` held before the call.
 * C = A^T B with A [K][M] and B [K][N] in bf16, C [M][N] in fp32; M, N
 * multiples of 8.  `together`: the first tile of each pair is given, as in the
 * backward of a layer without a branch.  The word is 0 when the work is complete.
 */
noble_status noble_test_late_counter(int64_t M, int64_t N, int64_t K,
                                     const void *A, const void *B, float *C,
                                     void *word, int together, uint64_t delay_ns,
                                     noble_stream stream);

/*
 * Instrumentation (no paper counterpart).  When enabled, every kernel the
 * library launches is bracketed by two CUDA events on its own stream and
 * attributed to a kernel class together with its algorithmic FLOPs and DRAM
 * bytes.  noble_profile_count() waits for the recorded events, aggregates
 * them and returns the number of classes; noble_profile_entry() reads class
 * i of that snapshot (bound: 0 tensor pipe, 1 HBM, 2 CUDA-core ALU).
 */
void noble_profile_enable(int on);
void noble_profile_reset(void);
int noble_profile_count(void);
noble_status noble_profile_entry(int i, char *name, size_t name_len,
                                 uint64_t *launches, double *ms,
                                 double *flops, double *bytes, int *bound);

#ifdef __cplusplus
}
#endif

#endif /* NOBLE_H */
