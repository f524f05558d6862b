/*
 * exo_fused.h -- C ABI of the B200 (sm_100a) operators that are matrix products with more than a product's epilogue.
 *
 *   exo_ffn_create / forward / backward   a gated feed-forward block, y = (act(x Wg^T) * (x Wu^T)) Wd^T
 *   exo_ce_create / forward / backward    softmax cross entropy of a head x W^T over a large vocabulary
 *   exo_i8_quantize, exo_gemm_i8_run      8-bit integers with a scale per row, and Y = alpha * X * W^T + beta * Y of them
 *
 * The status codes, types and conventions of exo_gemm.h hold here (exo_gemm_last_cuda_error included): all pointers to matrices are
 * DEVICE pointers owned by the caller, matrices are row-major with leading dimensions in elements, calls are enqueued on cuda_stream
 * (a cudaStream_t; NULL = the legacy default stream) and return without synchronising, every check happens before the first launch,
 * nothing runs on the CPU, and a device that is not compute capability 10.x is refused with EXO_GEMM_ERR_ARCH.  Calls may be captured
 * into a CUDA graph.  Launches use programmatic dependent launch: a kernel may begin while its predecessor in the stream drains, and
 * waits for it before it reads or writes anything.
 *
 * Every result is bitwise reproducible from run to run on the same inputs and plan: sums are taken in fixed orders, without atomics.
 *
 * A plan is for one device, on which its calls run whatever device is current (their stream has to be one of that device).  Calls of ONE
 * plan must not overlap on the GPU: they share its workspace.  Different plans share nothing.  The leading dimensions that a descriptor
 * takes may be 0, which stands for packed rows.  16-bit matrices whose rows do not start on 16-byte boundaries (leading dimension not a
 * multiple of 8) are read through aligned copies that the plan owns, one more pass over them per call; the other matrices have to be
 * 16-byte aligned, else ERR_ALIGNMENT.
 */
#ifndef EXO_FUSED_H_
#define EXO_FUSED_H_

#include "exo_gemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- gated feed-forward block */
typedef struct exo_ffn_plan* exo_ffn_handle_t; /* opaque; owned by the library */

typedef enum {
  EXO_ACT_SILU = 0,      /* g / (1 + exp(-g))                                               */
  EXO_ACT_GELU = 1,      /* g * Phi(g), Phi the normal distribution function                */
  EXO_ACT_GELU_TANH = 2  /* g * (1 + tanh(sqrt(2 / pi) * (g + 0.044715 g^3))) / 2            */
} exo_activation_t;

/*
 * For each of `tokens` rows x of `hidden` values:
 *
 *   g = Wg x,  u = Wu x         gate and up: the first and the last `inner` rows of one 2 * inner x hidden matrix
 *   h = act(g) * u
 *   y = Wd h                    down: hidden x inner
 */
typedef struct {
  int64_t tokens, hidden, inner; /* tokens >= 0; hidden, inner >= 1; each at most 2^24                       */
  int32_t dtype;                 /* BF16 or FP16: every matrix but the weights' gradients                    */
  int32_t activation;            /* exo_activation_t                                                         */
  int32_t training;              /* 0: forward only, without `saved`; 1: backward too                        */
  int32_t grad_dtype;            /* type of the weights' gradients: FP32 or dtype (not read if training == 0)*/
  int64_t ldx, ldy;              /* of x and dx, and of y and dy                                             */
  int64_t ld_gate_up, ld_down;   /* of the weights and their gradients                                       */
  int32_t device;                /* CUDA device ordinal; -1 = the current device                             */
} exo_ffn_desc_t;

/* Pure argument check; needs no GPU.  OK, ERR_NULL, ERR_INVALID_ARG or ERR_UNSUPPORTED. */
exo_gemm_status_t exo_ffn_validate(const exo_ffn_desc_t* desc);

/* Makes a plan with its workspace, which is ready for any stream when the call returns.  *out is written only on success. */
exo_gemm_status_t exo_ffn_create(exo_ffn_handle_t* out, const exo_ffn_desc_t* desc);

/* Bytes of the buffer that a forward call fills for the backward call (g and u, in dtype); 0 if training == 0. */
int64_t exo_ffn_saved_bytes(exo_ffn_handle_t plan);

/*
 * y = the block of x.  saved: NULL, or (training plans) exo_ffn_saved_bytes bytes, 32-byte aligned, that the backward call of these
 * tokens reads; the plan may be used for other tokens in between.  Both products are summed in fp32, act(g) * u is computed in fp32 and
 * rounded to dtype once, as the operand of the last product (a value beyond the largest finite one of fp16 becomes infinite); g and u
 * are rounded to dtype in `saved` only.  x and the weights must not overlap y or saved.
 */
exo_gemm_status_t exo_ffn_forward(exo_ffn_handle_t plan, const void* x, const void* gate_up, const void* down, void* y, void* saved,
                                  void* cuda_stream);

/*
 * Gradients, from dy (the gradient of y) and the saved g and u:
 *
 *   dh = dy Wd,   dg = dh * u * act'(g),   du = dh * act(g)
 *   dx = dg Wg + du Wu,   d_gate_up = (dg^T x, du^T x),   d_down = dy^T h
 *
 * dx, d_gate_up or d_down may be NULL: not wanted (x is then read only for d_gate_up, gate_up only for dx).  accumulate != 0 adds the
 * weights' gradients onto what is there.  dh is held in fp32; dg, du and the recomputed h are rounded to dtype once, as operands.
 * Outputs must not overlap inputs or each other.
 */
exo_gemm_status_t exo_ffn_backward(exo_ffn_handle_t plan, const void* x, const void* gate_up, const void* down, const void* saved,
                                   const void* dy, void* dx, void* d_gate_up, void* d_down, int32_t accumulate, void* cuda_stream);

/*
 * Waits for the plan's device and returns EXO_GEMM_ERR_DEVICE_TIMEOUT if a bounded device-side wait of one of this plan's kernels, its own
 * products' included, has given up since the last such call for this plan, else EXO_GEMM_OK.  What that call computed, and what the plan
 * computed from then on, is then wrong; other plans are not concerned.
 */
exo_gemm_status_t exo_ffn_check(exo_ffn_handle_t plan);
/* Device memory the plan owns, in bytes. */
int64_t exo_ffn_workspace_bytes(exo_ffn_handle_t plan);
/* Frees the plan and its workspace.  NULL is a no-op returning OK. */
exo_gemm_status_t exo_ffn_destroy(exo_ffn_handle_t plan);

/* ---------------------------------------------------------------- cross entropy over a vocabulary */
typedef struct exo_ce_plan* exo_ce_handle_t; /* opaque; owned by the library */

/*
 * For each of `tokens` rows x_i of `hidden` values with target t_i, and s = label_smoothing:
 *
 *   l_iv = w_v . x_i                                      the logits, for the `vocab` rows w_v of W; never stored
 *   lse_i = log sum_v exp(l_iv)
 *   loss_i = lse_i - (1 - s) * l_{i t_i} - s * mean_v l_iv
 *
 * A target that is ignore_index, or outside 0 .. vocab - 1, is ignored: loss_i = 0, dx_i = 0 and nothing of the row is added to W's gradient
 * (its x has to be finite all the same: 0 times an infinity or NaN is added).
 */
typedef struct {
  int64_t tokens, hidden, vocab; /* tokens >= 0; hidden, vocab >= 1; each at most 2^24                                   */
  int32_t dtype;                 /* BF16 or FP16: x, W and dx                                                           */
  int32_t training;              /* 0: forward only; 1: backward too                                                    */
  int32_t grad_dtype;            /* type of W's gradient: FP32 or dtype (not read if training == 0)                     */
  float label_smoothing;         /* 0 <= s < 1                                                                          */
  int64_t ignore_index;          /* a target that is ignored (one outside the vocabulary: none inside it is)            */
  int64_t ldx, ldw;              /* of x and dx, and of W and its gradient                                              */
  int64_t keep_bytes;            /* how large `saved` may be: -1 = up to 4 GiB, 0 = nothing is kept                     */
  int64_t piece;                 /* columns of the vocabulary that the backward call recomputes at a time; 0 = chosen   */
  int32_t device;                /* CUDA device ordinal; -1 = the current device                                        */
} exo_ce_desc_t;

/* Pure argument check; needs no GPU.  OK, ERR_NULL, ERR_INVALID_ARG or ERR_UNSUPPORTED. */
exo_gemm_status_t exo_ce_validate(const exo_ce_desc_t* desc);

/* Makes a plan with its workspace, which is ready for any stream when the call returns.  *out is written only on success. */
exo_gemm_status_t exo_ce_create(exo_ce_handle_t* out, const exo_ce_desc_t* desc);

/*
 * Bytes of the buffer in which a forward call leaves exponentials exp(l_iv - largest of the row's columns computed together), in dtype
 * (fp16: times 2^15, so that they are kept to 2^-29 of that largest with all bits), for the backward call: for as many columns of the
 * vocabulary as keep_bytes has room for.  The backward call recomputes the logits of
 * the other columns, a piece at a time: a third more arithmetic for the part that is not kept.
 */
int64_t exo_ce_saved_bytes(exo_ce_handle_t plan);

/*
 * loss and lse (fp32, `tokens` values each; either may be NULL) from x, W and target (int64, 8-byte aligned).  saved: NULL, or (training
 * plans) exo_ce_saved_bytes bytes, 16-byte aligned.  Logits, their exponentials' sums and the mean are held in fp32.  (The tensor core truncates
 * as it adds: products of depth 4096 come out 3e-6 of their deviation nearer to zero, and lse 1.6e-5 low where the logits' deviation is 2.)
 */
exo_gemm_status_t exo_ce_forward(exo_ce_handle_t plan, const void* x, const void* W, const int64_t* target, float* loss, float* lse,
                                 void* saved, void* cuda_stream);

/*
 * Gradients of sum_i dloss_i * loss_i, from the forward call's lse and dloss (fp32, `tokens` values each):
 *
 *   d_iv = dloss_i * (exp(l_iv - lse_i) - (1 - s) * [v == t_i] - s / vocab),    dx_i = sum_v d_iv w_v,    dW_v = sum_i d_iv x_i
 *
 * saved: what the forward call of the same x and W left (it is overwritten: one backward call per forward call; a second one, or one
 * without its forward call, finds that and gives NaN); not read if exo_ce_saved_bytes is 0.  dx or dW may be NULL: not wanted.  accumulate != 0 adds dW onto what is there.  d_iv is scaled to the range of dtype by the
 * largest finite |dloss_i|, rounded to dtype as the operand of both products (a kept exponential is rounded before that too), and the
 * scale is taken back in fp32; dx is summed in fp32 over all pieces.  Outputs must not overlap inputs or each other.
 */
exo_gemm_status_t exo_ce_backward(exo_ce_handle_t plan, const void* x, const void* W, const int64_t* target, const float* lse,
                                  const float* dloss, void* saved, void* dx, void* dW, int32_t accumulate, void* cuda_stream);

/* As exo_ffn_check. */
exo_gemm_status_t exo_ce_check(exo_ce_handle_t plan);
/* Device memory the plan owns, in bytes. */
int64_t exo_ce_workspace_bytes(exo_ce_handle_t plan);
/* Frees the plan and its workspace.  NULL is a no-op returning OK. */
exo_gemm_status_t exo_ce_destroy(exo_ce_handle_t plan);

/* ---------------------------------------------------------------- 8-bit integers */
/*
 * A matrix of `rows` x `K` values in 8 bits: value = scales[row] * codes[row * ld + k].  A row is a token of the activations or an output
 * channel of the weights.  ld is a multiple of 16 and codes are 16-byte aligned (ERR_ALIGNMENT); codes k >= K of a row may be anything.
 */
typedef struct {
  int64_t rows, K, ld;
  int8_t* codes;
  float* scales;
} exo_i8_t;

/*
 * Fills q's codes and scales from X (rows x K, leading dimension ldx >= K, x_dtype BF16, FP16 or FP32, aligned to its element), in fp32:
 *   scale = max |x| / 127,   code = clamp(rint(x / scale), -127, 127)
 * and code = 0 where the scale comes out as 0.  Values have to be finite (others give codes of no meaning).  Codes k >= K are not written.
 */
exo_gemm_status_t exo_i8_quantize(const exo_i8_t* q, const void* X, int64_t ldx, int32_t x_dtype, void* cuda_stream);

/*
 * Y = alpha * X * W^T + beta * Y: Y is X->rows x W->rows of y_dtype (BF16, FP16 or FP32), leading dimension ldy >= W->rows, aligned to its
 * element.  The sums of products of codes are exact 32-bit integers (K <= 131071; ERR_UNSUPPORTED above; codes may be -128); each is
 * converted to fp32 and multiplied by the token's scale, the channel's scale and alpha in this order.  beta == 0: Y is not read;
 * alpha == 0 or K == 0: X and W are not read.  X and W must not overlap Y.  Nothing is allocated; runs on the current device.
 */
exo_gemm_status_t exo_gemm_i8_run(const exo_i8_t* X, const exo_i8_t* W, void* Y, int64_t ldy, int32_t y_dtype, float alpha, float beta,
                                  void* cuda_stream);

/* ---------------------------------------------------------------- device-side waits */
/*
 * Waits for the current device and returns EXO_GEMM_ERR_DEVICE_TIMEOUT if a bounded device-side wait of a kernel of this header has
 * given up there since the last call of this function, else EXO_GEMM_OK.  Whose wait it was a plan's own check tells, and this call takes
 * nothing away from that.  The 8-bit products have no plan and share one report on a device, this one: from a wait that gave up until
 * this call, what any of them computes may be wrong.
 */
exo_gemm_status_t exo_fused_check(void);

/*
 * Test hook: in the next kernel of this header with tensor-core products, waits last `timeout_ms` (0 .. 10000; 0 stands for the usual
 * bound of 4 s), and with skip_copies 1 its first CTA leaves out the copies of its first k-block, so that a wait runs out.
 */
exo_gemm_status_t exo_fused_debug_set(int32_t timeout_ms, int32_t skip_copies);

#ifdef __cplusplus
}
#endif
#endif /* EXO_FUSED_H_ */
