/*
 * exo_decode.h -- C ABI of the B200 (sm_100a) operators that read a model's weights once for a few tokens.
 *
 *   exo_q4_quantize / exo_q4_dequantize   weights <-> 4-bit codes with a scale (and a zero point) per group
 *   exo_gemv_q4_run                       Y = alpha * X * W^T + beta * Y, W in 4 bits, 1 to 64 tokens
 *   exo_moe_create / run / destroy        a whole mixture-of-experts layer for 1 to 64 tokens, 16- or 4-bit experts
 *
 * For more tokens a 4-bit matrix goes through exo_q4_dequantize and exo_gemm_run (exo_gemm.h); a layer takes them 64 at a time.  The status codes,
 * types and conventions of exo_gemm.h hold here (exo_gemm_last_cuda_error included): all pointers to matrices are DEVICE pointers owned by the caller, calls are
 * enqueued on cuda_stream (a cudaStream_t; NULL = the legacy default stream) and return without synchronising, every
 * check happens before the first launch, nothing runs on the CPU, and a device that is not compute capability 10.x is
 * refused with EXO_GEMM_ERR_ARCH.  Calls may be captured into a CUDA graph.  Launches use programmatic dependent
 * launch: a kernel may begin while its predecessor in the stream drains, and waits for it before it reads or writes
 * anything.  The last of a layer's three kernels reads the routing tables and its first weights before the second one has ended: what
 * came before the layer, and the first kernel, have ended by then.
 *
 * Every result is bitwise reproducible from run to run on the same inputs: sums are taken in fixed orders.
 */
#ifndef EXO_DECODE_H_
#define EXO_DECODE_H_

#include "exo_gemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A matrix of `rows` x `K` weights in 4 bits.  With Kp = K rounded up to a multiple of 128 and G = Kp / group:
 *
 *   codes    rows of Kp / 2 bytes, 16-byte aligned.  Weight k = 128 b + 32 j + 8 t + i (j, t < 4, i < 8) of a row is
 *            bits 4 n .. 4 n + 3, n = i / 2 + 4 * (i % 2), of the row's little-endian 32-bit word 16 b + 4 t + j.
 *            (Lane t of four then finds its share of 128 weights in 16 consecutive bytes, and word & 0x000f000f is a
 *            pair of neighbours.)  Codes of the padding k >= K may be anything.
 *   scales   rows of G values of `dtype`, aligned to 256 / group bytes, one per `group` consecutive weights
 *   zeros    rows of G bytes 0 .. 15, aligned to 128 / group bytes, or NULL: 8 everywhere
 *
 * weight = scale * (code - zero).  group is 32, 64 or 128; dtype is EXO_GEMM_BF16 or EXO_GEMM_FP16 and also the
 * type of the activations the matrix is multiplied with.
 */
typedef struct {
  int64_t rows, K;
  int32_t group;
  int32_t dtype;
  void* codes;
  void* scales;
  uint8_t* zeros;
} exo_q4_t;

/*
 * Fills q's codes, scales and zeros from the row-major matrix W (rows x K, leading dimension ldw >= K elements,
 * w_dtype BF16, FP16 or FP32, aligned to its element).  Per group, in fp32 (r() rounds to q->dtype, an overflow to its largest finite
 * value):
 *   zeros == NULL   scale = r(max |w| / 7),             code = clamp(rint(w / scale), -8, 7) + 8
 *   else            lo = min(w, 0), hi = max(w, 0),     scale = r((hi - lo) / 15),
 *                   zero = clamp(rint(-lo / scale), 0, 15), code = clamp(rint(w / scale) + zero, 0, 15)
 * and where the scale comes out as 0, zero = 8 and code = zero.  The padding gets code = zero.  Weights have to be
 * finite (others give codes of no meaning).  Errors: ERR_NULL, ERR_INVALID_ARG, ERR_ALIGNMENT, ERR_ARCH, ERR_CUDA.
 */
exo_gemm_status_t exo_q4_quantize(const exo_q4_t* q, const void* W, int64_t ldw, int32_t w_dtype, void* cuda_stream);

/* W = the values of q, rounded to w_dtype (BF16, FP16 or FP32), row-major with leading dimension ldw >= K. */
exo_gemm_status_t exo_q4_dequantize(const exo_q4_t* q, void* W, int64_t ldw, int32_t w_dtype, void* cuda_stream);

/*
 * Y = alpha * X * W^T + beta * Y for `tokens` rows: X is tokens x K of W's dtype, Y is tokens x rows of y_dtype (FP32
 * or W's dtype), both row-major with leading dimensions ldx >= K and ldy >= rows (elements; no alignment beyond the
 * element's is needed, 16-byte aligned rows of X are read faster).  beta == 0: Y is not read; alpha == 0: W and X are
 * not read.  X and W must not overlap Y.  0 <= tokens <= 64 (ERR_UNSUPPORTED above).  Nothing is allocated.  Other
 * errors as above.
 *
 * Products are formed from the integers code - zero and a group's sum is multiplied by its scale in fp32; all further
 * sums are fp32.  The factors are the 16-bit activations and a group is summed in fp32; or, for one or two tokens and a large
 * matrix, they are integers of 30 bits that stand for the activations of 128 neighbouring k: exact for values down to 2^-22 (bf16) or
 * 2^-19 (fp16) of the largest of the 128, and off by at most 2^-30 of that largest below; their group sums are exact.  (Tokens with values
 * that are not finite, and results that come out so, are summed in fp32.)
 */
exo_gemm_status_t exo_gemv_q4_run(const exo_q4_t* W, int64_t tokens, const void* X, int64_t ldx, void* Y, int64_t ldy,
                                  int32_t y_dtype, float alpha, float beta, void* cuda_stream);

typedef struct exo_moe_plan* exo_moe_handle_t; /* opaque; owned by the library */

/*
 * A mixture-of-experts layer.  For each token x (a row of `hidden` values):
 *
 *   l = router * x                      (`experts` logits)
 *   taken = the top_k experts with the largest l; equal ones go to the lower index, NaN counts as the largest
 *   w_e = softmax(l)_e, divided by the sum over the taken ones if `renormalize`, times routed_scale
 *   y = sum over the taken experts e of w_e * down_e * (silu(gate_e * x) * (up_e * x))
 *     + the same with weight 1 for each of the `shared` experts
 *
 * The experts' matrices are stacked by rows, the routed experts first and the shared ones after them.
 */
typedef struct {
  int64_t hidden, inner;    /* columns of gate and up (rows of down), and rows of gate and up (columns of down)   */
  int32_t experts, shared;  /* 1 .. 512 routed experts, 0 .. 8 shared ones                                        */
  int32_t top_k;            /* 1 .. 16, at most `experts`                                                         */
  int32_t max_tokens;       /* 1 .. 64: the workspace is made for this many                                       */
  int32_t dtype;            /* BF16 or FP16: x, y, router, 16-bit expert weights, scales of 4-bit ones            */
  int32_t q4_group;         /* 0: 16-bit experts; 32, 64 or 128: 4-bit experts with this group                    */
  int32_t renormalize;      /* 0 or 1                                                                             */
  float routed_scale;
  int32_t device;           /* CUDA device ordinal; -1 = the current device                                       */
} exo_moe_desc_t;

/*
 * One stack of expert matrices: expert e's row r is row e * expert_rows + r.  16-bit experts: `w` is a row-major
 * matrix with leading dimension `ld` (elements), scales and zeros are NULL.  4-bit experts: `w`, `scales` and
 * `zeros` are the codes, scales and zeros of an exo_q4_t of (experts + shared) * expert_rows rows; `ld` is not read.
 * expert_rows is at least `inner` for gate and up and `hidden` for down; a larger one skips rows (a gate and an up
 * matrix stored in turn: up.w = gate.w + inner rows, expert_rows = 2 * inner for both).
 */
typedef struct {
  const void* w;
  int64_t ld;
  int64_t expert_rows;
  const void* scales;
  const uint8_t* zeros;
} exo_moe_matrix_t;

typedef struct {
  const void* router;      /* experts x hidden, row-major */
  int64_t ld_router;
  exo_moe_matrix_t gate, up, down;
} exo_moe_weights_t;

/* Pure argument check; needs no GPU.  OK, ERR_NULL, ERR_INVALID_ARG or ERR_UNSUPPORTED. */
exo_gemm_status_t exo_moe_validate(const exo_moe_desc_t* desc);

/*
 * Makes a plan: validates, allocates the workspace (routing tables and the taken experts' inner activations) and clears it, which is
 * done when the call returns: the plan may be run on any stream.  *out is written only on success.
 */
exo_gemm_status_t exo_moe_create(exo_moe_handle_t* out, const exo_moe_desc_t* desc);

/*
 * Enqueues the layer for `tokens` <= max_tokens tokens: x and y are tokens x hidden, row-major, leading dimensions
 * ldx, ldy >= hidden.  index (int32) and weight (fp32), tokens x top_k, receive the taken experts, largest first, and
 * their w_e; either may be NULL.  y, index and weight must not overlap the inputs or each other.  Runs of one plan
 * must not overlap on the GPU (they share its workspace).  silu(gate) * up * w_e is computed in fp32 and held in
 * `dtype` between the two products (for an expert of up to 4 tokens as the sum of two values of it), as the activations of a 16-bit
 * matrix product are; all sums are fp32.  Beyond the largest finite value of `dtype` (twice that, where it is held as a
 * sum) it is infinite.
 * Matrices of `dtype` need the alignment of their elements (16-byte aligned rows are read faster), the parts of 4-bit
 * ones that of exo_q4_t.
 */
exo_gemm_status_t exo_moe_run(exo_moe_handle_t plan, const exo_moe_weights_t* weights, int64_t tokens, const void* x,
                              int64_t ldx, void* y, int64_t ldy, int32_t* index, float* weight, void* cuda_stream);

/*
 * Waits for the current device and returns EXO_GEMM_ERR_DEVICE_TIMEOUT if a bounded device-side wait of a kernel of this
 * header has given up since the last call (what that launch computed is then wrong), else EXO_GEMM_OK.
 */
exo_gemm_status_t exo_decode_check(void);

/*
 * Test hook for the bounded waits: in the next exo_gemv_q4_run or exo_moe_run of this process a wait for copies lasts `timeout_ms` (0 ..
 * 10000; 0 stands for the usual bound of 4 s), and with skip_copies 1 (a product, an expert's gate and up) or 2 (an expert's down) the first
 * CTA's first warp issues none, so that its wait runs out and the kernel reports that without trapping.  Products and layers that
 * read their weights without copies ignore it.
 */
exo_gemm_status_t exo_decode_debug_set(int32_t timeout_ms, int32_t skip_copies);

/* Device memory the plan owns, in bytes. */
int64_t exo_moe_workspace_bytes(exo_moe_handle_t plan);

/* Frees the plan and its workspace.  NULL is a no-op returning OK. */
exo_gemm_status_t exo_moe_destroy(exo_moe_handle_t plan);

#ifdef __cplusplus
}
#endif
#endif /* EXO_DECODE_H_ */
