/*
 * adagc_ops.h -- C ABI of the training operators that stand next to the optimizer step of adagc.h: the loss of a
 * language model with its gradient, and activation checkpoints in 8 bits with their use in the backward pass.  They
 * produce the gradients that adagc_step consumes.
 *
 * Conventions are those of adagc.h: d_* are device pointers owned by the caller, `cuda_stream` is a cudaStream_t passed
 * as void*, every call only enqueues work on that stream (no synchronisation, no allocation of device memory), status
 * codes are adagc_status, and on an error nothing was enqueued.  The calls have no context: they run on the current
 * device, keep nothing between calls, and are thread-safe.  They can be captured in CUDA graphs.
 *   - Matrices are row-major with a leading dimension in ELEMENTS (ld >= columns); any element-aligned base and any ld
 *     are accepted.  Rows that start on 16-byte boundaries (for the logits' gradient: at the same distance from one as
 *     the logits' rows) are read and written faster.
 *   - Matrices have at most 2^30 columns; leading dimensions and offsets are 64-bit throughout.
 *   - dtype arguments are ADAGC_F32 or ADAGC_BF16.  Statistics are fp32; arithmetic is fp32 whatever the dtype, and an
 *     output is rounded once, to nearest even.
 *   - A call with no rows (or no columns where that leaves nothing to write) returns ADAGC_OK and enqueues nothing.
 *   - Results are deterministic: the same inputs give the same bits.
 */
#ifndef ADAGC_OPS_H_
#define ADAGC_OPS_H_

#include "adagc.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Log probabilities of given tokens under softmax(logits), with entropy and the most probable alternatives.
 * For row r with logits z_j, j = 0 .. vocab-1, and target t = d_targets[r]:
 *     lse = ln sum_j exp z_j       logprob = z_t - lse       entropy = -sum_j p_j ln p_j,  p_j = exp(z_j - lse)
 *     the top_k largest z_j in descending order, as ln p_j and j; of equal logits the lowest index comes first
 * in one pass over the logits.
 *   d_logits       [rows, vocab], logits_dtype, leading dimension ld;  1 <= vocab <= 2^30, rows < 2^31
 *   d_targets      rows int64.  A negative target means "no target" (padding): logprob is 0.  A target >= vocab is an
 *                  error of the caller that the call cannot return: logprob is NaN.
 *   d_logprob, d_lse, d_entropy   rows fp32 each.  d_entropy may be NULL.  d_targets and d_logprob may be NULL together.
 *   top_k          0 .. ADAGC_MAX_TOP_K;  d_top_logprob [rows, top_k] fp32 and d_top_index [rows, top_k] int32, ignored
 *                  (may be NULL) when top_k is 0
 * Masked entries (z_j = -inf) have p_j = 0, contribute nothing and are never listed; places of the list that nothing
 * fills hold index -1 and ln p = -inf.  A row with every entry masked: lse = -inf, logprob = -inf (0 without a target),
 * entropy = 0.  A row of equal finite values (the type's lowest among them) is uniform.  A row that holds a NaN or +inf
 * gives NaN in every output (but logprob 0 without a target) and -1 in every index.
 * Masks cost time where they are scattered over a row: with a tenth of the entries at -inf at random, 8192 x 128256 bf16 takes
 * about twice as long (fp32 a quarter longer); masked ends or long stretches cost little.
 */
#define ADAGC_MAX_TOP_K 32
int adagc_token_logprobs(const void* d_logits, int32_t logits_dtype, int64_t rows, int64_t vocab, int64_t ld,
                         const int64_t* d_targets, float* d_logprob, float* d_lse, float* d_entropy, int32_t top_k,
                         float* d_top_logprob, int32_t* d_top_index, void* cuda_stream);

/*
 * Gradient of the above: with a, b, c the upstream gradients of logprob, lse and entropy of a row,
 *     dz_j = a (delta_jt - p_j) + b p_j - c p_j (ln p_j + entropy)
 *   d_lse, d_entropy                 what the forward call wrote (d_entropy is needed, and read, only with d_grad_entropy)
 *   d_grad_logprob, d_grad_lse, d_grad_entropy   rows fp32 each; NULL means zero.  d_targets is needed with d_grad_logprob.
 *   d_grad_logits  [rows, vocab] in logits_dtype, leading dimension grad_ld.  It may be d_logits itself (same pointer and
 *                  ld: in place); any other overlap is ADAGC_E_OVERLAP.
 * Masked entries get 0 (a target that is masked itself, whose logprob is -inf, gets a) and so does a row with every entry
 * masked.  A row without a target ignores a.  A row whose three upstream gradients are zero (or absent) gets zeros whatever
 * its logits hold; they are not read.  A target >= vocab with a != 0 gives a row of NaN.  ln p_j is formed as z_j - lse, so
 * every p of a row shares the rounding of its fp32 lse, a relative error of |lse| 2^-24 at most (3e-5 where |lse| is from 512
 * to 1024).  Rows with |lse| >= 1024, where it would be larger (up to rows whose entries are all the type's lowest value),
 * take their sum anew from the logits, at the cost of a second pass.
 */
int adagc_token_logprobs_backward(const void* d_logits, int32_t logits_dtype, int64_t rows, int64_t vocab, int64_t ld,
                                  const int64_t* d_targets, const float* d_lse, const float* d_entropy,
                                  const float* d_grad_logprob, const float* d_grad_lse, const float* d_grad_entropy,
                                  void* d_grad_logits, int64_t grad_ld, void* cuda_stream);

/*
 * Activation checkpoints in 8 bits.  Groups of 32 consecutive elements of a row share one power of two:
 *     e    = the smallest integer with max|x| <= 127 * 2^e, kept within [-126, 121]
 *     code = rint(x * 2^-e) (ties to even), an int8 in [-127, 127]          x^ = code * 2^e
 * so |x^ - x| <= 2^(e-1) <= max|x| / 127 within a group.  (Two ends of the fp32 range differ: magnitudes above
 * 127 * 2^121 become 127 * 2^121, ones below 2^-127 become 0.)  Scaling by a power of two is exact, so the only rounding is
 * rint, and x^ is exactly representable in bfloat16.  The exponent is stored as the byte e + 127.  A group that holds a
 * NaN or an infinity is stored with the byte 255 and decodes to NaN throughout.
 *   codes  [rows, pitch] int8, pitch = adagc_act8_pitch(cols) = cols rounded up to a multiple of 128; 16-byte aligned
 *   exps   [rows, pitch / 32] uint8; 4-byte aligned
 * Both are dense (no other leading dimension), and rows [r0, r1) of a checkpoint are the checkpoint of rows [r0, r1).
 * Padding codes are 0, padding exponents 1.
 */
typedef struct {
  int8_t* codes;
  uint8_t* exps;
} adagc_act8;

/* Codes per row (0 for cols < 0).  Host-only. */
int64_t adagc_act8_pitch(int64_t cols);

/* x [rows, cols], dtype, leading dimension ld  ->  *out. */
int adagc_act8_encode(const void* d_x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const adagc_act8* out,
                      void* cuda_stream);
/* *in  ->  x^ [rows, cols] in dtype, leading dimension ld. */
int adagc_act8_decode(const adagc_act8* in, int64_t rows, int64_t cols, void* d_x, int32_t dtype, int64_t ld,
                      void* cuda_stream);

/*
 * Gated activation of a SwiGLU MLP, keeping its inputs in 8 bits for the backward pass:
 *     h = silu(gate) * up,  silu(x) = x / (1 + exp(-x)),  from the inputs as given;   *gate8 = act8(gate), *up8 = act8(up)
 * gate, up, h: [rows, cols] in dtype, each with its own leading dimension.
 * fp32: h is within 2^-21 of its value (relative) where 1 / (1 + exp(-gate)) is a normal number.  bf16: exp is taken with a
 * relative error of about |gate| 2^-24, far below the rounding of h.  The backward pass likewise.
 */
int adagc_act8_swiglu(const void* d_gate, int64_t ld_gate, const void* d_up, int64_t ld_up, int32_t dtype, int64_t rows,
                      int64_t cols, void* d_h, int64_t ld_h, const adagc_act8* gate8, const adagc_act8* up8,
                      void* cuda_stream);
/*
 * Its backward pass from the checkpoints: with g, u the values they stand for and s = 1 / (1 + exp(-g)),
 *     grad_gate = grad_h * u * s * (1 + g (1 - s))        grad_up = grad_h * g * s
 * and, if h8 is not NULL, *h8 = act8(g s u), the input of the down projection for adagc_act8_linear_wgrad (so h itself
 * need not be kept).
 */
int adagc_act8_swiglu_backward(const void* d_grad_h, int64_t ld_grad_h, int32_t dtype, int64_t rows, int64_t cols,
                               const adagc_act8* gate8, const adagc_act8* up8, void* d_grad_gate, int64_t ld_grad_gate,
                               void* d_grad_up, int64_t ld_grad_up, const adagc_act8* h8, void* cuda_stream);

/*
 * Weight gradient of a linear layer y = x W^T (W [out_features, in_features]) from the layer's input kept in 8 bits:
 *     dW[n, k] = sum over tokens t of grad_y[t, n] * x^[t, k]
 * on the tensor cores: both operands are exact in bfloat16, products are exact and sums are fp32.  The tensor core cuts when it
 * adds, so a sum leaves its accumulator every 1536 tokens at most (fp32 results: within 1e-6 of the result's norm for normal
 * values of any scale) or every 16384 (bf16 results: within 1.3e-4 of the sum of magnitudes before the rounding to bf16, and
 * as a rule 1e-5 of the result), and the parts are added with rounding.
 *   d_grad_y       [tokens, out_features] bfloat16 (grad_y_dtype must be ADAGC_BF16), leading dimension ld_grad_y
 *   x8             checkpoint of [tokens, in_features]
 *   d_grad_w       [out_features, in_features] in grad_w_dtype, leading dimension ld_grad_w: a tensor of the gradient arena
 *   accumulate     0: overwrite; 1: add to what d_grad_w holds (the finished sum is added to it in fp32 and rounded once; fp32
 *                  results below 2^-126 may become 0)
 *   d_workspace    adagc_act8_linear_wgrad_workspace_bytes(...) bytes, 256-byte aligned; its content is not kept
 * tokens = 0 gives dW = 0 (or leaves d_grad_w alone with accumulate).
 * The kernels wait on shared-memory barriers with a time limit of 2 s; a block that gives up writes NaN over its tile of
 * the result, so that a lost copy cannot pass unseen.
 * Returns 0 bytes if no workspace is needed; a negative adagc_status for invalid sizes.
 */
int64_t adagc_act8_linear_wgrad_workspace_bytes(int64_t tokens, int64_t out_features, int64_t in_features,
                                                const void* d_grad_y, int64_t ld_grad_y);
int adagc_act8_linear_wgrad(const void* d_grad_y, int32_t grad_y_dtype, int64_t ld_grad_y, const adagc_act8* x8,
                            int64_t tokens, int64_t out_features, int64_t in_features, void* d_grad_w,
                            int32_t grad_w_dtype, int64_t ld_grad_w, int32_t accumulate, void* d_workspace,
                            size_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* ADAGC_OPS_H_ */
