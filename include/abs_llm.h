/*
 * abs_llm.h -- operators of a language model's training micro-batch, for the gradients that abs_accumulate* take.
 *
 * The library's own gradient (abs_accumulate_mlp) is that of a small classifier.  A model that is trained with
 * Algorithm 1 but brings its own forward and backward pass hands its flat gradient to abs_accumulate; these calls are
 * the parts of such a pass that are not matrix products of plain operands:
 *     abs_policy_loss             clipped policy loss with a KL term, from logits to the gradient of the logits
 *     abs_preference_loss         paired preference loss, likewise
 *     abs_residual_norm           norm behind a block, gate, scaled residual, norm in front of the next block
 *     abs_residual_norm_backward  its gradients
 *     abs_ckpt8_quantize / _dequantize   an activation kept for the backward pass in 8 bits
 *     abs_ckpt8_wgrad             gradient of a linear layer's weight from such an activation
 *
 * Conventions
 *   - No context: a call works on the CURRENT device, enqueues on `stream` (a cudaStream_t, NULL = default stream) and
 *     returns an int status of abs_sgd.h.  Nothing is allocated, nothing blocks the host (abs_llm_check does).
 *     Arguments are checked before anything is enqueued; abs_last_error(NULL) gives the text of the last refusal on
 *     this thread.
 *   - The caller owns all buffers, the workspaces included.  A workspace (256-byte aligned) holds nothing between calls;
 *     two calls that may overlap on the GPU need two.
 *   - Matrices are row-major with a leading dimension `ld*` in elements (>= the row length); rows need the alignment of
 *     their element only.  16-byte aligned rows are moved by wider or asynchronous copies.
 *   - dtype: ABS_F32 or ABS_BF16, of the activations and logits and their gradients.  Parameters, their gradients and
 *     all per-token numbers are fp32; sums, softmax and norm statistics are held in fp32 or more.
 *   - Sums run in a fixed order: equal inputs give equal bits.
 *   - Sizes of zero are allowed: nothing is read, sums over nothing are zero (and are written).
 */
#ifndef ABS_LLM_H_
#define ABS_LLM_H_

#include "abs_sgd.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ABS_F32  ABS_GRAD_F32
#define ABS_BF16 ABS_GRAD_BF16

/* Clipped policy loss with a KL term, and its gradient with respect to the logits.  For token t with label y:
 *     logp = z_y - log sum_v exp z_v          r = exp(logp - logp_old)
 *     loss_t = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef (exp(logp_ref - logp) - (logp_ref - logp) - 1)
 *     L = sum_t weight_t loss_t
 *     dL/dz_v = g_t ([v = y] - softmax(z)_v),  g_t = weight_t (-(r A, 0 where clipped) + kl_coef (1 - exp(logp_ref - logp)))
 * (clipped: A > 0 and r > 1 + clip_high, or A < 0 and r < 1 - clip_low).
 *   logits    [tokens, vocab], ld >= vocab.  -inf entries have probability zero.  A row may have 2^32 - 2^16 bytes (ABS_ELIMIT).
 *   labels    [tokens] int32; weight [tokens]: the token's share of L (for the mean over n tokens 1/n).  A token whose
 *             weight is 0, whose label lies outside [0, vocab), or whose logits are all -inf is left out: its logp is 0, it
 *             adds nothing, its row of dlogits is zero.  (Logits of the first two kinds are not read.)
 *   logp_old, advantage [tokens]; logp_ref [tokens] or NULL (then no KL term, kl_coef must be 0);
 *             with kl_coef 0 it gives the statistic and nothing else
 *   stats     [3] out: L, sum weight_t kl_t (without kl_coef), sum weight_t [t clipped]
 *   logp      [tokens] out
 *   dlogits   [tokens, vocab] out, ld_d >= vocab, or NULL (loss only).  May be the logits themselves (then ld_d = ld);
 *             must not overlap them otherwise.
 *   workspace abs_policy_loss_workspace() bytes. */
size_t abs_policy_loss_workspace(void);
int abs_policy_loss(const void *logits, uint32_t dtype, uint64_t tokens, uint64_t vocab, uint64_t ld, const int32_t *labels,
                    const float *logp_old, const float *logp_ref, const float *advantage, const float *weight, float clip_low,
                    float clip_high, float kl_coef, float *stats, float *logp, void *dlogits, uint64_t ld_d, void *workspace,
                    size_t workspace_bytes, void *stream);

/* Paired preference loss, and its gradient with respect to the logits.  Answer q holds the rows offsets[q] .. offsets[q + 1] - 1;
 * answers 2 p and 2 p + 1 are the preferred and the other one of pair p:
 *     s_q = sum of logp over the answer's counted rows      h_p = beta ((s_2p - ref_2p) - (s_2p+1 - ref_2p+1))
 *     pair_loss_p = -(1 - smoothing) log sigmoid(h_p) - smoothing log sigmoid(-h_p)        L = scale sum_p pair_loss_p
 *     dL/dz_v = +-scale beta (sigmoid(h_p) - (1 - smoothing)) ([v = y] - softmax(z)_v)     (+ for the preferred answer)
 *   logits    as for abs_policy_loss; tokens up to 2^31 - 513 (ABS_ELIMIT)
 *   labels    [tokens] int32; a row whose label lies outside [0, vocab) (a prompt's token), whose logits are all -inf, or
 *             that belongs to no answer is not counted: its row of dlogits is zero.  (Logits of the first kind are not read.)
 *   offsets   [2 pairs + 1] int32 on the device, ascending; values outside [0, tokens] are clamped.  Empty answers are
 *             allowed (s = 0).
 *   logp_ref  [2 pairs]: the reference model's s_q
 *   stats     [1] out: L;  pair_loss [pairs] out;  seq_logp [2 pairs] out: s_q
 *   dlogits   as for abs_policy_loss
 *   workspace abs_preference_loss_workspace(tokens) bytes. */
size_t abs_preference_loss_workspace(uint64_t tokens);
int abs_preference_loss(const void *logits, uint32_t dtype, uint64_t tokens, uint64_t vocab, uint64_t ld, const int32_t *labels,
                        const int32_t *offsets, uint64_t pairs, const float *logp_ref, float beta, float smoothing, float scale,
                        float *stats, float *pair_loss, float *seq_logp, void *dlogits, uint64_t ld_d, void *workspace,
                        size_t workspace_bytes, void *stream);

#define ABS_GATE_NONE    0u  /* G = 1                                                                  */
#define ABS_GATE_CHANNEL 1u  /* G_td = gate[d], fp32: a learned gate, gradient summed over the tokens   */
#define ABS_GATE_ELEMENT 2u  /* G_td = sigmoid(gate[t, d]), dtype of the activations: a computed gate   */

/* Norm behind a block, gate and scaled residual, norm in front of the next block, in one pass:
 *     u = h / rms(h) * w_post  (w_post NULL: u = h)     y = scale x + G u     n = y / rms(y) * w_pre
 *     rms(v) = sqrt(mean_d v_d^2 + eps)
 * x, h, y, n [tokens, width] of `dtype` (y may be x, n may be h, with the same leading dimension; y and n are different); w_post, w_pre [width] fp32.  n is formed from y before
 * its rounding.  gate: see ABS_GATE_*; ld_gate is used with ABS_GATE_ELEMENT.  width <= 32768 (ABS_ELIMIT). */
int abs_residual_norm(const void *x, uint64_t ld_x, const void *h, uint64_t ld_h, const void *gate, uint64_t ld_gate,
                      uint32_t gate_kind, const float *w_post, const float *w_pre, float scale, float eps, uint32_t dtype,
                      uint64_t tokens, uint64_t width, void *y, uint64_t ld_y, void *n, uint64_t ld_n, void *stream);

/* Gradients of abs_residual_norm, from dn (of n) and dy (of y from elsewhere, NULL: none), at the stored y and h:
 *     dY = dy + (dn w_pre - yn mean(dn w_pre yn)) / rms(y), yn = y / rms(y)      dx = scale dY
 *     dU = G dY     dh = (dU w_post - hn mean(dU w_post hn)) / rms(h), hn = h / rms(h)   (dh = dU without w_post)
 *     dgate = dY u, summed over the tokens (channel) or times sigmoid' (element)
 *     dw_pre = sum_t dn yn      dw_post = sum_t dU hn
 * dx, dh and (element) dgate are of `dtype`, all with leading dimension width or more; dx may be dy or dn, dh may be h,
 * an element dgate may be the gate (each with the same leading dimension); with w_post dx and dgate may not be h, and no two
 * outputs may be the same (ABS_EINVAL).  dw_pre, dw_post, (channel) dgate: fp32 [width], 4-byte aligned (slices of a flat
 * gradient); accumulate != 0 adds to what they hold.  dw_post must be given exactly when w_post is, dgate exactly when
 * there is a gate.  workspace: abs_residual_norm_workspace(tokens, width) bytes. */
size_t abs_residual_norm_workspace(uint64_t tokens, uint64_t width);
int abs_residual_norm_backward(const void *dn, uint64_t ld_dn, const void *dy, uint64_t ld_dy, const void *y, uint64_t ld_y,
                               const void *h, uint64_t ld_h, const void *gate, uint64_t ld_gate, uint32_t gate_kind,
                               const float *w_post, const float *w_pre, float scale, float eps, uint32_t dtype, uint64_t tokens,
                               uint64_t width, void *dx, uint64_t ld_dx, void *dh, uint64_t ld_dh, void *dgate, uint64_t ld_dgate,
                               float *dw_pre, float *dw_post, int accumulate, void *workspace, size_t workspace_bytes,
                               void *stream);

/* An activation in 8 bits.  A row of `width` values is cut into blocks of 32 (the last one may be short; it is filled up
 * with zeros, so that a stored row has width rounded up to 32 values).  A block holds 32 int8 values q and one exponent
 * byte e: value = q 2^(e - 127), with the smallest e in 0..254 for which the block's largest magnitude is at most
 * 127 2^(e - 127), q rounded to nearest even.  Every such value is a bf16 number, so that a bf16 tensor-core product
 * takes it without a rounding.  A block that holds an infinity or NaN gets e = 255 and stands for NaNs.
 *   x [tokens, width] of `dtype`;  q [tokens, W] int8, e [tokens, W / 32] uint8, W = width rounded up to 32, both packed
 *   (no gaps between rows), q 16-byte aligned. */
int abs_ckpt8_quantize(const void *x, uint64_t ld_x, uint32_t dtype, uint64_t tokens, uint64_t width, int8_t *q, uint8_t *e,
                       void *stream);
int abs_ckpt8_dequantize(const int8_t *q, const uint8_t *e, uint64_t tokens, uint64_t width, void *x, uint64_t ld_x,
                         uint32_t dtype, void *stream);

/* dw[i, o] (+)= sum_t x^[t, i] dy[t, o]: the gradient of a weight stored [in, out] (as the library's own layers are) from
 * the 8-bit activation q, e [tokens, width] and dy [tokens, out] bf16, on the tcgen05 tensor cores with fp32 accumulation.
 *   dw [width, out] fp32, ld_dw >= out, 4-byte aligned (a slice of a flat gradient); accumulate != 0 adds to what it holds.
 *   workspace: abs_ckpt8_wgrad_workspace(tokens, width, out, dy, ld_dy) bytes: partial sums where the tokens are split
 *             over the GPU, and a packed copy of a dy whose rows are not 16-byte aligned.  May be 0 (NULL is taken then).
 * tokens, width and out up to 2^31 - 64 (ABS_ELIMIT).  The kernel's waits are bounded; see abs_llm_check. */
size_t abs_ckpt8_wgrad_workspace(uint64_t tokens, uint64_t width, uint64_t out, const void *dy, uint64_t ld_dy);
int abs_ckpt8_wgrad(const int8_t *q, const uint8_t *e, const void *dy, uint64_t ld_dy, uint64_t tokens, uint64_t width,
                    uint64_t out, float *dw, uint64_t ld_dw, int accumulate, void *workspace, size_t workspace_bytes,
                    void *stream);

/* Blocks until `stream` has finished and reports the device-side status of the calls of this header on the current
 * device: ABS_OK, ABS_ECUDA, or once ABS_ETIMEOUT (a bounded wait inside a kernel ran out; its tile was not written). */
int abs_llm_check(void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ABS_LLM_H_ */
