/*
 * kvr_policy.h -- the clipped policy loss of given tokens, and the gradient of its logits.
 *
 * The rollouts that this library brings back are a trainer's samples: beside each token
 * stands the log probability it was taken with (kv_logprobs, kvr_logprob.h), its advantage
 * and, where the loss holds the policy near a reference, the reference's log probability.
 * kv_policy_loss takes these and the present policy's logits to the loss of every token,
 * their sum and the logits' gradient.  Same conventions as kvr.h (status codes, void*
 * streams, host-side validation before any device work, thread-compatible).
 */
#ifndef KVR_POLICY_H
#define KVR_POLICY_H

#include <stdint.h>

#include "kvr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Workspace bytes of kv_policy_loss, enough for every call of fewer rows or a smaller
 * vocabulary too; 0 for sizes it does not take (rows 1 .. 2^20, vocab 1 .. 2^21, rows *
 * ceil(vocab / 8192) below 2^24). */
uint64_t kv_policy_loss_workspace_bytes(int64_t rows, int32_t vocab);

/* With x_v = scale * z_v of row i's logits z (0 < scale <= 2^127, the inverse temperature),
 * t = tokens[i], A = advantages[i], w = weights[i]:
 *   lp    = x_t - log sum_v e^(x_v)                        the token's log probability
 *   rho   = e^(lp - old_logprobs[i])                       1 where old_logprobs is NULL
 *   gain  = min(rho A, clip(rho, 1 - clip_low, 1 + clip_high) A)
 *   kl    = e^D - D - 1, D = ref_logprobs[i] - lp          0 where ref_logprobs is NULL
 *   loss  = w (kl_coef kl - gain)
 *   dloss / dz_v = scale w (-(rho A where rho A <= the clipped one, else 0)
 *                           + kl_coef (1 - e^D)) (1[v = t] - p_v),  p = softmax(x)
 * old_logprobs, ref_logprobs, advantages and weights are constants of the loss.
 *   logits       device [rows][vocab] of dtype (KV_F32 or KV_BF16), rows `stride`
 *                elements apart, on any boundary of their elements
 *   tokens       device int32 [rows]; one outside [0, vocab) leaves its row out
 *   old_logprobs, ref_logprobs, weights  device float [rows] or NULL (weights: all 1)
 *   advantages   device float [rows]
 *   clip_low     0 .. 1; clip_high at least 0, infinity: not clipped
 *   kl_coef      finite; 0 without ref_logprobs
 *   total        device float [1], NULL = not wanted: the sum of the rows' losses
 *   losses, logprobs, kls  device float [rows], NULL = not wanted: loss, lp and kl
 *                (kls needs ref_logprobs)
 *   grad         device [rows][vocab] of dtype, rows grad_stride elements apart, NULL = not
 *                wanted: dtotal / dlogits, every entry written.  May be the logits
 *                themselves with the same stride, which it then takes the place of
 *   workspace    device scratch, on a boundary of 16 bytes; calls in flight at once
 *                need one each
 * A row with weight 0 has loss and kl 0 and a gradient of zeros, whatever its logits,
 * advantage and log probabilities are; one left out has logprob 0 besides.  An entry of
 * probability 0 has gradient 0, also where e^D or rho and the row's slope with it are
 * infinite (past 2^1023): a masked token, its logit -infinity or so far below the largest
 * that fp64 holds no e^(x_v - x_max), and every entry beside a token of probability 1.  The
 * row's own token, where that is masked, is not meant: 1 - p_t is 1 there, lp = -infinity
 * makes rho 0 (1 without old_logprobs) and D infinite, and loss, kl and the token's entry
 * are the formula's.  A NaN or +infinity makes its row's results NaN, and the total with
 * them.  Elsewhere infinite inputs go the formula's way.  1 - p_t and log p_t are taken
 * from the other tokens' sum, so that for all but certain tokens too they are off by at most
 * (50 + 2 T) 2^-24 of themselves, T the largest log2 e (max x - x_v) that counts, below 150
 * (a few 2^-24 in ordinary rows).  Sums are fp32 over what a thread takes at once, or over
 * 8192 neighbouring entries and up to four such parts, and joined in fp64; entries below 2^-126
 * of the largest are left out.  grad is rounded once; results do not depend on timing.
 * The arrays on the device are read when the call runs there, so a captured call follows
 * their contents.
 *   KV_EINVAL  null arrays, rows or vocab out of range, a stride < vocab, an unknown dtype, a
 *              scale, clip bound or kl_coef out of range, kls or kl_coef without
 *              ref_logprobs, a pointer not on its boundary
 *   KV_ENOMEM  workspace smaller than kv_policy_loss_workspace_bytes
 *   KV_EDEVICE device not selectable, or a device error */
kv_status kv_policy_loss(const void* logits, int32_t dtype, int64_t rows, int32_t vocab, int64_t stride,
                         float scale, const int32_t* tokens, const float* old_logprobs,
                         const float* ref_logprobs, const float* advantages, const float* weights,
                         float clip_low, float clip_high, float kl_coef, float* total, float* losses,
                         float* logprobs, float* kls, void* grad, int64_t grad_stride,
                         void* workspace, uint64_t workspace_bytes, int32_t device, void* stream);

#ifdef __cplusplus
}
#endif
#endif
