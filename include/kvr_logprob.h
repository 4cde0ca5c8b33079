/*
 * kvr_logprob.h -- log probabilities of given tokens, entropy, likeliest tokens.
 *
 * A rollout records, beside every token it takes, that token's log probability
 * under the model (and often the distribution's entropy and the likeliest
 * alternatives); kv_decode_step returns the logits, and kv_logprobs reads them once
 * for all three.  Same conventions as kvr.h (status codes, void* streams, host-side
 * validation before any device work, thread-compatible).
 */
#ifndef KVR_LOGPROB_H
#define KVR_LOGPROB_H

#include <stdint.h>

#include "kvr.h"

#ifdef __cplusplus
extern "C" {
#endif

#define KV_LOGPROBS_MAX_TOP 64

/* Workspace bytes of kv_logprobs; 0 for sizes it does not take (rows 1 .. 2^20, vocab
 * 1 .. 2^21, rows * ceil(vocab / 8192) below 2^24, top_n 0 .. KV_LOGPROBS_MAX_TOP and at
 * most vocab). */
uint64_t kv_logprobs_workspace_bytes(int64_t rows, int32_t vocab, int32_t top_n);

/* With x_v = scale * z_v of a row's logits z (0 < scale <= 2^127, the inverse temperature):
 *   logprobs[i]     = x_t - log sum_v e^(x_v), t = tokens[i]
 *   entropy[i]      = - sum_v p_v log p_v, p = softmax(x); terms with p_v = 0 are 0
 *   top_tokens[i][] the top_n tokens of largest z_v in falling order, the lower
 *                   index first among equals, top_logprobs[i][] their log
 *                   probabilities
 *   logits       device [rows][vocab] of dtype (KV_F32 or KV_BF16), rows `stride`
 *                elements apart, on any boundary of their elements
 *   tokens       device int32 [rows], NULL only with logprobs NULL; a negative one
 *                marks a row without a token (logprobs 0), one >= vocab has
 *                probability 0 (-infinity)
 *   logprobs, entropy            device float [rows], NULL = not wanted
 *   top_logprobs, top_tokens     device float / int32 [rows][top_n]; top_n 0 ..
 *                KV_LOGPROBS_MAX_TOP and at most vocab, 0 = not wanted
 *   workspace    device scratch, on a boundary of 16 bytes; calls in flight at once
 *                need one each
 * Logits of -infinity (masked tokens) and of the dtype's lowest value count like any
 * other; where all of a row are -infinity its log probabilities are -infinity, its
 * entropy 0 and its likeliest tokens the first ones.  A NaN or +infinity in a row
 * makes its log probabilities and entropy NaN; its likeliest tokens rank NaN below
 * every number.  Sums are fp32; results do not depend on timing.
 *   KV_EINVAL  null arrays, rows or vocab out of range, stride < vocab, an unknown dtype, a
 *              scale that is not positive or above 2^127, top_n out of range, a pointer not
 *              on its boundary
 *   KV_ENOMEM  workspace smaller than kv_logprobs_workspace_bytes
 *   KV_EDEVICE device not selectable, or a device error */
kv_status kv_logprobs(const void* logits, int32_t dtype, int64_t rows, int32_t vocab, int64_t stride,
                      float scale, const int32_t* tokens, int32_t top_n, float* logprobs,
                      float* entropy, float* top_logprobs, int32_t* top_tokens, void* workspace,
                      uint64_t workspace_bytes, int32_t device, void* stream);

#ifdef __cplusplus
}
#endif
#endif
