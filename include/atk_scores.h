/*
 * atk_scores.h - C ABI of the scores of tokens: log probabilities of given tokens with the entropy of their distribution and its likeliest tokens, and the gradient of the
 * first two.  Conventions are atk_decode.h's: device pointers, everything the host sees checked, nothing allocated or waited for, all calls may be captured.
 *
 * Rows of logits x (batch, tokens, vocab) of `dtype`, vocab contiguous, strides in elements for the first two (rows begin where elements may):
 *   lse = log sum_i exp(x_i),   log p_i = x_i - lse,   entropy = -sum_i p_i log p_i (with 0 log 0 = 0), all f32.
 * A log probability is as good as its size allows wherever the row lies: it is taken from a logit near the largest one, not from lse, which in f32 is off by |lse| 2^-24.
 * A logit of -inf has no probability.  A row without any (all -inf) has lse -inf, log probabilities of -inf and entropy 0; with a NaN or +inf all of these are NaN.
 */
#ifndef ATK_SCORES_H
#define ATK_SCORES_H

#include "atk_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * chosen       (batch, tokens) int32: the token that is asked for; outside 0..vocab-1 (padding) its log probability is -inf.
 * logprobs, entropy, lse   (batch, tokens) f32.
 * top          0 to 32, at most vocab.  top_logprobs (batch, tokens, top) f32 and top_tokens int32: the likeliest tokens, equally likely ones by their numbers; NaN counts as -inf in this order.
 * vocab        1 to 2^24.  work: atk_token_logprobs_workspace_bytes() bytes on 16 bytes.
 */
int64_t atk_token_logprobs_workspace_bytes(int64_t batch, int64_t tokens, int64_t vocab, int64_t top, int dtype);
int atk_token_logprobs(const void *logits, const int64_t stride[2], const int32_t *chosen, int64_t batch, int64_t tokens, int64_t vocab,
                       int64_t top, int dtype, float *logprobs, float *entropy, float *lse, float *top_logprobs, int32_t *top_tokens,
                       void *work, int64_t work_bytes, void *stream);

/*
 * grad (batch, tokens, vocab) of `dtype`, strides in elements for the first two: with a = grad_logprobs and b = grad_entropy (batch, tokens) f32 (either may be NULL: 0)
 *   grad_i = a ([i = chosen] - p_i) - b p_i (log p_i + entropy),   p_i = exp(x_i - lse)
 * of the lse and the entropy that the call above gave (entropy may be NULL where grad_entropy is).  With |lse| below 1024 p is off by |lse| 2^-24 relatively, as lse itself is; from there on (a row of
 * the type's lowest value) what lse lost in its rounding is found from the row and put in again, if it is no more than that.  A chosen token outside 0..vocab-1 has a = 0; a row without any
 * probability has gradients of 0.  Rows of grad do not overlap; it may be the logits' own memory, in the same places.
 */
int atk_token_logprobs_grad(const void *logits, const int64_t stride[2], const int32_t *chosen, const float *lse, const float *entropy,
                            const float *grad_logprobs, const float *grad_entropy, int64_t batch, int64_t tokens, int64_t vocab, int dtype,
                            void *grad, const int64_t grad_stride[2], void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ATK_SCORES_H */
