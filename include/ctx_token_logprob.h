/*
 * ctx_token_logprob.h -- log probabilities of given tokens with the entropy of
 * their distribution and its top alternatives, and the gradient by the logits, on
 * one AMD Instinct MI355X (gfx950).
 *
 * The OPD loss (ctx_opd_loss.h) takes stored log probabilities of the sampler and
 * of the teacher; these calls find them.  Row j of the logits z_j has V entries,
 * x_j = scale * z_j (scale = 1 / temperature), p_j = softmax(x_j):
 *
 *   logp[j, i] = x_j[tokens[j, i]] - log sum_v exp(x_j[v])
 *   entropy[j] = -sum_v p_j[v] log p_j[v]
 *   the `top` largest logits of the row: their columns, the lowest first among equal
 *   ones, and their log probabilities
 *
 * and, for upstream gradients a of logp and b of the entropy,
 *
 *   grad_logits[j, v] = scale (sum_i a[j, i] ([tokens[j, i] = v] - p_j[v])
 *                              - b[j] p_j[v] (log p_j[v] + entropy[j]))
 *
 * A logit of -1e38 or less is masked (-inf, and the lowest value of a type): it has
 * probability 0 and logp -inf and is no alternative.  A row without others has entropy 0
 * and a gradient of zeros.  A row with a NaN or +inf gives NaN throughout, and no
 * alternatives.  A token below 0 stands for none: its logp is 0, its
 * gradient is not used; one past the vocabulary has logp NaN and is as none for the
 * gradient.  Masked rows are not read: their outputs are 0, without alternatives.
 * Where a row has no more alternatives the column is -1, the log probability -inf (NaN
 * in a row of NaN, 0 in a masked one).
 *
 * Arithmetic: fp32 (differences to the largest logit in one FMA each, or two roundings where its
 * product is 2^24 or more, so that no result grows worse with an offset of all logits; sums over lanes
 * and then in a fixed order); gradients are rounded to the logits' type once, nearest even.
 * Deterministic.
 *
 * Conventions as in ctx_decode_attn.h: device pointers unless stated, owned by the
 * caller until the work queued on `stream` completes; asynchronous, no allocation,
 * no host read of device data; status codes of ctx_status, and
 * ctx_decode_attn_last_error() for the message.  All memory is on the current device.
 */
#ifndef CTX_TOKEN_LOGPROB_H_
#define CTX_TOKEN_LOGPROB_H_

#include <stddef.h>
#include <stdint.h>

#include "ctx_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CTX_LOGPROB_MAX_TOKENS 64 /* given tokens per row */
#define CTX_LOGPROB_MAX_TOP 64    /* alternatives per row */

/*
 * Bytes of workspace that a ctx_token_logprob_run call with these arguments on the
 * current device needs (0 for many rows), written to the HOST pointer `bytes`.
 * Errors: INVALID_ARG, UNSUPPORTED, HIP.
 */
int ctx_token_logprob_workspace(ctx_dtype dtype, int32_t vocab, int32_t num_rows, int32_t top, size_t* bytes);

/*
 * Queue the log probabilities of one batch of rows.
 *
 *   logits      `dtype` (bf16 or fp32) [num_rows, row_stride]; columns 0 .. vocab-1 used
 *   row_stride  elements between rows, at least vocab, a multiple of 16 bytes
 *   vocab       1 .. 2^28
 *   tokens      int32 [num_rows, num_tokens], or NULL with num_tokens = 0
 *   num_tokens  0 .. CTX_LOGPROB_MAX_TOKENS
 *   mask        uint8 [num_rows], zero: a masked row; NULL: none is
 *   num_rows    0 .. 2^24 - 1
 *   scale       1e-30 .. 1e30
 *   top         0 .. CTX_LOGPROB_MAX_TOP
 *   token_logp  float [num_rows, num_tokens] out (NULL with num_tokens = 0)
 *   entropy     float [num_rows] out, or NULL
 *   stats       float [num_rows, 2] out, or NULL: what the gradient needs of a row, its
 *               largest logit and the sum of exp(x - scale * that) (0 in rows without any)
 *   top_tokens, top_logp  int32 and float [num_rows, top] out (NULL with top = 0)
 *   workspace   at least what ctx_token_logprob_workspace says, 16-byte aligned; calls
 *               that may overlap need one each.  NULL if that is 0
 * Errors: INVALID_ARG, UNSUPPORTED (vocab, num_tokens, num_rows, top), CAPACITY (workspace_bytes),
 * ALIGNMENT (16 bytes: logits, workspace), HIP.
 */
int ctx_token_logprob_run(const void* logits, ctx_dtype dtype, int64_t row_stride, int32_t vocab, const int32_t* tokens,
                          int32_t num_tokens, const uint8_t* mask, int32_t num_rows, float scale, int32_t top,
                          float* token_logp, float* entropy, float* stats, int32_t* top_tokens, float* top_logp,
                          void* workspace, size_t workspace_bytes, void* stream);

/*
 * Queue the gradient by the logits.  logits, dtype, row_stride, vocab, tokens,
 * num_tokens, mask, num_rows and scale as in the call that gave stats and entropy.
 *
 *   stats         float [num_rows, 2] of that call
 *   grad_logp     float [num_rows, num_tokens]: a (NULL with num_tokens = 0)
 *   entropy, grad_entropy  float [num_rows]: that call's, and b; both NULL: b = 0
 *   grad_logits   `dtype` [num_rows, grad_row_stride] out; columns >= vocab are not
 *                 written.  It may not overlap the logits (INVALID_ARG)
 * A row whose sum of a and whose b are 0, and whose tokens' gradients all are, gets zeros
 * without being read.  Errors: INVALID_ARG, UNSUPPORTED, ALIGNMENT (16 bytes: logits,
 * grad_logits), HIP.
 */
int ctx_token_logprob_grad_run(const void* logits, ctx_dtype dtype, int64_t row_stride, int32_t vocab,
                               const int32_t* tokens, int32_t num_tokens, const uint8_t* mask, int32_t num_rows,
                               float scale, const float* stats, const float* entropy, const float* grad_logp,
                               const float* grad_entropy, void* grad_logits, int64_t grad_row_stride, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CTX_TOKEN_LOGPROB_H_ */
