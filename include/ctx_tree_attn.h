/*
 * ctx_tree_attn.h -- attention of a tree of drafted tokens over paged key-value caches
 * on one AMD Instinct MI355X (gfx950): the step that verifies the drafts of a
 * smaller model, many tokens of a sequence in one pass over its cache.
 *
 * The drafts are appended first (ctx_kv_append_run_paged, with their positions), attend
 * to the cache here, and the accepted ones are moved together
 * (ctx_kv_compact_run_paged in ctx_kv_pages.h).
 *
 * Sequence b holds L_b tokens, of which the last n_b = q_lens[b] are its drafts: draft i is token
 * H_b + i, H_b = L_b - n_b, and row q_starts[b] + i of the packed rows.  Its parent is
 * a draft before it or, for a root, the last token before the drafts.  depth_i = 0 for roots,
 * depth of the parent + 1 for others; position p_i = H_b + depth_i.  Draft i sees
 *   token t < H_b   if t < prefix_b or p_i - t < window (any t without a window),
 *   draft a         if a = i or a is an ancestor of i, and depth_i - depth_a < window.
 * Its score with a token at position p (t, or p_a) is
 *
 *   s = scale * q . k,   then, if softcap > 0, s = softcap * tanh(s / softcap),
 *   then, if slopes are given, s -= slopes[h] * (p_i - p)
 *
 * and its output the softmax over the tokens that it sees times their values.
 *
 * Common arguments and conventions as in ctx_paged_attn.h; a handle whose page_tokens is positive.
 */
#ifndef CTX_TREE_ATTN_H_
#define CTX_TREE_ATTN_H_

#include <stddef.h>
#include <stdint.h>

#include "ctx_decode_attn.h"
#include "ctx_paged_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CTX_TREE_MAX_DRAFTS 256 /* drafts per sequence */

/*
 * Bytes of workspace that a call on `num_seqs` sequences with up to max_q_len drafts each
 * needs, written to the HOST pointer `bytes`.
 * Errors: INVALID_ARG, UNSUPPORTED, CAPACITY.
 */
int ctx_tree_attn_workspace(ctx_decode_attn* handle, int32_t num_seqs, int32_t max_q_len, size_t* bytes);

/*
 * Queue the attention of the sequences' drafts.
 *
 *   q        bf16 [total_q, Hq, D], contiguous
 *   parents  int32 [total_q]: -1 for a root, or the index 0 .. i - 1 of draft i's parent among
 *            its sequence's drafts.  Any other value marks a padding row, and so are the
 *            drafts below one: nothing of their q, keys and values is used, and they get zeros
 *   max_q_len  host bound on q_lens, up to CTX_TREE_MAX_DRAFTS; drafts past it are not touched
 *   scores   NULL: s = scale * q . k, every token.  Without doc_starts; a prefix counts up to
 *            H_b tokens.  CTX_SCORES_SPLIT_P asks for two-term softmax weights with bf16
 *            outputs; without it they are of one term, whatever the cap (the prefill takes
 *            two for caps above 512)
 *   out      [total_q, Hq, D] of desc.out_dtype, contiguous
 *   workspace, workspace_bytes  at least what ctx_tree_attn_workspace says, 16-byte aligned;
 *            calls that may overlap need one each
 * Arithmetic: fp32 scores and softmax statistics, fp32 accumulation.  With bf16 outputs the softmax
 * weights enter the product with V rounded to bf16, and each row is normalised by the
 * sum of the rounded weights; with CTX_SCORES_SPLIT_P as two bf16 terms (16 significant
 * bits); with fp32 outputs as three (24 bits).
 * Keys and values that some draft of the sequence sees must be finite, their scores too; what
 * none sees may hold anything.  The batch's blocks of tokens are shared out evenly, so the
 * order of sums depends on the other sequences' lengths: the same request alone and
 * in a batch may differ by fp32 rounding.
 * Errors: INVALID_ARG (also for doc_starts), UNSUPPORTED (max_q_len), CAPACITY (also
 * workspace_bytes), ALIGNMENT, HIP.
 */
int ctx_tree_attn_run_paged(ctx_decode_attn* handle, const void* q, const void* k_pages, const void* v_pages,
                            int32_t num_pages, const int32_t* block_tables, int32_t max_pages_per_seq,
                            const int32_t* seq_lens, const int32_t* q_starts, const int32_t* q_lens,
                            const int32_t* parents, int32_t num_seqs, int32_t total_q, int32_t max_q_len, float scale,
                            const ctx_attn_scores* scores, void* out, void* workspace, size_t workspace_bytes,
                            void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CTX_TREE_ATTN_H_ */
