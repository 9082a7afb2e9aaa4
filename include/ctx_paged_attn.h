/*
 * ctx_paged_attn.h -- operators over paged key-value caches on one AMD Instinct
 * MI355X (gfx950), beside ctx_decode_attn_run_paged: the append of new keys
 * and values with the head norm and the rotation of positions applied on the
 * way, and the causal prefill and the decode step with changed scores (capped
 * by a tanh, biased by distance, masked by a window, a prefix or documents).
 *
 * A serving loop over a handle whose page_tokens P is positive: the new tokens of a
 * turn are appended (ctx_kv_append_run_paged), attend to the cache
 * (ctx_prefill_attn_run_paged), and every decoded token after them is appended
 * and attends (ctx_decode_attn_run_paged_scored).
 *
 * Common arguments:
 *   k_pages, v_pages  bf16 [num_pages, P, Hkv, D], D = 128
 *   block_tables      int32 [num_seqs, max_pages_per_seq]: token t of sequence b is slot
 *                     t % P of page block_tables[b][t / P].  Entries of tokens that a call
 *                     does not touch are not used.  An entry outside 0 .. num_pages - 1, or
 *                     a token past max_pages_per_seq, is no fault: nothing is appended
 *                     there, and no query sees the tokens that would be there
 *   seq_lens          int32 [num_seqs]: L_b, tokens of sequence b in the cache, the new
 *                     ones included; a value below 0 counts as 0
 *   q_starts, q_lens  int32 [num_seqs]: the new tokens of sequence b are its last
 *                     q_lens[b] and rows q_starts[b] .. q_starts[b] + q_lens[b] - 1 of the
 *                     packed rows (any order, no overlap, gaps allowed).  Row
 *                     q_starts[b] + i has position p = L_b - q_lens[b] + i
 *   total_q           rows of the packed arrays; rows outside 0 .. total_q - 1 are not touched
 * Packed rows of no sequence are neither read nor written.  0 <= q_lens[b] <= L_b is the
 * caller's to keep; otherwise what the sequence's rows get is unspecified.
 *
 * Conventions as in ctx_decode_attn.h: device pointers unless stated, owned by
 * the caller until the work queued on `stream` completes; asynchronous, no
 * allocation, no host read of device data (every call can be captured in a HIP
 * graph); deterministic; status codes of ctx_status, and
 * ctx_decode_attn_last_error() for the message.  The handle's device must be the
 * current one.
 */
#ifndef CTX_PAGED_ATTN_H_
#define CTX_PAGED_ATTN_H_

#include <stdint.h>

#include "ctx_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * What the append does to queries and keys (a HOST struct, read during the call).
 *
 *   normed(x)_d  = x_d * weight_d / sqrt(sum_d x_d^2 / D + norm_eps)   per head, if a weight is given
 *   rotated(x):  the pairs (a, c) of the first rotary_dim dimensions become
 *                (a cos u - c sin u, c cos u + a sin u) with u = position * inv_freq[i];
 *                pair i is dimensions (i, i + rotary_dim / 2), or (2 i, 2 i + 1) with
 *                CTX_ROTARY_INTERLEAVED.  The other dimensions stay.
 *
 * The result is computed in fp32 from the bf16 inputs and rounded to bf16 once;
 * the angle is reduced in fp64, so far positions are as exact as near ones.  The sum of
 * squares is an fp32 one: a normed head holds values up to 1e18, and with norm_eps = 0
 * some of 1e-18 or more.
 */
#define CTX_ROTARY_INTERLEAVED 1u
typedef struct {
  const float* inv_freq;    /* float [rotary_dim / 2], or NULL with rotary_dim = 0: no rotation */
  const int32_t* positions; /* int32 [total_q]: the rows' rotary positions, or NULL: p */
  const void* q_norm;       /* bf16 [D]: norm weight of the queries' heads, or NULL: no norm */
  const void* k_norm;       /* the same of the keys' */
  float norm_eps;           /* >= 0; used with a norm weight */
  int32_t rotary_dim;       /* 0, or a multiple of 16 up to D */
  uint32_t flags;           /* 0 or CTX_ROTARY_INTERLEAVED */
} ctx_rotary;

/*
 * Queue the append of the new tokens: their keys and values go to their cache
 * slots, their queries (optional) to q_out, queries and keys normed and then
 * rotated as `rotary` says (NULL: neither).
 *
 *   q, k, v    bf16 rows [total_q] of Hq (Hkv, Hkv) heads of D: row j starts at element
 *              j * q_stride (k_stride, v_stride), so that the three may be slices of the rows
 *              of one projection.  q may be NULL (then q_out too)
 *   strides    in elements, multiples of 8, at least the row's Hq * D (Hkv * D)
 *   q_out      bf16 [total_q, Hq, D], contiguous; may be q itself if q_stride = Hq * D,
 *              otherwise it may not overlap an input
 *   q_starts, q_lens  both NULL: one new token per sequence, row b being sequence b's
 *              (none where L_b = 0); total_q is then num_seqs
 * No two tokens of a call may share a cache slot.  Nothing else in the caches changes.
 * Errors: INVALID_ARG, UNSUPPORTED (handle without page_tokens, rotary_dim),
 * CAPACITY, ALIGNMENT (16 bytes: q, k, v, pages, q_out, norm weights), HIP.
 */
int ctx_kv_append_run_paged(ctx_decode_attn* handle, const void* q, int64_t q_stride, const void* k,
                            int64_t k_stride, const void* v, int64_t v_stride, void* k_pages, void* v_pages,
                            int32_t num_pages, const int32_t* block_tables, int32_t max_pages_per_seq,
                            const int32_t* seq_lens, const int32_t* q_starts, const int32_t* q_lens,
                            int32_t num_seqs, int32_t total_q, const ctx_rotary* rotary, void* q_out,
                            void* stream);

/*
 * Scores and masks of the two attention calls below (a HOST struct, read during
 * the call).  A query of head h at position p has with token t of its sequence
 *
 *   s = scale * q . k,   then, if softcap > 0, s = softcap * tanh(s / softcap),
 *   then, if slopes are given, s -= slopes[h] * |p - t|
 *
 * and sees the token if t < L_b and (t < prefix_b or max(doc, p - window + 1) <= t <= p).
 * A prefix is thus seen by every query of its sequence, its own ones included, whatever
 * the window and the documents are.  The output is the softmax over the seen tokens
 * times their values; a query that sees none gets zeros.
 */
#define CTX_SCORES_SPLIT_P 1u
typedef struct {
  float softcap;              /* > 0 (up to 1e38, and scale / softcap too), or 0: no cap */
  int32_t window;             /* > 0, or 0: no window */
  const float* slopes;        /* float [Hq], |slope| * L_b up to 1e37, or NULL: no bias */
  const int32_t* prefix_lens; /* int32 [num_seqs] or NULL: no prefix; a value past L_b counts as L_b */
  const int32_t* doc_starts;  /* int32, the first token of each query's document, one per packed
                                 row (prefill) or sequence (decode), or NULL: 0.  A value above p
                                 (a padding row) leaves the query its prefix alone */
  uint32_t flags;             /* 0 or CTX_SCORES_SPLIT_P: the prefill with bf16 outputs carries its
                                 softmax weights as two bf16 terms instead of one, as it does
                                 for a softcap above 512 in any case */
} ctx_attn_scores;

/*
 * Queue the causal prefill of each sequence's newest tokens against its pages,
 * which already hold their keys and values.
 *
 *   q       bf16 [total_q, Hq, D], contiguous
 *   max_q_len  host bound on q_lens (sizes the grid); rows past it are not touched
 *   scores  NULL: s = scale * q . k, every token up to p
 *   out     [total_q, Hq, D] of desc.out_dtype, contiguous
 * Arithmetic: fp32 scores and softmax statistics, fp32 accumulation.  With bf16
 * outputs the softmax weights enter the product with V rounded to bf16, and each
 * row is normalised by the sum of the rounded weights (an error of the size of the
 * outputs' own rounding); CTX_SCORES_SPLIT_P carries them as two bf16 terms (16
 * significant bits), for a second product with V.  With fp32 outputs they are three
 * bf16 terms (24 significant bits), whatever the flag.
 * Keys and values that some query of the sequence sees must be finite, their scores
 * too; what no query sees may hold anything.
 * Calls with few rows share a long context out over workgroups that meet in the
 * handle's workspace: as for ctx_decode_attn_run, calls that may overlap need separate
 * handles.
 * The kernel, and with it the order of sums and the roundings of weights, is chosen by num_seqs,
 * total_q, max_q_len, desc, the device's CU count and, of the scores, by the flags, the window, whether
 * prefix_lens and slopes are given, and the softcap (none, up to 512, above; a cap so large that
 * scale / softcap is below the smallest normal float counts as none).  So the same request alone and
 * in a batch may differ by those roundings.  desc.max_seq_len counts as the longest context: on a
 * handle for far longer ones, calls of a few rows over short contexts take 2 to 3 times as long.
 * Errors: INVALID_ARG, UNSUPPORTED, CAPACITY, ALIGNMENT, HIP.
 */
int ctx_prefill_attn_run_paged(ctx_decode_attn* handle, const void* q, const void* k_pages, const void* v_pages,
                               int32_t num_pages, const int32_t* block_tables, int32_t max_pages_per_seq,
                               const int32_t* seq_lens, const int32_t* q_starts, const int32_t* q_lens,
                               int32_t num_seqs, int32_t total_q, int32_t max_q_len, float scale,
                               const ctx_attn_scores* scores, void* out, void* stream);

/*
 * Queue one decode step: the newest token of every sequence (p = L_b - 1, its key
 * and value already in the pages) attends to what it sees.  Only pages with seen
 * tokens are read.  Uses the handle's workspace, as ctx_decode_attn_run_paged does:
 * calls that may overlap need separate handles.
 *
 *   q       bf16 [num_seqs, Hq, D], contiguous
 *   scores  as above; NULL: none
 *   out     [num_seqs, Hq, D] of desc.out_dtype, contiguous; zeros where L_b = 0
 * Keys and values of seen tokens must be finite; what is not seen may hold anything.
 * With split_tokens > 0, seq_lens[b] <= max_seq_len as for ctx_decode_attn_run.
 * Errors: INVALID_ARG, UNSUPPORTED, CAPACITY, ALIGNMENT, HIP.
 */
int ctx_decode_attn_run_paged_scored(ctx_decode_attn* handle, const void* q, const void* k_pages,
                                     const void* v_pages, int32_t num_pages, const int32_t* block_tables,
                                     int32_t max_pages_per_seq, const int32_t* seq_lens, int32_t num_seqs,
                                     float scale, const ctx_attn_scores* scores, void* out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CTX_PAGED_ATTN_H_ */
