/*
 * ctx_kv_pages.h -- the pages of paged key-value caches on one AMD Instinct MI355X
 * (gfx950): rows of a block table forked, grown, trimmed and freed, with the
 * pages' use counted on the device, and the data of the caches copied and compacted.
 *
 * An act-first rollout asks for a fast action and for a full response over the same
 * context c_t (Sec. 4.1): the second request forks the first one's pages.  A serving
 * loop (ctx_paged_attn.h) makes room for new tokens (ctx_kv_resize_run_paged), copies
 * the pages that forks still share and that the tokens go to
 * (ctx_kv_copy_run_paged, once per layer), appends, attends, keeps the
 * drafts that were accepted (ctx_kv_compact_run_paged, once per layer) and gives the
 * rest of the room back (ctx_kv_resize_run_paged).  Nothing of it waits for the
 * host, so a step can be captured in a HIP graph.
 *
 * Common arguments (with those of ctx_paged_attn.h):
 *   block_tables  int32 [num_seqs, max_pages_per_seq].  Row b holds the pages of its
 *                 first ceil(seq_lens[b] / P) entries, P the handle's page_tokens
 *   seq_lens      int32 [num_seqs]: a value below 0 counts as 0.  Forks and resizes count one past
 *                 the row's max_pages_per_seq * P tokens as that; for a compaction the
 *                 tokens past them are on no page
 *   page_refs     int32 [num_pages]: how many rows hold each page; 0 is a free one.  The
 *                 caller sets it up (zeros, if all rows are empty) and leaves it to
 *                 ctx_kv_fork_run_paged and ctx_kv_resize_run_paged
 * An entry outside 0 .. num_pages - 1 is no fault: it holds no page, and no token is read or
 * written there.  Arrays that a call writes may not overlap each other or those that it
 * reads, unless said otherwise (INVALID_ARG).
 *
 * Conventions as in ctx_decode_attn.h: device pointers unless stated, owned by the
 * caller until the work queued on `stream` completes; asynchronous, no allocation, no
 * host read of device data; results do not depend on the order in which the device
 * works; status codes of ctx_status, and ctx_decode_attn_last_error() for the
 * message.  The handle's device must be the current one.
 */
#ifndef CTX_KV_PAGES_H_
#define CTX_KV_PAGES_H_

#include <stddef.h>
#include <stdint.h>

#include "ctx_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Queue forks: row b of the table and seq_lens[b] become those of row parents[b], whose pages
 * it then holds too.  The pages that row b held before are given back; its entries
 * past the parent's pages become -1.
 *
 *   parents  int32 [num_seqs]; outside 0 .. num_seqs - 1, or b: row b stays as it is.  So does
 *            a row whose parent is itself to be forked
 * Errors: INVALID_ARG, UNSUPPORTED (handle without page_tokens), CAPACITY, HIP.
 */
int ctx_kv_fork_run_paged(ctx_decode_attn* handle, int32_t* block_tables, int32_t max_pages_per_seq,
                          int32_t* seq_lens, int32_t num_seqs, const int32_t* parents, int32_t* page_refs,
                          int32_t num_pages, void* stream);

/* Bytes of workspace of a ctx_kv_resize_run_paged call. */
size_t ctx_kv_resize_workspace(int32_t num_seqs, int32_t num_pages);

/*
 * Queue a change of every row's length from seq_lens[b] to new_lens[b] (below 0: 0).
 *
 * Shorter rows first give back the pages past their new length (entries -1).  Then, in the
 * order of rows, longer ones get the lowest free pages; one whose last page is not
 * full and held by other rows too gets a page in its place first, so that what is
 * appended is its own.  A row that the free pages do not suffice for, and each
 * later one that needs pages, keeps its length and pages; so does one whose new length is past
 * max_pages_per_seq * P.  Pages replaced in this call are free in the next.
 *
 *   granted  int32 [num_seqs] out: the rows' lengths from now on.  May be seq_lens or new_lens,
 *            the same array and no part of it
 *   copies   int32 [num_seqs, 2] out: the page that was replaced and the one in its
 *            place, whose data ctx_kv_copy_run_paged has to copy; -1, -1 where none was
 *   workspace, workspace_bytes  at least ctx_kv_resize_workspace, 16-byte aligned; calls that
 *            may overlap need one each
 * Errors: INVALID_ARG, UNSUPPORTED, CAPACITY (also workspace_bytes), ALIGNMENT, HIP.
 */
int ctx_kv_resize_run_paged(ctx_decode_attn* handle, int32_t* block_tables, int32_t max_pages_per_seq,
                            const int32_t* seq_lens, const int32_t* new_lens, int32_t num_seqs, int32_t* page_refs,
                            int32_t num_pages, int32_t* granted, int32_t* copies, void* workspace,
                            size_t workspace_bytes, void* stream);

/*
 * Queue copies of whole pages: page copies[i, 1] of both caches becomes page copies[i, 0].
 * A pair with a page outside 0 .. num_pages - 1, or with the same one twice, copies
 * nothing.  No page may be written twice, or read and written, in one call.
 *
 *   k_pages, v_pages  bf16 [num_pages, P, Hkv, D]
 *   copies            int32 [num_copies, 2]
 * Errors: INVALID_ARG, UNSUPPORTED, ALIGNMENT (16 bytes: pages), HIP.
 */
int ctx_kv_copy_run_paged(ctx_decode_attn* handle, void* k_pages, void* v_pages, int32_t num_pages,
                          const int32_t* copies, int32_t num_copies, void* stream);

/*
 * Queue the compaction of each sequence's newest tokens: of the last q_lens[b] of its
 * seq_lens[b] tokens those listed in `keep` move together, in order, and the others are
 * lost.  Token i of them goes to position seq_lens[b] - q_lens[b] + i.  (The accepted path
 * of drafted tokens; with q_lens = seq_lens, a context without some of its turns.)
 *
 *   q_starts, q_lens  int32 [num_seqs]: 0 <= q_lens[b] <= seq_lens[b]; rows q_starts[b] ..
 *                     q_starts[b] + q_lens[b] - 1 of the packed rows are the sequence's
 *   keep        int32 [total_q]: entry q_starts[b] + i, i < keep_lens[b], is which of the
 *               sequence's last q_lens[b] tokens is kept as its i-th: rising, from 0 ..
 *               q_lens[b] - 1.  A token outside them leaves its place unspecified, and so do
 *               entries that do not rise
 *   keep_lens   int32 [num_seqs], 0 .. q_lens[b]
 *   new_lens    int32 [num_seqs] out, or NULL: seq_lens[b] - q_lens[b] + keep_lens[b].
 * Pages that tokens move within or to must not be shared with other sequences.  Tables and
 * counts stay as they are: ctx_kv_resize_run_paged to new_lens gives pages back.
 * Errors: INVALID_ARG, UNSUPPORTED, CAPACITY, ALIGNMENT (16 bytes: pages), HIP.
 */
int ctx_kv_compact_run_paged(ctx_decode_attn* handle, void* k_pages, void* v_pages, int32_t num_pages,
                             const int32_t* block_tables, int32_t max_pages_per_seq, const int32_t* seq_lens,
                             const int32_t* q_starts, const int32_t* q_lens, const int32_t* keep,
                             const int32_t* keep_lens, int32_t num_seqs, int32_t total_q, int32_t* new_lens,
                             void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CTX_KV_PAGES_H_ */
