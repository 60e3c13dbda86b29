/*
 * atk_decode.h - C ABI of the operators that a decoder needs beside the selection of approx_topk.h: attention of a
 * batch that shares a long prefix, verification of drafted tokens, and the pages of the cache between them.
 *
 * Conventions of approx_topk.h: device pointers on the current device, buffers owned by the caller, calls asynchronous
 * on `stream`, every argument that the host sees checked before any HIP call, ATK_OK or a negative code returned.  Unlike
 * approx_topk no call here allocates, waits or uses the library's pool: scratch comes with the call, and all calls may be
 * captured into a graph.  What only the device sees - page numbers, sequence numbers, lengths - is checked by the
 * kernels: a bad one is never used as an address, and is reported by a bit of *status (device, one int32, only ever
 * or-ed to, may be NULL).
 *
 * Sizes whose launches would have 2^32 threads and more are ATK_ERR_ARGS: batch * tokens * heads from 2^26 on, 2^24 sequences of a call on
 * pages, 2^22 requests of up to 128 KB of probabilities each.
 */
#ifndef ATK_DECODE_H
#define ATK_DECODE_H

#include <stdint.h>

#include "approx_topk.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { ATK_F16 = 2 }; /* element type of the functions of this header, beside ATK_F32 and ATK_BF16 */

enum { ATK_ERR_ARGS = -9 }; /* an argument of a function of this header is out of the range that it states */

/* bits of *status */
enum {
    ATK_STATUS_NO_PAGES = 1, /* fork, append: fewer free pages than the call needs; nothing of it was done */
    ATK_STATUS_BAD_SEQ = 2,  /* a row number outside the table; fork: a child that is not empty (nothing was done) */
    ATK_STATUS_BAD_PAGE = 4, /* a page number outside the cache, or a page given back more often than it was taken */
    ATK_STATUS_BAD_LEN = 8   /* a length below 0 or past the row's pages; append: a row too short for the new tokens (nothing was done) */
};

/*
 * Attention of `tokens` new tokens of each of `batch` sequences over a paged cache, the first prefix_len keys of which
 * all sequences share.
 *
 *   Sequence i is row s = seqs[i] of the table (NULL: s = i) and has lens[s] keys, its new tokens' among them: key j lies in
 *   page page_table[s * table_stride + j / page_size], at j % page_size.  Query t of it sees the keys
 *   j < lens[s] - (tokens - 1 - t).  Keys j < prefix_len are read through the row of the first sequence of the call, once
 *   for all of them: the caller sees to it that the others hold the same there.
 *   out = sum_j softmax_j(scale * q.k_j) * v_j over the visible keys, lse = log sum_j exp(scale * q.k_j); a query that sees
 *   no key, or whose scores are all -inf, gets 0 and -inf.  (Beside others a visible key with a score of -inf weighs 0, and 0 times NaN or infinity is NaN.)  What is not visible has no influence, NaN and infinities included.  Nor is a key
 *   whose page is outside the cache visible, nor any of a sequence whose row number is outside the table; a length past the row's pages counts as all of them.
 *
 *   q, out     (batch, tokens, heads, dim) of `dtype`, dim contiguous, strides in elements for the first three.
 *   k, v       (n_pages, page_size, kv_heads, dim) of `dtype`, dim contiguous, strides in elements for the first three: token
 *              by token or head by head in a page.  heads is a multiple of kv_heads, query head h reads head h / (heads / kv_heads).
 *   lse        (batch, tokens, heads) f32, contiguous, or NULL.
 *   dim        a multiple of 16 bytes / element size, up to 256.  Pointers of q, k, v, out on 16 bytes, strides (but a single one's) of whole 16 bytes.
 *   work       atk_attention_workspace_bytes() bytes on 16 bytes.
 * Scores, statistics and accumulators are f32; the weights are rounded to `dtype` for the product with v, their sum is not.
 */
typedef struct {
    const void *q, *k, *v;
    void *out;
    float *lse;
    const int32_t *page_table, *lens, *seqs;
    int32_t *status;
    int64_t batch, tokens, heads, kv_heads, dim;
    int64_t page_size, n_pages;
    int64_t rows, row_pages, table_stride; /* of the table: rows, pages in a row, int32 words between rows */
    int64_t prefix_len;
    int64_t q_stride[3], out_stride[3];    /* sequence, token, head */
    int64_t k_stride[3], v_stride[3];      /* page, token, head */
    double scale;                          /* FLT_MIN to 1e30 */
    int32_t dtype;
} atk_attention_args;
int64_t atk_attention_workspace_bytes(const atk_attention_args *args);
int atk_shared_prefix_attention(const atk_attention_args *args, void *work, int64_t work_bytes, void *stream);

/*
 * Verification of drafted tokens against the target's probabilities, from given random numbers.
 *
 *   Request b has n = n_drafts[b] drafted tokens (NULL: `drafts`; clamped to 0..drafts).  Token i is accepted while all
 *   before it were and accept_random[b, i] * q_i(d_i) < p_i(d_i); the products and sums are f64.  Then one token is drawn:
 *   with weights max(p_i - q_i, 0) after a rejection at i (p_i where those are all 0), with p_n if all were accepted; it is the
 *   first index at which the running sum of the weights exceeds final_random[b] times their total.  NaN weighs nothing.
 *   draft_probs NULL: the drafts were certain, q_i is 1 at d_i and 0 elsewhere.  A drafted token outside 0..vocab-1 has
 *   probability 0 on both sides.
 *
 *   target_probs  (batch, drafts + 1, vocab), draft_probs (batch, drafts, vocab) of `dtype`, vocab contiguous, strides in
 *                 elements for the first two.  draft_tokens (batch, drafts) int32, accept_random (batch, drafts) f32,
 *                 final_random (batch) f32, contiguous, random numbers in [0, 1).
 *   accepted      (batch) int32: how many drafted tokens were accepted.
 *   tokens        (batch, drafts + 1) int32: those, the drawn one (-1 where no token has a weight), then -1.
 *   work          atk_verify_workspace_bytes() bytes on 16 bytes.
 */
int64_t atk_verify_workspace_bytes(int64_t batch, int64_t drafts, int64_t vocab);
int atk_verify_drafts(const void *target_probs, const int64_t target_stride[2], const void *draft_probs,
                      const int64_t draft_stride[2], const int32_t *draft_tokens, const float *accept_random,
                      const float *final_random, const int32_t *n_drafts, int64_t batch, int64_t drafts, int64_t vocab, int dtype,
                      int32_t *accepted, int32_t *tokens, void *work, int64_t work_bytes, void *stream);

/*
 * The pages of a cache.  A pool is n_pages pages of page_size tokens, page_size * token_bytes contiguous bytes each; a cache is
 * several pools (keys and values of each layer) under one table:
 *   page_table  rows x row_pages int32: pages of each sequence in order, -1 past them.
 *   lens        rows int32: tokens of each sequence, which hold ceil(len / page_size) pages.
 *   refs        n_pages int32: how many rows hold a page.
 *   free_pages  n_pages int32, a stack of n_free[0] pages: the last is taken first.  Pages given back together are put
 *               with the lowest on top.
 *   work        atk_pages_work_bytes() bytes on 16 bytes, zeroed once and the table's own from then on.
 * All calls on one table are one stream's, or ordered by the caller.  Results do not depend on the order in which workgroups run.
 */
typedef struct {
    int32_t *page_table, *lens, *refs, *free_pages, *n_free, *status;
    void *work;
    int64_t rows, row_pages, n_pages, page_size;
    int64_t work_bytes;
} atk_page_tables;
int64_t atk_pages_work_bytes(int64_t n_pages);

/* Copies whole pages: dst pool p, page dst_ids[i] from src pool p, page src_ids[i], i < n, for n_pools pools (host arrays of
 * device pointers).  Destinations are distinct and no source of the same call.  (16 bytes at a time where page_bytes and all pools are multiples of 16, else 4 or 1.) */
int atk_copy_pages(const void *const *src_pools, void *const *dst_pools, int64_t n_pools, int64_t page_bytes, int64_t src_pages,
                   int64_t dst_pages, const int32_t *src_ids, const int32_t *dst_ids, int64_t n, int32_t *status, void *stream);

/* Makes row children[i], empty before, a copy of row parents[i] as it is at the call (a parent that is a child of the same call is empty):
 * whole pages are shared, a last page that is filled in part is copied (its filled tokens) to a fresh one.  children are distinct.  All or nothing. */
int atk_fork_sequences(const atk_page_tables *t, void *const *pools, int64_t n_pools, int64_t token_bytes, const int32_t *parents,
                       const int32_t *children, int64_t n, void *stream);

/* Adds `tokens` tokens to each of the distinct rows seqs[i]: takes fresh pages, copies a part-filled last page that other rows
 * hold too, and stores values[p] (n, tokens, token_bytes; value_strides[p] bytes between sequences) into pool p.  Rows that all hold
 * one part-filled page at the call each get a copy of it.  All or nothing.  n * (ceil(tokens / page_size) + 1) is below 2^31. */
int atk_append_tokens(const atk_page_tables *t, void *const *pools, const void *const *values, const int64_t *value_strides,
                      int64_t n_pools, int64_t token_bytes, const int32_t *seqs, int64_t n, int64_t tokens, void *stream);

/* Drops the last drop[i] tokens of each of the distinct rows seqs[i] (drop NULL: all of them) and gives back the pages that
 * hold none of the rest.  seqs that are out of range are passed over. */
int atk_free_sequences(const atk_page_tables *t, const int32_t *seqs, const int32_t *drop, int64_t n, void *stream);

/* Moves the held pages to the lowest numbers: with L of them, the i-th held page at or past L goes to the i-th page below L that
 * is not held; table, refs and stack (n_pages-1, ..., L) follow.  remap (n_pages int32): new number of each page, -1 of those
 * that were free. */
int atk_compact_pages(const atk_page_tables *t, void *const *pools, int64_t n_pools, int64_t token_bytes, int32_t *remap, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ATK_DECODE_H */
