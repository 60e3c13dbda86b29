/*
 * atk_quant.h - C ABI of a cache in few bits beside that of atk_decode.h: tokens are quantised as they are appended, read
 * back, and attended to.  Conventions, status bits and page tables are atk_decode.h's.
 *
 * A pool has page_size rows to a page, one for a token, so that atk_fork_sequences, atk_compact_pages and atk_copy_pages move
 * it as it is (token_bytes: atk_quant_token_bytes()).  With `bits` 4 an element is an e2m1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), with 8
 * an e4m3 code (up to 448; 0x7f is no number); 32 elements of a head are a block with one power of two for a unit:
 *   codes      head after head, element after element; 4 bits: the even element in a byte's low half.
 *   exponents  behind all codes, head after head, a byte for each block: its unit is 2^(byte - 127), 255: its elements are NaN.
 *   padding    to whole 16 bytes, neither written nor read.
 * A block's unit is 2^max(floor(log2 a) - top, -117) of its largest magnitude a, top 2 for 4 bits and 8 for 8; an element is x / unit
 * rounded to the nearest code, ties to the even one, at most the largest.  (Scaling by a power of two is exact, so nothing else is rounded.)  A block with a NaN or an
 * infinity has the exponent 255 and codes of 0.
 */
#ifndef ATK_QUANT_H
#define ATK_QUANT_H

#include "atk_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of a token's row; negative: kv_heads below 1, dim no multiple of 32 or outside 32..256, kv_heads * dim past 2^20 (ATK_ERR_ARGS), bits neither 4 nor 8
 * (ATK_ERR_UNSUPPORTED).  The functions below refuse the same. */
int64_t atk_quant_token_bytes(int64_t kv_heads, int64_t dim, int bits);

/* atk_append_tokens of values (n, tokens, kv_heads, dim) of `dtype` that are quantised as they are stored.  value_strides: for each pool the bytes from a sequence's values
 * to the next one's and from a token's to the next one's (heads and dim are contiguous), addresses and strides (but a single one's) of whole 16 bytes. */
int atk_append_quantized(const atk_page_tables *t, void *const *pools, const void *const *values, const int64_t *value_strides,
                         int64_t n_pools, int64_t kv_heads, int64_t dim, int bits, int dtype, const int32_t *seqs, int64_t n,
                         int64_t tokens, void *stream);

/* outs[p] (n, tokens, kv_heads, dim) of `dtype`, contiguous, on 16 bytes: tokens starts[i], starts[i] + 1, ... (NULL: 0, 1, ...) of row seqs[i] out of pool p, rounded to the
 * nearest.  Places before the first and behind the last token of the row, and those of pages that are none, are 0.  A row may be read more than once; the tables are only read. */
int atk_read_quantized(const atk_page_tables *t, const void *const *pools, void *const *outs, int64_t n_pools, int64_t kv_heads,
                       int64_t dim, int bits, int dtype, const int32_t *seqs, const int32_t *starts, int64_t n, int64_t tokens,
                       void *stream);

/*
 * Attention of `tokens` new tokens of each of `batch` sequences over such pools k and v.
 *   Which keys a query sees, what it gets from none, and what status reports are as for atk_shared_prefix_attention, with all keys the sequence's own.  Keys and values are
 *   those that atk_read_quantized gives in `dtype`.  (In f32 a unit that is never written, of 2^120 and more for e4m3 or 2^126 for e2m1, may give NaN in place of an infinity.)
 *   q, out     (batch, tokens, heads, dim) of `dtype`, dim contiguous, strides in elements for the first three (whole 16 bytes but for a single one's).
 *   k, v       n_pages * page_size rows of atk_quant_token_bytes() bytes, on 16 bytes; fewer than 2^36 bytes each.
 *   heads      a multiple of kv_heads; query head h reads head h / (heads / kv_heads).
 *   lse        (batch, tokens, heads) f32, contiguous, or NULL.
 *   work       atk_quant_attention_workspace_bytes() bytes on 16 bytes.
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
    int64_t q_stride[3], out_stride[3];    /* sequence, token, head */
    double scale;                          /* FLT_MIN to 1e30 */
    int32_t dtype, bits;
} atk_quant_attention_args;
int64_t atk_quant_attention_workspace_bytes(const atk_quant_attention_args *args);
int atk_quant_attention(const atk_quant_attention_args *args, void *work, int64_t work_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ATK_QUANT_H */
