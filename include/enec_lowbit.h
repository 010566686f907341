/*
 * libenec, second part -- what a decoding step reads, held in few bits, on AMD MI355X (gfx950): weights and activations in
 * microscaled 4-bit floating point with the products that read them, and a paged 8-bit cache of keys and values with the
 * attention that reads it.  The codec of enec.h brings a layer's weights back bit for bit; this part is for the layers that are
 * kept in 4 bits instead, and for the cache, which has no exact form to return to.
 *
 * Conventions are those of enec.h: plain pointers and sizes, status codes of enec_status, all work enqueued on `stream`, no
 * device memory allocated by the library, a call returns as soon as its work is enqueued, and errors that the host can see return
 * before anything is enqueued.  A workspace here is scratch memory: it needs no initialisation, and nothing is kept in it between
 * calls; calls that share one must not run concurrently.  No call synchronises or makes an allocation, so all of them can be
 * captured into a graph.  Results do not depend on the timing of a run: no atomics, sums in a fixed order.
 *
 * dtype is an enec_dtype, the format of 16- or 32-bit values: bf16 and fp16 everywhere, fp32 where stated.  Strides count
 * elements, and need no alignment beyond an element's own.
 *
 * Forward only: codes are whole numbers, and no call here has a gradient.
 */
#ifndef ENEC_LOWBIT_H
#define ENEC_LOWBIT_H

#include "enec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- Microscaled 4-bit floating point -----------------------------------------------------------------------------------
 * A matrix of rows x cols values is held in blocks of 32 consecutive values of a row.  A block has a scale 2^(byte - 127) and 32
 * E2M1 codes: sign << 3 | index into (0, 0.5, 1, 1.5, 2, 3, 4, 6).  With a = the largest magnitude of the block:
 *   byte = 255 (every value reads back as NaN, codes 0) if the block holds a NaN or an infinity, else
 *   byte = max(0, floor(log2 a) - 2 + 127), 0 for a block of zeros
 *   code = the nearest value to x / 2^(byte - 127), ties to the even index, at most 6
 * Rows are padded with blocks of zeros to a multiple of 128 values:
 *   codes   rows x padded / 2 bytes, the value of even column in the low half of a byte
 *   scales  rows x padded / 32 bytes
 * both without gaps between rows. */
#define ENEC_MX4_BLOCK 32u
#define ENEC_MX4_ROW_GROUP 128u

/* Bytes of a matrix's codes and scales (either pointer may be NULL).  ENEC_E_ARG if cols exceeds 2^31 or rows x padded 2^34. */
int enec_mx4_bytes(size_t rows, size_t cols, size_t *code_bytes, size_t *scale_bytes);

/* Quantise.
 *   in      DEVICE, rows x cols values (bf16, fp16 or fp32), row_stride elements from row to row (>= cols)
 *   codes   DEVICE, 16-byte aligned;  scales  DEVICE, 4-byte aligned; sizes as enec_mx4_bytes says, padding included */
int enec_mx4_quantize(const void *in, size_t rows, size_t cols, size_t row_stride, int dtype, void *codes, void *scales,
                      void *stream);

/* The values that the codes stand for, rounded once to dtype (bf16, fp16 or fp32). */
int enec_mx4_dequantize(const void *codes, const void *scales, size_t rows, size_t cols, void *out, size_t row_stride,
                        int dtype, void *stream);

/* y = x w^T with weights in 4 bits: y[i][j] = sum over c of x[i][c] w[j][c], i < m, j < n, c < k.
 *   x       DEVICE, m x k values (bf16 or fp16), x_stride elements from row to row (>= k)
 *   codes, scales  DEVICE, an n x k matrix as enec_mx4_quantize writes it
 *   y       DEVICE, m x n values of the same dtype, y_stride (>= n); must not overlap the inputs
 *   workspace      DEVICE, 16-byte aligned, or NULL if workspace_bytes = enec_mx4_linear_workspace(m, n, k) is 0.  What it says serves
 *                  every product of fewer rows with the same n and k as well, in either format.
 * Products are exact and summed in 32 bits; y is rounded once.
 * ENEC_E_ARG also beyond m = 2^21, n = 2^26, k = 2^21, m k = 2^34 or m n = 2^40. */
size_t enec_mx4_linear_workspace(size_t m, size_t n, size_t k);
int enec_mx4_linear(const void *x, size_t m, size_t x_stride, int dtype, const void *codes, const void *scales, size_t n, size_t k,
                    void *y, size_t y_stride, void *workspace, size_t workspace_bytes, void *stream);

/* y = x w^T with both in 4 bits: x is an m x k matrix, w an n x k matrix as enec_mx4_quantize writes them; y and the
 * workspace as above, y of any dtype (bf16, fp16 or fp32). */
size_t enec_mx4_matmul_workspace(size_t m, size_t n, size_t k);
int enec_mx4_matmul(const void *x_codes, const void *x_scales, size_t m, const void *codes, const void *scales, size_t n, size_t k,
                    void *y, size_t y_stride, int dtype, void *workspace, size_t workspace_bytes, void *stream);

/* ---- A paged cache of keys and values in 8 bits ---------------------------------------------------------------------------
 * A page holds page_tokens consecutive tokens of one sequence.  For each page and head there are E4M3 codes (the format without
 * infinities, largest value 448) and one scale 2^(byte - 127), for keys and for values:
 *   k_codes   n_pages x kv_heads x page_tokens x head_dim bytes
 *   v_codes   n_pages x kv_heads x head_dim x page_tokens bytes   (a head's values, transposed: a product over tokens reads runs)
 *   k_scales, v_scales  n_pages x kv_heads bytes
 * n_pages is at least 1, page_tokens a power of two from 16 to 256, head_dim 64, 128 or 256.  Which pages a sequence owns says
 *   table     DEVICE, int32, batch rows of table_stride entries: entry i is the page of tokens i page_tokens ...
 * A batch of sequences is described by
 *   starts    DEVICE, int32, batch + 1 entries, ascending from 0 to n_tokens: where the sequence's tokens begin among those the
 *             call takes or returns, which are the newest of their sequence
 *   lengths   DEVICE, int32, batch entries: tokens of the sequence, those of the call among them
 * batch and kv_heads are at most 65535 and n_tokens below 2^24.
 * Token i of a sequence's t tokens in the call has position lengths[b] - t + i.  A negative position (an idle slot of a batch,
 * with length 0) belongs to no page: such a token is not stored, reads back as zeros, and its attention is zeros.
 * What only the device can see is checked there.  A sequence whose two starts are out of order or beyond the call's tokens, or whose length exceeds
 * table_stride * page_tokens or 2^30 (attention: or max_length, or whose tokens in the call exceed max_new), is left out: nothing of
 * it is stored or returned.  The tokens of a page whose number lies outside the cache are not stored, read back as zeros and are not
 * seen.  In both cases ENEC_E_ARG is stored to
 *   status    NULL, or a DEVICE-ACCESSIBLE word that the caller has set to 0
 */
typedef struct {
    void *k_codes, *k_scales, *v_codes, *v_scales;       /* DEVICE; codes 16-byte aligned */
    uint32_t n_pages, page_tokens, kv_heads, head_dim;
} enec_cache;

typedef struct {
    const int32_t *table, *starts, *lengths;             /* DEVICE */
    uint32_t table_stride, batch, n_tokens;              /* n_tokens = starts[batch] */
    uint32_t *status;                                    /* DEVICE-ACCESSIBLE, or NULL */
} enec_cache_batch;

/* Quantise new tokens into their pages.
 *   k, v    DEVICE, n_tokens x kv_heads x head_dim values (bf16 or fp16), token_stride and head_stride elements apart
 * For each page and head that receives tokens, with a = the largest finite magnitude among them: the smallest e >= -127 with
 * a <= 448 2^e; a page that already holds earlier tokens of its sequence keeps at least its scale, and where the scale grows its
 * earlier codes are divided by as much (exact, but for codes that reach E4M3's subnormal range: to nearest, ties to even).
 * code = nearest of x / 2^e, ties to even; an infinity takes the largest code, a NaN stays one.  Codes behind the sequence's end are
 * not written.  A page that is written must belong to one sequence of the batch only. */
int enec_cache_write(const enec_cache *cache, const enec_cache_batch *batch, const void *k, size_t k_token_stride, size_t k_head_stride,
                     const void *v, size_t v_token_stride, size_t v_head_stride, int dtype, void *stream);

/* The values that the newest tokens' codes stand for, rounded once to dtype (bf16, fp16 or fp32); layout as for enec_cache_write.  starts
 * of whole lengths read everything. */
int enec_cache_read(const enec_cache *cache, const enec_cache_batch *batch, void *k, size_t k_token_stride, size_t k_head_stride,
                    void *v, size_t v_token_stride, size_t v_head_stride, int dtype, void *stream);

/* Attention of the newest tokens over the cache (which holds their own keys and values already):
 *   out[i][h] = sum over j <= p of softmax_j(scale q[i][h] . k[j][h']) v[j][h'],   h' = h div (q_heads / kv_heads)
 * for token i at position p; zeros if p < 0.
 *   q, out  DEVICE, n_tokens x q_heads x head_dim values (bf16 or fp16), token and head strides; must not overlap
 *   q_heads a multiple of kv_heads
 *   max_new, max_length  HOST: no sequence has more tokens in the call, or more in all (they shape the launch)
 *           ENEC_E_ARG from max_new (q_heads / kv_heads) = 2^21 or batch kv_heads = 2^23 on
 *   scale   above zero and at most 2^127, usually head_dim^-1/2
 *   workspace  DEVICE, 16-byte aligned, or NULL if workspace_bytes = enec_cache_attention_workspace(...) is 0.  What it says serves every
 *           call with no more sequences, tokens, max_new and max_length as well (n_tokens at most batch max_new, as in any call that leaves
 *           no sequence out); it is 35 MB at most then.
 * Scores, softmax and sums are held in 32 bits (queries from 2^110 on may leave their range: a score's sum is one over codes, which
 * takes the page's scale last); for the product with v the probabilities are rounded to the sum of two bf16 numbers (16
 * significant bits). */
size_t enec_cache_attention_workspace(const enec_cache *cache, uint32_t batch, uint32_t n_tokens, uint32_t q_heads, uint32_t max_new,
                                      uint32_t max_length);
int enec_cache_attention(const enec_cache *cache, const enec_cache_batch *batch, const void *q, size_t q_token_stride,
                         size_t q_head_stride, void *out, size_t out_token_stride, size_t out_head_stride, int dtype, uint32_t q_heads,
                         uint32_t max_new, uint32_t max_length, float scale, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ENEC_LOWBIT_H */
