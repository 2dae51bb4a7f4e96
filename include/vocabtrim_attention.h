/*
 * vocabtrim_attention.h -- the attention of a drafter's layer, the step ahead of
 * the trimmed head: norms of queries and keys with the position rotation (and
 * their gradients), a paged key-value cache in 16 or 8 bits, and the attention
 * of a draft step's new tokens over it.
 *
 * The general conventions of vocabtrim.h hold: device pointers of the caller's,
 * nothing allocated, kept or synchronised, work enqueued on `stream`, errors
 * that the host can see returned with nothing enqueued.
 *
 * Tensors of heads.  q, k, v and the like are [n, heads, head_dim] with the last
 * two dimensions contiguous and rows `*_stride` ELEMENTS apart (the views q, k, v
 * of one projection's output rows, say).  Strides are multiples of 8 and at
 * least heads * head_dim, pointers are 16-byte aligned.  An output may be its
 * input (same pointer, same stride); other overlaps are not allowed.
 */
#ifndef VOCABTRIM_ATTENTION_H_
#define VOCABTRIM_ATTENTION_H_

#include "vocabtrim.h"

#ifdef __cplusplus
extern "C" {
#endif

#define VT_MAX_HEAD_DIM 256
#define VT_MAX_ATTENTION_HEADS 1024
#define VT_MAX_REQUESTS 65535

/* ------------------------------------------------------------------------
 * Norm and rotation.  For every head x in R^head_dim of q (and k likewise):
 *
 *   z = x * (mean(x^2) + eps)^(-1/2) * q_weight          (z = x without weights)
 *   every pair (a, b) of the first rotary_dim values of z, at the row's angle:
 *       (a * cos - b * sin,  b * cos + a * sin)
 *
 * computed in fp32 and rounded once.  Pair i is (z[i], z[i + rotary_dim / 2])
 * for VT_ROPE_HALVES and (z[2 i], z[2 i + 1]) for VT_ROPE_NEIGHBOURS.
 *
 *   type          VT_BF16 or VT_F32: of q, k, the weights and the outputs
 *   n             rows (tokens), >= 0
 *   q_heads       >= 0, k_heads >= 0, together 1 .. VT_MAX_ATTENTION_HEADS
 *   head_dim      a multiple of 8, <= VT_MAX_HEAD_DIM
 *   q_weight, k_weight  [head_dim], both or neither (neither: no norm)
 *   eps           > 0 with weights
 *   table         [table_rows, rotary_dim] fp32: cosines of a position's angles in
 *                 the first half of its row, sines in the second; NULL: no rotation
 *   rotary_dim    a multiple of 8, 8 .. head_dim
 *   positions     [n] int32 or int64 (pos_type): row of the table for every row.  A
 *                 position outside the table has no angle: the rotated values of
 *                 that row are NaN.
 * ---------------------------------------------------------------------- */
typedef enum { VT_ROPE_HALVES = 0, VT_ROPE_NEIGHBOURS = 1 } vt_rope_style;

int vt_qk_norm_rope(const void *q, int64_t q_stride, const void *k, int64_t k_stride, int type, int64_t n,
                    int32_t q_heads, int32_t k_heads, int32_t head_dim, const void *q_weight, const void *k_weight,
                    float eps, const float *table, int64_t table_rows, int32_t rotary_dim, int style,
                    const void *positions, int pos_type, void *q_out, int64_t q_out_stride, void *k_out,
                    int64_t k_out_stride, void *stream);

/* Its gradients.  q, k, weights, table and positions as given to the forward
 * call; gq and gk are the gradients of its outputs.
 *   dq, dk   gradients of q and k, in their type; may be gq and gk
 *   dqw, dkw [head_dim] fp32, gradients of the weights: sums over all rows and
 *            heads, in an order that depends on the sizes alone; with weights only
 *   ws       >= vt_qk_norm_rope_backward_ws_bytes(n, head_dim) bytes, with weights only
 * n == 0 gives weight gradients of zero. */
int vt_qk_norm_rope_backward(const void *gq, int64_t gq_stride, const void *gk, int64_t gk_stride, const void *q,
                             int64_t q_stride, const void *k, int64_t k_stride, int type, int64_t n, int32_t q_heads,
                             int32_t k_heads, int32_t head_dim, const void *q_weight, const void *k_weight, float eps,
                             const float *table, int64_t table_rows, int32_t rotary_dim, int style,
                             const void *positions, int pos_type, void *dq, int64_t dq_stride, void *dk,
                             int64_t dk_stride, float *dqw, float *dkw, void *ws, size_t ws_bytes, void *stream);
size_t vt_qk_norm_rope_backward_ws_bytes(int64_t n, int32_t head_dim);

/* ------------------------------------------------------------------------
 * A paged key-value cache: caller's memory, described by this struct (HOST).
 *
 *   k, v              [pages, heads, page_size, head_dim] of type VT_BF16 or VT_E4M3
 *   k_scale, v_scale  [pages, heads, page_size] exponents of the scales, VT_E4M3
 *                     only (else NULL): code c stands for c * 2^(scale - 127).  (255 has
 *                     no place in fp32 but for the least codes: what reads or sees such
 *                     a token may get infinities and NaN.)
 *   page_size         a power of two, 16 .. 65536
 *   head_dim          a multiple of 16, <= VT_MAX_HEAD_DIM
 *
 * A head's tokens of a page are one stretch of memory.  A SLOT is
 * page * page_size + place.  An e4m3 row has the smallest scale 2^e, e >= -126,
 * with max |x| <= 448 * 2^e over its finite values; a value is then rounded to
 * nearest even, at most +-448 * 2^e (240 * 2^120, the scale of the largest fp32
 * values: no held value is infinite), infinities to those; NaN is held as NaN.  A power of two
 * makes the scaling exact and every held value exact in bf16.
 * ---------------------------------------------------------------------- */
typedef struct {
    void *k, *v;
    uint8_t *k_scale, *v_scale;
    int32_t type;
    int64_t pages;
    int32_t heads, page_size, head_dim;
} vt_kv_cache;

/* vt_qk_norm_rope on q and k, with k and v written into the cache in the same
 * launch (k rounded once, from fp32 to what the cache holds).
 *   q        NULL with q_heads == 0 writes the cache only
 *   k, v     [n, cache->heads, cache->head_dim]
 *   slots    [n] int32 or int64 (slot_type): where each row's k and v go.  A slot
 *            outside the cache (-1, say) leaves its row out.  A slot that
 *            occurs twice holds no more than a mixture of its rows. */
int vt_qkv_to_cache(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                    int type, int64_t n, int32_t q_heads, const void *q_weight, const void *k_weight, float eps,
                    const float *table, int64_t table_rows, int32_t rotary_dim, int style, const void *positions,
                    int pos_type, void *q_out, int64_t q_out_stride, const vt_kv_cache *cache, const void *slots,
                    int slot_type, void *stream);

/* Rows of the cache back as values: k_out, v_out [n, heads, head_dim] contiguous,
 * VT_BF16 or VT_F32 (exact in both, down to their smallest normal values).  A slot
 * outside the cache gives zeros. */
int vt_kv_cache_read(const vt_kv_cache *cache, const void *slots, int slot_type, int64_t n, void *k_out, void *v_out,
                     int out_type, void *stream);

/* ------------------------------------------------------------------------
 * Attention of a draft step's new tokens over the cache.  Request b has
 * lengths[b] cached tokens; token t of it is in page page_table[b, t / page_size]
 * at place t % page_size.  Row i of request b, head h, kv head g = h / (q_heads / heads):
 *
 *   s[t] = scale * sum_d q[i, h, d] * k[t, g, d]    over the tokens t that row i sees
 *   out[i, h, :] = sum_t exp(s[t] - lse) * v[t, g, :],   lse[i, h] = log sum_t exp(s[t])
 *
 * in fp32 (a weight times an 8-bit row's scale counts as less, or not at all, below
 * 2^-126).  A row that sees nothing (or whose scores are all -inf) has out = 0 and
 * lse = -inf.  What a row does not see does not reach it, NaN, infinities and any scale
 * included.
 *
 *   q, out       [n, q_heads, head_dim], type VT_BF16 or VT_F32; n <= n_requests * max_rows
 *   page_table   [n_requests, table_pages] int32; entries past a request's tokens are
 *                not used.  Tokens of a page outside [0, cache->pages) are not seen.
 *   lengths      [n_requests] int32, n_requests <= VT_MAX_REQUESTS; below 0 counts as 0, above
 *                min(max_length, table_pages * page_size) as that
 *   row_start    [n_requests + 1] int32: rows row_start[b] .. row_start[b + 1] - 1 are
 *                request b's, at most max_rows of them (more, and rows of no
 *                request, are not computed: their out and lse stay as they are);
 *                NULL: row i is the one row of request i, n == n_requests, max_rows == 1
 *   tail_mask    [n] uint64, nullable: bit j says whether the row sees token
 *                lengths[b] - 64 + j; tokens before those are seen by all rows
 *   max_length   0 .. 2^30
 *   scale        of the scores, finite
 *   out_lse      [n, q_heads] fp32, nullable
 *   ws           >= vt_paged_attention_ws_bytes(...) bytes, no initialisation; may be
 *                NULL where that is 0.  One for the largest batch serves smaller ones.
 * n_requests, max_rows and max_length decide how the work is cut up (many requests of
 * few tokens are taken whole, a workgroup each, others in even shares of their
 * lengths): near the largest that occur is fastest.  Only kernels are enqueued: the call may be captured in a graph.
 * ---------------------------------------------------------------------- */
int vt_paged_attention(const void *q, int64_t q_stride, int type, int64_t n, int32_t q_heads, const vt_kv_cache *cache,
                       const int32_t *page_table, int32_t table_pages, const int32_t *lengths, int32_t n_requests,
                       const int32_t *row_start, int32_t max_rows, const uint64_t *tail_mask, int64_t max_length,
                       float scale, void *out, int64_t out_stride, float *out_lse, void *ws, size_t ws_bytes,
                       void *stream);
/* Enough for every call of up to these sizes (kv_heads and head_dim as they are); 0 also for arguments out of range. */
size_t vt_paged_attention_ws_bytes(int64_t n, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t n_requests,
                                   int32_t max_rows, int64_t max_length);

#ifdef __cplusplus
}
#endif
#endif /* VOCABTRIM_ATTENTION_H_ */
