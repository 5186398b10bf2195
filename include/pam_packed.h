/*
 * pam_packed.h -- C ABI of softmax attention over packed sequences and of
 * serving an attention layer from a paged cache, in the MI355X (gfx950)
 * permutohedral-lattice filter library (libpam_lattice.so).  They stand next
 * to pam_attn.h, whose differential attention takes padded batches:
 *
 *   attention            out = softmax(scale q k^T) v over sequences of
 *                        different lengths that lie behind each other, with
 *                        its gradients
 *   head norms, rotary   the norm of every head of the queries and keys and
 *                        the rotation of pam_rotary, in one pass
 *   a paged cache        keys and values of many sequences in pages of one
 *                        pool, as they are or in 8 bits with a scale per row
 *   attention of new     over that cache, with one softmax map or
 *   tokens               differential
 *
 * Conventions as in pam_attn.h: device pointers owned by the caller, work
 * enqueued and not waited for, argument errors found on the host before
 * anything is enqueued, nothing allocated and no state kept between calls;
 * sums, softmax statistics and norms in fp32.  What lies on the device
 * (starts, lengths, page tables) is clamped or checked by the kernels, as each
 * call says: no content of it makes a kernel leave an array.
 */
#ifndef PAM_PACKED_H
#define PAM_PACKED_H

#include "pam_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ */
/* Attention over packed sequences                                    */

/*
 * Sequence b has the queries q_start[b] .. q_start[b + 1] - 1 of `tokens` and
 * the keys k_start[b] .. k_start[b + 1] - 1 of `keys` (n_q, n_k of them).  For
 * head h (keys and values of key head h / (heads / kv_heads)):
 *   out_i = sum_j p_ij v_j,  p_i = softmax over the keys that i sees of
 *   scale <q_i, k_j>;
 * query i of a sequence sees its key j if, with PAM_ATTN_CAUSAL,
 * j <= i + n_k - n_q (the last query sees every key), without it always.  A
 * query that sees nothing has output and gradients 0; rows of no sequence
 * (before q_start[0], from q_start[sequences] on; of k likewise) have output
 * and gradients 0 and are part of nothing, whatever they hold.  Keys and
 * values that the causal rule hides from a query must be finite.
 *   q   : element (t, h, x) at q + t q_stride[0] + h q_stride[1] + x, strides
 *         in elements; k and v likewise (key heads).  Any strides; rows whose
 *         start and strides are multiples of 16 bytes are read wide.
 *   out : tokens x heads x dim_v, contiguous.
 *   q_start, k_start : sequences + 1 ascending int32 on the device; with one
 *         sequence NULL: all rows.  They are clamped to [0, tokens] and
 *         [0, keys], and a sequence that would end before it starts is empty;
 *         where they do not ascend, out's rows are not specified.
 * Limits: 1 <= dim, dim_v <= PAM_ATTN_MAX_DIM, kv_heads divides heads,
 * sequences >= 1, tokens and keys less than 2^30 (0 allowed), tokens heads and
 * keys kv_heads less than 2^31, scale positive and finite.
 */
typedef struct {
    int32_t dtype; /* pam_dtype_t */
    int32_t sequences, heads, kv_heads;
    int32_t dim, dim_v;
    uint32_t flags; /* PAM_ATTN_CAUSAL */
    float scale;
    int64_t tokens, keys;
    int64_t q_stride[2], k_stride[2], v_stride[2]; /* token, head */
} pam_attn_desc_t;

/* Bytes of device workspace, by the descriptor alone (0: none); SIZE_MAX on
 * invalid arguments. */
size_t pam_attn_fwd_workspace(const pam_attn_desc_t *desc);
size_t pam_attn_bwd_workspace(const pam_attn_desc_t *desc);

/*
 * Forward.  For a backward pass give saved_o (tokens x heads x dim_v fp32: out
 * before it is rounded) and saved_lse (heads x tokens fp32: the logarithms of
 * the softmax sums); both NULL otherwise; their rows of no sequence are left as
 * they are.  workspace: 16-byte aligned, overwritten (NULL if 0 bytes).
 * Outputs must not overlap inputs.  Asynchronous.
 */
pam_status_t pam_attn_fwd(const pam_attn_desc_t *desc, const void *q, const void *k, const void *v,
                          const int32_t *q_start, const int32_t *k_start, void *out, float *saved_o, float *saved_lse,
                          void *workspace, void *stream);

/*
 * Backward, with D_i = <grad_out_i, o_i>, dp = grad_out v^T, ds = scale p (dp - D):
 *   grad_q = ds k, grad_k = sum over the key head's heads of ds^T q,
 *   grad_v = sum p^T grad_out.
 *   grad_out : tokens x heads x dim_v with strides do_stride (token, head);
 *         grad_q, grad_k, grad_v contiguous, of type dtype, written in full.
 * Other arguments as the forward call's, which saved_o and saved_lse are from.
 * Sums run in a fixed order (the results of two calls are equal).  With 16 bits
 * the matrix units take p and ds rounded to dtype, but for grad_q of dim and
 * dim_v up to 64 ds with what its rounding left: that is off by little more than
 * its own rounding, the others by about 1.4 times as much.  Asynchronous.
 */
pam_status_t pam_attn_bwd(const pam_attn_desc_t *desc, const void *q, const void *k, const void *v,
                          const int32_t *q_start, const int32_t *k_start, const float *saved_o, const float *saved_lse,
                          const void *grad_out, const int64_t do_stride[2], void *grad_q, void *grad_k, void *grad_v,
                          void *workspace, void *stream);

/* ------------------------------------------------------------------ */
/* Norms of the heads of queries and keys, with rotary positions      */

#define PAM_HEAD_NORM_MAX_DIM 512

/*
 * For every head x (dim channels) of q and of k, n = x / sqrt(mean x^2 + eps)
 * (PAM_NORM_RMS) or the same of x - mean x (PAM_NORM_LAYER), y = n w, and the
 * first 2 pairs channels of y turned as pam_rotary does, by the token's entry
 * of the table (pos, start, entries and PAM_ROTARY_INTERLEAVED as there; a
 * token whose entry is not in [0, entries) gets NaN in its turned channels).
 *   w_q, w_k : dim fp32 each for all heads, or heads (kv_heads) x dim with
 *           w_per_head; NULL: 1.
 *   q_out, k_out : contiguous; they may be q and k themselves if those are
 *           contiguous, and overlap nothing else.
 * Other arguments and limits as pam_rotary's, with 1 <= dim <=
 * PAM_HEAD_NORM_MAX_DIM, batch length (heads + kv_heads) less than 2^31, eps
 * finite and not negative.  Asynchronous.
 */
typedef struct {
    int32_t dtype;
    int32_t norm; /* pam_norm_t */
    int32_t batch, length, heads, kv_heads, dim, pairs;
    uint32_t flags; /* PAM_ROTARY_INTERLEAVED */
    int32_t w_per_head;
    float eps;
    int64_t start, entries;
    int64_t q_stride[3], k_stride[3];
} pam_head_norm_desc_t;

pam_status_t pam_head_norm_rotary_fwd(const pam_head_norm_desc_t *desc, const void *q, const void *k, const float *w_q,
                                      const float *w_k, const float *table, const int32_t *pos, void *q_out,
                                      void *k_out, void *stream);

/* Bytes of device workspace for the backward call; SIZE_MAX on invalid
 * arguments. */
size_t pam_head_norm_rotary_bwd_workspace(const pam_head_norm_desc_t *desc);

/*
 * Backward from grad_q_out and grad_k_out (contiguous, the outputs' shapes), with
 * dy = the gradient turned back and dn = dy w:
 *   grad_x = (dn - n mean(dn n)) / sqrt(mean x^2 + eps)   (layer: less mean dn),
 *   grad_w = sum dy n over the tokens (and, without w_per_head, the heads).
 * grad_q, grad_k (contiguous, dtype) are written in full and may be grad_q_out
 * and grad_k_out; grad_w_q and grad_w_k (the weights' shapes, fp32; summed in a
 * fixed order) may be NULL.  workspace 16-byte aligned.  Asynchronous.
 */
pam_status_t pam_head_norm_rotary_bwd(const pam_head_norm_desc_t *desc, const void *q, const void *k, const float *w_q,
                                      const float *w_k, const float *table, const int32_t *pos,
                                      const void *grad_q_out, const void *grad_k_out, void *grad_q, void *grad_k,
                                      float *grad_w_q, float *grad_w_k, void *workspace, void *stream);

/* ------------------------------------------------------------------ */
/* A paged cache of keys and values                                   */

/* how rows are stored: as pam_dtype_t says, or in 8 bits with a scale per row */
typedef enum {
    PAM_STORE_F32 = PAM_F32,
    PAM_STORE_F16 = PAM_F16,
    PAM_STORE_BF16 = PAM_BF16,
    PAM_STORE_E4M3 = 3, /* sign, 4 bits of exponent, 3 of mantissa; largest 448 */
    PAM_STORE_INT8 = 4  /* -127 .. 127 */
} pam_store_t;

#define PAM_CACHE_MAX_ROW 256 /* channels of a row of keys (maps dim) and of values */

/*
 * A pool of `pages` pages of page_size tokens:
 *   k_pages : pages x kv_heads x page_size x maps x dim, of the stored type,
 *   v_pages : pages x kv_heads x page_size x dim_v,
 *   k_scale : pages x kv_heads x page_size x maps fp32, v_scale without the
 *             last axis; NULL for types that have none.
 * All contiguous and 16-byte aligned (scales: 4).  maps is 2 for the keys of
 * differential attention, else 1.  A sequence's token at position p is token
 * p mod page_size of page table[b, p / page_size]; table is sequences x
 * table_width int32 on the device.  A page number that is not in [0, pages)
 * names no page: its tokens are not written, read as 0 and seen by no query.
 *   k_len : sequences int32 on the device: tokens of each sequence, the new ones
 *           included; clamped to [0, table_width page_size] by what reads the
 *           cache.  Positions of tokens that are written count from it as it is.
 * Stored rows of 8 bits: scale = max(largest magnitude / top, 2^-126) with top
 * 448 or 127, number = x / scale, clamped to [-top, top], rounded to nearest,
 * ties to even; quotients in fp32.  A row of keys is its dim channels of one map.  The
 * value is number scale.  A row that holds an infinity or NaN is stored with
 * the scale NaN, and its values are NaN.
 * Limits: 1 <= maps <= 2, maps dim and dim_v in [1, PAM_CACHE_MAX_ROW], pages
 * kv_heads page_size less than 2^31, table_width page_size less than 2^30.
 */
typedef struct {
    int32_t dtype; /* of what is written and read: pam_dtype_t */
    int32_t store; /* pam_store_t: dtype itself, or one of 8 bits */
    int32_t pages, page_size, kv_heads, dim, dim_v, maps;
    int32_t sequences, table_width;
} pam_cache_desc_t;

/*
 * Writes new tokens: sequence b has the last n_b of its k_len[b] tokens in the
 * rows (b, 0) .. (b, n_b - 1) of k and v, n_b = new_len[b] (device int32,
 * clamped to [0, length]; NULL: length), or, with starts (sequences + 1
 * ascending int32 on the device, clamped to [0, rows]), in rows starts[b] ..
 * starts[b + 1] - 1 of `rows`.  Tokens at positions less than 0 or past the table are
 * not written.  Two new tokens must not have the same place.
 *   k : element (b, i, head, map, x) at strides k_stride (sequence, token, head,
 *       map) and v without the map axis; with starts the sequence axis is not
 *       there, its stride not looked at.
 * Without starts `rows` is not looked at, with them `length` is not.  (rows + 16)
 * kv_heads maps less than 2^31 (rows: sequences length).  Asynchronous.
 */
typedef struct {
    int64_t rows;
    int32_t length;
    int64_t k_stride[4], v_stride[3];
} pam_cache_rows_t;

pam_status_t pam_cache_write(const pam_cache_desc_t *desc, const pam_cache_rows_t *rows, const void *k, const void *v,
                             const int32_t *starts, const int32_t *new_len, const int32_t *table, const int32_t *k_len,
                             void *k_pages, void *v_pages, float *k_scale, float *v_scale, void *stream);

/*
 * Reads the first `length` positions of every sequence back: k is sequences x
 * length x kv_heads x maps x dim, v sequences x length x kv_heads x dim_v,
 * contiguous, of type dtype; 0 from k_len[b] on.  Values of 8 bits are the
 * fp32 products of number and scale, rounded to dtype.  k or v may be NULL: not
 * asked for.  (sequences length + 16) kv_heads maps less than 2^31.  Asynchronous.
 */
pam_status_t pam_cache_read(const pam_cache_desc_t *desc, int32_t length, const int32_t *table, const int32_t *k_len,
                            const void *k_pages, const void *v_pages, const float *k_scale, const float *v_scale,
                            void *k, void *v, void *stream);

/*
 * Attention of new tokens: query i of the n_q = q_len[b] (device int32, clamped
 * to [0, len_q]; NULL: len_q) of sequence b sees the keys j <= i + k_len[b] - n_q
 * of its sequence (the new tokens' own are in the cache already).
 *   maps 1: out = softmax(scale q k^T) v; lambda NULL.
 *   maps 2: pam_diff_attn_fwd's out = o^0 - lambda[h] o^1; lambda: heads values
 *           of type dtype.
 * Rows from n_q on, and rows that see nothing, are 0.  Cached rows that the causal
 * rule alone hides from a query must be finite.
 *   q   : element (b, i, h, m, x) at strides q_stride (sequence, token, head,
 *         map); out: sequences x len_q x heads x dim_v, contiguous.
 *   key_bound : a length that most sequences reach at the most, 0 for that of
 *         the table.  It decides how finely the keys are split, for speed alone.
 * With dtype of 16 bits and numbers of 8, a product of a probability and a value's
 * scale is rounded to 11 bits or to 2^-31 of the largest scale that a new token of
 * the sequence sees, whichever is more.  Every 32 rows of a key head (its heads,
 * tokens and maps) read the sequence's keys again: for one token or a few.
 * kv_heads divides heads; sequences heads len_q maps at most 2^30, len_q less than 2^20; scale
 * positive and finite.  The workspace is 16-byte aligned; by the descriptors.
 */
typedef struct {
    int32_t heads, len_q;
    int32_t key_bound;
    float scale;
    int64_t q_stride[4];
} pam_paged_attn_desc_t;

size_t pam_paged_attn_workspace(const pam_cache_desc_t *cache, const pam_paged_attn_desc_t *desc);

pam_status_t pam_paged_attn(const pam_cache_desc_t *cache, const pam_paged_attn_desc_t *desc, const void *q,
                            const void *lambda, const int32_t *q_len, const int32_t *table, const int32_t *k_len,
                            const void *k_pages, const void *v_pages, const float *k_scale, const float *v_scale,
                            void *out, void *workspace, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PAM_PACKED_H */
