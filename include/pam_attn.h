/*
 * pam_attn.h -- C ABI of the operators around an exact attention layer, in
 * the MI355X (gfx950) permutohedral-lattice filter library
 * (libpam_lattice.so).  A network that filters its fine feature maps through
 * the lattice (pam_lattice.h) can afford exact softmax attention on its
 * coarse ones; these are the parts of such a residual block:
 *
 *   differential attention   out = (P1 - lambda P2) v, two softmax maps per
 *                            head over shared values, the second subtracted
 *                            with a learned weight
 *   rotary positions         of its queries and keys
 *   norm, gate, residual     the norms before and after the block, with its
 *                            gate, residual scale and dropout
 *   dropout                  from a counter-based generator, with no mask
 *
 * Conventions as in pam_lattice.h: device pointers owned by the caller,
 * streams as void*, work enqueued and not waited for, argument errors found
 * on the host before anything is enqueued, a text in pam_last_error().  The
 * lengths, masks and positions that live on the device are clamped or
 * checked by the kernels, as each call says.  Nothing here allocates device
 * memory or keeps state between calls, so every call may be captured in a
 * graph.  Activations are fp32, fp16 or bf16 (pam_dtype_t); every sum, softmax
 * statistic and norm is held in fp32.
 */
#ifndef PAM_ATTN_H
#define PAM_ATTN_H

#include "pam_lattice.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PAM_F32 = 0, PAM_F16 = 1, PAM_BF16 = 2 } pam_dtype_t;

/* ------------------------------------------------------------------ */
/* Differential attention                                             */

/* flags */
#define PAM_ATTN_CAUSAL 1u

#define PAM_ATTN_MAX_DIM 128

/*
 * For sequence b, head h (its keys and values are those of key head
 * h / (heads / kv_heads)), query i and map m in {0, 1}:
 *   s_ij^m = scale <q_i^m, k_j^m>,   p^m = softmax of s_i^m over the keys j
 *   that query i sees,   o_i^m = sum_j p_ij^m v_j,
 *   out_i = o_i^0 - lambda[h] o_i^1.
 * Query i (of q_len[b]) sees key j (of k_len[b]) if key_mask[b, j] is not 0
 * and, with PAM_ATTN_CAUSAL, j <= i + k_len[b] - q_len[b] (the last query
 * sees every key).  A query that sees nothing, and every row from q_len[b]
 * on, has output and gradients 0.  Keys and values from k_len[b] on or
 * hidden by key_mask are never part of a result, whatever they hold; those
 * hidden by the causal rule alone must be finite.  Their gradients are 0.
 *   q   : element (b, i, h, m, x) at q + b q_stride[0] + i q_stride[1]
 *         + h q_stride[2] + m q_stride[3] + x, strides in elements; k
 *         likewise (key heads); v without the map axis.  Any strides; rows
 *         whose start and strides are multiples of 16 bytes are read wide.
 *   out : batch x len_q x heads x dim_v, contiguous; all types as dtype.
 *   lambda : heads values of type dtype.
 *   q_len, k_len : batch int32 on the device, clamped to [0, len]; NULL: all
 *         of len_q, len_k.
 *   key_mask : batch x len_k bytes on the device, NULL: every key is seen.
 * Limits: 1 <= dim <= PAM_ATTN_MAX_DIM, 1 <= dim_v <= 2 PAM_ATTN_MAX_DIM,
 * kv_heads divides heads; batch, len_q and len_k may be 0 and are less than
 * 2^30; batch heads len_q and batch kv_heads len_k less than 2^31; scale
 * positive.
 */
typedef struct {
    int32_t dtype; /* pam_dtype_t */
    int32_t batch, heads, kv_heads;
    int32_t dim, dim_v;
    int32_t len_q, len_k;
    uint32_t flags;
    float scale;
    int64_t q_stride[4]; /* sequence, token, head, map */
    int64_t k_stride[4];
    int64_t v_stride[3]; /* sequence, token, head */
} pam_diff_attn_desc_t;

/* Bytes of device workspace for pam_diff_attn_fwd and pam_diff_attn_bwd, by the
 * descriptor alone; SIZE_MAX on invalid arguments.  Always to be asked for:
 * where the queries do not fill the card in whole rounds, prompts and training
 * among them, the keys are split into parts that meet there (0 elsewhere). */
size_t pam_diff_attn_fwd_workspace(const pam_diff_attn_desc_t *desc);
size_t pam_diff_attn_bwd_workspace(const pam_diff_attn_desc_t *desc);

/*
 * Forward.  For a backward pass give saved_o (2 x batch x len_q x heads x
 * dim_v fp32: o^0, then o^1) and saved_lse (2 x batch x heads x len_q fp32:
 * the logarithms of the softmax sums); both NULL otherwise.  workspace: 16-byte
 * aligned, pam_diff_attn_fwd_workspace bytes, overwritten (NULL if 0).
 * Outputs must not overlap inputs.  Asynchronous.
 */
pam_status_t pam_diff_attn_fwd(const pam_diff_attn_desc_t *desc, const void *q, const void *k, const void *v,
                               const void *lambda, const int32_t *q_len, const int32_t *k_len,
                               const uint8_t *key_mask, void *out, float *saved_o, float *saved_lse, void *workspace,
                               void *stream);

/*
 * Backward, with D^m = <grad_out, o^m>, dp = grad_out v^T:
 *   ds^0 = scale p^0 (dp - D^0),  ds^1 = -lambda scale p^1 (dp - D^1),
 *   grad_q^m = ds^m k^m,  grad_k^m = sum over the key head's heads of
 *   ds^m^T q^m,  grad_v = sum (p^0 - lambda p^1)^T grad_out,
 *   grad_lambda = -sum p^1 dp.
 *   grad_out : batch x len_q x heads x dim_v with strides do_stride
 *         (sequence, token, head), grad_q, grad_k, grad_v contiguous in the
 *         order of q, k and v, grad_lambda heads values; all of type dtype and
 *         written in full.  Rows of grad_out from q_len[b] on are not part of
 *         any result.
 * Other arguments as the forward call's, which saved_o and saved_lse are
 * from.  Sums run in a fixed order (the results of two calls are equal).
 * Asynchronous.
 */
pam_status_t pam_diff_attn_bwd(const pam_diff_attn_desc_t *desc, const void *q, const void *k, const void *v,
                               const void *lambda, const int32_t *q_len, const int32_t *k_len,
                               const uint8_t *key_mask, const float *saved_o, const float *saved_lse,
                               const void *grad_out, const int64_t do_stride[3], void *grad_q, void *grad_k,
                               void *grad_v, void *grad_lambda, void *workspace, void *stream);

/* ------------------------------------------------------------------ */
/* Rotary positions                                                   */

/* how angles are scaled for contexts longer than the trained one */
typedef enum {
    PAM_ROPE_PLAIN = 0,
    PAM_ROPE_LINEAR = 1, /* positions divided by factor */
    PAM_ROPE_NTK = 2,    /* base times factor^(rot / (rot - 2)): the slowest pair is stretched by factor, the
                            fastest not at all */
    PAM_ROPE_YARN = 3    /* by parts (Peng et al. 2023, YaRN): pairs of fewer than beta_slow turns over
                            original_len stretched by factor, of more than beta_fast not at all, a ramp between
                            them; cosines and sines times 0.1 ln(factor) + 1 */
} pam_rope_scaling_t;

/*
 * Host function: the rot / 2 angles per unit of position, base^(-2 i / rot)
 * scaled as asked, to freq (host, rot / 2 doubles), and what cosines and
 * sines are multiplied by to *magnitude (host).  rot even, 2 <= rot <= 512;
 * base > 1; factor >= 1; for PAM_ROPE_NTK rot > 2; for PAM_ROPE_YARN
 * original_len > 0 and 0 < beta_slow < beta_fast.
 */
pam_status_t pam_rotary_frequencies(int32_t rot, double base, int32_t scaling, double factor, double original_len,
                                    double beta_slow, double beta_fast, double *freq, double *magnitude);

/*
 * Table of cosines and sines: for entry t < entries and pair i < pairs
 *   angle = freq[i] coord[t, axis[i]],  table[t, i] = magnitude (cos, sin)
 * with the product and its reduction in 64 bits.
 *   freq  : pairs doubles (device).
 *   coord : entries x axes fp32 positions (device), or NULL: the entry's
 *           number (axes 1).
 *   axis  : pairs int32 (device) in [0, axes) (others count as 0), or NULL: 0.
 *           A voxel's x, y and z take three axes, each with its share of the
 *           pairs.
 *   table : entries x pairs x 2 fp32 (device).
 * 1 <= pairs <= 256, 1 <= axes <= 16, entries pairs < 2^31.  Asynchronous.
 */
pam_status_t pam_rotary_table(const double *freq, const float *coord, const int32_t *axis, int64_t entries,
                              int32_t pairs, int32_t axes, double magnitude, float *table, void *stream);

#define PAM_ROTARY_INTERLEAVED 1u /* pairs (2 i, 2 i + 1); else (i, rot / 2 + i) */
#define PAM_ROTARY_INVERSE 2u     /* by the negative angle: the gradient of the rotation (with a magnitude 1 also
                                     its inverse) */

/*
 * Rotates the first 2 pairs channels of every head of q and, in the same
 * launch, of k:  (a, b) -> (a c - b s, a s + b c); the others are copied.
 * Token (b, l) takes entry pos[b, l] of the table (device int32), or start + l
 * if pos is NULL; a token whose entry is not in [0, entries) gets NaN in its
 * rotated channels.
 *   q     : batch x length x heads x dim at strides q_stride (sequence,
 *           token, head; elements), k likewise with kv_heads (NULL with
 *           kv_heads = 0: none).
 *   q_out, k_out : contiguous; they may be q and k themselves if those are
 *           contiguous, and must not overlap otherwise, nor with table or
 *           pos.
 * 1 <= dim <= 1024, 1 <= pairs <= dim / 2, batch length (heads + kv_heads)
 * dim < 2^40.  Asynchronous.
 */
typedef struct {
    int32_t dtype;
    int32_t batch, length, heads, kv_heads, dim, pairs;
    uint32_t flags;
    int64_t start, entries;
    int64_t q_stride[3], k_stride[3];
} pam_rotary_desc_t;

pam_status_t pam_rotary(const pam_rotary_desc_t *desc, const void *q, const void *k, const float *table,
                        const int32_t *pos, void *q_out, void *k_out, void *stream);

/* ------------------------------------------------------------------ */
/* Dropout                                                            */

/*
 * y_e = x_e * (u_e >= T ? 65536 / (65536 - T) : 0) for the n elements of x,
 * T = rint(65536 p), u_e a 16-bit number: elements 8 j .. 8 j + 7 take the low
 * and high halves of the four 32-bit words, in order, that Philox4x32-10
 * (Salmon et al. 2011) makes of the counter (j mod 2^32, j / 2^32, offset mod
 * 2^32, offset / 2^32) and the key (seed mod 2^32, seed / 2^32).  The mask
 * depends on nothing else, so the gradient is the same call on the upstream
 * gradient.  A dropped element is 0 whatever x holds.  y may be x.
 * 0 <= p <= 1 (p = 1: all are dropped).  Asynchronous.
 */
pam_status_t pam_dropout(const void *x, int64_t n, int32_t dtype, double p, uint64_t seed, uint64_t offset, void *y,
                         void *stream);

/* ------------------------------------------------------------------ */
/* Norms before and after a block, gate, residual scale, dropout      */

typedef enum { PAM_NORM_RMS = 0, PAM_NORM_LAYER = 1 } pam_norm_t;

#define PAM_NORM_MAX_CHANNELS 8192

/*
 * For a block's output z and the residual stream x, row by row,
 *   r = x + drop(scale * gate * (N(z) w_post + b_post)),
 *   h = N(r) w_pre + b_pre          (the next block's input),
 * N(t) = t / sqrt(mean t^2 + eps) (PAM_NORM_RMS) or the same of t - mean t
 * (PAM_NORM_LAYER), drop as pam_dropout's over the row-major elements.  h is
 * taken from r before r is rounded to dtype.
 *   x, z  : rows x channels at row strides x_stride, z_stride (elements);
 *           r, h contiguous.  z NULL: no block, r = x (pass r NULL).  h NULL:
 *           no norm after.
 *   gate  : rows / gate_rows rows of channels values of type dtype,
 *           contiguous; row i takes gate row i / gate_rows (gate_rows divides
 *           rows).  NULL: 1.
 *   w_post, b_post, scale, w_pre, b_pre : channels fp32 each, NULL: 1 or 0.
 * 1 <= channels <= PAM_NORM_MAX_CHANNELS, rows channels < 2^40.  r may be x
 * or z if those are contiguous; outputs overlap nothing else.  Asynchronous.
 */
typedef struct {
    int32_t dtype;
    int32_t norm; /* pam_norm_t */
    int64_t rows;
    int32_t channels;
    float eps;
    int64_t gate_rows;
    int64_t x_stride, z_stride;
    double p; /* dropout: 0 = none */
    uint64_t seed, offset;
} pam_norm_desc_t;

pam_status_t pam_norm_gate_fwd(const pam_norm_desc_t *desc, const void *x, const void *z, const float *w_post,
                               const float *b_post, const void *gate, const float *scale, const float *w_pre,
                               const float *b_pre, void *r, void *h, void *stream);

/* Bytes of device workspace for pam_norm_gate_bwd; SIZE_MAX on invalid
 * arguments. */
size_t pam_norm_gate_bwd_workspace(const pam_norm_desc_t *desc);

/*
 * Backward from grad_r (NULL: 0) and grad_h (NULL: there was no h), both
 * contiguous.  r is formed again from x and z, so its rounding enters no
 * gradient.  Outputs, each written in full, NULL to skip: grad_x, grad_z
 * (contiguous), grad_gate (gate's shape), dtype; grad_w_post, grad_b_post,
 * grad_scale, grad_w_pre, grad_b_pre, channels fp32 each, summed over the rows
 * in a fixed order.  Gradients of what the call has not (z, gate, h NULL) must
 * be NULL.  grad_x may be grad_r; outputs overlap nothing else.
 * Asynchronous.
 */
pam_status_t pam_norm_gate_bwd(const pam_norm_desc_t *desc, const void *x, const void *z, const float *w_post,
                               const float *b_post, const void *gate, const float *scale, const float *w_pre,
                               const void *grad_r, const void *grad_h, void *grad_x, void *grad_z, float *grad_w_post,
                               float *grad_b_post, void *grad_gate, float *grad_scale, float *grad_w_pre,
                               float *grad_b_pre, void *workspace, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PAM_ATTN_H */
