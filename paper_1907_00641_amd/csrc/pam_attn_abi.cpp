// C ABI of the operators around the attention layer (include/pam_attn.h):
// argument checks; the kernels live in pam_attn_kernels.h, pam_rotary.hip and
// pam_norm.hip.
#include "pam_checks.h"

using namespace pam;

namespace {

pam_status_t check_attn(const pam_diff_attn_desc_t *d)
{
    REQUIRE(d, "desc is NULL");
    REQUIRE(known_type(d->dtype), "dtype must be PAM_F32, PAM_F16 or PAM_BF16");
    REQUIRE(d->batch >= 0 && d->len_q >= 0 && d->len_k >= 0, "batch, len_q and len_k must not be negative");
    REQUIRE(d->heads >= 1 && d->kv_heads >= 1 && d->heads % d->kv_heads == 0, "kv_heads must divide heads");
    REQUIRE(d->dim >= 1 && d->dim <= PAM_ATTN_MAX_DIM, "dim must be in [1, 128]");
    REQUIRE(d->dim_v >= 1 && d->dim_v <= 2 * PAM_ATTN_MAX_DIM, "dim_v must be in [1, 256]");
    REQUIRE((d->flags & ~PAM_ATTN_CAUSAL) == 0, "unknown flag");
    REQUIRE(d->scale > 0.0f && d->scale < INFINITY, "scale must be positive and finite");
    const int64_t most = ((int64_t)1 << 31) - 1;
    REQUIRE((__int128)d->batch * d->heads * d->len_q <= most, "batch heads len_q must be less than 2^31");
    REQUIRE((__int128)d->batch * d->kv_heads * d->len_k <= most, "batch kv_heads len_k must be less than 2^31");
    // sums of two lengths and a tile are formed in 32 bits
    REQUIRE(d->len_q < 1 << 30 && d->len_k < 1 << 30, "len_q and len_k must be less than 2^30");
    return PAM_OK;
}

constexpr int kAttnInputs = 7;
pam_status_t attn_spans(const pam_diff_attn_desc_t *d, const void *q, const void *k, const void *v, const void *lambda,
                        const int32_t *q_len, const int32_t *k_len, const uint8_t *key_mask, Span in[kAttnInputs])
{
    in[3] = bytes_at(lambda, d->heads * bytes_of(d->dtype));
    in[4] = bytes_at(q_len, d->batch * (int64_t)sizeof(int32_t));
    in[5] = bytes_at(k_len, d->batch * (int64_t)sizeof(int32_t));
    in[6] = bytes_at(key_mask, (int64_t)d->batch * d->len_k);
    const int64_t ql[4] = {d->batch, d->len_q, d->heads, 2}, kl[4] = {d->batch, d->len_k, d->kv_heads, 2};
    REQUIRE(span_of(q, d->dtype, ql, d->q_stride, 4, d->dim, &in[0]) &&
                span_of(k, d->dtype, kl, d->k_stride, 4, d->dim, &in[1]) &&
                span_of(v, d->dtype, kl, d->v_stride, 3, d->dim_v, &in[2]),
            "strides reach too far");
    return PAM_OK;
}

pam_status_t check_norm(const pam_norm_desc_t *d)
{
    REQUIRE(d, "desc is NULL");
    REQUIRE(known_type(d->dtype), "dtype must be PAM_F32, PAM_F16 or PAM_BF16");
    REQUIRE(d->norm == PAM_NORM_RMS || d->norm == PAM_NORM_LAYER, "norm must be PAM_NORM_RMS or PAM_NORM_LAYER");
    REQUIRE(d->channels >= 1 && d->channels <= PAM_NORM_MAX_CHANNELS, "channels must be in [1, 8192]");
    REQUIRE(d->rows >= 0 && d->rows < ((int64_t)1 << 40) / d->channels, "rows channels must be less than 2^40");
    REQUIRE(d->eps >= 0.0f && d->eps < INFINITY, "eps must be finite and not negative");
    REQUIRE(d->p >= 0.0 && d->p <= 1.0, "p must be in [0, 1]");
    return PAM_OK;
}

// z's stride means nothing without z
pam_norm_desc_t without_z(pam_norm_desc_t d, const void *z)
{
    if (!z)
        d.z_stride = d.x_stride;
    return d;
}

}  // namespace

extern "C" {

size_t pam_diff_attn_fwd_workspace(const pam_diff_attn_desc_t *desc)
{
    return check_attn(desc) == PAM_OK ? attn_fwd_workspace(*desc) : SIZE_MAX;
}

size_t pam_diff_attn_bwd_workspace(const pam_diff_attn_desc_t *desc)
{
    return check_attn(desc) == PAM_OK ? attn_bwd_workspace(*desc) : SIZE_MAX;
}

pam_status_t pam_diff_attn_fwd(const pam_diff_attn_desc_t *desc, const void *q, const void *k, const void *v,
                               const void *lambda, const int32_t *q_len, const int32_t *k_len,
                               const uint8_t *key_mask, void *out, float *saved_o, float *saved_lse, void *workspace,
                               void *stream)
{
    pam_status_t st = check_attn(desc);
    if (st != PAM_OK)
        return st;
    const int64_t rows = (int64_t)desc->batch * desc->heads * desc->len_q;
    const int64_t keys = (int64_t)desc->batch * desc->len_k;
    if (rows == 0)
        return PAM_OK;
    REQUIRE(q && lambda && out && (keys == 0 || (k && v)), "a pointer is NULL");
    REQUIRE(!saved_o == !saved_lse, "saved_o and saved_lse must be given together");
    const size_t ws = attn_fwd_workspace(*desc);
    REQUIRE(ws == 0 || (workspace && (uintptr_t)workspace % 16 == 0), "workspace is NULL or not 16-byte aligned");
    Span in[kAttnInputs];
    if ((st = attn_spans(desc, q, k, v, lambda, q_len, k_len, key_mask, in)) != PAM_OK)
        return st;
    const int64_t ob = rows * desc->dim_v * bytes_of(desc->dtype);
    const Span outs[4] = {bytes_at(out, ob), bytes_at(saved_o, rows * desc->dim_v * 8), bytes_at(saved_lse, rows * 8),
                          bytes_at(workspace, (int64_t)ws)};
    for (int i = 0; i < 4; ++i) {
        for (const Span &x : in)
            REQUIRE(!meet(outs[i], x), "an output overlaps an input");
        for (int j = 0; j < i; ++j)
            REQUIRE(!meet(outs[i], outs[j]), "outputs overlap");
    }
    LAUNCH(launch_attn_fwd(*desc, q, k, v, lambda, q_len, k_len, key_mask, out, saved_o, saved_lse, workspace,
                           (hipStream_t)stream),
           "differential attention forward");
    return PAM_OK;
}

pam_status_t pam_diff_attn_bwd(const pam_diff_attn_desc_t *desc, const void *q, const void *k, const void *v,
                               const void *lambda, const int32_t *q_len, const int32_t *k_len,
                               const uint8_t *key_mask, const float *saved_o, const float *saved_lse,
                               const void *grad_out, const int64_t do_stride[3], void *grad_q, void *grad_k,
                               void *grad_v, void *grad_lambda, void *workspace, void *stream)
{
    pam_status_t st = check_attn(desc);
    if (st != PAM_OK)
        return st;
    const int64_t rows = (int64_t)desc->batch * desc->heads * desc->len_q;
    const int64_t keys = (int64_t)desc->batch * desc->kv_heads * desc->len_k;
    REQUIRE(lambda && grad_lambda, "a pointer is NULL");
    REQUIRE(rows == 0 || (q && saved_o && saved_lse && grad_out && do_stride && grad_q), "a pointer is NULL");
    REQUIRE(keys == 0 || (k && v && grad_k && grad_v), "a pointer is NULL");
    const size_t ws = attn_bwd_workspace(*desc);
    REQUIRE(ws == 0 || (workspace && (uintptr_t)workspace % 16 == 0), "workspace is NULL or not 16-byte aligned");
    const int64_t e = bytes_of(desc->dtype);
    Span in[kAttnInputs + 3] = {};
    if ((st = attn_spans(desc, q, k, v, lambda, q_len, k_len, key_mask, in)) != PAM_OK)
        return st;
    if (rows) {
        const int64_t ol[3] = {desc->batch, desc->len_q, desc->heads};
        REQUIRE(span_of(grad_out, desc->dtype, ol, do_stride, 3, desc->dim_v, &in[kAttnInputs]),
                "strides reach too far");
        in[kAttnInputs + 1] = bytes_at(saved_o, rows * desc->dim_v * 8);
        in[kAttnInputs + 2] = bytes_at(saved_lse, rows * 8);
    }
    const Span outs[5] = {bytes_at(grad_q, rows * 2 * desc->dim * e), bytes_at(grad_k, keys * 2 * desc->dim * e),
                          bytes_at(grad_v, keys * desc->dim_v * e), bytes_at(grad_lambda, desc->heads * e),
                          bytes_at(workspace, (int64_t)ws)};
    for (int i = 0; i < 5; ++i) {
        for (const Span &x : in)
            REQUIRE(!meet(outs[i], x), "an output overlaps an input");
        for (int j = 0; j < i; ++j)
            REQUIRE(!meet(outs[i], outs[j]), "outputs overlap");
    }
    const int64_t none[3] = {0, 0, 0};
    LAUNCH(launch_attn_bwd(*desc, q, k, v, lambda, q_len, k_len, key_mask, saved_o, saved_lse, grad_out,
                           do_stride ? do_stride : none, grad_q, grad_k, grad_v, grad_lambda, workspace,
                           (hipStream_t)stream),
           "differential attention backward");
    return PAM_OK;
}

pam_status_t pam_rotary_frequencies(int32_t rot, double base, int32_t scaling, double factor, double original_len,
                                    double beta_slow, double beta_fast, double *freq, double *magnitude)
{
    REQUIRE(freq && magnitude, "a pointer is NULL");
    REQUIRE(rot >= 2 && rot <= 512 && rot % 2 == 0, "rot must be even and in [2, 512]");
    REQUIRE(base > 1.0 && base < INFINITY, "base must be finite and more than 1");
    REQUIRE(scaling >= PAM_ROPE_PLAIN && scaling <= PAM_ROPE_YARN, "unknown scaling");
    REQUIRE(scaling == PAM_ROPE_PLAIN || (factor >= 1.0 && factor < INFINITY), "factor must be finite and at least 1");
    REQUIRE(scaling != PAM_ROPE_NTK || rot > 2, "rot must be more than 2");
    REQUIRE(scaling != PAM_ROPE_YARN ||
                (original_len > 0.0 && original_len < INFINITY && beta_slow > 0.0 && beta_fast > beta_slow &&
                 beta_fast < INFINITY),
            "original_len must be positive and 0 < beta_slow < beta_fast");
    if (scaling == PAM_ROPE_NTK)
        base *= pow(factor, (double)rot / (rot - 2));
    *magnitude = scaling == PAM_ROPE_YARN ? 0.1 * log(factor) + 1.0 : 1.0;
    for (int32_t i = 0; i < rot / 2; ++i) {
        const double f = pow(base, -2.0 * i / rot);
        if (scaling == PAM_ROPE_LINEAR) {
            freq[i] = f / factor;
        } else if (scaling == PAM_ROPE_YARN) {
            const double turns = original_len * f / (2.0 * M_PI);
            double kept = (turns - beta_slow) / (beta_fast - beta_slow);
            kept = kept < 0.0 ? 0.0 : (kept > 1.0 ? 1.0 : kept);
            freq[i] = (1.0 - kept) * f / factor + kept * f;
        } else {
            freq[i] = f;
        }
    }
    return PAM_OK;
}

pam_status_t pam_rotary_table(const double *freq, const float *coord, const int32_t *axis, int64_t entries,
                              int32_t pairs, int32_t axes, double magnitude, float *table, void *stream)
{
    REQUIRE(pairs >= 1 && pairs <= 256, "pairs must be in [1, 256]");
    REQUIRE(axes >= 1 && axes <= 16 && (coord || axes == 1), "axes must be in [1, 16], and 1 without coordinates");
    REQUIRE(entries >= 0 && entries < ((int64_t)1 << 31) / pairs, "entries pairs must be less than 2^31");
    REQUIRE(isfinite(magnitude), "magnitude must be finite");
    if (entries == 0)
        return PAM_OK;
    REQUIRE(freq && table, "a pointer is NULL");
    REQUIRE((uintptr_t)freq % 8 == 0 && (uintptr_t)table % 8 == 0, "freq and table must be 8-byte aligned");
    REQUIRE(!meet_any(bytes_at(table, entries * pairs * 8),
                      {bytes_at(freq, 8ll * pairs), bytes_at(coord, entries * axes * 4), bytes_at(axis, 4ll * pairs)}),
            "table overlaps an input");
    LAUNCH(launch_rotary_table(freq, coord, axis, entries, pairs, axes, magnitude, table, (hipStream_t)stream),
           "rotary table");
    return PAM_OK;
}

pam_status_t pam_rotary(const pam_rotary_desc_t *desc, const void *q, const void *k, const float *table,
                        const int32_t *pos, void *q_out, void *k_out, void *stream)
{
    REQUIRE(desc, "desc is NULL");
    const pam_rotary_desc_t &d = *desc;
    REQUIRE(known_type(d.dtype), "dtype must be PAM_F32, PAM_F16 or PAM_BF16");
    REQUIRE(d.batch >= 0 && d.length >= 0, "batch and length must not be negative");
    REQUIRE(d.heads >= 1 && d.kv_heads >= 0 && d.heads < (1 << 20) && d.kv_heads < (1 << 20),
            "heads must be positive, kv_heads not negative, both less than 2^20");
    REQUIRE(d.dim >= 1 && d.dim <= 1024, "dim must be in [1, 1024]");
    REQUIRE(d.pairs >= 1 && d.pairs <= d.dim / 2, "pairs must be in [1, dim / 2]");
    REQUIRE((d.flags & ~(PAM_ROTARY_INTERLEAVED | PAM_ROTARY_INVERSE)) == 0, "unknown flag");
    REQUIRE((__int128)d.batch * d.length * (d.heads + d.kv_heads) * d.dim < ((__int128)1 << 40),
            "batch length (heads + kv_heads) dim must be less than 2^40");
    REQUIRE(d.entries >= 0 && d.start > -((int64_t)1 << 62) && d.start < ((int64_t)1 << 62),
            "entries must not be negative, start less than 2^62 in size");
    if (d.batch == 0 || d.length == 0)
        return PAM_OK;
    REQUIRE(d.entries >= 1, "the table is empty");
    REQUIRE(q && q_out && table && (d.kv_heads == 0 || (k && k_out)), "a pointer is NULL");
    REQUIRE((uintptr_t)table % 8 == 0, "table must be 8-byte aligned");
    if (d.kv_heads == 0)
        k = k_out = nullptr;
    const int64_t ql[3] = {d.batch, d.length, d.heads}, kl[3] = {d.batch, d.length, d.kv_heads};
    Span in[2];
    REQUIRE(span_of(q, d.dtype, ql, d.q_stride, 3, d.dim, &in[0]) &&
                span_of(k, d.dtype, kl, d.k_stride, 3, d.dim, &in[1]),
            "strides reach too far");
    const int64_t tok = (int64_t)d.batch * d.length * d.dim * bytes_of(d.dtype);
    const Span outs[2] = {bytes_at(q_out, tok * d.heads), bytes_at(k_out, tok * d.kv_heads)};
    auto contiguous = [&](const int64_t s[3], int64_t h) {
        return (d.batch == 1 || s[0] == d.length * h * d.dim) && (d.length == 1 || s[1] == h * d.dim) &&
               (h == 1 || s[2] == d.dim);
    };
    REQUIRE(!meet(outs[0], in[0]) || (q == q_out && contiguous(d.q_stride, d.heads)), "q_out overlaps q");
    REQUIRE(!meet(outs[1], in[1]) || (k == k_out && contiguous(d.k_stride, d.kv_heads)), "k_out overlaps k");
    REQUIRE(!meet(outs[0], in[1]) && !meet(outs[1], in[0]) && !meet(outs[0], outs[1]), "outputs overlap");
    // a table of which no entry past 2^40 is reached counts as that long
    const Span st = bytes_at(table, std::min(d.entries, (int64_t)1 << 40) * d.pairs * 8),
               sp = bytes_at(pos, (int64_t)d.batch * d.length * 4);
    REQUIRE(!meet_any(outs[0], {st, sp}) && !meet_any(outs[1], {st, sp}), "an output overlaps the table or pos");
    LAUNCH(launch_rotary(d, q, k, table, pos, q_out, k_out, (hipStream_t)stream), "rotary positions");
    return PAM_OK;
}

pam_status_t pam_dropout(const void *x, int64_t n, int32_t dtype, double p, uint64_t seed, uint64_t offset, void *y,
                         void *stream)
{
    REQUIRE(known_type(dtype), "dtype must be PAM_F32, PAM_F16 or PAM_BF16");
    REQUIRE(n >= 0 && n < (int64_t)1 << 40, "n must be in [0, 2^40)");
    REQUIRE(p >= 0.0 && p <= 1.0, "p must be in [0, 1]");
    if (n == 0)
        return PAM_OK;
    REQUIRE(x && y, "a pointer is NULL");
    const int64_t b = n * bytes_of(dtype);
    REQUIRE(x == y || !meet(bytes_at(x, b), bytes_at(y, b)), "y overlaps x");
    LAUNCH(launch_dropout(x, n, dtype, p, seed, offset, y, (hipStream_t)stream), "dropout");
    return PAM_OK;
}

pam_status_t pam_norm_gate_fwd(const pam_norm_desc_t *desc, const void *x, const void *z, const float *w_post,
                               const float *b_post, const void *gate, const float *scale, const float *w_pre,
                               const float *b_pre, void *r, void *h, void *stream)
{
    pam_status_t st = check_norm(desc);
    if (st != PAM_OK)
        return st;
    const pam_norm_desc_t d = without_z(*desc, z);
    if (d.rows == 0)
        return PAM_OK;
    REQUIRE(!gate || (d.gate_rows >= 1 && d.rows % d.gate_rows == 0), "gate_rows must divide rows");
    REQUIRE(z || (!gate && !scale && !w_post && !b_post), "gate, scale, w_post and b_post need z");
    REQUIRE(!z == !r, "r goes with z");
    REQUIRE(h || (!w_pre && !b_pre), "w_pre and b_pre need h");
    REQUIRE(r || h, "there is no output");
    REQUIRE(x, "x is NULL");
    const int64_t len[1] = {d.rows}, out = d.rows * d.channels * bytes_of(d.dtype);
    Span sx, sz;
    REQUIRE(span_of(x, d.dtype, len, &d.x_stride, 1, d.channels, &sx) &&
                span_of(z, d.dtype, len, &d.z_stride, 1, z ? d.channels : 0, &sz),
            "strides reach too far");
    if (!z)
        sz = bytes_at(nullptr, 0);
    const Span sr = bytes_at(r, out), shh = bytes_at(h, out);
    const bool dense_x = d.x_stride == d.channels || d.rows == 1, dense_z = d.z_stride == d.channels || d.rows == 1;
    REQUIRE(!meet(sr, sx) || (r == x && dense_x), "r overlaps x");
    REQUIRE(!meet(sr, sz) || (r == z && dense_z), "r overlaps z");
    REQUIRE(!meet(shh, sx) && !meet(shh, sz) && !meet(shh, sr), "h overlaps another array");
    const int64_t vec = 4ll * d.channels;
    const std::initializer_list<Span> rest = {
        bytes_at(gate, gate ? d.rows / d.gate_rows * d.channels * bytes_of(d.dtype) : 0), bytes_at(w_post, vec),
        bytes_at(b_post, vec), bytes_at(scale, vec), bytes_at(w_pre, vec), bytes_at(b_pre, vec)};
    REQUIRE(!meet_any(sr, rest) && !meet_any(shh, rest), "an output overlaps the gate or a vector");
    LAUNCH(launch_norm_fwd(d, x, z, w_post, b_post, gate, scale, w_pre, b_pre, r, h, (hipStream_t)stream),
           "norm and gate forward");
    return PAM_OK;
}

size_t pam_norm_gate_bwd_workspace(const pam_norm_desc_t *desc)
{
    if (check_norm(desc) != PAM_OK)
        return SIZE_MAX;
    if (desc->gate_rows < 0 || (desc->gate_rows > 0 && desc->rows % desc->gate_rows)) {
        abi_fail(PAM_ERR_INVALID_ARGUMENT, "gate_rows must divide rows");
        return SIZE_MAX;
    }
    return norm_bwd_workspace(*desc);
}

pam_status_t pam_norm_gate_bwd(const pam_norm_desc_t *desc, const void *x, const void *z, const float *w_post,
                               const float *b_post, const void *gate, const float *scale, const float *w_pre,
                               const void *grad_r, const void *grad_h, void *grad_x, void *grad_z, float *grad_w_post,
                               float *grad_b_post, void *grad_gate, float *grad_scale, float *grad_w_pre,
                               float *grad_b_pre, void *workspace, void *stream)
{
    pam_status_t st = check_norm(desc);
    if (st != PAM_OK)
        return st;
    const pam_norm_desc_t d = without_z(*desc, z);
    REQUIRE(!gate || (d.gate_rows >= 1 && d.rows % d.gate_rows == 0), "gate_rows must divide rows");
    REQUIRE(d.gate_rows >= 0 && (d.gate_rows == 0 || d.rows % d.gate_rows == 0), "gate_rows must divide rows");
    // arrays of no rows may be NULL, and the vectors' gradients are 0 then
    const bool none = d.rows == 0;
    REQUIRE(none || z || (!gate && !scale && !w_post && !b_post), "gate, scale, w_post and b_post need z");
    REQUIRE(none || z || (!grad_z && !grad_w_post && !grad_b_post && !grad_scale), "a gradient of z's norm without z");
    REQUIRE(none || gate || !grad_gate, "grad_gate without a gate");
    REQUIRE(none || grad_h || (!w_pre && !grad_w_pre && !grad_b_pre), "w_pre or a gradient of h's norm without grad_h");
    REQUIRE(none || x, "x is NULL");
    REQUIRE(workspace && (uintptr_t)workspace % 16 == 0, "workspace is NULL or not 16-byte aligned");
    const int64_t len[1] = {d.rows}, dense = d.rows * d.channels * bytes_of(d.dtype), vec = 4ll * d.channels;
    Span in[9];
    REQUIRE(span_of(x, d.dtype, len, &d.x_stride, 1, d.channels, &in[0]) &&
                span_of(z, d.dtype, len, &d.z_stride, 1, z ? d.channels : 0, &in[1]),
            "strides reach too far");
    if (!z)
        in[1] = bytes_at(nullptr, 0);
    in[2] = bytes_at(grad_r, dense);
    in[3] = bytes_at(grad_h, dense);
    const int64_t gb = gate ? d.rows / d.gate_rows * d.channels * bytes_of(d.dtype) : 0;
    in[4] = bytes_at(gate, gb);
    in[5] = bytes_at(w_post, vec);
    in[6] = bytes_at(b_post, vec);
    in[7] = bytes_at(scale, vec);
    in[8] = bytes_at(w_pre, vec);
    const Span outs[9] = {bytes_at(grad_x, dense),     bytes_at(grad_z, dense),      bytes_at(grad_gate, gb),
                          bytes_at(grad_w_post, vec),  bytes_at(grad_b_post, vec),   bytes_at(grad_scale, vec),
                          bytes_at(grad_w_pre, vec),   bytes_at(grad_b_pre, vec),
                          bytes_at(workspace, (int64_t)norm_bwd_workspace(d))};
    for (int i = 0; i < 9; ++i) {
        for (int j = 0; j < 9; ++j)
            REQUIRE(!meet(outs[i], in[j]) || (i == 0 && j == 2 && grad_x == grad_r), "an output overlaps an input");
        for (int j = 0; j < i; ++j)
            REQUIRE(!meet(outs[i], outs[j]), "outputs overlap");
    }
    LAUNCH(launch_norm_bwd(d, x, z, w_post, b_post, gate, scale, w_pre, grad_r, grad_h, grad_x, grad_z, grad_w_post,
                           grad_b_post, grad_gate, grad_scale, grad_w_pre, grad_b_pre, workspace,
                           (hipStream_t)stream),
           "norm and gate backward");
    return PAM_OK;
}

}  // extern "C"
