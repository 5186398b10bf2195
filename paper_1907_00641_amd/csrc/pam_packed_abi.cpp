// C ABI of attention over packed sequences and from a paged cache
// (include/pam_packed.h): argument checks; the kernels live in
// pam_packed_kernels.h, pam_head_norm.hip, pam_cache.hip and pam_paged_kernels.h.
#include "pam_checks.h"

using namespace pam;

namespace {

constexpr int64_t kMost31 = ((int64_t)1 << 31) - 1;

// whether an output meets an input or another output
pam_status_t apart(const Span *outs, int n, const Span *ins, int m)
{
    for (int i = 0; i < n; ++i) {
        for (int j = 0; j < m; ++j)
            REQUIRE(!meet(outs[i], ins[j]), "an output overlaps an input");
        for (int j = 0; j < i; ++j)
            REQUIRE(!meet(outs[i], outs[j]), "outputs overlap");
    }
    return PAM_OK;
}

#define CHECK(call)                                                                               \
    do {                                                                                          \
        const pam_status_t st_ = (call);                                                          \
        if (st_ != PAM_OK)                                                                        \
            return st_;                                                                           \
    } while (0)

pam_status_t check_packed(const pam_attn_desc_t *d)
{
    REQUIRE(d, "desc is NULL");
    REQUIRE(known_type(d->dtype), "dtype must be PAM_F32, PAM_F16 or PAM_BF16");
    REQUIRE(d->sequences >= 1 && d->sequences < 1 << 24, "sequences must be in [1, 2^24)");
    REQUIRE(d->heads >= 1 && d->kv_heads >= 1 && d->heads % d->kv_heads == 0, "kv_heads must divide heads");
    REQUIRE(d->dim >= 1 && d->dim <= PAM_ATTN_MAX_DIM, "dim must be in [1, 128]");
    REQUIRE(d->dim_v >= 1 && d->dim_v <= PAM_ATTN_MAX_DIM, "dim_v must be in [1, 128]");
    REQUIRE((d->flags & ~PAM_ATTN_CAUSAL) == 0, "unknown flag");
    REQUIRE(d->scale > 0.0f && d->scale < INFINITY, "scale must be positive and finite");
    REQUIRE(d->tokens >= 0 && d->tokens < 1 << 30 && d->keys >= 0 && d->keys < 1 << 30,
            "tokens and keys must be in [0, 2^30)");
    REQUIRE(d->tokens * d->heads <= kMost31 && d->keys * d->kv_heads <= kMost31,
            "tokens heads and keys kv_heads must be less than 2^31");
    // a tile of every sequence and head is a number of 32 bits
    REQUIRE((d->tokens / 128 + d->sequences) * d->heads <= (int64_t)1 << 27 &&
                (d->keys / 128 + d->sequences) * d->kv_heads <= (int64_t)1 << 27,
            "sequences heads must be less than 2^26");
    return PAM_OK;
}

constexpr int kPackedInputs = 5;
pam_status_t packed_spans(const pam_attn_desc_t *d, const void *q, const void *k, const void *v, const int32_t *q_start,
                          const int32_t *k_start, Span in[kPackedInputs])
{
    REQUIRE((q_start && k_start) || d->sequences == 1, "q_start and k_start go with more than one sequence");
    const int64_t ql[2] = {d->tokens, d->heads}, kl[2] = {d->keys, d->kv_heads};
    REQUIRE(span_of(q, d->dtype, ql, d->q_stride, 2, d->dim, &in[0]) &&
                span_of(k, d->dtype, kl, d->k_stride, 2, d->dim, &in[1]) &&
                span_of(v, d->dtype, kl, d->v_stride, 2, d->dim_v, &in[2]),
            "strides reach too far");
    in[3] = bytes_at(q_start, 4ll * (d->sequences + 1));
    in[4] = bytes_at(k_start, 4ll * (d->sequences + 1));
    return PAM_OK;
}

pam_status_t check_head_norm(const pam_head_norm_desc_t *desc)
{
    REQUIRE(desc, "desc is NULL");
    const pam_head_norm_desc_t &d = *desc;
    REQUIRE(known_type(d.dtype), "dtype must be PAM_F32, PAM_F16 or PAM_BF16");
    REQUIRE(d.norm == PAM_NORM_RMS || d.norm == PAM_NORM_LAYER, "norm must be PAM_NORM_RMS or PAM_NORM_LAYER");
    REQUIRE(d.batch >= 0 && d.length >= 0, "batch and length must not be negative");
    REQUIRE(d.heads >= 1 && d.kv_heads >= 0 && d.heads < (1 << 20) && d.kv_heads < (1 << 20),
            "heads must be positive, kv_heads not negative, both less than 2^20");
    REQUIRE(d.dim >= 1 && d.dim <= PAM_HEAD_NORM_MAX_DIM, "dim must be in [1, 512]");
    REQUIRE(d.pairs >= 1 && d.pairs <= d.dim / 2, "pairs must be in [1, dim / 2]");
    REQUIRE((d.flags & ~PAM_ROTARY_INTERLEAVED) == 0, "unknown flag");
    REQUIRE((__int128)d.batch * d.length * (d.heads + d.kv_heads) <= kMost31,
            "batch length (heads + kv_heads) must be less than 2^31");
    REQUIRE(d.eps >= 0.0f && d.eps < INFINITY, "eps must be finite and not negative");
    REQUIRE(d.entries >= 0 && d.start > -((int64_t)1 << 62) && d.start < ((int64_t)1 << 62),
            "entries must not be negative, start less than 2^62 in size");
    return PAM_OK;
}

struct HeadNormSpans {
    Span q, k;        // inputs
    Span rest[4];     // weights, table, positions
    int64_t bytes_q, bytes_k, bytes_wq, bytes_wk;
    bool dense_q, dense_k;
};
pam_status_t head_norm_spans(const pam_head_norm_desc_t &d, const void *q, const void *k, const float *w_q,
                             const float *w_k, const float *table, const int32_t *pos, HeadNormSpans *s)
{
    REQUIRE(d.entries >= 1, "the table is empty");
    REQUIRE(q && table && (d.kv_heads == 0 || k), "a pointer is NULL");
    REQUIRE((uintptr_t)table % 8 == 0, "table must be 8-byte aligned");
    const int64_t ql[3] = {d.batch, d.length, d.heads}, kl[3] = {d.batch, d.length, d.kv_heads};
    REQUIRE(span_of(q, d.dtype, ql, d.q_stride, 3, d.dim, &s->q) && span_of(k, d.dtype, kl, d.k_stride, 3, d.dim, &s->k),
            "strides reach too far");
    const int64_t tok = (int64_t)d.batch * d.length * d.dim * bytes_of(d.dtype);
    s->bytes_q = tok * d.heads;
    s->bytes_k = tok * d.kv_heads;
    s->bytes_wq = 4ll * d.dim * (d.w_per_head ? d.heads : 1);
    s->bytes_wk = d.kv_heads ? 4ll * d.dim * (d.w_per_head ? d.kv_heads : 1) : 0;
    auto contiguous = [&](const int64_t st[3], int64_t h) {
        return (d.batch == 1 || st[0] == d.length * h * d.dim) && (d.length == 1 || st[1] == h * d.dim) &&
               (h == 1 || st[2] == d.dim);
    };
    s->dense_q = contiguous(d.q_stride, d.heads);
    s->dense_k = contiguous(d.k_stride, d.kv_heads);
    s->rest[0] = bytes_at(w_q, s->bytes_wq);
    s->rest[1] = bytes_at(w_k, s->bytes_wk);
    // a table of which no entry past 2^40 is reached counts as that long
    s->rest[2] = bytes_at(table, std::min(d.entries, (int64_t)1 << 40) * d.pairs * 8);
    s->rest[3] = bytes_at(pos, (int64_t)d.batch * d.length * 4);
    return PAM_OK;
}

bool scaled(int32_t store) { return store == PAM_STORE_E4M3 || store == PAM_STORE_INT8; }

pam_status_t check_cache(const pam_cache_desc_t *d)
{
    REQUIRE(d, "cache is NULL");
    REQUIRE(known_type(d->dtype), "dtype must be PAM_F32, PAM_F16 or PAM_BF16");
    REQUIRE(d->store == d->dtype || scaled(d->store), "store must be dtype, PAM_STORE_E4M3 or PAM_STORE_INT8");
    REQUIRE(d->maps == 1 || d->maps == 2, "maps must be 1 or 2");
    REQUIRE(d->dim >= 1 && d->dim <= PAM_CACHE_MAX_ROW / d->maps, "maps dim must be in [1, 256]");
    REQUIRE(d->dim_v >= 1 && d->dim_v <= PAM_CACHE_MAX_ROW, "dim_v must be in [1, 256]");
    REQUIRE(d->kv_heads >= 1 && d->page_size >= 1 && d->pages >= 0, "kv_heads and page_size must be positive, pages not negative");
    REQUIRE((__int128)d->pages * d->kv_heads * d->page_size <= kMost31, "pages kv_heads page_size must be less than 2^31");
    REQUIRE(d->sequences >= 0 && d->table_width >= 0, "sequences and table_width must not be negative");
    REQUIRE((int64_t)d->table_width * d->page_size < 1 << 30, "table_width page_size must be less than 2^30");
    return PAM_OK;
}

// The pool's arrays and what names a sequence's tokens: 6 spans, k_pages first.
pam_status_t pool_of(const pam_cache_desc_t &d, const int32_t *table, const int32_t *k_len, const void *k_pages,
                     const void *v_pages, const float *k_scale, const float *v_scale, Pool *p, Span s[6])
{
    const int64_t rows = (int64_t)d.pages * d.kv_heads * d.page_size;
    const int64_t e = scaled(d.store) ? 1 : bytes_of(d.dtype);
    REQUIRE(k_len && (d.table_width == 0 || table), "a pointer is NULL");
    REQUIRE(rows == 0 || (k_pages && v_pages), "a pointer is NULL");
    REQUIRE(((uintptr_t)k_pages | (uintptr_t)v_pages) % 16 == 0, "k_pages and v_pages must be 16-byte aligned");
    if (scaled(d.store)) {
        REQUIRE(rows == 0 || (k_scale && v_scale), "k_scale and v_scale go with stored types of 8 bits");
    } else {
        REQUIRE(!k_scale && !v_scale, "k_scale and v_scale go with stored types of 8 bits");
    }
    *p = Pool{const_cast<void *>(k_pages), const_cast<void *>(v_pages), const_cast<float *>(k_scale),
              const_cast<float *>(v_scale), table, k_len, d.pages, d.page_size, d.kv_heads, d.dim, d.dim_v, d.maps,
              d.sequences, d.table_width};
    s[0] = bytes_at(k_pages, rows * d.maps * d.dim * e);
    s[1] = bytes_at(v_pages, rows * d.dim_v * e);
    s[2] = bytes_at(k_scale, rows * d.maps * 4);
    s[3] = bytes_at(v_scale, rows * 4);
    s[4] = bytes_at(table, (int64_t)d.sequences * d.table_width * 4);
    s[5] = bytes_at(k_len, d.sequences * 4ll);
    return PAM_OK;
}

pam_status_t check_paged(const pam_cache_desc_t *c, const pam_paged_attn_desc_t *d)
{
    CHECK(check_cache(c));
    REQUIRE(d, "desc is NULL");
    REQUIRE(d->heads >= 1 && d->heads % c->kv_heads == 0, "kv_heads must divide heads");
    REQUIRE(d->len_q >= 0 && d->len_q < 1 << 20, "len_q must be in [0, 2^20)");
    REQUIRE((__int128)c->sequences * d->heads * d->len_q * c->maps <= 1 << 30,
            "sequences heads len_q maps must be at most 2^30");  // rows and units are numbers of 32 bits
    REQUIRE(d->key_bound >= 0, "key_bound must not be negative");
    REQUIRE(d->scale > 0.0f && d->scale < INFINITY, "scale must be positive and finite");
    return PAM_OK;
}

}  // namespace

extern "C" {

size_t pam_attn_fwd_workspace(const pam_attn_desc_t *desc)
{
    return check_packed(desc) == PAM_OK ? packed_fwd_workspace(*desc) : SIZE_MAX;
}

size_t pam_attn_bwd_workspace(const pam_attn_desc_t *desc)
{
    return check_packed(desc) == PAM_OK ? packed_bwd_workspace(*desc) : SIZE_MAX;
}

pam_status_t pam_attn_fwd(const pam_attn_desc_t *desc, const void *q, const void *k, const void *v,
                          const int32_t *q_start, const int32_t *k_start, void *out, float *saved_o, float *saved_lse,
                          void *workspace, void *stream)
{
    CHECK(check_packed(desc));
    if (desc->tokens == 0)
        return PAM_OK;
    REQUIRE(q && out && (desc->keys == 0 || (k && v)), "a pointer is NULL");
    REQUIRE(!saved_o == !saved_lse, "saved_o and saved_lse must be given together");
    const size_t ws = packed_fwd_workspace(*desc);
    REQUIRE(ws == 0 || (workspace && (uintptr_t)workspace % 16 == 0), "workspace is NULL or not 16-byte aligned");
    Span in[kPackedInputs];
    CHECK(packed_spans(desc, q, k, v, q_start, k_start, in));
    const int64_t rows = desc->tokens * desc->heads;
    const Span outs[4] = {bytes_at(out, rows * desc->dim_v * bytes_of(desc->dtype)),
                          bytes_at(saved_o, rows * desc->dim_v * 4), bytes_at(saved_lse, rows * 4),
                          bytes_at(workspace, (int64_t)ws)};
    CHECK(apart(outs, 4, in, kPackedInputs));
    LAUNCH(launch_packed_fwd(*desc, q, k, v, q_start, k_start, out, saved_o, saved_lse, workspace, (hipStream_t)stream),
           "attention forward");
    return PAM_OK;
}

pam_status_t pam_attn_bwd(const pam_attn_desc_t *desc, const void *q, const void *k, const void *v,
                          const int32_t *q_start, const int32_t *k_start, const float *saved_o, const float *saved_lse,
                          const void *grad_out, const int64_t do_stride[2], void *grad_q, void *grad_k, void *grad_v,
                          void *workspace, void *stream)
{
    CHECK(check_packed(desc));
    const int64_t rows = desc->tokens * desc->heads, keys = desc->keys * desc->kv_heads;
    if (rows == 0 && keys == 0)
        return PAM_OK;
    REQUIRE(rows == 0 || (q && saved_o && saved_lse && grad_out && do_stride && grad_q), "a pointer is NULL");
    REQUIRE(keys == 0 || (k && v && grad_k && grad_v), "a pointer is NULL");
    const size_t ws = packed_bwd_workspace(*desc);
    REQUIRE(ws == 0 || (workspace && (uintptr_t)workspace % 16 == 0), "workspace is NULL or not 16-byte aligned");
    const int64_t e = bytes_of(desc->dtype);
    Span in[kPackedInputs + 3] = {};
    CHECK(packed_spans(desc, q, k, v, q_start, k_start, in));
    if (rows) {
        const int64_t ol[2] = {desc->tokens, desc->heads};
        REQUIRE(span_of(grad_out, desc->dtype, ol, do_stride, 2, desc->dim_v, &in[kPackedInputs]), "strides reach too far");
        in[kPackedInputs + 1] = bytes_at(saved_o, rows * desc->dim_v * 4);
        in[kPackedInputs + 2] = bytes_at(saved_lse, rows * 4);
    }
    const Span outs[4] = {bytes_at(grad_q, rows * desc->dim * e), bytes_at(grad_k, keys * desc->dim * e),
                          bytes_at(grad_v, keys * desc->dim_v * e), bytes_at(workspace, (int64_t)ws)};
    CHECK(apart(outs, 4, in, kPackedInputs + 3));
    const int64_t none[2] = {0, 0};
    LAUNCH(launch_packed_bwd(*desc, q, k, v, q_start, k_start, saved_o, saved_lse, grad_out, do_stride ? do_stride : none,
                             grad_q, grad_k, grad_v, workspace, (hipStream_t)stream),
           "attention backward");
    return PAM_OK;
}

pam_status_t pam_head_norm_rotary_fwd(const pam_head_norm_desc_t *desc, const void *q, const void *k, const float *w_q,
                                      const float *w_k, const float *table, const int32_t *pos, void *q_out,
                                      void *k_out, void *stream)
{
    CHECK(check_head_norm(desc));
    const pam_head_norm_desc_t &d = *desc;
    if (d.batch == 0 || d.length == 0)
        return PAM_OK;
    REQUIRE(q_out && (d.kv_heads == 0 || k_out), "a pointer is NULL");
    if (d.kv_heads == 0)
        k = k_out = nullptr, w_k = nullptr;
    HeadNormSpans s;
    CHECK(head_norm_spans(d, q, k, w_q, w_k, table, pos, &s));
    const Span outs[2] = {bytes_at(q_out, s.bytes_q), bytes_at(k_out, s.bytes_k)};
    REQUIRE(!meet(outs[0], s.q) || (q == q_out && s.dense_q), "q_out overlaps q");
    REQUIRE(!meet(outs[1], s.k) || (k == k_out && s.dense_k), "k_out overlaps k");
    REQUIRE(!meet(outs[0], s.k) && !meet(outs[1], s.q), "an output overlaps an input");
    CHECK(apart(outs, 2, s.rest, 4));
    LAUNCH(launch_head_norm_fwd(d, q, k, w_q, w_k, table, pos, q_out, k_out, (hipStream_t)stream),
           "head norms and rotary positions forward");
    return PAM_OK;
}

size_t pam_head_norm_rotary_bwd_workspace(const pam_head_norm_desc_t *desc)
{
    return check_head_norm(desc) == PAM_OK ? head_norm_bwd_workspace(*desc) : SIZE_MAX;
}

pam_status_t pam_head_norm_rotary_bwd(const pam_head_norm_desc_t *desc, const void *q, const void *k, const float *w_q,
                                      const float *w_k, const float *table, const int32_t *pos,
                                      const void *grad_q_out, const void *grad_k_out, void *grad_q, void *grad_k,
                                      float *grad_w_q, float *grad_w_k, void *workspace, void *stream)
{
    CHECK(check_head_norm(desc));
    const pam_head_norm_desc_t &d = *desc;
    if (d.kv_heads == 0) {
        k = grad_k_out = grad_k = nullptr;
        w_k = grad_w_k = nullptr;
    }
    const size_t ws = head_norm_bwd_workspace(d);
    REQUIRE(workspace && (uintptr_t)workspace % 16 == 0, "workspace is NULL or not 16-byte aligned");
    HeadNormSpans s = {};
    s.bytes_wq = 4ll * d.dim * (d.w_per_head ? d.heads : 1);
    s.bytes_wk = d.kv_heads ? 4ll * d.dim * (d.w_per_head ? d.kv_heads : 1) : 0;
    if (d.batch && d.length) {  // without rows the weights' gradients are 0
        REQUIRE(grad_q_out && grad_q && (d.kv_heads == 0 || (grad_k_out && grad_k)), "a pointer is NULL");
        CHECK(head_norm_spans(d, q, k, w_q, w_k, table, pos, &s));
    }
    const Span outs[5] = {bytes_at(grad_q, s.bytes_q), bytes_at(grad_k, s.bytes_k), bytes_at(grad_w_q, s.bytes_wq),
                          bytes_at(grad_w_k, s.bytes_wk), bytes_at(workspace, (int64_t)ws)};
    const Span in[8] = {bytes_at(grad_q_out, s.bytes_q), bytes_at(grad_k_out, s.bytes_k), s.q, s.k,
                        s.rest[0], s.rest[1], s.rest[2], s.rest[3]};
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < 8; ++j)
            REQUIRE(!meet(outs[i], in[j]) || (i == j && i < 2 && outs[i].from == in[j].from), "an output overlaps an input");
        for (int j = 0; j < i; ++j)
            REQUIRE(!meet(outs[i], outs[j]), "outputs overlap");
    }
    LAUNCH(launch_head_norm_bwd(d, q, k, w_q, w_k, table, pos, grad_q_out, grad_k_out, grad_q, grad_k, grad_w_q, grad_w_k,
                                workspace, (hipStream_t)stream),
           "head norms and rotary positions backward");
    return PAM_OK;
}

pam_status_t pam_cache_write(const pam_cache_desc_t *desc, const pam_cache_rows_t *rows, const void *k, const void *v,
                             const int32_t *starts, const int32_t *new_len, const int32_t *table, const int32_t *k_len,
                             void *k_pages, void *v_pages, float *k_scale, float *v_scale, void *stream)
{
    CHECK(check_cache(desc));
    REQUIRE(rows, "rows is NULL");
    pam_cache_rows_t r = *rows;
    const pam_cache_desc_t &d = *desc;
    REQUIRE(!starts || !new_len, "new_len does not go with starts");
    REQUIRE(starts || r.length >= 0, "length must not be negative");
    if (starts) {
        r.length = 1;
        r.k_stride[0] = r.v_stride[0] = 0;
    } else {
        r.rows = (int64_t)d.sequences * r.length;
    }
    // tokens are taken in whole blocks of 16
    REQUIRE(r.rows >= 0 && ((__int128)r.rows + 16) * d.kv_heads * d.maps <= kMost31,
            "(rows + 16) kv_heads maps must be less than 2^31");
    if (r.rows == 0 || d.sequences == 0 || d.table_width == 0)
        return PAM_OK;
    REQUIRE(k && v, "a pointer is NULL");
    Pool p;
    Span outs[6], in[5];
    CHECK(pool_of(d, table, k_len, k_pages, v_pages, k_scale, v_scale, &p, outs));
    const int64_t len[4] = {starts ? 1 : d.sequences, starts ? r.rows : r.length, d.kv_heads, d.maps};
    REQUIRE(span_of(k, d.dtype, len, r.k_stride, 4, d.dim, &in[0]) &&
                span_of(v, d.dtype, len, r.v_stride, 3, d.dim_v, &in[1]),
            "strides reach too far");
    in[2] = bytes_at(starts ? starts : new_len, starts ? 4ll * (d.sequences + 1) : 4ll * d.sequences);
    in[3] = outs[4];
    in[4] = outs[5];
    CHECK(apart(outs, 4, in, 5));
    LAUNCH(launch_cache_write(d, r, p, k, v, starts, new_len, (hipStream_t)stream), "cache write");
    return PAM_OK;
}

pam_status_t pam_cache_read(const pam_cache_desc_t *desc, int32_t length, const int32_t *table, const int32_t *k_len,
                            const void *k_pages, const void *v_pages, const float *k_scale, const float *v_scale,
                            void *k, void *v, void *stream)
{
    CHECK(check_cache(desc));
    const pam_cache_desc_t &d = *desc;
    REQUIRE(length >= 0, "length must not be negative");
    REQUIRE(((__int128)d.sequences * length + 16) * d.kv_heads * d.maps <= kMost31,
            "(sequences length + 16) kv_heads maps must be less than 2^31");
    if (length == 0 || d.sequences == 0 || (!k && !v))
        return PAM_OK;
    Pool p;
    Span in[6];
    CHECK(pool_of(d, table, k_len, k_pages, v_pages, k_scale, v_scale, &p, in));
    REQUIRE(((uintptr_t)k | (uintptr_t)v) % bytes_of(d.dtype) == 0, "k and v must be aligned to their type");
    const int64_t rows = (int64_t)d.sequences * length * d.kv_heads * bytes_of(d.dtype);
    const Span outs[2] = {bytes_at(k, rows * d.maps * d.dim), bytes_at(v, rows * d.dim_v)};
    CHECK(apart(outs, 2, in, 6));
    LAUNCH(launch_cache_read(d, length, p, k, v, (hipStream_t)stream), "cache read");
    return PAM_OK;
}

size_t pam_paged_attn_workspace(const pam_cache_desc_t *cache, const pam_paged_attn_desc_t *desc)
{
    return check_paged(cache, desc) == PAM_OK ? paged_workspace(*cache, *desc) : SIZE_MAX;
}

pam_status_t pam_paged_attn(const pam_cache_desc_t *cache, const pam_paged_attn_desc_t *desc, const void *q,
                            const void *lambda, const int32_t *q_len, const int32_t *table, const int32_t *k_len,
                            const void *k_pages, const void *v_pages, const float *k_scale, const float *v_scale,
                            void *out, void *workspace, void *stream)
{
    CHECK(check_paged(cache, desc));
    const pam_cache_desc_t &c = *cache;
    const int64_t rows = (int64_t)c.sequences * desc->heads * desc->len_q;
    if (rows == 0)
        return PAM_OK;
    REQUIRE(q && out, "a pointer is NULL");
    REQUIRE(!lambda == (c.maps == 1), "lambda goes with two maps");
    const size_t ws = paged_workspace(c, *desc);
    REQUIRE(ws == 0 || (workspace && (uintptr_t)workspace % 16 == 0), "workspace is NULL or not 16-byte aligned");
    Pool p;
    Span in[9];
    CHECK(pool_of(c, table, k_len, k_pages, v_pages, k_scale, v_scale, &p, in));
    const int64_t ql[4] = {c.sequences, desc->len_q, desc->heads, c.maps};
    REQUIRE(span_of(q, c.dtype, ql, desc->q_stride, 4, c.dim, &in[6]), "strides reach too far");
    in[7] = bytes_at(lambda, desc->heads * bytes_of(c.dtype));
    in[8] = bytes_at(q_len, c.sequences * 4ll);
    const Span outs[2] = {bytes_at(out, rows * c.dim_v * bytes_of(c.dtype)), bytes_at(workspace, (int64_t)ws)};
    CHECK(apart(outs, 2, in, 9));
    LAUNCH(launch_paged(c, *desc, p, q, lambda, q_len, out, workspace, (hipStream_t)stream), "attention over pages");
    return PAM_OK;
}

}  // extern "C"
