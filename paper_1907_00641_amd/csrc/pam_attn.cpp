// Differential attention: from a call's descriptor to the kernels' arguments,
// and the choice of kernel (pam_attn_kernels.h, compiled per element type).
#include "pam_attn.h"

#include <algorithm>

namespace pam {

namespace {

AttnArgs attn_args(const pam_diff_attn_desc_t &d, const void *q, const void *k, const void *v, const void *lam,
                   const int32_t *q_len, const int32_t *k_len, const uint8_t *key_mask)
{
    AttnArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.lam = lam;
    a.q_len = q_len;
    a.k_len = k_len;
    a.key_mask = key_mask;
    for (int i = 0; i < 4; ++i) {
        a.qs[i] = d.q_stride[i];
        a.ks[i] = d.k_stride[i];
    }
    for (int i = 0; i < 3; ++i)
        a.vs[i] = d.v_stride[i];
    a.batch = d.batch;
    a.heads = d.heads;
    a.kv_heads = d.kv_heads;
    a.group = d.heads / d.kv_heads;
    a.dim = d.dim;
    a.dim_v = d.dim_v;
    a.len_q = d.len_q;
    a.len_k = d.len_k;
    a.causal = (d.flags & PAM_ATTN_CAUSAL) != 0;
    a.scale = d.scale;
    a.lse_map = (int64_t)d.batch * d.heads * d.len_q;
    a.so_map = a.lse_map * d.dim_v;
    return a;
}

// Whether every row of every array may be read 16 bytes at a time, with the
// offsets of a tile of 64 rows, in bytes, in 32 bits.
struct Wide {
    int per;
    bool ok = true;
    void at(const void *p) { ok = ok && (uintptr_t)p % 16 == 0; }
    void rows(const void *p, const int64_t *stride, int axes, int dim)
    {
        at(p);
        for (int i = 0; i < axes; ++i)
            ok = ok && stride[i] % per == 0;
        ok = ok && dim % per == 0 && stride[1] >= 0 && stride[1] <= 1 << 23 &&
             (axes < 4 || (stride[3] >= 0 && stride[3] <= 1 << 28));
    }
};

Wide wide_of(const pam_diff_attn_desc_t &d, const void *q, const void *k, const void *v)
{
    Wide w{d.dtype == PAM_F32 ? 4 : 8};
    w.rows(q, d.q_stride, 4, d.dim);
    w.rows(k, d.k_stride, 4, d.dim);
    w.rows(v, d.v_stride, 3, d.dim_v);
    return w;
}

// Whether the keys' gradients are formed per head and then added up: heads
// that share keys, and too few blocks of 128 keys for the card without (two per
// CU: 256 blocks of unequal length leave half the card idle at the end).
bool split_heads(const pam_diff_attn_desc_t &d)
{
    const int64_t blocks = (int64_t)((d.len_k + 127) / 128) * d.kv_heads * d.batch;
    return d.heads > d.kv_heads && blocks < 1024 && d.len_q > 0;
}

int64_t rows_of(const pam_diff_attn_desc_t &d) { return (int64_t)d.batch * d.heads * d.len_q; }
// the rows' statistics and their parts of grad_lambda, whole groups of four floats
int64_t row_floats(const pam_diff_attn_desc_t &d) { return (5 * rows_of(d) + 3) / 4 * 4; }

}  // namespace

size_t attn_fwd_workspace(const pam_diff_attn_desc_t &) { return 0; }

size_t attn_bwd_workspace(const pam_diff_attn_desc_t &d)
{
    int64_t n = row_floats(d);
    if (split_heads(d))
        n += (int64_t)d.batch * d.len_k * d.heads * (2 * d.dim + d.dim_v);
    return (size_t)n * sizeof(float);
}

hipError_t launch_attn_fwd(const pam_diff_attn_desc_t &d, const void *q, const void *k, const void *v,
                           const void *lam, const int32_t *q_len, const int32_t *k_len, const uint8_t *key_mask,
                           void *out, void *so, float *lse, void *workspace, hipStream_t s)
{
    AttnArgs a = attn_args(d, q, k, v, lam, q_len, k_len, key_mask);
    a.out = out;
    a.so = so;
    a.lse = lse;
    Wide w = wide_of(d, q, k, v);
    w.at(out);
    w.at(so);
    if (d.dtype == PAM_F32)
        return attn_fwd_f32(a, w.ok, s);
    return d.dtype == PAM_F16 ? attn_fwd_f16(a, w.ok, s) : attn_fwd_bf16(a, w.ok, s);
}

hipError_t launch_attn_bwd(const pam_diff_attn_desc_t &d, const void *q, const void *k, const void *v,
                           const void *lam, const int32_t *q_len, const int32_t *k_len, const uint8_t *key_mask,
                           const void *so, const float *lse, const void *dout, const int64_t *dos, void *gq, void *gk,
                           void *gv, void *glam, void *workspace, hipStream_t s)
{
    AttnArgs a = attn_args(d, q, k, v, lam, q_len, k_len, key_mask);
    a.so = const_cast<void *>(so);
    a.lse = const_cast<float *>(lse);
    a.dout = dout;
    for (int i = 0; i < 3; ++i)
        a.dos[i] = dos[i];
    a.gq = gq;
    a.gk = gk;
    a.gv = gv;
    a.glam = glam;
    a.stats = (float *)workspace;
    a.dlam = a.stats + 4 * a.lse_map;
    if (split_heads(d)) {
        a.parts = a.stats + row_floats(d);
        a.parts_v = (int64_t)d.batch * d.len_k * d.heads * 2 * d.dim;
    }
    Wide w = wide_of(d, q, k, v);
    w.rows(dout, dos, 3, d.dim_v);
    w.at(so);
    w.at(gq);
    w.at(gk);
    w.at(gv);
    if (d.dtype == PAM_F32)
        return attn_bwd_f32(a, w.ok, s);
    return d.dtype == PAM_F16 ? attn_bwd_f16(a, w.ok, s) : attn_bwd_bf16(a, w.ok, s);
}

}  // namespace pam
