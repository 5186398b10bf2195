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

// Blocks that the card holds at once: 256 CUs with two (one, where a lane's
// registers or a block's LDS are for one) of four waves.
constexpr int64_t kCUs = 256;

int64_t at_once(const pam_diff_attn_desc_t &d)
{
    const int cls = attn_class(d.dim, d.dim_v);
    return kCUs * (cls == 0 || (cls == 1 && d.dtype != PAM_F32) ? 2 : 1);
}

// Units beyond whole rounds of `room` blocks are cut into parts that fill one
// more round, of at least `least` of the unit's `trips` each (`slow`: in fp32), or
// of `shortest` where they do not come to one block per CU: waiting for a longer
// part takes longer there than joining more of them.  (fp32, 1 x 500, 8 heads of
// 64: 43 us for 74, backward 79 for 160; bf16, backward, 44 for 54, but 4 x 500, a
// block per CU without it, 74 for 67.)
// Causal units are of unequal lengths: from a round and a half on (a quarter, with
// two blocks on a CU) they fill the rounds by themselves, longest first; fewer
// would wait for the longest, so they are all cut, where two blocks share a CU if
// they are long.
// bf16, 8 heads of 64, 8192 tokens: 320 us cut for 338 whole, backward 715 for 903;
// 2 x 4800: 209 for 186; fp32, 4096 tokens (one block per CU): 538 for 933.
Plan plan_of(int64_t tiles, int64_t heads, int64_t batch, int64_t room, int64_t trips, int64_t least, int64_t shortest,
             bool causal, bool slow)
{
    Plan p{};
    p.tiles = (uint32_t)tiles;
    p.heads = (uint32_t)heads;
    p.rows_of_heads = causal ? (uint32_t)(heads * batch) : 0;
    const int64_t units = tiles * heads * batch;
    p.units = p.full = (uint32_t)units;
    p.parts = 1;
    const int64_t most = trips / least;
    const bool two = room == 2 * kCUs;
    const bool enough = causal && (units >= (two ? room * 5 / 4 : room * 3 / 2) || (two && units >= room && most < 20));
    p.fold = enough && two ? (uint32_t)kCUs : 0;
    if (units == 0 || trips / shortest < 2 || enough)
        return p;
    const int64_t full = causal ? 0 : units / room * room, rest = units - full;
    if (rest == 0)
        return p;
    // Parts of causal units fill two rounds, longest first, or one where joining
    // more would cost more: short units of 16-bit types with two blocks on a CU
    // (bf16, 8 heads of 64, forward and backward, one round for two: 1 x 2000 55 us
    // for 87 and 113 for 137, 1 x 2500 65 for 80 and 141 for 163; 1 x 2900 81 for 85
    // and 194 for 176, 1 x 3300 92 for 88 and 218 for 187)
    const bool one_round = two && !slow && most < 12;
    const int64_t fill = causal ? std::max<int64_t>((one_round ? room : 2 * room) / rest, 2) : room / rest;
    const int64_t parts = std::max(std::min(most, fill), std::min(trips / shortest, kCUs / rest));
    if (parts < 2)
        return p;
    p.full = (uint32_t)full;
    p.parts = (uint32_t)parts;
    return p;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct FwdPlan {
    Plan plan;
    bool few;
    int value_parts, rows, dvp;
    int64_t floats() const { return plan.parts > 1 ? (int64_t)plan.slots() * rows * (2 * dvp + 4) : 0; }
};

FwdPlan fwd_plan(const pam_diff_attn_desc_t &d)
{
    FwdPlan f;
    const int cls = attn_class(d.dim, d.dim_v);
    f.dvp = cls == 0 ? 64 : 128;
    f.value_parts = (int)ceil_div(d.dim_v, f.dvp);
    // The kernel for few queries: a block of 128 rows of one head would be half
    // empty, or (16-bit types) all its blocks of 32 rows fit the card at once and
    // the keys are few, so that nothing has to be cut and joined (bf16, 1 x 500, 8
    // heads of 64: 22 us for 26; 4 x 500, of 32: 18 for 27; but 1 x 1000, 4 of 64,
    // 30 for 27), or it still has more blocks for the same cut (2000 keys, 26 blocks:
    // 25 us for 29, 32: 26 for 28, 48: 32 for 30; 8000 keys 35 for 46, 37 for 45, 50
    // for 51).
    const bool half = d.dtype != PAM_F32;
    const int64_t tiles = ceil_div((int64_t)(d.heads / d.kv_heads) * d.len_q, 32),
                  blocks = tiles * d.kv_heads * d.batch * f.value_parts;
    const bool empty = d.len_q <= 64 || (half && cls < 2 && d.len_q <= 128 && blocks <= 32);
    const bool whole = !empty && half && blocks <= (cls == 0 ? 2 : 1) * kCUs &&
                       d.len_k <= (cls == 0 ? 1024 : (cls == 1 ? 768 : 384));
    f.few = empty || whole;
    const bool causal = d.flags & PAM_ATTN_CAUSAL;
    if (f.few) {
        f.rows = 32;
        // a block's four waves take a part each already
        f.plan = plan_of(tiles, (int64_t)d.kv_heads * f.value_parts, d.batch, kCUs, whole ? 1 : ceil_div(d.len_k, 128),
                         2, half ? 2 : 1, false, false);
    } else {
        f.rows = 128;
        f.plan = plan_of(ceil_div(d.len_q, 128), (int64_t)d.heads * f.value_parts, d.batch, at_once(d),
                         ceil_div(d.len_k, 64), 4, d.dtype == PAM_F32 ? 1 : 4, causal, d.dtype == PAM_F32);
    }
    return f;
}

struct BwdPlan {
    Plan rows, keys;
    int64_t stats, dlam, row_part, key_part;  // floats
};

BwdPlan bwd_plan(const pam_diff_attn_desc_t &d)
{
    BwdPlan p;
    const bool causal = d.flags & PAM_ATTN_CAUSAL;
    const int cls = attn_class(d.dim, d.dim_v), dp = cls == 0 ? 32 : (cls == 1 ? 64 : 128);
    p.rows = plan_of(ceil_div(d.len_q, 128), d.heads, d.batch, at_once(d), ceil_div(d.len_k, 64), 4, 1, causal,
                     d.dtype == PAM_F32);
    p.keys = plan_of(ceil_div(d.len_k, 128), d.kv_heads, d.batch, at_once(d),
                     ceil_div(d.len_q, 32) * (d.heads / d.kv_heads), 8, 2, causal, d.dtype == PAM_F32);
    p.stats = 4 * (int64_t)d.batch * d.heads * d.len_q;
    p.dlam = (int64_t)p.rows.items() * 4;
    p.row_part = (int64_t)p.rows.slots() * 128 * 2 * dp;
    p.key_part = (int64_t)p.keys.slots() * 128 * 4 * dp;
    return p;
}

}  // namespace

size_t attn_fwd_workspace(const pam_diff_attn_desc_t &d)
{
    return d.batch && d.len_q ? (size_t)fwd_plan(d).floats() * sizeof(float) : 0;
}

size_t attn_bwd_workspace(const pam_diff_attn_desc_t &d)
{
    const BwdPlan p = bwd_plan(d);
    return (size_t)(p.row_part + p.key_part + p.stats + p.dlam) * sizeof(float);
}

hipError_t launch_attn_fwd(const pam_diff_attn_desc_t &d, const void *q, const void *k, const void *v,
                           const void *lam, const int32_t *q_len, const int32_t *k_len, const uint8_t *key_mask,
                           void *out, float *so, float *lse, void *workspace, hipStream_t s)
{
    AttnArgs a = attn_args(d, q, k, v, lam, q_len, k_len, key_mask);
    a.out = out;
    a.so = so;
    a.lse = lse;
    const FwdPlan f = fwd_plan(d);
    a.plan = f.plan;
    a.value_parts = f.value_parts;
    a.part = (float *)workspace;
    Wide w = wide_of(d, q, k, v);
    w.at(out);
    w.at(so);
    a.wide = w.ok;
    if (d.dtype == PAM_F32)
        return attn_fwd_f32(a, w.ok, f.few, s);
    return d.dtype == PAM_F16 ? attn_fwd_f16(a, w.ok, f.few, s) : attn_fwd_bf16(a, w.ok, f.few, s);
}

hipError_t launch_attn_bwd(const pam_diff_attn_desc_t &d, const void *q, const void *k, const void *v,
                           const void *lam, const int32_t *q_len, const int32_t *k_len, const uint8_t *key_mask,
                           const float *so, const float *lse, const void *dout, const int64_t *dos, void *gq, void *gk,
                           void *gv, void *glam, void *workspace, hipStream_t s)
{
    AttnArgs a = attn_args(d, q, k, v, lam, q_len, k_len, key_mask);
    a.so = const_cast<float *>(so);
    a.lse = const_cast<float *>(lse);
    a.dout = dout;
    for (int i = 0; i < 3; ++i)
        a.dos[i] = dos[i];
    a.gq = gq;
    a.gk = gk;
    a.gv = gv;
    a.glam = glam;
    // whole groups of four floats first
    const BwdPlan p = bwd_plan(d);
    a.plan = p.rows;
    a.key_plan = p.keys;
    a.part = (float *)workspace;
    a.key_part = a.part + p.row_part;
    a.stats = a.key_part + p.key_part;
    a.dlam = a.stats + p.stats;
    a.value_parts = 1;
    Wide w = wide_of(d, q, k, v);
    w.rows(dout, dos, 3, d.dim_v);
    w.at(so);
    w.at(gq);
    w.at(gk);
    w.at(gv);
    a.wide = w.ok;
    if (d.dtype == PAM_F32)
        return attn_bwd_f32(a, w.ok, s);
    return d.dtype == PAM_F16 ? attn_bwd_f16(a, w.ok, s) : attn_bwd_bf16(a, w.ok, s);
}

}  // namespace pam
