// Attention over a paged cache: from a call's descriptors to the kernels'
// arguments, and how finely the keys are split (pam_paged_kernels.h, compiled per
// element type).
#include "pam_paged.h"

#include <algorithm>

namespace pam {

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// blocks of four waves that the card holds at once
int64_t at_once(const pam_cache_desc_t &c)
{
    const int cls = paged_class(c.maps * c.dim, c.dim_v);
    return 256 * (cls == 256 || (c.dtype == PAM_F32 && cls == 128) ? 1 : 2);
}

struct PagedPlan {
    int32_t rows, live, tiles, parts;
    int64_t units, floats;
};

// The keys are split so that the units fill the card once with two blocks per CU, unless a wave
// of a part had fewer than two tiles of 32 keys then.  One, two and three blocks per CU: 16 sequences of up
// to 16384, 32 heads of 128 over 8, e4m3, 164, 94 and 112 us; 8 of up to 9000, 4 tokens, 8 heads over 4, 2 maps of
// 64, int8, 34, 29 and 40; 32 of up to 2000 39, 35 and 42; one of 65536, bf16, 33, 35 and 40.
PagedPlan plan_of(const pam_cache_desc_t &c, const pam_paged_attn_desc_t &d)
{
    PagedPlan p;
    p.rows = d.heads / c.kv_heads * d.len_q * c.maps;
    p.live = std::min(p.rows, 32);
    p.tiles = (int32_t)ceil_div(p.rows, 32);
    p.units = (int64_t)c.sequences * c.kv_heads * p.tiles;
    const int64_t table = (int64_t)c.table_width * c.page_size;
    const int64_t bound = d.key_bound ? std::min<int64_t>(d.key_bound, table) : table;
    const int64_t most = bound / (32 * 4 * 2), fill = p.units ? at_once(c) / p.units : 1;
    p.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>({most, fill, 256}));
    const int64_t width = paged_class(c.maps * c.dim, c.dim_v);
    // the blocks' sums, and two numbers for every unit
    p.floats = p.parts > 1 ? p.units * (p.parts * p.live * (width + 2) + 2) : 0;
    return p;
}

}  // namespace

size_t paged_workspace(const pam_cache_desc_t &c, const pam_paged_attn_desc_t &d)
{
    return c.sequences && d.len_q ? (size_t)plan_of(c, d).floats * sizeof(float) : 0;
}

hipError_t launch_paged(const pam_cache_desc_t &c, const pam_paged_attn_desc_t &d, const Pool &pool, const void *q,
                        const void *lam, const int32_t *q_len, void *out, void *workspace, hipStream_t s)
{
    const PagedPlan p = plan_of(c, d);
    PagedArgs a{};
    a.pool = pool;
    a.q = q;
    a.lam = lam;
    a.q_len = q_len;
    a.out = out;
    a.part = (float *)workspace;
    a.cuts = (int2 *)(a.part + p.floats - 2 * p.units);
    a.heads = d.heads;
    a.group = d.heads / c.kv_heads;
    a.len_q = d.len_q;
    a.rows = p.rows;
    a.live = p.live;
    a.tiles = p.tiles;
    a.parts = p.parts;
    a.units = (int32_t)p.units;
    a.scale = d.scale;
    const int per = c.dtype == PAM_F32 ? 4 : 8;
    a.q_wide = (uintptr_t)q % 16 == 0 && c.dim % per == 0;
    for (int i = 0; i < 4; ++i) {
        a.qs[i] = i == 3 && c.maps == 1 ? 0 : d.q_stride[i];
        a.q_wide = a.q_wide && a.qs[i] % per == 0;
    }
    a.by_page = Divisor::of(c.page_size);
    // rows of whole pieces, which begin at multiples of them
    const int both = c.maps * c.dim | c.dim_v;
    const int piece = both % 16 == 0 && (c.store == PAM_STORE_E4M3 || c.store == PAM_STORE_INT8) ? 16 : (both % 8 ? 0 : 8);
    if (c.dtype == PAM_F32)
        return paged_f32(a, c.store, piece, s);
    return c.dtype == PAM_F16 ? paged_f16(a, c.store, piece, s) : paged_bf16(a, c.store, piece, s);
}

}  // namespace pam
