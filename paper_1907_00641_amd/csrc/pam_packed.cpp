// Attention over packed sequences: from a call's descriptor to the kernels'
// arguments, and how the work is dealt out (pam_packed_kernels.h, compiled per
// element type).
#include "pam_packed.h"

#include <algorithm>

namespace pam {

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int64_t kCUs = 256;

// blocks of four waves that the card holds at once
int64_t at_once(const pam_attn_desc_t &d)
{
    return kCUs * (d.dtype != PAM_F32 || packed_class(d.dim, d.dim_v) == 64 ? 2 : 1);
}

// rows: of all sequences, on the axis that is dealt out; walked: tiles of the other
// axis that a unit of an average sequence walks over, `many` of which are a long walk; least:
// tiles of a part, of one team, of two, and of two with so few units that the card is mostly idle
// (keys, 3 x 1000, 2 key heads, 36 units, 8 tiles 26 us for 32; 4 x 500, 8 heads, 128 units, 42 for 37).
//
// Teams (bf16, forward and backward, one team or two): 1 x 500, 8 heads of 64, causal 17 and 34 us
// for 13 and 36; 4 x 500 20 and 44 for 13 and 38; 2 x 1000, 16 of 128, 39 and 122 for 28 and 84; 3 x 2000, 8
// of 128, 65 and 185 for 46 and 146. A block of two teams has a CU to itself: beyond 256 blocks, or
// beyond half of that where causal units are long and only the order of more, shorter items evens
// them out, one team is better: 8 x 300, 16 heads of 64, 12 and 44 us for 16 and 53; 1 x 4000, 8 of 64, causal,
// backward 120 for 143; 3 x 2000, 8 of 128, not causal, 70 and 226 for 83 and 249.
//
// Parts: units beyond whole rounds of the blocks that the card holds are cut, to fill one more
// round; of causal units, which are of unequal lengths, all or none, longest first, and
// `rounds` rounds of them (keys, 16384 tokens, 2 key heads of 128: one round 1774 us, two 1132).
// Each part has a place for its sums, also those of places that hold no tile, of which there are up to
// one per sequence and head: with four times the parts of those rounds nothing is cut. Not causal, 16 heads,
// cut and whole: 52 x 512 tokens, heads of 64, 2176 parts of 2048, 110 and 96 us, backward 385 and 372; 60 x 512, of
// 128, 269 and 229, 860 and 831; below, 36 x 512, of 64, 1664 parts,
// 91 and 275 cut. (4097 x 512 took 4.4 GB for 64 units.)
PackedPlan plan_of(const pam_attn_desc_t &d, int64_t rows, int64_t heads, int64_t walked, int64_t many,
                   const int64_t (&least)[3], int64_t rounds)
{
    PackedPlan p{};
    if (rows == 0)
        return p;
    const bool causal = d.flags & PAM_ATTN_CAUSAL;
    p.slots = (uint32_t)(rows / kPackedRows + d.sequences);
    p.heads = (uint32_t)heads;
    p.full = p.units();
    p.parts = 1;
    // units of sequences of the average length
    const int64_t units = ceil_div(std::max<int64_t>(rows / d.sequences, 1), kPackedRows) * d.sequences * heads;
    const bool two = at_once(d) == 2 * kCUs &&
                     (units <= kCUs / 2 || (causal ? units < 2 * kCUs && walked < many && walked >= 8 : units <= kCUs));
    p.teams = two ? 2 : 1;
    const int64_t room = at_once(d) / p.teams, full = causal ? 0 : units / room * room, rest = units - full;
    const int64_t fill = causal ? (units < room ? rounds * room / units : 1) : (rest ? room / rest : 1);
    const int64_t parts = std::min(walked / least[two ? (units <= kCUs / 4 ? 2 : 1) : 0], fill);
    const int64_t most = 4 * (causal ? rounds : 1) * room;
    if (parts > 1 && ((int64_t)p.units() - full) * parts <= most) {
        p.full = (uint32_t)full;
        p.parts = (uint32_t)parts;
    } else if (causal && room == 2 * kCUs && units >= 2 * kCUs) {
        p.fold = (uint32_t)kCUs;
    }
    return p;
}

struct Plans {
    PackedPlan rows, keys;
    int64_t row_part, key_part, stats, places;  // numbers of 4 bytes; places: of an axis
};

Plans plans_of(const pam_attn_desc_t &d, bool backward)
{
    Plans p{};
    p.places = d.sequences > kScanned ? d.sequences + 1 : 0;
    const int64_t cls = packed_class(d.dim, d.dim_v);
    p.rows = plan_of(d, d.tokens, d.heads, ceil_div(d.keys / d.sequences, 64), 48, {4, 8, 8}, 1);
    p.row_part = (int64_t)p.rows.cut() * p.rows.parts * kPackedRows * (cls + (backward ? 0 : 2));
    if (backward) {
        p.keys = plan_of(d, d.keys, d.kv_heads, ceil_div(d.tokens / d.sequences, 32) * (d.heads / d.kv_heads), 96,
                         {8, 16, 8}, 2);
        p.key_part = (int64_t)p.keys.cut() * p.keys.parts * kPackedRows * 2 * cls;
        p.stats = 2 * (int64_t)d.heads * d.tokens;
    }
    return p;
}

PackedArgs args_of(const pam_attn_desc_t &d, const void *q, const void *k, const void *v, const int32_t *q_start,
                   const int32_t *k_start)
{
    PackedArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_start = q_start;
    a.k_start = k_start;
    for (int i = 0; i < 2; ++i) {
        a.qs[i] = d.q_stride[i];
        a.ks[i] = d.k_stride[i];
        a.vs[i] = d.v_stride[i];
    }
    a.sequences = d.sequences;
    a.heads = d.heads;
    a.kv_heads = d.kv_heads;
    a.group = d.heads / d.kv_heads;
    a.dim = d.dim;
    a.dim_v = d.dim_v;
    a.tokens = (int32_t)d.tokens;
    a.keys = (int32_t)d.keys;
    a.causal = (d.flags & PAM_ATTN_CAUSAL) != 0;
    a.scale = d.scale;
    return a;
}

// Whether every row may be read 16 bytes at a time, with the offsets of a tile of
// 64 rows, in bytes, in 32 bits.
bool wide_rows(const pam_attn_desc_t &d, const void *p, const int64_t *stride, int dim)
{
    const int per = d.dtype == PAM_F32 ? 4 : 8;
    return (uintptr_t)p % 16 == 0 && stride[0] % per == 0 && stride[1] % per == 0 && dim % per == 0 && stride[0] >= 0 &&
           stride[0] <= 1 << 23;
}
bool wide_of(const pam_attn_desc_t &d, const void *q, const void *k, const void *v)
{
    return wide_rows(d, q, d.q_stride, d.dim) && wide_rows(d, k, d.k_stride, d.dim) && wide_rows(d, v, d.v_stride, d.dim_v);
}
bool at16(const void *p) { return (uintptr_t)p % 16 == 0; }

}  // namespace

size_t packed_fwd_workspace(const pam_attn_desc_t &d)
{
    const Plans p = plans_of(d, false);
    return d.tokens ? (size_t)(p.row_part + p.places) * sizeof(float) : 0;
}

size_t packed_bwd_workspace(const pam_attn_desc_t &d)
{
    const Plans p = plans_of(d, true);
    return (size_t)(p.row_part + p.key_part + p.stats + 2 * p.places) * sizeof(float);
}

hipError_t launch_packed_fwd(const pam_attn_desc_t &d, const void *q, const void *k, const void *v,
                             const int32_t *q_start, const int32_t *k_start, void *out, float *so, float *lse,
                             void *workspace, hipStream_t s)
{
    PackedArgs a = args_of(d, q, k, v, q_start, k_start);
    const Plans p = plans_of(d, false);
    a.plan = p.rows;
    a.part = (float *)workspace;
    a.q_places = p.places ? (uint32_t *)(a.part + p.row_part) : nullptr;
    a.out = out;
    a.so = so;
    a.lse = lse;
    a.wide = wide_of(d, q, k, v) && at16(out) && at16(so);
    if (d.dtype == PAM_F32)
        return packed_fwd_f32(a, s);
    return d.dtype == PAM_F16 ? packed_fwd_f16(a, s) : packed_fwd_bf16(a, s);
}

hipError_t launch_packed_bwd(const pam_attn_desc_t &d, const void *q, const void *k, const void *v,
                             const int32_t *q_start, const int32_t *k_start, const float *so, const float *lse,
                             const void *dout, const int64_t *dos, void *gq, void *gk, void *gv, void *workspace,
                             hipStream_t s)
{
    PackedArgs a = args_of(d, q, k, v, q_start, k_start);
    const Plans p = plans_of(d, true);
    a.plan = p.rows;
    a.key_plan = p.keys;
    a.part = (float *)workspace;
    a.key_part = a.part + p.row_part;
    a.stats = a.key_part + p.key_part;
    a.q_places = p.places ? (uint32_t *)(a.stats + p.stats) : nullptr;
    a.k_places = p.places ? a.q_places + p.places : nullptr;
    a.so = const_cast<float *>(so);
    a.lse = const_cast<float *>(lse);
    a.dout = dout;
    a.dos[0] = dos[0];
    a.dos[1] = dos[1];
    a.gq = gq;
    a.gk = gk;
    a.gv = gv;
    a.wide = wide_of(d, q, k, v) && wide_rows(d, dout, dos, d.dim_v) && at16(so) && at16(gq) && at16(gk) && at16(gv);
    if (d.dtype == PAM_F32)
        return packed_bwd_f32(a, s);
    return d.dtype == PAM_F16 ? packed_bwd_f16(a, s) : packed_bwd_bf16(a, s);
}

}  // namespace pam
