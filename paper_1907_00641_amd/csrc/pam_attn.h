// What the differential attention's kernels and its host code share.
#pragma once

#include "pam_rows.h"

namespace pam {

struct AttnArgs {
    const void *q, *k, *v, *lam;
    const int32_t *q_len, *k_len;
    const uint8_t *key_mask;
    int64_t qs[4], ks[4], vs[3];  // strides in elements: sequence, token, head, map
    int32_t batch, heads, kv_heads, group, dim, dim_v, len_q, len_k;
    int32_t causal;
    float scale;
    // forward
    void *out, *so;   // so: o^0, then o^1 at so_map elements
    float *lse;       // of map m at m * lse_map
    int64_t so_map, lse_map;
    // backward
    const void *dout;
    int64_t dos[3];
    void *gq, *gk, *gv, *glam;
    float *stats;     // lse^0 and lse^1 (base 2; infinity where a row sees nothing), D^0, D^1, each laid out as lse
    float *dlam;      // per row sum_j p^1 dp: batch x heads x len_q
    float *parts;     // grad_k and, parts_v floats on, grad_v per head, or null: no heads to add up
    int64_t parts_v;
};

// per element type (pam_attn_f32.hip, pam_attn_f16.hip, pam_attn_bf16.hip)
hipError_t attn_fwd_f32(const AttnArgs &a, bool wide, hipStream_t s);
hipError_t attn_fwd_f16(const AttnArgs &a, bool wide, hipStream_t s);
hipError_t attn_fwd_bf16(const AttnArgs &a, bool wide, hipStream_t s);
hipError_t attn_bwd_f32(const AttnArgs &a, bool wide, hipStream_t s);
hipError_t attn_bwd_f16(const AttnArgs &a, bool wide, hipStream_t s);
hipError_t attn_bwd_bf16(const AttnArgs &a, bool wide, hipStream_t s);

// lengths of sequence b, clamped to the arrays
__device__ __forceinline__ int q_len_of(const AttnArgs &a, int b)
{
    return a.q_len ? min(max(a.q_len[b], 0), a.len_q) : a.len_q;
}
__device__ __forceinline__ int k_len_of(const AttnArgs &a, int b)
{
    return a.k_len ? min(max(a.k_len[b], 0), a.len_k) : a.len_k;
}

}  // namespace pam
