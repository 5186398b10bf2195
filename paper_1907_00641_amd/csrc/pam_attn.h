// What the differential attention's kernels and its host code share.
#pragma once

#include "pam_rows.h"

namespace pam {

// How a launch's work is dealt out (see Item in pam_attn_kernels.h).
struct Plan {
    uint32_t tiles, heads;  // row tiles per head, heads per sequence
    uint32_t units, full, parts;
    uint32_t rows_of_heads;  // 0: units are numbered head by head; else the number of heads in all sequences, and
                             // units are numbered tile by tile
    uint32_t fold;           // units [fold, 2 fold) are taken in reverse; 0: none
    __host__ __device__ uint32_t unit(uint32_t bh, uint32_t tile) const
    {
        return rows_of_heads ? tile * rows_of_heads + bh : bh * tiles + tile;
    }
    __host__ __device__ uint32_t bh_of(uint32_t unit) const
    {
        return rows_of_heads ? unit % rows_of_heads : unit / tiles;
    }
    __host__ __device__ uint32_t tile_of(uint32_t unit) const
    {
        return rows_of_heads ? unit / rows_of_heads : unit % tiles;
    }
    __host__ __device__ uint32_t items() const { return full + (units - full) * parts; }
    __host__ __device__ uint32_t slots() const { return parts > 1 ? (units - full) * parts : 0; }  // items that are parts
};

struct AttnArgs {
    const void *q, *k, *v, *lam;
    const int32_t *q_len, *k_len;
    const uint8_t *key_mask;
    int64_t qs[4], ks[4], vs[3];  // strides in elements: sequence, token, head, map
    int32_t batch, heads, kv_heads, group, dim, dim_v, len_q, len_k;
    int32_t causal, wide;  // wide: every row of every array allows 16-byte accesses
    float scale;
    Plan plan;        // of the launch: queries, or keys
    float *part;      // what the plan's parts leave, and the plan of the other pass with its own
    Plan key_plan;
    float *key_part;
    // forward
    int32_t value_parts;  // of up to 128 channels, each an item of its own
    void *out;
    float *so;        // o^0, then o^1 at so_map elements
    float *lse;       // of map m at m * lse_map
    int64_t so_map, lse_map;
    // backward
    const void *dout;
    int64_t dos[3];
    void *gq, *gk, *gv, *glam;
    float *stats;     // (sequence, head) x 4 x len_q: lse^0 and lse^1 (base 2; infinity where a row sees nothing), D^0,
                      // D^1
    float *dlam;      // sum_ij p^1 dp of every wave of every item of the queries' pass
};

// Head sizes are padded to a class: 32 channels of keys and 64 of values (0), 64
// and 128 (1), 128 and 256 (2; forward: the values in two parts of 128).
inline int attn_class(int dim, int dim_v) { return dim <= 32 && dim_v <= 64 ? 0 : (dim <= 64 && dim_v <= 128 ? 1 : 2); }

// per element type (pam_attn_f32.hip, pam_attn_f16.hip, pam_attn_bf16.hip)
hipError_t attn_fwd_f32(const AttnArgs &a, bool wide, bool few, hipStream_t s);
hipError_t attn_fwd_f16(const AttnArgs &a, bool wide, bool few, hipStream_t s);
hipError_t attn_fwd_bf16(const AttnArgs &a, bool wide, bool few, hipStream_t s);
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
