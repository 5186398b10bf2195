// What the kernels of attention over a paged cache and their host code share.
#pragma once

#include "pam_rows.h"

namespace pam {

struct PagedArgs {
    Pool pool;
    const void *q, *lam;
    const int32_t *q_len;
    void *out;
    float *part;  // sums of the blocks: (block, row, channel), then tops and sums: (block, row, 2)
    int2 *cuts;   // of every unit: its first block, and their number
    int64_t qs[4];  // sequence, token, head, map
    int32_t heads, group, len_q, rows;  // rows: of a key head, group len_q maps
    int32_t live;                       // rows of a tile that are there at the most
    int32_t tiles, parts, units;        // tiles of 32 rows per key head; parts of a unit on average; units: sequences
                                        // kv_heads tiles
    bool q_wide;
    Divisor by_page;
    float scale;
};

// channels that a row of keys and one of values are padded to
inline int paged_class(int row, int dim_v) { return row <= 64 && dim_v <= 64 ? 64 : (row <= 128 && dim_v <= 128 ? 128 : 256); }

// per element type (pam_paged_f32.hip, pam_paged_f16.hip, pam_paged_bf16.hip)
hipError_t paged_f32(const PagedArgs &a, int store, int piece, hipStream_t s);
hipError_t paged_f16(const PagedArgs &a, int store, int piece, hipStream_t s);
hipError_t paged_bf16(const PagedArgs &a, int store, int piece, hipStream_t s);

}  // namespace pam
