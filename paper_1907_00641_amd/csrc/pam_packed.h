// What the kernels of attention over packed sequences and their host code share.
#pragma once

#include "pam_rows.h"

namespace pam {

constexpr int kPackedRows = 128;  // rows (queries, or keys) of a block
constexpr int kScanned = 256;     // sequences that a block looks through for its place

// How a launch's work is dealt out.  A unit is a place for a tile of 128 rows, of one head:
// there are as many places as the sequences' tiles at the most (which sequence's tile a place
// has is known on the device alone).  The first `full` units are an item each, the others
// `parts` items along the walked axis, whose sums a second kernel joins.
struct PackedPlan {
    uint32_t slots, heads, full, parts, teams;  // teams: of four waves, in a block
    uint32_t fold;  // items [fold, 2 fold) are taken in reverse; 0: none
    __host__ __device__ uint32_t units() const { return slots * heads; }
    __host__ __device__ uint32_t cut() const { return slots * heads - full; }
    __host__ __device__ uint32_t items() const { return full + cut() * parts; }
};

struct PackedArgs {
    const void *q, *k, *v;
    const int32_t *q_start, *k_start;
    int64_t qs[2], ks[2], vs[2], dos[2];  // strides in elements: token, head
    int32_t sequences, heads, kv_heads, group, dim, dim_v, tokens, keys;
    int32_t causal;
    float scale;
    PackedPlan plan, key_plan;
    float *part, *key_part;
    uint32_t *q_places, *k_places;  // more than kScanned sequences: tiles before each, and in all
    void *out;
    float *so, *lse;
    const void *dout;
    void *gq, *gk, *gv;
    float *stats;  // head x 2 x tokens: lse (base 2; infinity where a row sees nothing), D
    int32_t wide;  // every row of every array allows 16-byte accesses
};

// head sizes are padded to 64, or 128
inline int packed_class(int dim, int dim_v) { return dim <= 64 && dim_v <= 64 ? 64 : 128; }

// per element type (pam_packed_f32.hip, pam_packed_f16.hip, pam_packed_bf16.hip)
hipError_t packed_fwd_f32(const PackedArgs &a, hipStream_t s);
hipError_t packed_fwd_f16(const PackedArgs &a, hipStream_t s);
hipError_t packed_fwd_bf16(const PackedArgs &a, hipStream_t s);
hipError_t packed_bwd_f32(const PackedArgs &a, hipStream_t s);
hipError_t packed_bwd_f16(const PackedArgs &a, hipStream_t s);
hipError_t packed_bwd_bf16(const PackedArgs &a, hipStream_t s);

}  // namespace pam
