// Kernels of differential attention for one element type (included by one
// source file per type, so that they compile side by side).
//
// With two maps m of scores s^m = scale q^m k^m^T and shared values v,
//   out = o^0 - lambda o^1,  o^m = softmax(s^m) v.
// A block of four waves takes 128 rows (queries; in the keys' gradient pass:
// keys), 32 per wave, and walks over tiles of the other axis that the block's
// loads bring to LDS a tile ahead, straight from memory.  The rows' operands stay
// in registers.
#pragma once

#include "pam_attn_common.h"

namespace pam {

namespace {

constexpr int kBlockRows = 32 * kAttnWaves;
// Sizes of a class of head sizes: keys' channels padded to DP, values' to DVP.
template <class T, int DP, int DVP>
struct Sizes {
    using RK = Rows<T, 2 * DP>;  // both maps of a key (query) side by side
    using RV = Rows<T, DVP>;
    static constexpr int kKeys = RK::kBytes <= 256 ? 64 : 32;  // keys per tile
    static constexpr int kQueries = 32;                        // queries per tile of the keys' pass
    static constexpr int CK = DP / kChunk<T>, CV = DVP / kChunk<T>;
    static constexpr int TK = DP / 32, TV = DVP / 32;
    static constexpr int CP = 32 / kChunk<T>;  // chunks of 32 rows
    // 32-bit registers that a lane's operands and sums take decide how many
    // waves fit a SIMD's 512: two where they are fewer than 256 with room
    // for the scores
    static constexpr bool kSmall = (sizeof(T) == 2 && DP <= 64) || (sizeof(T) == 4 && DP <= 32);
    static constexpr int kWavesPerSimd = kSmall ? 2 : 1;
    // Whether a wave skips the part of a tile that none of its rows sees.  With one
    // wave the sums lie in registers that only the matrix units reach, and a
    // branch around the products costs a copy of them all for every tile: those
    // classes form the products and hide them (bf16, 2 x 4800, 8 heads of 128,
    // backward: 2810 us for 3254).
    static constexpr bool kSkip = kSmall;
    // LDS: a tile of keys and values; of queries and dout with 4 statistics
    // each; the block's values of the keys' pass
    static constexpr int kKeyTile = RK::size(kKeys) + RV::size(kKeys);
    // a wave's own tile of 32 keys in the kernel for few queries, and the waves
    // of a block that have LDS for two of them, and for their sums
    static constexpr int kFewTile = RK::size(32) + RV::size(32);
    static constexpr int kFewWaves = (2 * kFewTile + 512) * 4 <= (160 << 10) ? 4 : ((2 * kFewTile + 512) * 2 <= (160 << 10) ? 2 : 1);
    static constexpr int kQueryTile = RK::size(kQueries) + RV::size(kQueries) + 4 * kQueries * 4;
    static constexpr bool kKeepValues = 2 * kQueryTile + RV::size(kBlockRows) <= (160 << 10);
    static constexpr int kValues = kKeepValues ? RV::size(kBlockRows) : 0;
};

// Work items.  A unit is a tile of rows of one head of one sequence.  Units come
// in an order that starts with the longest; the first `full` of them are one item
// each, whole rounds of the blocks that the card holds at once; the others, which
// would leave most of the card idle, are `parts` items each, cut along the
// walked axis, whose 32-bit sums a second kernel joins.
struct Item {
    int tile, b, h, part, parts;
    uint32_t slot;  // items that are parts: their number
    // The dispatcher deals blocks to the eight dies in turn.  Units of one length:
    // consecutive ones, which share keys and values, go to one die, so that its L2
    // serves them.  Causal units are numbered tile by tile, the longest first, and
    // taken as they come: every die gets as many long ones (and the same heads,
    // where those are a multiple of eight).  Where two blocks share a CU, the
    // second ones of the first round are taken in reverse: the longest unit is
    // paired with the shortest of the round.
    __device__ __forceinline__ static uint32_t order(const Plan &p, uint32_t n, uint32_t total)
    {
        if (p.rows_of_heads)
            return n >= p.fold && n < 2 * p.fold ? 3 * p.fold - 1 - n : n;
        const uint32_t per = total / 8, rest = total - per * 8, die = n % 8;
        return die * per + min(die, rest) + n / 8;
    }
    __device__ __forceinline__ Item(const Plan &p, uint32_t n)
    {
        const bool whole = n < p.full;
        const uint32_t m = uniform(order(p, whole ? n : n - p.full, whole ? p.full : (p.units - p.full) * p.parts));
        const uint32_t cut = uniform(m / p.parts), unit = whole ? m : p.full + cut;
        parts = whole ? 1 : p.parts;
        part = whole ? 0 : m - cut * p.parts;
        slot = whole ? 0 : m;
        const uint32_t bh = p.bh_of(unit);
        tile = uniform(p.tile_of(unit));
        b = uniform(bh / p.heads);
        h = uniform(bh - bh / p.heads * p.heads);
    }
    // the walked tiles of this item, of `trips` of its unit
    __device__ __forceinline__ void range(int trips, int &from, int &to) const
    {
        const int per = (trips + parts - 1) / parts;
        from = min(part * per, trips);
        to = min(from + per, trips);
    }
};

// Bits of the tile's keys that are part of the sequence and not hidden.
__device__ __forceinline__ bool key_seen(const AttnArgs &a, int b, int nk, int j)
{
    return j < nk && (!a.key_mask || a.key_mask[(int64_t)b * a.len_k + j]);
}

// The first of 128 keys from k0 on of which that is so, nk if there is none; the same in
// every lane.
__device__ __forceinline__ int first_key_seen(const AttnArgs &a, int b, int nk, int k0)
{
    if (!a.key_mask)
        return min(k0, nk);
    const int l = lane_id();
    const uint64_t lo = __ballot(key_seen(a, b, nk, k0 + l)), hi = __ballot(key_seen(a, b, nk, k0 + 64 + l));
    return lo ? k0 + __builtin_ctzll(lo) : (hi ? k0 + 64 + __builtin_ctzll(hi) : nk);
}

// Both maps' scores of this lane's rows to -inf where a bit is 0.  bits: of the
// 32 rows; a lane holds rows 8 x + y + 4 (l / 32).
__device__ __forceinline__ void hide(f32x16 (&s)[2], uint32_t bits)
{
    bits >>= 4 * (lane_id() >> 5);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const bool see = bits >> (8 * (r >> 2) + (r & 3)) & 1;
        s[0][r] = see ? s[0][r] : -INFINITY;
        s[1][r] = see ? s[1][r] : -INFINITY;
    }
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------

// What a wave has of its 32 queries (a lane: query l % 32), and a step over 32
// keys.  Scores are formed transposed (rows keys, columns queries), so a lane
// holds one query: its statistics need an exchange with the lane 32 away alone,
// and scaling the sums of values, which are formed transposed too, needs none.
// The maximum is followed only when it grew by more than 2^8 (then the sums are
// scaled): the probabilities are at most 2^8 then, and nothing is lost, since both
// sums carry the same factor.
// The sums of the two maps are kept apart, since their normalisers are known
// only at the end; a first pass for those would allow one product with
// p^0 - lambda p^1 instead of two, and take as many products and twice the
// exponentials.
template <class T, int DP, int DVP>
struct Queries {
    using S = Sizes<T, DP, DVP>;
    uint4v q[2][S::CK];
    f32x16 o[2][S::TV];
    float top[2], sum[2];  // base 2; a lane's own keys' share of the sum

    template <bool WIDE>
    __device__ __forceinline__ void start(const AttnArgs &a, const T *row, bool in)
    {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
            for (int s = 0; s < S::CK; ++s)
                q[m][s] = memory_chunk<T, WIDE>(row + m * a.qs[3], s, a.dim, in);
#pragma unroll
            for (int v = 0; v < S::TV; ++v)
                o[m][v] = f32x16{};
            top[m] = -INFINITY;
            sum[m] = 0.0f;
        }
    }
    // keys and values from row r0 of a tile (kr, vc: this lane's places in it);
    // `some`: keys from j0 on that are past `limit` or not in `seen` are hidden
    __device__ __forceinline__ void step(uint32_t kr, uint32_t vc, int r0, float c, bool some, int j0, int limit,
                                         uint32_t seen)
    {
        using RK = typename S::RK;
        using RV = typename S::RV;
        f32x16 s[2] = {};
#pragma unroll
        for (int x = 0; x < S::CK; ++x)
#pragma unroll
            for (int m = 0; m < 2; ++m)
                mma<T>(s[m], RK::row_chunk(kr, r0, m * S::CK + x), q[m][x]);
        if (some)
            hide(s, seen & low_bits(limit - j0));
        uint4v p[2][S::CP];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            float mx = s[m][0];
#pragma unroll
            for (int r = 1; r < 16; ++r)
                mx = __builtin_fmaxf(mx, s[m][r]);
            mx *= c;
            if (__any(mx > top[m] + 8.0f)) {
                const float to = __builtin_fmaxf(top[m], xor32_max(mx));
                const float f = top[m] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top[m] - to);
                top[m] = to;
                sum[m] *= f;
#pragma unroll
                for (int v = 0; v < S::TV; ++v)
                    o[m][v] *= f;
            }
            const float base = top[m] == -INFINITY ? 0.0f : top[m] - kLift<T>;
            float add = 0.0f;  // a step's sum first: shorter chains of rounded additions
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[m][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[m][r], c, -base));
                add += s[m][r];
            }
            sum[m] += add;
#pragma unroll
            for (int x = 0; x < S::CP; ++x)
                p[m][x] = operand<T>(s[m], x);
        }
#pragma unroll
        for (int x = 0; x < S::CP; ++x)
#pragma unroll
            for (int v = 0; v < S::TV; ++v) {
                const uint4v vf = RV::col_chunk(vc, r0, x, 32 * v);
                mma<T>(o[0][v], vf, p[0][x]);
                mma<T>(o[1][v], vf, p[1][x]);
            }
    }
    __device__ __forceinline__ void whole_sums()
    {
#pragma unroll
        for (int m = 0; m < 2; ++m)
            sum[m] = xor32_add(sum[m]);
    }
    // A channel's sum, after whole_sums.  A query that saw nothing has 0 times its
    // tiles' values there, which others may see and which need not be finite.
    __device__ __forceinline__ float value(int m, int v, int r) const { return sum[m] != 0.0f ? o[m][v][r] : 0.0f; }
    // unnormalised sums and statistics of this lane's query, for a later join:
    // o as [map][DVP], then the tops and sums
    __device__ __forceinline__ void leave(float *sums, float *stats) const
    {
        const int l = lane_id();
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int v = 0; v < S::TV; ++v)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<float4v *>(sums + m * DVP + 32 * v + 8 * g + 4 * (l >> 5)) =
                        float4v{value(m, v, 4 * g), value(m, v, 4 * g + 1), value(m, v, 4 * g + 2), value(m, v, 4 * g + 3)};
        if (l < 32)
            *reinterpret_cast<float4v *>(stats) = float4v{top[0], top[1], sum[0], sum[1]};
    }
};

// The keys of a tile that are part of the sequence and not hidden, as bits.
// The mask's byte of a lane's key is loaded with the tile and compared only when
// that has arrived: a comparison before would wait for all the loads.
struct KeyMask {
    const uint8_t *mask;
    int nk, next = 1;
    __device__ __forceinline__ KeyMask(const AttnArgs &a, int b, int keys)
        : mask(a.key_mask ? a.key_mask + (int64_t)b * a.len_k : nullptr), nk(keys)
    {
    }
    template <int KT>
    __device__ __forceinline__ void fetch(int k0)
    {
        const int l = lane_id(), j = k0 + l;
        next = mask && l < KT && j < nk ? (int)mask[j] : 1;
    }
    template <int KT>
    __device__ __forceinline__ uint64_t seen(int k0) const
    {
        const int l = lane_id();
        return __ballot(next != 0 && l < KT && k0 + l < nk);
    }
};
template <int KT>
constexpr uint64_t kAllSeen = KT == 64 ? ~0ull : (1ull << KT) - 1;

// Forward: blocks of four waves, 128 queries of one head; the waves share the
// tiles of keys and values, which are loaded straight to LDS a tile ahead.  The
// probabilities never leave the registers: the scores' layout, rounded, is the
// operand of the second product.  They are rounded to the activations' type
// for it, before they are divided by their sum (by a relative 2^-8 at most in bf16,
// 2^-11 in fp16, and at random: about what rounding the output takes, so that out is
// off by 1.1 to 1.45 times as much as by that alone); the sums are of the 32-bit
// values.
// Head sizes over 64 take the values' channels 128 at a time (a.value_parts):
// both maps' sums of 256 did not fit the registers, and spilling them cost more
// than forming the scores twice.
// Bound by instructions: 220 vector operations (64 of them for the softmax's
// sums and maxima, 32 exponentials) for 24 products of 32 x 32 x 16, which take
// as long again; two waves per SIMD hide a part of either behind the other.  bf16, 8
// heads of 64, 2 x 4800: 325 us with its join, 870 TFLOP/s (a large product of the
// library: 1185), 330 with o saved; 16384 causal, 2 key heads: 835 us, 990.  Heads of
// 128, one wave per SIMD: 1470 us, 385.  fp32, 2197, 4 heads of 32: 75 us, 99 (154).
template <class T, int DP, int DVP, bool WIDE>
__global__ __launch_bounds__(kAttnThreads, (Sizes<T, DP, DVP>::kWavesPerSimd)) void k_attn_fwd(AttnArgs a)
{
    using S = Sizes<T, DP, DVP>;
    using RK = typename S::RK;
    using RV = typename S::RV;
    constexpr int KT = S::kKeys;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id();
    const float c = a.scale * kLog2e;
    if (a.dim < DP || a.dim_v % DVP) {  // the channels that no load writes
        for (int e = threadIdx.x; e < 2 * S::kKeyTile / 16; e += kAttnThreads)
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
        __syncthreads();
    }
    const uint32_t items = a.plan.items();
    for (uint32_t n = blockIdx.x; n < items; n += gridDim.x) {
        const Item item(a.plan, n);
        const int q0 = ((int)a.plan.tiles - 1 - item.tile) * kBlockRows;  // causal: the longest first
        const int b = item.b, h = uniform(item.h / a.value_parts), hk = uniform(h / a.group);
        const int v0 = (item.h - h * a.value_parts) * DVP, dim_v = min(a.dim_v - v0, DVP);
        const int nq = q_len_of(a, b), nk = k_len_of(a, b);
        const int i = q0 + 32 * w + (l & 31);  // this lane's query
        const bool in = i < nq;
        const int limit = in ? (a.causal ? min(nk, i + nk - nq + 1) : nk) : 0;
        // keys that a row of the block, and of the wave, sees at the most; and
        // that every row of the wave sees
        const int last = min(q0 + kBlockRows, nq) - 1, wlast = min(q0 + 32 * w + 31, nq - 1);
        const int end = q0 < nq ? (a.causal ? min(nk, last + nk - nq + 1) : nk) : 0;
        const int wend = q0 + 32 * w < nq ? (a.causal ? min(nk, wlast + nk - nq + 1) : nk) : 0;
        const int wall = q0 + 32 * w + 31 < nq ? (a.causal ? min(nk, q0 + 32 * w + nk - nq + 1) : nk) : 0;
        int from, to;
        item.range(max(end + KT - 1, 0) / KT, from, to);
        const T *kp = uniform_ptr((const T *)a.k + b * a.ks[0] + hk * a.ks[2] + (int64_t)from * KT * a.ks[1]);
        const T *vp = uniform_ptr((const T *)a.v + b * a.vs[0] + hk * a.vs[2] + v0 + (int64_t)from * KT * a.vs[1]);

        Queries<T, DP, DVP> Q;
        Q.template start<WIDE>(a, (const T *)a.q + b * a.qs[0] + i * a.qs[1] + h * a.qs[2], in);
        KeyMask mask(a, b, nk);
        auto issue = [&](int t) {  // tiles in order
            char *at = lds + (t & 1) * S::kKeyTile;
            mask.template fetch<KT>(t * KT);
            load_rows<T, 2 * DP, 2, KT, kAttnWaves, WIDE>(at, kp, a.ks[1], a.ks[3], nk - 1 - t * KT, a.dim);
            load_rows<T, DVP, 1, KT, kAttnWaves, WIDE>(at + RK::size(KT), vp, a.vs[1], 0, nk - 1 - t * KT, dim_v);
            kp = uniform_ptr(kp + KT * a.ks[1]);
            vp = uniform_ptr(vp + KT * a.vs[1]);
        };
        if (from < to)
            issue(from);
        for (int t = from; t < to; ++t) {
            const int k0 = t * KT;
            char *kb = lds + (t & 1) * S::kKeyTile, *vb = kb + RK::size(KT);
            wait_loads();
            __syncthreads();  // tile t is there for every wave, and tile t - 1 done with
            const uint64_t seen = mask.template seen<KT>(k0);
            if (t + 1 < to)
                issue(t + 1);
            const bool some_hidden = seen != kAllSeen<KT>;
            if (some_hidden) {  // the same in every wave of the block; of keys, the scores are hidden
                clear_rows<T, DVP, KT, kAttnWaves>(vb, seen);
                __syncthreads();
            }
            const uint32_t kr = lds_address(kb) + RK::row_lane(), vc = lds_address(vb) + RV::col_lane();
#pragma unroll
            for (int kt = 0; kt < KT / 32; ++kt) {
                const int j0 = k0 + 32 * kt;
                if (!S::kSkip || j0 < wend)
                    Q.step(kr, vc, 32 * kt, c, some_hidden || j0 + 32 > wall, j0, limit, (uint32_t)(seen >> (32 * kt)));
            }
        }
        __syncthreads();  // the next item's loads write where this one's were read
        Q.whole_sums();
        if (item.parts > 1) {
            const int64_t at = ((int64_t)item.slot * kAttnWaves + w) * 32 + (l & 31);
            Q.leave(a.part + at * 2 * DVP, a.part + (int64_t)a.plan.slots() * kBlockRows * 2 * DVP + at * 4);
            continue;
        }
        if (i >= a.len_q)
            continue;
        const float inv[2] = {Q.sum[0] != 0.0f ? 1.0f / Q.sum[0] : 0.0f, Q.sum[1] != 0.0f ? 1.0f / Q.sum[1] : 0.0f};
        const float lam = (float)((const T *)a.lam)[h];
        const int64_t row = (((int64_t)b * a.len_q + i) * a.heads + h) * a.dim_v + v0;
#pragma unroll
        for (int v = 0; v < S::TV; ++v)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float x0[4], x1[4], y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x0[j] = Q.value(0, v, 4 * g + j) * inv[0];
                    x1[j] = Q.value(1, v, 4 * g + j) * inv[1];
                    y[j] = x0[j] - lam * x1[j];
                }
                const int ch = 32 * v + 8 * g + 4 * (l >> 5);
                store4<T, WIDE>((T *)a.out + row, ch, dim_v, y);
                if (a.so) {
                    store4<float, WIDE>(a.so + row, ch, dim_v, x0);
                    store4<float, WIDE>(a.so + a.so_map + row, ch, dim_v, x1);
                }
            }
        if (a.lse && l < 32 && v0 == 0) {
            const int64_t at = ((int64_t)b * a.heads + h) * a.len_q + i;
            a.lse[at] = lse_of<T>(Q.top[0], Q.sum[0]);
            a.lse[a.lse_map + at] = lse_of<T>(Q.top[1], Q.sum[1]);
        }
    }
}

// Four channels of a row, wide where the arrays allow it.
template <class T>
__device__ __forceinline__ void put4(const AttnArgs &a, T *row, int c, int dim, const float (&x)[4])
{
    if (a.wide)
        store4<T, true>(row, c, dim, x);
    else
        store4<T, false>(row, c, dim, x);
}

// A row's outputs from its parts, channels ch .. ch + 3 of both maps by one
// thread: stats(p) are part p's tops and sums, sums(p, m) its unnormalised
// channels.
template <class T, class GetStats, class GetSums>
__device__ __forceinline__ void join_row(const AttnArgs &a, int parts, const GetStats &stats, const GetSums &sums, int b,
                                         int h, int i, int v0, int ch, int dim_v)
{
    float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};
    float4v o[2] = {};
    for (int p = 0; p < parts; ++p) {
        const float4v st = stats(p);
#pragma unroll
        for (int m = 0; m < 2; ++m)
            top[m] = st[2 + m] != 0.0f ? __builtin_fmaxf(top[m], st[m]) : top[m];
    }
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
        const float4v st = stats(p);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const float4v x = sums(p, m);
            // a part whose top is -inf and whose sum is not 0 has a NaN in it; one
            // whose sum is 0 saw nothing, and its channels are 0
            const float f = st[2 + m] == 0.0f ? 0.0f : (st[m] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st[m] - top[m]));
            sum[m] += f * st[2 + m];
            o[m] += f * x;
        }
    }
    const float i0 = sum[0] != 0.0f ? 1.0f / sum[0] : 0.0f, i1 = sum[1] != 0.0f ? 1.0f / sum[1] : 0.0f;
    const float lam = (float)((const T *)a.lam)[h];
    const int64_t at = (((int64_t)b * a.len_q + i) * a.heads + h) * a.dim_v + v0;
    float x0[4], x1[4], y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x0[j] = o[0][j] * i0;
        x1[j] = o[1][j] * i1;
        y[j] = x0[j] - lam * x1[j];
    }
    put4<T>(a, (T *)a.out + at, ch, dim_v, y);
    if (a.so) {
        put4<float>(a, a.so + at, ch, dim_v, x0);
        put4<float>(a, a.so + a.so_map + at, ch, dim_v, x1);
    }
    if (a.lse && ch == 0 && v0 == 0) {
        const int64_t r = ((int64_t)b * a.heads + h) * a.len_q + i;
        a.lse[r] = lse_of<T>(top[0], sum[0]);
        a.lse[a.lse_map + r] = lse_of<T>(top[1], sum[1]);
    }
}

// Few queries over many keys (a decoding step).  The rows of a tile are the
// queries of all heads of a key head, 32 at a time; the waves of a block walk over
// their own keys, without waiting for each other, and join their sums in LDS.
// What bounds it is reading the cache: every wave has two tiles of 32 keys under
// way (bf16, 8 x 16384 keys, all full, 8 key heads of 64, 32 query heads: 110 us,
// 4.9 TB/s, joining included).  A short cache is bound by the steps' latency: 300
// keys, three steps of a wave, 10.8 us.
template <class T, int DP, int DVP, bool WIDE>
__global__ __launch_bounds__((64 * Sizes<T, DP, DVP>::kFewWaves)) void k_attn_few(AttnArgs a)
{
    using S = Sizes<T, DP, DVP>;
    using RK = typename S::RK;
    using RV = typename S::RV;
    constexpr int KT = 32, W = S::kFewWaves;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id();
    const float c = a.scale * kLog2e;
    char *mine = lds + w * 2 * S::kFewTile;
    float *stats = reinterpret_cast<float *>(lds + W * 2 * S::kFewTile);
    const uint32_t items = a.plan.items();
    for (uint32_t n = blockIdx.x; n < items; n += gridDim.x) {
        const Item item(a.plan, n);
        const int b = item.b, hk = uniform(item.h / a.value_parts);
        const int v0 = (item.h - hk * a.value_parts) * DVP, dim_v = min(a.dim_v - v0, DVP);
        const int nq = q_len_of(a, b), nk = k_len_of(a, b);
        const int r = item.tile * 32 + (l & 31), g = r / a.len_q, i = r - g * a.len_q, h = hk * a.group + g;
        const bool in = g < a.group && i < nq;
        const int limit = in ? (a.causal ? min(nk, i + nk - nq + 1) : nk) : 0;
        // over the wave's rows: the most, the least; lanes without a row do not ask
        // that anything be hidden from them
        int wend = limit, wall = g < a.group ? limit : nk;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            wend = max(wend, __shfl_xor(wend, s));
            wall = min(wall, __shfl_xor(wall, s));
        }
        wend = uniform(wend);
        wall = uniform(wall);
        int from, to;
        item.range(max(wend + KT - 1, 0) / KT, from, to);
        {
            const int per = (to - from + W - 1) / W;
            from = min(from + w * per, to);
            to = min(from + per, to);
        }
        if (a.dim < DP || a.dim_v % DVP) {  // the channels that no load writes
            for (int e = l; e < 2 * S::kFewTile / 16; e += 64)
                store16(mine + e * 16, uint4v{0, 0, 0, 0});
        }
        const T *kp = uniform_ptr((const T *)a.k + b * a.ks[0] + hk * a.ks[2] + (int64_t)from * KT * a.ks[1]);
        const T *vp = uniform_ptr((const T *)a.v + b * a.vs[0] + hk * a.vs[2] + v0 + (int64_t)from * KT * a.vs[1]);
        Queries<T, DP, DVP> Q;
        KeyMask mask(a, b, nk);
        auto issue = [&](int t) {
            char *at = mine + (t & 1) * S::kFewTile;
            mask.template fetch<KT>(t * KT);
            load_rows<T, 2 * DP, 2, KT, 1, WIDE>(at, kp, a.ks[1], a.ks[3], nk - 1 - t * KT, a.dim);
            load_rows<T, DVP, 1, KT, 1, WIDE>(at + RK::size(KT), vp, a.vs[1], 0, nk - 1 - t * KT, dim_v);
            kp = uniform_ptr(kp + KT * a.ks[1]);
            vp = uniform_ptr(vp + KT * a.vs[1]);
        };
        wave_fence();
        if (from < to)
            issue(from);
        Q.template start<WIDE>(a, (const T *)a.q + b * a.qs[0] + i * a.qs[1] + h * a.qs[2], in);
        for (int t = from; t < to; ++t) {
            const int k0 = t * KT;
            char *kb = mine + (t & 1) * S::kFewTile, *vb = kb + RK::size(KT);
            wait_loads();
            wave_fence();
            const uint64_t seen = mask.template seen<KT>(k0);
            if (t + 1 < to)
                issue(t + 1);
            const bool some_hidden = seen != kAllSeen<KT>;
            if (some_hidden) {
                clear_rows<T, DVP, KT, 1>(vb, seen);
                wave_fence();
            }
            Q.step(lds_address(kb) + RK::row_lane(), lds_address(vb) + RV::col_lane(), 0, c,
                   some_hidden || k0 + KT > wall, k0, limit, (uint32_t)seen);
            wave_fence();
        }
        Q.whole_sums();
        // [row][map][DVP] of this wave where its tiles were
        float *sums = reinterpret_cast<float *>(mine);
        static_assert(32 * 2 * DVP * 4 <= 2 * S::kFewTile, "a wave's sums fit its tiles");
        Q.leave(sums + (l & 31) * 2 * DVP, stats + (w * 32 + (l & 31)) * 4);
        __syncthreads();
        auto sums_of = [&](int p, int row, int at) {
            return *reinterpret_cast<const float4v *>(reinterpret_cast<const float *>(lds + p * 2 * S::kFewTile) +
                                                      row * 2 * DVP + at);
        };
        auto stats_of = [&](int p, int row) { return *reinterpret_cast<const float4v *>(stats + (p * 32 + row) * 4); };
        const int rows = min(a.group * a.len_q - item.tile * 32, 32);
        for (int e = threadIdx.x; e < rows * (DVP / 4); e += 64 * W) {
            const int row = e / (DVP / 4), ch = e % (DVP / 4) * 4;
            const int rr = item.tile * 32 + row, gg = rr / a.len_q, ii = rr - gg * a.len_q;
            if (item.parts == 1) {
                join_row<T>(
                    a, W, [&](int p) { return stats_of(p, row); },
                    [&](int p, int m) { return sums_of(p, row, m * DVP + ch); }, b, hk * a.group + gg, ii, v0, ch, dim_v);
            } else {  // the block's sums, relative to the largest top of its waves
                float4v st = {-INFINITY, -INFINITY, 0.0f, 0.0f};
                const int64_t at = (int64_t)item.slot * 32 + row;
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    for (int p = 0; p < W; ++p)
                        if (stats_of(p, row)[2 + m] != 0.0f)
                            st[m] = __builtin_fmaxf(st[m], stats_of(p, row)[m]);
                    float4v y = {};
                    for (int p = 0; p < W; ++p) {
                        const float4v sp = stats_of(p, row);
                        const float f =
                            sp[2 + m] == 0.0f ? 0.0f : (sp[m] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(sp[m] - st[m]));
                        st[2 + m] += f * sp[2 + m];
                        y += f * sums_of(p, row, m * DVP + ch);
                    }
                    *reinterpret_cast<float4v *>(a.part + at * 2 * DVP + m * DVP + ch) = y;
                }
                if (ch == 0)
                    *reinterpret_cast<float4v *>(a.part + (int64_t)a.plan.slots() * 32 * 2 * DVP + at * 4) = st;
            }
        }
        __syncthreads();
    }
}

// Joins the parts of a launch's last units: a thread per four channels of a row;
// FEW (up to 256 parts of few rows): a block per row, G threads per four
// channels that take every G-th part each; what bounds it is the loads' latency, so
// there are enough for each to wait for one or two rounds of them (8 rows of 156
// parts: 16.5 us with 8 threads that take a part at a time, 12.6 so).
constexpr int kJoinThreads = 1024;  // FEW: the most

template <class T, int DVP, bool FEW>
__global__ __launch_bounds__((FEW ? kJoinThreads : kAttnThreads)) void k_attn_join(AttnArgs a)
{
    constexpr int ROWS = FEW ? 32 : kBlockRows, QUADS = DVP / 4;
    const float *stats = a.part + (int64_t)a.plan.slots() * ROWS * 2 * DVP;
    auto stats_of = [&](int64_t at) { return *reinterpret_cast<const float4v *>(stats + at * 4); };
    auto sums_of = [&](int64_t at, int m, int ch) {
        return *reinterpret_cast<const float4v *>(a.part + at * 2 * DVP + m * DVP + ch);
    };
    if constexpr (FEW) {
        constexpr int MOST = kJoinThreads / QUADS;
        __shared__ float4v gs[MOST], go[MOST][2][QUADS];
        const int G = blockDim.x / QUADS;
        const uint32_t per = min(a.group * a.len_q, ROWS), rows = (a.plan.units - a.plan.full) * per;
        const int g = threadIdx.x / QUADS, ch = threadIdx.x % QUADS * 4;
        for (uint32_t x = blockIdx.x; x < rows; x += gridDim.x) {
            const uint32_t u = x / per, row = x - u * per, unit = a.plan.full + u;
            const uint32_t bh = a.plan.bh_of(unit), tile = a.plan.tile_of(unit);
            const int b = bh / a.plan.heads, hv = bh - b * a.plan.heads, hk = hv / a.value_parts;
            const int v0 = (hv - hk * a.value_parts) * DVP;
            const int r = tile * 32 + row, q = r / a.len_q, i = r - q * a.len_q, h = hk * a.group + q;
            if (q >= a.group)  // the same in every thread of the block
                continue;
            auto at = [&](int p) { return ((int64_t)u * a.plan.parts + p) * ROWS + row; };
            float4v st = {-INFINITY, -INFINITY, 0.0f, 0.0f}, o[2] = {};
            for (int p0 = g; p0 < (int)a.plan.parts; p0 += 4 * G) {
                float4v sp[4], x[4][2];  // four parts' loads are under way together
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int p = min(p0 + k * G, (int)a.plan.parts - 1);
                    sp[k] = stats_of(at(p));
                    x[k][0] = sums_of(at(p), 0, ch);
                    x[k][1] = sums_of(at(p), 1, ch);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        if (p0 + k * G >= (int)a.plan.parts || sp[k][2 + m] == 0.0f)  // saw nothing
                            continue;
                        const float to = __builtin_fmaxf(st[m], sp[k][m]);
                        const float f0 =
                            st[m] == -INFINITY ? (st[2 + m] == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(st[m] - to);
                        const float f1 = sp[k][m] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(sp[k][m] - to);
                        o[m] = o[m] * f0 + x[k][m] * f1;
                        st[2 + m] = st[2 + m] * f0 + sp[k][2 + m] * f1;
                        st[m] = to;
                    }
            }
            __syncthreads();
            if (ch == 0)
                gs[g] = st;
            go[g][0][ch / 4] = o[0];
            go[g][1][ch / 4] = o[1];
            __syncthreads();
            if (g == 0)
                join_row<T>(
                    a, G, [&](int p) { return gs[p]; }, [&](int p, int m) { return go[p][m][ch / 4]; }, b, h, i, v0, ch,
                    min(a.dim_v - v0, DVP));
        }
    } else {
        const uint32_t rows = (a.plan.units - a.plan.full) * ROWS;
        for (uint32_t e = blockIdx.x * kAttnThreads + threadIdx.x; e < rows * QUADS; e += gridDim.x * kAttnThreads) {
            const uint32_t x = e / QUADS, ch = e % QUADS * 4;
            const uint32_t u = x / ROWS, row = x % ROWS, unit = a.plan.full + u;
            const uint32_t bh = a.plan.bh_of(unit), tile = a.plan.tile_of(unit);
            const int b = bh / a.plan.heads, hv = bh - b * a.plan.heads, h = hv / a.value_parts;
            const int v0 = (hv - h * a.value_parts) * DVP;
            const int i = (a.plan.tiles - 1 - tile) * kBlockRows + row;
            if (i >= a.len_q)
                continue;
            auto at = [&](int p) { return ((int64_t)u * a.plan.parts + p) * ROWS + row; };
            join_row<T>(
                a, a.plan.parts, [&](int p) { return stats_of(at(p)); },
                [&](int p, int m) { return sums_of(at(p), m, ch); }, b, h, i, v0, ch, min(a.dim_v - v0, DVP));
        }
    }
}

// ---------------------------------------------------------------------------
// backward: queries
// ---------------------------------------------------------------------------

// D, dq and the rows' part of grad_lambda.  Transposed as the forward pass is, so
// a lane holds one query.  sum_j p^1 dp is taken from the 32-bit probabilities and
// dp, not from the saved o^1, whose rounding would be all its error.
// D is taken from o in 32 bits: it is the difference of dp and D that counts, which
// may be far smaller than either (values around 4 times their deviation, bf16: dq off
// by 0.003 of its norm, of which the rounding of the probabilities that o is made of
// has a part; with o rounded to bf16 0.011).
// Score gradients are rounded to the activations' type for their product: about as
// much again as rounding dq itself (bf16: 0.0024 for 0.0017 of its norm; with 32-bit
// operands the product would take eight times as long).
// Bound as the forward pass is: bf16, 8 heads of 64, 2 x 4800: 348 us, 810 TFLOP/s;
// 16384 causal 939, 880; heads of 128 975 us; fp32, 2197, 4 heads of 32: 81 us.
template <class T, int DP, int DVP, bool WIDE>
__global__ __launch_bounds__(kAttnThreads, (Sizes<T, DP, DVP>::kWavesPerSimd)) void k_attn_dq(AttnArgs a)
{
    using S = Sizes<T, DP, DVP>;
    using RK = typename S::RK;
    using RV = typename S::RV;
    constexpr int KT = S::kKeys;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id();
    const float c = a.scale * kLog2e;
    if (a.dim < DP || a.dim_v < DVP) {
        for (int e = threadIdx.x; e < 2 * S::kKeyTile / 16; e += kAttnThreads)
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
        __syncthreads();
    }
    const uint32_t items = a.plan.items();
    for (uint32_t n = blockIdx.x; n < items; n += gridDim.x) {
        const Item item(a.plan, n);
        const int q0 = ((int)a.plan.tiles - 1 - item.tile) * kBlockRows;
        const int b = item.b, h = item.h, hk = uniform(h / a.group);
        const int nq = q_len_of(a, b), nk = k_len_of(a, b);
        const int i = q0 + 32 * w + (l & 31);
        const bool in = i < nq;
        const int limit = in ? (a.causal ? min(nk, i + nk - nq + 1) : nk) : 0;
        const int last = min(q0 + kBlockRows, nq) - 1, wlast = min(q0 + 32 * w + 31, nq - 1);
        const int end = q0 < nq ? (a.causal ? min(nk, last + nk - nq + 1) : nk) : 0;
        const int wend = q0 + 32 * w < nq ? (a.causal ? min(nk, wlast + nk - nq + 1) : nk) : 0;
        const int wall = q0 + 32 * w + 31 < nq ? (a.causal ? min(nk, q0 + 32 * w + nk - nq + 1) : nk) : 0;
        int from, to;
        item.range(max(end + KT - 1, 0) / KT, from, to);
        const T *kp = uniform_ptr((const T *)a.k + b * a.ks[0] + hk * a.ks[2] + (int64_t)from * KT * a.ks[1]);
        const T *vp = uniform_ptr((const T *)a.v + b * a.vs[0] + hk * a.vs[2] + (int64_t)from * KT * a.vs[1]);
        const int64_t row = ((int64_t)b * a.len_q + i) * a.heads + h,
                      at = ((int64_t)b * a.heads + h) * a.len_q + i;

        KeyMask mask(a, b, nk);
        auto issue = [&](int t) {  // tiles in order
            char *at = lds + (t & 1) * S::kKeyTile;
            mask.template fetch<KT>(t * KT);
            load_rows<T, 2 * DP, 2, KT, kAttnWaves, WIDE>(at, kp, a.ks[1], a.ks[3], nk - 1 - t * KT, a.dim);
            load_rows<T, DVP, 1, KT, kAttnWaves, WIDE>(at + RK::size(KT), vp, a.vs[1], 0, nk - 1 - t * KT, a.dim_v);
            kp = uniform_ptr(kp + KT * a.ks[1]);
            vp = uniform_ptr(vp + KT * a.vs[1]);
        };
        if (from < to)
            issue(from);
        uint4v q[2][S::CK], g[S::CV];
        const T *qrow = (const T *)a.q + b * a.qs[0] + i * a.qs[1] + h * a.qs[2];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int s = 0; s < S::CK; ++s)
                q[m][s] = memory_chunk<T, WIDE>(qrow + m * a.qs[3], s, a.dim, in);
        const T *grow = (const T *)a.dout + b * a.dos[0] + i * a.dos[1] + h * a.dos[2];
        float D[2] = {0.0f, 0.0f}, lse[2] = {INFINITY, INFINITY};
#pragma unroll
        for (int s = 0; s < S::CV; ++s) {
            g[s] = memory_chunk<T, WIDE>(grow, s, a.dim_v, in);
#pragma unroll
            for (int m = 0; m < 2; ++m)
                D[m] += piece_dot<T, WIDE>(g[s], a.so + m * a.so_map + row * a.dim_v, s, a.dim_v, in);
            if (sizeof(T) == 2 && s % 4 == 3)  // no more of o under way than the registers hold
                asm volatile("" : "+v"(D[0]), "+v"(D[1]));
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            D[m] = xor32_add(D[m]);
            if (in) {  // a row that sees nothing has probabilities 0
                const float x = a.lse[m * a.lse_map + at];
                lse[m] = x == -INFINITY ? INFINITY : x * kLog2e;
            }
            D[m] = lse[m] == INFINITY ? 0.0f : D[m];
            if (l < 32 && i < a.len_q && item.part == 0) {
                float *st = a.stats + ((int64_t)b * a.heads + h) * 4 * a.len_q + i;
                st[(int64_t)m * a.len_q] = lse[m];
                st[(int64_t)(2 + m) * a.len_q] = D[m];
            }
        }
        f32x16 acc[2][S::TK] = {};
        float dlam = 0.0f;
        Range range;
        for (int t = from; t < to; ++t) {
            const int k0 = t * KT;
            char *kb = lds + (t & 1) * S::kKeyTile, *vb = kb + RK::size(KT);
            wait_loads();
            __syncthreads();
            const uint64_t seen = mask.template seen<KT>(k0);
            if (t + 1 < to)
                issue(t + 1);
            const bool some_hidden = seen != kAllSeen<KT>;
            if (some_hidden) {
                clear_rows<T, 2 * DP, KT, kAttnWaves>(kb, seen);
                clear_rows<T, DVP, KT, kAttnWaves>(vb, seen);
                __syncthreads();
            }
            const uint32_t kr = lds_address(kb) + RK::row_lane(), kc = lds_address(kb) + RK::col_lane();
            const uint32_t vr = lds_address(vb) + RV::row_lane();
#pragma unroll
            for (int kt = 0; kt < KT / 32; ++kt) {
                const int j0 = k0 + 32 * kt;
                // (fp16's branch in Range costs the copies anyhow)
                if ((S::kSkip || std::is_same<T, f16>::value) && j0 >= wend)
                    break;
                f32x16 s[2] = {}, dp = {};
#pragma unroll
                for (int x = 0; x < S::CK; ++x)
#pragma unroll
                    for (int m = 0; m < 2; ++m)
                        mma<T>(s[m], RK::row_chunk(kr, 32 * kt, m * S::CK + x), q[m][x]);
#pragma unroll
                for (int x = 0; x < S::CV; ++x)
                    mma<T>(dp, RV::row_chunk(vr, 32 * kt, x), g[x]);
                if (some_hidden || j0 + 32 > wall)
                    hide(s, (uint32_t)(seen >> (32 * kt)) & low_bits(limit - j0));
                uint4v ds[2][S::CP];
                float add = 0.0f;  // a step's sum first: shorter chains of rounded additions
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[m][r], c, -lse[m]));
                        if (m == 1)
                            add = __builtin_fmaf(p, dp[r], add);
                        s[m][r] = p * (dp[r] - D[m]);
                    }
                dlam += add;
                if constexpr (std::is_same<T, f16>::value)
                    range.fit(s, [&](float f) {
#pragma unroll
                        for (int m = 0; m < 2; ++m)
#pragma unroll
                            for (int v = 0; v < S::TK; ++v)
                                acc[m][v] *= f;
                    });
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int x = 0; x < S::CP; ++x)
                        ds[m][x] = operand<T>(s[m], x);
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int x = 0; x < S::CP; ++x)
#pragma unroll
                        for (int v = 0; v < S::TK; ++v)
                            mma<T>(acc[m][v], RK::col_chunk(kc, 32 * kt, x, m * DP + 32 * v), ds[m][x]);
            }
        }
        __syncthreads();
        // A row that sees nothing has sums of 0 times its own grad_out and its tiles' keys
        // and values, none of which need be finite: it adds nothing, and dq is 0.
        dlam = lanes_sum<64>(lse[1] == INFINITY ? 0.0f : dlam);
        if (l == 0)
            a.dlam[(item.parts > 1 ? a.plan.full + item.slot : a.plan.unit(b * a.heads + h, item.tile)) * (int64_t)kAttnWaves + w] =
                dlam;
        if (i >= a.len_q)
            continue;
        const float lam = (float)((const T *)a.lam)[h];
        float *part = a.part + (((int64_t)item.slot * kAttnWaves + w) * 32 + (l & 31)) * 2 * DP;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const float f = (m ? -lam * a.scale : a.scale) * range.down();
#pragma unroll
            for (int v = 0; v < S::TK; ++v)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    float x[4];
#pragma unroll
                    for (int z = 0; z < 4; ++z)
                        x[z] = lse[m] == INFINITY ? 0.0f : acc[m][v][4 * y + z] * f;
                    const int ch = 32 * v + 8 * y + 4 * (l >> 5);
                    if (item.parts > 1)
                        store4<float, true>(part + m * DP, ch, DP, x);
                    else
                        store4<T, WIDE>((T *)a.gq + (row * 2 + m) * a.dim, ch, a.dim, x);
                }
        }
    }
}

// ---------------------------------------------------------------------------
// backward: keys and values
// ---------------------------------------------------------------------------

// dk and dv of 128 keys, over the queries of every head of the key head.  Scores
// are formed with queries as rows here: a lane holds one key.  WHAT: both (3), or
// dv (1) and dk (2) by themselves: head sizes over 64 have no registers for the
// sums of both, and form the scores twice.
// A kernel of its own, apart from dq's: one pass would save two of the seven
// products, but either dq or dk and dv would have to be summed over blocks, by
// atomics in an order that changes from run to run, or by parts of 32 bits as
// large as the scores' rows over 128.
// Bound by the same, and by LDS, which the queries, dout and the block's values
// are read from in two orders each: bf16, 8 heads of 64, 2 x 4800: 453 us, 830
// TFLOP/s; 16384 causal, 2 key heads 1283, 860; heads of 128, dv 737 and dk 1025 us; fp32,
// 2197, 4 heads of 32: 100 us.
template <class T, int DP, int DVP, bool WIDE, int WHAT>
__global__ __launch_bounds__(kAttnThreads, (Sizes<T, DP, DVP>::kWavesPerSimd)) void k_attn_dkv(AttnArgs a)
{
    using S = Sizes<T, DP, DVP>;
    using RK = typename S::RK;
    using RV = typename S::RV;
    constexpr int QT = S::kQueries;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id();
    const float c = a.scale * kLog2e;
    if (a.dim < DP || a.dim_v < DVP) {
        for (int e = threadIdx.x; e < (2 * S::kQueryTile + S::kValues) / 16; e += kAttnThreads)
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
        __syncthreads();
    }
    const uint32_t items = a.key_plan.items();
    for (uint32_t n = blockIdx.x; n < items; n += gridDim.x) {
        const Item item(a.key_plan, n);
        const int k0 = item.tile * kBlockRows;  // causal: the longest first
        const int b = item.b, hk = item.h, h0 = hk * a.group, h1 = h0 + a.group;
        const int nq = q_len_of(a, b), nk = k_len_of(a, b);
        const int j = k0 + 32 * w + (l & 31);  // this lane's key
        const bool seen = key_seen(a, b, nk, j);
        // the first query that sees this lane's key, one of the block's (the queries
        // before it may see nothing at all), the first of its tile, the wave's first
        const int off = a.causal ? nk - nq : (1 << 30);
        const int from = seen ? j - off : 0x7fffffff;
        const int key0 = first_key_seen(a, b, nk, k0);
        const int lowest = key0 - off, first = max(lowest, 0) / QT * QT, wfirst = k0 + 32 * w - off;
        const bool all = __all(seen);
        const bool wany = __any(seen);

        uint4v kf[2][S::CK];
        {
            const T *krow = (const T *)a.k + b * a.ks[0] + j * a.ks[1] + hk * a.ks[2];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int s = 0; s < S::CK; ++s)
                    kf[m][s] = memory_chunk<T, WIDE>(krow + m * a.ks[3], s, a.dim, seen);
        }
        // The wave's 32 rows of values stay in LDS: with them in registers too, two
        // maps of 64 bf16 channels did not fit 256.  (The largest class has no LDS
        // for them and reads them again and again, through the caches.)
        char *vrows = lds + 2 * S::kQueryTile + RV::size(32) * w;
        const T *vrow = (const T *)a.v + b * a.vs[0] + j * a.vs[1] + hk * a.vs[2];
        if constexpr (S::kKeepValues && (WHAT & 2))
            for (int s = 0; s < S::CV; ++s)
                store16(vrows + RV::at(l & 31, 2 * s + (l >> 5)), memory_chunk<T, WIDE>(vrow, s, a.dim_v, seen));
        f32x16 gk[2][S::TK] = {}, gv[S::TV] = {};
        Range range;
        // fp16: probabilities, at most 1 + |lambda| together, go into the product
        // 2^lift times larger, at most 2^14
        float lift = 0.0f;
        if constexpr (std::is_same<T, f16>::value) {
            float most = 0.0f;
            for (int h = h0; h < h1; ++h)
                most = __builtin_fmaxf(most, __builtin_fabsf((float)((const T *)a.lam)[h]));
            // (with scores so small that what their sums would start from passes 32 bits
            // there is nothing to lift)
            lift = c > 0x1p-100f ? (float)(14 - __builtin_amdgcn_frexp_expf(1.0f + most)) : 0.0f;
        }
        const float lifted = lift / c;  // what the scores' sums start from

        // tiles of all heads in one run, loads a tile ahead
        const int per = key0 < nk && nq > first ? (nq - first + QT - 1) / QT : 0;
        int t0, t1;
        item.range(per * a.group, t0, t1);
        // head and first query of the next tile to load
        int nh = h0 + (per ? t0 / per : 0), ni = first + (per ? t0 % per : 0) * QT;
        nh = uniform(nh);
        ni = uniform(ni);
        const T *qp, *gp;
        const float *sp;
        auto head = [&](int h) {
            qp = uniform_ptr((const T *)a.q + b * a.qs[0] + ni * a.qs[1] + h * a.qs[2]);
            gp = uniform_ptr((const T *)a.dout + b * a.dos[0] + ni * a.dos[1] + h * a.dos[2]);
            sp = uniform_ptr(a.stats + ((int64_t)b * a.heads + h) * 4 * a.len_q + ni);
        };
        auto issue = [&](int buf) {
            char *to = lds + buf * S::kQueryTile;
            load_rows<T, 2 * DP, 2, QT, kAttnWaves, WIDE>(to, qp, a.qs[1], a.qs[3], nq - 1 - ni, a.dim);
            load_rows<T, DVP, 1, QT, kAttnWaves, WIDE>(to + RK::size(QT), gp, a.dos[1], 0, nq - 1 - ni, a.dim_v);
            // 4 statistics of 32 queries, one by half of each wave: an offset from one
            // to the next would pass 32 bits in the longest sequences
            const int y = again(l);
            if (y < 32)
                load_lds4(uniform_ptr(sp + w * (int64_t)a.len_q), 4u * (uint32_t)min(y, nq - 1 - ni),
                          lds_address(to + RK::size(QT) + RV::size(QT)) + w * 128);
            ni += QT;
            qp = uniform_ptr(qp + QT * a.qs[1]);
            gp = uniform_ptr(gp + QT * a.dos[1]);
            sp += QT;
            if (ni >= nq && ++nh < h1) {
                ni = first;
                head(nh);
            }
        };
        int i0 = ni - QT, ch = nh;  // of the tile at hand
        if (t0 < t1) {
            head(nh);
            issue(t0 & 1);
        }
        float lam = -uniform_float((float)((const T *)a.lam)[min(ch, a.heads - 1)]);
        for (int t = t0; t < t1; ++t) {
            const int buf = t & 1;
            char *qb = lds + buf * S::kQueryTile, *gb = qb + RK::size(QT);
            const float *st = reinterpret_cast<const float *>(gb + RV::size(QT));
            i0 += QT;
            if (i0 >= nq) {
                i0 = first;
                lam = -uniform_float((float)((const T *)a.lam)[++ch]);
            }
            wait_loads();
            __syncthreads();
            if (t + 1 < t1)
                issue(buf ^ 1);
            const bool tail = i0 + QT > nq;
            if (tail || i0 < lowest) {  // rows past the sequence, or before the first that sees a key of the block
                const uint32_t live = low_bits(nq - i0) & ~low_bits(lowest - i0);
                clear_rows<T, 2 * DP, QT, kAttnWaves>(qb, live);
                clear_rows<T, DVP, QT, kAttnWaves>(gb, live);
                __syncthreads();
            }
            if (!S::kSkip || (wany && i0 + QT > wfirst)) {
                const uint32_t qr = lds_address(qb) + RK::row_lane(), qc = lds_address(qb) + RK::col_lane();
                const uint32_t gr = lds_address(gb) + RV::row_lane(), gc = lds_address(gb) + RV::col_lane();
                const uint32_t vr = lds_address(vrows) + RV::row_lane();
                f32x16 s[2] = {}, dp = {};
                if constexpr (std::is_same<T, f16>::value) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[0][r] = s[1][r] = lifted;
                }
#pragma unroll
                for (int x = 0; x < S::CK; ++x)
#pragma unroll
                    for (int m = 0; m < 2; ++m)
                        mma<T>(s[m], RK::row_chunk(qr, 0, m * S::CK + x), kf[m][x]);
#pragma unroll
                for (int x = 0; x < ((WHAT & 2) ? S::CV : 0); ++x)
                    if constexpr (S::kKeepValues)
                        mma<T>(dp, RV::row_chunk(gr, 0, x), RV::row_chunk(vr, 0, x));
                    else
                        mma<T>(dp, RV::row_chunk(gr, 0, x), memory_chunk<T, WIDE>(vrow, x, a.dim_v, seen));
                if (!all || i0 < wfirst + 31 || tail)
                    hide(s, low_bits(nq - i0) & ~low_bits(from > i0 ? from - i0 : 0));
                uint4v wf[S::CP], ds[2][S::CP];
                f32x16 wt;
#pragma unroll
                for (int x = 0; x < S::CP; ++x) {
#pragma unroll
                    for (int g = x * 4 / S::CP; g < (x + 1) * 4 / S::CP; ++g) {
                        const int at = 8 * g + 4 * (l >> 5);
                        const float4v l0 = *reinterpret_cast<const float4v *>(st + at);
                        const float4v l1 = *reinterpret_cast<const float4v *>(st + QT + at);
                        const float4v d0 = *reinterpret_cast<const float4v *>(st + 2 * QT + at);
                        const float4v d1 = *reinterpret_cast<const float4v *>(st + 3 * QT + at);
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const int r = 4 * g + y;
                            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][r], c, -l0[y]));
                            const float p1 = lam * __builtin_amdgcn_exp2f(__builtin_fmaf(s[1][r], c, -l1[y]));
                            wt[r] = p0 + p1;
                            s[0][r] = p0 * (dp[r] - d0[y]);
                            s[1][r] = p1 * (dp[r] - d1[y]);
                        }
                    }
                    if constexpr (WHAT & 1)
                        wf[x] = operand<T>(wt, x);
                    if constexpr (!std::is_same<T, f16>::value && (WHAT & 2)) {
                        ds[0][x] = operand<T>(s[0], x);
                        ds[1][x] = operand<T>(s[1], x);
                    }
                }
                if constexpr (std::is_same<T, f16>::value && (WHAT & 2)) {
                    range.fit(s, [&](float f) {
#pragma unroll
                        for (int m = 0; m < 2; ++m)
#pragma unroll
                            for (int v = 0; v < S::TK; ++v)
                                gk[m][v] *= f;
                    });
#pragma unroll
                    for (int x = 0; x < S::CP; ++x) {
                        ds[0][x] = operand<T>(s[0], x);
                        ds[1][x] = operand<T>(s[1], x);
                    }
                }
#pragma unroll
                for (int x = 0; x < S::CP; ++x) {
#pragma unroll
                    for (int v = 0; v < ((WHAT & 1) ? S::TV : 0); ++v)
                        mma<T>(gv[v], RV::col_chunk(gc, 0, x, 32 * v), wf[x]);
#pragma unroll
                    for (int m = 0; m < ((WHAT & 2) ? 2 : 0); ++m)
#pragma unroll
                        for (int v = 0; v < S::TK; ++v)
                            mma<T>(gk[m][v], RK::col_chunk(qc, 0, x, m * DP + 32 * v), ds[m][x]);
                }
            }
        }
        __syncthreads();
        if (j >= a.len_k)
            continue;
        const int64_t row = ((int64_t)b * a.len_k + j) * a.kv_heads + hk;
        float *part = a.key_part + (((int64_t)item.slot * kAttnWaves + w) * 32 + (l & 31)) * (2 * DP + DVP);
        auto put = [&](T *to, float *to_part, const f32x16 &x, int v, int dim, float f) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float y[4];  // a hidden key has sums of 0 times what the queries hold
#pragma unroll
                for (int z = 0; z < 4; ++z)
                    y[z] = seen ? x[4 * g + z] * f : 0.0f;
                const int at = 32 * v + 8 * g + 4 * (l >> 5);
                if (item.parts > 1)
                    store4<float, true>(to_part, at, 1 << 20, y);
                else
                    store4<T, WIDE>(to, at, dim, y);
            }
        };
        const float fv = __builtin_amdgcn_exp2f(-lift), fk = a.scale * range.down() * fv;
        if constexpr (WHAT & 2) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int v = 0; v < S::TK; ++v)
                    put((T *)a.gk + (row * 2 + m) * a.dim, part + m * DP, gk[m][v], v, a.dim, fk);
        }
        if constexpr (WHAT & 1) {
#pragma unroll
            for (int v = 0; v < S::TV; ++v)
                put((T *)a.gv + row * a.dim_v, part + 2 * DP, gv[v], v, a.dim_v, fv);
        }
    }
}

// What is left after both passes, in a fixed order: grad_lambda, a block per
// head; and the sums of the parts of both passes' last units.
template <class T, int DP, int DVP>
__global__ __launch_bounds__(kAttnThreads) void k_attn_finish(AttnArgs a)
{
    if ((int)blockIdx.x < a.heads) {
        __shared__ float s[kAttnWaves];
        const uint32_t h = blockIdx.x, tiles = a.plan.tiles;
        float y = 0.0f;
        for (uint32_t e = threadIdx.x; e < (uint32_t)a.batch * tiles; e += kAttnThreads) {
            const uint32_t b = e / tiles, unit = a.plan.unit(b * a.heads + h, e - b * tiles);
            const bool one = unit < a.plan.full;
            const uint32_t from = one ? unit : a.plan.full + (unit - a.plan.full) * a.plan.parts;
            const uint32_t n = (one ? 1 : a.plan.parts) * kAttnWaves;
            for (uint32_t x = 0; x < n; ++x)
                y += a.dlam[(int64_t)from * kAttnWaves + x];
        }
        y = lanes_sum<64>(y);
        if (lane_id() == 0)
            s[threadIdx.x >> 6] = y;
        __syncthreads();
        if (threadIdx.x == 0)
            ((T *)a.glam)[h] = (T)(-(((s[0] + s[1]) + s[2]) + s[3]));
        return;
    }
    constexpr int WQ = 2 * DP, WK = 2 * DP + DVP;
    const uint32_t nq = a.plan.parts > 1 ? (a.plan.units - a.plan.full) * kBlockRows * (WQ / 4) : 0;
    const uint32_t nk = a.key_plan.parts > 1 ? (a.key_plan.units - a.key_plan.full) * kBlockRows * (WK / 4) : 0;
    for (uint32_t e = (blockIdx.x - a.heads) * kAttnThreads + threadIdx.x; e < nq + nk;
         e += (gridDim.x - a.heads) * kAttnThreads) {
        const bool key = e >= nq;
        const Plan &p = key ? a.key_plan : a.plan;
        const int width = key ? WK : WQ;
        const uint32_t x = key ? e - nq : e;
        const uint32_t at = key ? x / (WK / 4) : x / (WQ / 4), ch = (x - at * (width / 4)) * 4;
        const uint32_t u = at / kBlockRows, row = at % kBlockRows, unit = p.full + u;
        const uint32_t bh = p.bh_of(unit), tile = p.tile_of(unit), b = bh / p.heads, h = bh - b * p.heads;
        const int len = key ? a.len_k : a.len_q, i = (key ? tile : p.tiles - 1 - tile) * kBlockRows + row;
        const bool value = ch >= 2 * DP;
        const uint32_t m = value ? 0 : ch / DP, cc = value ? ch - 2 * DP : ch % DP;
        if (i >= len || (int)cc >= (value ? a.dim_v : a.dim))
            continue;
        const float *from = (key ? a.key_part : a.part) + ((int64_t)u * p.parts * kBlockRows + row) * width + ch;
        float4v s = {};
#pragma unroll 4
        for (uint32_t q = 0; q < p.parts; ++q)
            s += *reinterpret_cast<const float4v *>(from + (int64_t)q * kBlockRows * width);
        const float y[4] = {s[0], s[1], s[2], s[3]};
        const int64_t out = ((int64_t)b * len + i) * p.heads + h;
        if (value)
            put4<T>(a, (T *)a.gv + out * a.dim_v, cc, a.dim_v, y);
        else
            put4<T>(a, (T *)(key ? a.gk : a.gq) + (out * 2 + m) * a.dim, cc, a.dim, y);
    }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

template <class T, int DP, int DVP, bool WIDE>
hipError_t fwd_class(const AttnArgs &a, bool few, hipStream_t s)
{
    using S = Sizes<T, DP, DVP>;
    hipError_t e;
    if (few)
        e = launch_lds<k_attn_few<T, DP, DVP, WIDE>>(item_blocks(a.plan.items()), 64 * S::kFewWaves,
                       S::kFewWaves * (2 * S::kFewTile + 32 * 16), a, s);
    else
        e = launch_lds<k_attn_fwd<T, DP, DVP, WIDE>>(item_blocks(a.plan.items()), kAttnThreads, 2 * S::kKeyTile, a, s);
    if (e != hipSuccess || a.plan.parts == 1)
        return e;
    const unsigned cut = a.plan.units - a.plan.full;
    if (few) {
        const unsigned rows = cut * std::min(a.group * a.len_q, 32);
        hipLaunchKernelGGL((k_attn_join<T, DVP, true>), dim3(rows), dim3(a.plan.parts > 32 ? kJoinThreads : 256), 0, s, a);
    } else {
        const unsigned blocks = sum_blocks((int64_t)cut * kBlockRows * DVP / 4);
        hipLaunchKernelGGL((k_attn_join<T, DVP, false>), dim3(blocks), dim3(kAttnThreads), 0, s, a);
    }
    return hipGetLastError();
}

template <class T, int DP, int DVP, bool WIDE>
hipError_t bwd_class(const AttnArgs &a, hipStream_t s)
{
    using S = Sizes<T, DP, DVP>;
    hipError_t e = hipSuccess;
    const unsigned rows = item_blocks(a.plan.items()), keys = item_blocks(a.key_plan.items());
    if (rows)
        e = launch_lds<k_attn_dq<T, DP, DVP, WIDE>>(rows, kAttnThreads, 2 * S::kKeyTile, a, s);
    if (e != hipSuccess)
        return e;
    constexpr int lds = 2 * S::kQueryTile + S::kValues;
    if constexpr (DP <= 64) {
        if (keys)
            e = launch_lds<k_attn_dkv<T, DP, DVP, WIDE, 3>>(keys, kAttnThreads, lds, a, s);
    } else if (keys) {
        e = launch_lds<k_attn_dkv<T, DP, DVP, WIDE, 1>>(keys, kAttnThreads, lds, a, s);
        if (e == hipSuccess)
            e = launch_lds<k_attn_dkv<T, DP, DVP, WIDE, 2>>(keys, kAttnThreads, lds, a, s);
    }
    if (e != hipSuccess)
        return e;
    int64_t sums = 0;
    if (a.plan.parts > 1)
        sums += (int64_t)(a.plan.units - a.plan.full) * kBlockRows * 2 * DP;
    if (a.key_plan.parts > 1)
        sums += (int64_t)(a.key_plan.units - a.key_plan.full) * kBlockRows * (2 * DP + DVP);
    hipLaunchKernelGGL((k_attn_finish<T, DP, DVP>), dim3(a.heads + sum_blocks(sums / 4)), dim3(kAttnThreads), 0, s, a);
    return hipGetLastError();
}

// by the class of head sizes that attn_class names
template <class T, bool WIDE>
hipError_t fwd_wide(const AttnArgs &a, bool few, hipStream_t s)
{
    switch (attn_class(a.dim, a.dim_v)) {
    case 0: return fwd_class<T, 32, 64, WIDE>(a, few, s);
    case 1: return fwd_class<T, 64, 128, WIDE>(a, few, s);
    default: return fwd_class<T, 128, 128, WIDE>(a, few, s);
    }
}
template <class T, bool WIDE>
hipError_t bwd_wide(const AttnArgs &a, hipStream_t s)
{
    switch (attn_class(a.dim, a.dim_v)) {
    case 0: return bwd_class<T, 32, 64, WIDE>(a, s);
    case 1: return bwd_class<T, 64, 128, WIDE>(a, s);
    default: return bwd_class<T, 128, 256, WIDE>(a, s);
    }
}

template <class T>
hipError_t attn_fwd(const AttnArgs &a, bool wide, bool few, hipStream_t s)
{
    return wide ? fwd_wide<T, true>(a, few, s) : fwd_wide<T, false>(a, few, s);
}
template <class T>
hipError_t attn_bwd(const AttnArgs &a, bool wide, hipStream_t s)
{
    return wide ? bwd_wide<T, true>(a, s) : bwd_wide<T, false>(a, s);
}

}  // namespace

}  // namespace pam
