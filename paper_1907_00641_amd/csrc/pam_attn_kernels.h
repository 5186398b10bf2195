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

#include <algorithm>
#include <type_traits>

#include "pam_attn_tiles.h"

namespace pam {

namespace {

constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = 4;
constexpr int kBlockRows = 32 * kAttnWaves;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

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
    // LDS: a tile of keys and values; of queries and dout with 4 statistics
    // each; the block's values of the keys' pass
    static constexpr int kKeyTile = RK::size(kKeys) + RV::size(kKeys);
    static constexpr int kQueryTile = RK::size(kQueries) + RV::size(kQueries) + 4 * kQueries * 4;
    static constexpr bool kKeepValues = 2 * kQueryTile + RV::size(kBlockRows) <= (160 << 10);
    static constexpr int kValues = kKeepValues ? RV::size(kBlockRows) : 0;
};

// fp16 has 2^-14 as its smallest full-precision value.  Probabilities are at
// most 2^8 of the running maximum's: 2^7 more keeps them under 2^15 and gives
// small ones 7 bits of room.
template <class T>
constexpr float kLift = std::is_same<T, f16>::value ? 7.0f : 0.0f;

// Score gradients have no such bound.  In fp16 a lane (a query, or a key)
// multiplies its own by a power of two that puts the first tile's largest at
// 2^7 .. 2^8, and takes a smaller one, scaling what it has summed, if a later
// tile would pass 2^15.
struct Range {
    float up = 0.0f;  // 0: not chosen yet
    // x: this lane's results of a tile; both lanes of a column agree
    template <int N, class F>
    __device__ __forceinline__ void fit(f32x16 (&x)[N], const F &scale_sums)
    {
        float mx = 0.0f;
#pragma unroll
        for (int m = 0; m < N; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                mx = __builtin_fmaxf(mx, __builtin_fabsf(x[m][r]));
        mx = xor32_max(mx);
        const bool change = up == 0.0f ? mx > 0.0f : mx * up > 32768.0f;
        if (__any(change)) {
            const float to = change ? __builtin_ldexpf(1.0f, min(8 - __builtin_amdgcn_frexp_expf(mx), 100)) : up;
            scale_sums(up == 0.0f ? 1.0f : to / up);
            up = to;
        }
#pragma unroll
        for (int m = 0; m < N; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                x[m][r] *= up;
    }
    __device__ __forceinline__ float down() const { return up == 0.0f ? 1.0f : 1.0f / up; }
};

// Work item n of `total` for the block that the dispatcher hands out as number
// n: consecutive items, which share keys and values, go to one of the eight
// dies (blocks go round them), so that its L2 serves them.
__device__ __forceinline__ uint32_t die_order(uint32_t n, uint32_t total)
{
    const uint32_t per = total / 8, rest = total - per * 8, die = n % 8;
    return die * per + min(die, rest) + n / 8;
}

// A value that is the same in every lane, in a scalar register: divisions are
// vector code, and what is computed from their results would stay there.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uniform_float(float x)
{
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}

// Item n: its tile of 128 rows, sequence and head.
struct Item {
    int tile, b, h;
    __device__ __forceinline__ Item(uint32_t n, uint32_t total, uint32_t tiles, uint32_t heads)
    {
        const uint32_t x = die_order(n, total), bh = x / tiles;
        tile = uniform(x - bh * tiles);
        b = uniform(bh / heads);
        h = uniform(bh - bh / heads * heads);
    }
};

// Bits of the tile's keys that are part of the sequence and not hidden.
__device__ __forceinline__ bool key_seen(const AttnArgs &a, int b, int nk, int j)
{
    return j < nk && (!a.key_mask || a.key_mask[(int64_t)b * a.len_k + j]);
}

// scores of this lane's keys to -inf where they are not seen: keys from
// `limit` on and those whose bit in `seen` (bit 0: the first key of the 32) is 0
__device__ __forceinline__ void hide(f32x16 &s, int key0, int limit, uint32_t seen)
{
    const int h4 = 4 * (lane_id() >> 5);
    const uint32_t bits = seen >> h4;
    const int lim = limit - key0 - h4;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int j = 8 * (r >> 2) + (r & 3);
        s[r] = (j < lim && (bits >> j & 1)) ? s[r] : -INFINITY;
    }
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------

// One pass over the keys with a running maximum and sum per map.  Scores are
// formed transposed (rows keys, columns queries), so a lane holds one query: its
// statistics need one exchange with the lane 32 away per tile, and scaling the
// sums of values, which are formed transposed too, needs none.  The maximum
// is followed only when it grew by more than 2^8 (then the sums are scaled): the
// probabilities are at most 2^8 then, and nothing is lost, since both sums
// carry the same factor.
template <class T, int DP, int DVP, bool WIDE>
__global__ __launch_bounds__(kAttnThreads, (Sizes<T, DP, DVP>::kWavesPerSimd)) void k_attn_fwd(AttnArgs a)
{
    using S = Sizes<T, DP, DVP>;
    using RK = typename S::RK;
    using RV = typename S::RV;
    constexpr int KT = S::kKeys;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id();
    const uint32_t tiles = (a.len_q + kBlockRows - 1) / kBlockRows, total = tiles * a.heads * a.batch;
    const float c = a.scale * kLog2e;
    if (a.dim < DP || a.dim_v < DVP) {  // the channels that no load writes
        for (int e = threadIdx.x; e < 2 * S::kKeyTile / 16; e += kAttnThreads)
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
        __syncthreads();
    }
    for (uint32_t n = blockIdx.x; n < total; n += gridDim.x) {
        const Item item(n, total, tiles, a.heads);
        const int q0 = ((int)tiles - 1 - item.tile) * kBlockRows;  // causal: the longest first
        const int b = item.b, h = item.h, hk = uniform(h / a.group);
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
        const T *kp = uniform_ptr((const T *)a.k + b * a.ks[0] + hk * a.ks[2]);
        const T *vp = uniform_ptr((const T *)a.v + b * a.vs[0] + hk * a.vs[2]);

        uint4v q[2][S::CK];
        {
            const T *row = (const T *)a.q + b * a.qs[0] + i * a.qs[1] + h * a.qs[2];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int s = 0; s < S::CK; ++s)
                    q[m][s] = memory_chunk<T, WIDE>(row + m * a.qs[3], s, a.dim, in);
        }
        f32x16 o[2][S::TV] = {};
        float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};

        auto issue = [&](int k0, int buf) {  // tiles in order
            char *at = lds + buf * S::kKeyTile;
            load_rows<T, 2 * DP, 2, KT, kAttnWaves, WIDE>(at, kp, a.ks[1], a.ks[3], nk - 1 - k0, a.dim);
            load_rows<T, DVP, 1, KT, kAttnWaves, WIDE>(at + RK::size(KT), vp, a.vs[1], 0, nk - 1 - k0, a.dim_v);
            kp = uniform_ptr(kp + KT * a.ks[1]);
            vp = uniform_ptr(vp + KT * a.vs[1]);
        };
        const int trips = (end + KT - 1) / KT;
        // the mask's byte of this lane's key of the next tile, compared only when
        // that tile is there: a comparison here would wait for all the loads
        const uint8_t *mask = a.key_mask ? a.key_mask + (int64_t)b * a.len_k : nullptr;
        auto mask_byte = [&](int j) { return mask && l < KT && j < nk ? (int)mask[j] : 1; };
        int next = 1;
        if (trips > 0) {
            next = mask_byte(l);
            issue(0, 0);
        }
        for (int t = 0; t < trips; ++t) {
            const int k0 = t * KT, buf = t & 1;
            char *kb = lds + buf * S::kKeyTile, *vb = kb + RK::size(KT);
            wait_loads();
            __syncthreads();  // tile t is there for every wave, and tile t - 1 done with
            const uint64_t seen = __ballot(next != 0 && l < KT && k0 + l < nk);
            if (t + 1 < trips) {
                next = mask_byte(k0 + KT + l);
                issue(k0 + KT, buf ^ 1);
            }
            const bool some_hidden = seen != (KT == 64 ? ~0ull : (1ull << KT) - 1);
            if (some_hidden) {  // the same in every wave of the block
                clear_rows<T, 2 * DP, KT, kAttnWaves>(kb, seen);
                clear_rows<T, DVP, KT, kAttnWaves>(vb, seen);
                __syncthreads();
            }
            const uint32_t kr = lds_address(kb) + RK::row_lane(), vc = lds_address(vb) + RV::col_lane();
#pragma unroll
            for (int kt = 0; kt < KT / 32; ++kt) {
                const int j0 = k0 + 32 * kt;
                if (j0 >= wend)
                    break;
                f32x16 s[2] = {};
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int x = 0; x < S::CK; ++x)
                        mma<T>(s[m], RK::row_chunk(kr, 32 * kt, m * S::CK + x), q[m][x]);
                if (some_hidden || j0 + 32 > wall) {
                    hide(s[0], j0, limit, (uint32_t)(seen >> (32 * kt)));
                    hide(s[1], j0, limit, (uint32_t)(seen >> (32 * kt)));
                }
                uint4v p[2][S::CP];
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    float mx = s[m][0];
#pragma unroll
                    for (int r = 1; r < 16; ++r)
                        mx = __builtin_fmaxf(mx, s[m][r]);
                    mx = xor32_max(mx) * c;
                    if (__any(mx > top[m] + 8.0f)) {
                        const float to = __builtin_fmaxf(top[m], mx);
                        const float f = top[m] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top[m] - to);
                        top[m] = to;
                        sum[m] *= f;
#pragma unroll
                        for (int v = 0; v < S::TV; ++v)
                            o[m][v] *= f;
                    }
                    const float base = top[m] == -INFINITY ? 0.0f : top[m] - kLift<T>;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[m][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[m][r], c, -base));
                        sum[m] += s[m][r];
                    }
#pragma unroll
                    for (int x = 0; x < S::CP; ++x)
                        p[m][x] = operand<T>(s[m], x);
                }
#pragma unroll
                for (int x = 0; x < S::CP; ++x)
#pragma unroll
                    for (int v = 0; v < S::TV; ++v) {
                        const uint4v vf = RV::col_chunk(vc, 32 * kt, x, 32 * v);
                        mma<T>(o[0][v], vf, p[0][x]);
                        mma<T>(o[1][v], vf, p[1][x]);
                    }
            }
        }
        __syncthreads();  // the next item's loads write where this one's were read
        if (i >= a.len_q)
            continue;
        float inv[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            sum[m] = __shfl_xor(sum[m], 32) + sum[m];
            inv[m] = sum[m] != 0.0f ? 1.0f / sum[m] : 0.0f;
        }
        const float lam = (float)((const T *)a.lam)[h];
        const int64_t row = ((int64_t)b * a.len_q + i) * a.heads + h;
        T *out = (T *)a.out + row * a.dim_v;
#pragma unroll
        for (int v = 0; v < S::TV; ++v)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float x0[4], x1[4], y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x0[j] = o[0][v][4 * g + j] * inv[0];
                    x1[j] = o[1][v][4 * g + j] * inv[1];
                    y[j] = x0[j] - lam * x1[j];
                }
                const int ch = 32 * v + 8 * g + 4 * (l >> 5);
                store4<T, WIDE>(out, ch, a.dim_v, y);
                if (a.so) {
                    store4<T, WIDE>((T *)a.so + row * a.dim_v, ch, a.dim_v, x0);
                    store4<T, WIDE>((T *)a.so + a.so_map + row * a.dim_v, ch, a.dim_v, x1);
                }
            }
        if (a.lse && l < 32) {
            const int64_t at = ((int64_t)b * a.heads + h) * a.len_q + i;
#pragma unroll
            for (int m = 0; m < 2; ++m)
                a.lse[m * a.lse_map + at] =
                    sum[m] != 0.0f ? (top[m] - kLift<T> + __builtin_amdgcn_logf(sum[m])) * kLn2 : -INFINITY;
        }
    }
}

// ---------------------------------------------------------------------------
// backward: queries
// ---------------------------------------------------------------------------

// D, dq and the rows' part of grad_lambda.  Transposed as the forward pass is, so
// a lane holds one query.  sum_j p^1 dp is taken from the 32-bit probabilities and
// dp, not from the saved o^1, whose rounding would be all its error.
template <class T, int DP, int DVP, bool WIDE>
__global__ __launch_bounds__(kAttnThreads, (Sizes<T, DP, DVP>::kWavesPerSimd)) void k_attn_dq(AttnArgs a)
{
    using S = Sizes<T, DP, DVP>;
    using RK = typename S::RK;
    using RV = typename S::RV;
    constexpr int KT = S::kKeys;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id();
    const uint32_t tiles = (a.len_q + kBlockRows - 1) / kBlockRows, total = tiles * a.heads * a.batch;
    const float c = a.scale * kLog2e;
    if (a.dim < DP || a.dim_v < DVP) {
        for (int e = threadIdx.x; e < 2 * S::kKeyTile / 16; e += kAttnThreads)
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
        __syncthreads();
    }
    for (uint32_t n = blockIdx.x; n < total; n += gridDim.x) {
        const Item item(n, total, tiles, a.heads);
        const int q0 = ((int)tiles - 1 - item.tile) * kBlockRows;  // causal: the longest first
        const int b = item.b, h = item.h, hk = uniform(h / a.group);
        const int nq = q_len_of(a, b), nk = k_len_of(a, b);
        const int i = q0 + 32 * w + (l & 31);
        const bool in = i < nq;
        const int limit = in ? (a.causal ? min(nk, i + nk - nq + 1) : nk) : 0;
        const int last = min(q0 + kBlockRows, nq) - 1, wlast = min(q0 + 32 * w + 31, nq - 1);
        const int end = q0 < nq ? (a.causal ? min(nk, last + nk - nq + 1) : nk) : 0;
        const int wend = q0 + 32 * w < nq ? (a.causal ? min(nk, wlast + nk - nq + 1) : nk) : 0;
        const int wall = q0 + 32 * w + 31 < nq ? (a.causal ? min(nk, q0 + 32 * w + nk - nq + 1) : nk) : 0;
        const T *kp = uniform_ptr((const T *)a.k + b * a.ks[0] + hk * a.ks[2]);
        const T *vp = uniform_ptr((const T *)a.v + b * a.vs[0] + hk * a.vs[2]);
        const int64_t row = ((int64_t)b * a.len_q + i) * a.heads + h,
                      at = ((int64_t)b * a.heads + h) * a.len_q + i;

        auto issue = [&](int k0, int buf) {  // tiles in order
            char *to = lds + buf * S::kKeyTile;
            load_rows<T, 2 * DP, 2, KT, kAttnWaves, WIDE>(to, kp, a.ks[1], a.ks[3], nk - 1 - k0, a.dim);
            load_rows<T, DVP, 1, KT, kAttnWaves, WIDE>(to + RK::size(KT), vp, a.vs[1], 0, nk - 1 - k0, a.dim_v);
            kp = uniform_ptr(kp + KT * a.ks[1]);
            vp = uniform_ptr(vp + KT * a.vs[1]);
        };
        const int trips = (end + KT - 1) / KT;
        // the mask's byte of this lane's key of the next tile, compared only when
        // that tile is there: a comparison here would wait for all the loads
        const uint8_t *mask = a.key_mask ? a.key_mask + (int64_t)b * a.len_k : nullptr;
        auto mask_byte = [&](int j) { return mask && l < KT && j < nk ? (int)mask[j] : 1; };
        int next = 1;
        if (trips > 0) {
            next = mask_byte(l);
            issue(0, 0);
        }
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
                D[m] += piece_dot<T>(g[s], memory_chunk<T, WIDE>((const T *)a.so + m * a.so_map + row * a.dim_v, s,
                                                                 a.dim_v, in));
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            D[m] = xor32_add(D[m]);
            if (in) {  // a row that sees nothing has probabilities 0
                const float x = a.lse[m * a.lse_map + at];
                lse[m] = x == -INFINITY ? INFINITY : x * kLog2e;
            }
            if (l < 32 && i < a.len_q) {
                a.stats[m * a.lse_map + at] = lse[m];
                a.stats[(2 + m) * a.lse_map + at] = D[m];
            }
        }
        f32x16 acc[2][S::TK] = {};
        float dlam = 0.0f;
        Range range;
        for (int t = 0; t < trips; ++t) {
            const int k0 = t * KT, buf = t & 1;
            char *kb = lds + buf * S::kKeyTile, *vb = kb + RK::size(KT);
            wait_loads();
            __syncthreads();
            const uint64_t seen = __ballot(next != 0 && l < KT && k0 + l < nk);
            if (t + 1 < trips) {
                next = mask_byte(k0 + KT + l);
                issue(k0 + KT, buf ^ 1);
            }
            const bool some_hidden = seen != (KT == 64 ? ~0ull : (1ull << KT) - 1);
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
                if (j0 >= wend)
                    break;
                f32x16 s[2] = {}, dp = {};
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int x = 0; x < S::CK; ++x)
                        mma<T>(s[m], RK::row_chunk(kr, 32 * kt, m * S::CK + x), q[m][x]);
#pragma unroll
                for (int x = 0; x < S::CV; ++x)
                    mma<T>(dp, RV::row_chunk(vr, 32 * kt, x), g[x]);
                if (some_hidden || j0 + 32 > wall) {
                    hide(s[0], j0, limit, (uint32_t)(seen >> (32 * kt)));
                    hide(s[1], j0, limit, (uint32_t)(seen >> (32 * kt)));
                }
                uint4v ds[2][S::CP];
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[m][r], c, -lse[m]));
                        if (m == 1)
                            dlam = __builtin_fmaf(p, dp[r], dlam);
                        s[m][r] = p * (dp[r] - D[m]);
                    }
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
        if (i >= a.len_q)
            continue;
        const float lam = (float)((const T *)a.lam)[h];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const float f = (m ? -lam * a.scale : a.scale) * range.down();
#pragma unroll
            for (int v = 0; v < S::TK; ++v)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float x[4] = {acc[m][v][4 * y] * f, acc[m][v][4 * y + 1] * f, acc[m][v][4 * y + 2] * f,
                                        acc[m][v][4 * y + 3] * f};
                    store4<T, WIDE>((T *)a.gq + (row * 2 + m) * a.dim, 32 * v + 8 * y + 4 * (l >> 5), a.dim, x);
                }
        }
        dlam += __shfl_xor(dlam, 32);
        if (l < 32)
            a.dlam[at] = dlam;
    }
}

// ---------------------------------------------------------------------------
// backward: keys and values
// ---------------------------------------------------------------------------

// dk and dv of 128 keys, over the queries of every head of the key head; or of
// one head (a.parts: 32-bit sums per head, added up by k_attn_parts), where the
// key heads alone are too few blocks.  Scores are formed with queries as rows
// here: a lane holds one key.
template <class T, int DP, int DVP, bool WIDE>
__global__ __launch_bounds__(kAttnThreads, (Sizes<T, DP, DVP>::kWavesPerSimd)) void k_attn_dkv(AttnArgs a)
{
    using S = Sizes<T, DP, DVP>;
    using RK = typename S::RK;
    using RV = typename S::RV;
    constexpr int QT = S::kQueries;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id();
    const int heads = a.parts ? a.heads : a.kv_heads;
    const uint32_t tiles = (a.len_k + kBlockRows - 1) / kBlockRows, total = tiles * heads * a.batch;
    const float c = a.scale * kLog2e;
    if (a.dim < DP || a.dim_v < DVP) {
        for (int e = threadIdx.x; e < (2 * S::kQueryTile + S::kValues) / 16; e += kAttnThreads)
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
        __syncthreads();
    }
    for (uint32_t n = blockIdx.x; n < total; n += gridDim.x) {
        const Item item(n, total, tiles, heads);
        const int k0 = item.tile * kBlockRows;  // causal: the longest first
        const int b = item.b, hx = item.h, hk = a.parts ? uniform(hx / a.group) : hx;
        const int h0 = a.parts ? hx : hx * a.group, h1 = a.parts ? hx + 1 : h0 + a.group;
        const int nq = q_len_of(a, b), nk = k_len_of(a, b);
        const int j = k0 + 32 * w + (l & 31);  // this lane's key
        const bool seen = key_seen(a, b, nk, j);
        // the first query that sees this lane's key, the block's first, the wave's first
        const int off = a.causal ? nk - nq : (1 << 30);
        const int from = seen ? j - off : 0x7fffffff;
        const int first = max(k0 - off, 0) / QT * QT, wfirst = k0 + 32 * w - off;
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
        if constexpr (S::kKeepValues)
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
            lift = (float)(14 - __builtin_amdgcn_frexp_expf(1.0f + most));
        }
        const float lifted = lift / c;  // what the scores' sums start from

        // tiles of all heads in one run, loads a tile ahead
        const int per = nk > k0 && nq > first ? (nq - first + QT - 1) / QT : 0;
        const int trips = per * (h1 - h0);
        int nh = h0, ni = first;  // head and first query of the next tile to load
        const T *qp, *gp;
        const float *sp;
        auto head = [&](int h) {
            qp = uniform_ptr((const T *)a.q + b * a.qs[0] + first * a.qs[1] + h * a.qs[2]);
            gp = uniform_ptr((const T *)a.dout + b * a.dos[0] + first * a.dos[1] + h * a.dos[2]);
            sp = uniform_ptr(a.stats + ((int64_t)b * a.heads + h) * a.len_q + first);
        };
        auto issue = [&](int buf) {
            char *to = lds + buf * S::kQueryTile;
            load_rows<T, 2 * DP, 2, QT, kAttnWaves, WIDE>(to, qp, a.qs[1], a.qs[3], nq - 1 - ni, a.dim);
            load_rows<T, DVP, 1, QT, kAttnWaves, WIDE>(to + RK::size(QT), gp, a.dos[1], 0, nq - 1 - ni, a.dim_v);
            if (w < 2) {  // 4 statistics of 32 queries: a wave takes two of them
                const int y = again(l);
                const float *p = sp + (2 * w + (y >> 5)) * a.lse_map + min(y & 31, nq - 1 - ni);
                __builtin_amdgcn_global_load_lds((const PAM_GLOBAL void *)p,
                                                 (PAM_LDS void *)(to + RK::size(QT) + RV::size(QT) + w * 256), 4, 0, 0);
            }
            ni += QT;
            qp = uniform_ptr(qp + QT * a.qs[1]);
            gp = uniform_ptr(gp + QT * a.dos[1]);
            sp += QT;
            if (ni >= nq && ++nh < h1) {
                ni = first;
                head(nh);
            }
        };
        if (trips > 0) {
            head(h0);
            issue(0);
        }
        int i0 = first - QT, ch = h0;  // of the tile at hand
        float lam = -uniform_float((float)((const T *)a.lam)[h0]);
        for (int t = 0; t < trips; ++t) {
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
            if (t + 1 < trips)
                issue(buf ^ 1);
            const bool tail = i0 + QT > nq;
            if (tail) {  // rows past the sequence
                clear_rows<T, 2 * DP, QT, kAttnWaves>(qb, (1ull << (nq - i0)) - 1);
                clear_rows<T, DVP, QT, kAttnWaves>(gb, (1ull << (nq - i0)) - 1);
                __syncthreads();
            }
            if (wany && i0 + QT > wfirst) {
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
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int x = 0; x < S::CK; ++x)
                        mma<T>(s[m], RK::row_chunk(qr, 0, m * S::CK + x), kf[m][x]);
#pragma unroll
                for (int x = 0; x < S::CV; ++x)
                    if constexpr (S::kKeepValues)
                        mma<T>(dp, RV::row_chunk(gr, 0, x), RV::row_chunk(vr, 0, x));
                    else
                        mma<T>(dp, RV::row_chunk(gr, 0, x), memory_chunk<T, WIDE>(vrow, x, a.dim_v, seen));
                if (!all || i0 < wfirst + 31 || tail) {
                    const int lim = from - i0 - 4 * (l >> 5), rows = nq - i0 - 4 * (l >> 5);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool see = 8 * (r >> 2) + (r & 3) >= lim && 8 * (r >> 2) + (r & 3) < rows;
                        s[0][r] = see ? s[0][r] : -INFINITY;
                        s[1][r] = see ? s[1][r] : -INFINITY;
                    }
                }
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
                    wf[x] = operand<T>(wt, x);
                    if constexpr (!std::is_same<T, f16>::value) {
                        ds[0][x] = operand<T>(s[0], x);
                        ds[1][x] = operand<T>(s[1], x);
                    }
                }
                if constexpr (std::is_same<T, f16>::value) {
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
                    for (int v = 0; v < S::TV; ++v)
                        mma<T>(gv[v], RV::col_chunk(gc, 0, x, 32 * v), wf[x]);
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int v = 0; v < S::TK; ++v)
                            mma<T>(gk[m][v], RK::col_chunk(qc, 0, x, m * DP + 32 * v), ds[m][x]);
                }
            }
        }
        __syncthreads();
        if (j >= a.len_k)
            continue;
        const int64_t row = ((int64_t)b * a.len_k + j) * heads + hx;
        auto put = [&](auto *to, const f32x16 &x, int v, int dim, float f) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float y[4] = {x[4 * g] * f, x[4 * g + 1] * f, x[4 * g + 2] * f, x[4 * g + 3] * f};
                store4<std::remove_reference_t<decltype(*to)>, WIDE>(to, 32 * v + 8 * g + 4 * (l >> 5), dim, y);
            }
        };
        const float fv = __builtin_amdgcn_exp2f(-lift), fk = a.scale * range.down() * fv;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int v = 0; v < S::TK; ++v) {
                if (a.parts)
                    put(a.parts + (row * 2 + m) * a.dim, gk[m][v], v, a.dim, fk);
                else
                    put((T *)a.gk + (row * 2 + m) * a.dim, gk[m][v], v, a.dim, fk);
            }
#pragma unroll
        for (int v = 0; v < S::TV; ++v) {
            if (a.parts)
                put(a.parts + a.parts_v + row * a.dim_v, gv[v], v, a.dim_v, fv);
            else
                put((T *)a.gv + row * a.dim_v, gv[v], v, a.dim_v, fv);
        }
    }
}

// Sums of the heads' parts of a key head, in order, and of grad_lambda's rows.
// Blocks up to `heads` take one lambda each, the others the parts.
template <class T>
__global__ __launch_bounds__(kAttnThreads) void k_attn_finish(AttnArgs a)
{
    if ((int)blockIdx.x < a.heads) {
        __shared__ float s[kAttnWaves];
        const int h = blockIdx.x;
        float y = 0.0f;
        for (int b = 0; b < a.batch; ++b) {
            const float *x = a.dlam + ((int64_t)b * a.heads + h) * a.len_q;
            for (int i = threadIdx.x; i < a.len_q; i += kAttnThreads)
                y += x[i];
        }
        y = lanes_sum<64>(y);
        if (lane_id() == 0)
            s[threadIdx.x >> 6] = y;
        __syncthreads();
        if (threadIdx.x == 0)
            ((T *)a.glam)[h] = (T)(-(((s[0] + s[1]) + s[2]) + s[3]));
        return;
    }
    const int64_t rows = (int64_t)a.batch * a.len_k * a.kv_heads;
    const int wk = 2 * a.dim, wv = a.dim_v;
    const int64_t nk = rows * wk, total = nk + rows * wv;
    for (int64_t e = (int64_t)(blockIdx.x - a.heads) * kAttnThreads + threadIdx.x; e < total;
         e += (int64_t)(gridDim.x - a.heads) * kAttnThreads) {
        const bool key = e < nk;
        const int64_t x = key ? e : e - nk;
        const int width = key ? wk : wv;
        const int64_t row = x / width;
        const int ch = (int)(x - row * width);
        const float *p = a.parts + (key ? 0 : a.parts_v) + row * a.group * width + ch;
        float y = 0.0f;
        for (int g = 0; g < a.group; ++g)
            y += p[(int64_t)g * width];
        ((T *)(key ? a.gk : a.gv))[x] = (T)y;
    }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

// blocks of a launch: fewer than 2^32 work items, the rest in turns
inline unsigned item_blocks(int64_t items) { return (unsigned)std::min<int64_t>(items, 1 << 23); }

template <class K>
hipError_t launch_lds(K kernel, unsigned blocks, int lds, const AttnArgs &a, hipStream_t s)
{
    if (lds > (64 << 10)) {
        const hipError_t e =
            hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kAttnThreads), lds, s, a);
    return hipGetLastError();
}

template <class T, int DP, int DVP, bool WIDE>
hipError_t fwd_class(const AttnArgs &a, hipStream_t s)
{
    using S = Sizes<T, DP, DVP>;
    const int64_t items = (int64_t)((a.len_q + kBlockRows - 1) / kBlockRows) * a.heads * a.batch;
    return launch_lds(k_attn_fwd<T, DP, DVP, WIDE>, item_blocks(items), 2 * S::kKeyTile, a, s);
}

template <class T, int DP, int DVP, bool WIDE>
hipError_t bwd_class(const AttnArgs &a, hipStream_t s)
{
    using S = Sizes<T, DP, DVP>;
    hipError_t e = hipSuccess;
    const int64_t rows = (int64_t)((a.len_q + kBlockRows - 1) / kBlockRows) * a.heads * a.batch;
    if (rows)
        e = launch_lds(k_attn_dq<T, DP, DVP, WIDE>, item_blocks(rows), 2 * S::kKeyTile, a, s);
    const int64_t keys = (int64_t)((a.len_k + kBlockRows - 1) / kBlockRows) * (a.parts ? a.heads : a.kv_heads) * a.batch;
    if (e == hipSuccess && keys)
        e = launch_lds(k_attn_dkv<T, DP, DVP, WIDE>, item_blocks(keys), 2 * S::kQueryTile + S::kValues, a, s);
    return e;
}

// The class is the smallest that holds both head sizes.
template <class F>
hipError_t with_class(const AttnArgs &a, const F &f)
{
    using std::integral_constant;
    if (a.dim <= 32 && a.dim_v <= 64)
        return f(integral_constant<int, 32>(), integral_constant<int, 64>());
    if (a.dim <= 64 && a.dim_v <= 128)
        return f(integral_constant<int, 64>(), integral_constant<int, 128>());
    return f(integral_constant<int, 128>(), integral_constant<int, 256>());
}

template <class T>
hipError_t attn_fwd(const AttnArgs &a, bool wide, hipStream_t s)
{
    return with_class(a, [&](auto d, auto dv) {
        return wide ? fwd_class<T, d, dv, true>(a, s) : fwd_class<T, d, dv, false>(a, s);
    });
}

template <class T>
hipError_t attn_bwd(const AttnArgs &a, bool wide, hipStream_t s)
{
    const hipError_t e = with_class(a, [&](auto d, auto dv) {
        return wide ? bwd_class<T, d, dv, true>(a, s) : bwd_class<T, d, dv, false>(a, s);
    });
    if (e != hipSuccess)
        return e;
    const int64_t sums = a.parts ? (int64_t)a.batch * a.len_k * a.kv_heads * (2 * a.dim + a.dim_v) : 0;
    const unsigned blocks = (unsigned)std::min<int64_t>((sums + kAttnThreads - 1) / kAttnThreads, 4096);
    hipLaunchKernelGGL(k_attn_finish<T>, dim3(a.heads + blocks), dim3(kAttnThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

}  // namespace pam
