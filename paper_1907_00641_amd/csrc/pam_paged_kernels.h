// Kernels of attention over a paged cache for one element type of queries
// (included by one source file per type, so that they compile side by side).
//
// The queries of all heads of a key head, and both maps of differential
// attention, are the rows of one tile of 32: a row of map m is padded with zeros to
// the channels of both maps' keys, so that one product forms every row's scores
// with its own map, and both maps meet the values in one product.
//   s_rj = scale <q_r, number_j> kscale_j,   p_rj = softmax over the keys that r sees,
//   o_r = sum_j p_rj vscale_j number_j,      out = o, or o^0 - lambda o^1.
// Scores are formed transposed, as in pam_attn_kernels.h: a lane holds one row.
#pragma once

#include "pam_attn_common.h"
#include "pam_paged.h"
#include "pam_store.h"

namespace pam {

namespace {

constexpr int kPagedWaves = 4;
constexpr int kPagedLeast = 2;  // tiles of 32 keys that a wave of a part has at the least

template <class T, int C>
struct PagedSizes {
    using R = Rows<T, C>;
    static constexpr int CK = C / kChunk<T>, TV = C / 32, CP = 32 / kChunk<T>;
    static constexpr int kTile = R::size(32);
    static constexpr int kScales = 3 * 32 * 4;   // of a tile: both maps' keys, values
    // waves per SIMD that the registers are for
    static constexpr int kWavesPerSimd = C == 256 || (sizeof(T) == 4 && C == 128) ? 1 : 2;
    // LDS of a wave: its tile, or its sums of `live` rows; its scales, or tops and sums
    static constexpr int wave_bytes(int live) { return std::max(kTile, live * C * 4); }
    static constexpr int bytes(int live) { return kPagedWaves * (wave_bytes(live) + kScales); }
};

// A tile's rows on their way from the pool, in registers: pieces of PE elements, read in
// accesses of up to 16 bytes from wherever there is a row (rows that there are not, and channels
// past a row's, repeat others and are cleared on their way to LDS); PE 0: pieces of
// eight, element by element.
template <class T, class S, int C, int PE>
struct Staged {
    static constexpr int E = PE ? PE : 8, kPer = C / E, N = C / (2 * E);  // pieces of a row, of a lane
    static constexpr int kWords = E * sizeof(S) / 4;
    uint32_t x[N][kWords], live;  // live: bit n: piece n is a row's
    __device__ __forceinline__ static int row_of(int n) { return n * (64 / kPer) + lane_id() / kPer; }
    __device__ __forceinline__ static int channel() { return lane_id() % kPer * E; }
    // rows of `dim` elements from `pool`; lane j has the number of row j of the tile,
    // negative: there is none
    __device__ __forceinline__ void load(const S *pool, int rid, int dim)
    {
        const int c = channel();
        live = 0;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int r = __shfl(rid, row_of(n));
            live |= (r >= 0 && c < dim ? 1u : 0u) << n;
            if constexpr (PE != 0) {
                const S *p = pool + (int64_t)max(r, 0) * dim + min(c, dim - E);
                __builtin_memcpy(x[n], __builtin_assume_aligned(p, sizeof(x[n]) > 16 ? 16 : sizeof(x[n])), sizeof(x[n]));
            } else {
                const Stored8<S> y = load_stored_some(pool + (int64_t)r * dim + c, r >= 0 ? max(min(dim - c, 8), 0) : 0);
#pragma unroll
                for (int i = 0; i < kWords; ++i)
                    x[n][i] = y.w[i];
            }
        }
    }
    // to the tile, as T
    __device__ __forceinline__ void put(char *tile)
    {
        using R = typename PagedSizes<T, C>::R;
        if (__any(live != (1u << N) - 1)) {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < kWords; ++i)
                    x[n][i] = live >> n & 1 ? x[n][i] : 0;
        }
        const int c = channel();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int row = row_of(n);
            uint32_t y[E * sizeof(T) / 4];
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                if constexpr (kScaled<S>) {
                    uint32_t z[sizeof(T)];
                    widen<T, S>(x[n][i], z);
#pragma unroll
                    for (int k = 0; k < (int)sizeof(T); ++k)
                        y[i * sizeof(T) + k] = z[k];
                } else {
                    y[i] = x[n][i];
                }
            }
#pragma unroll
            for (int i = 0; i < E * (int)sizeof(T) / 16; ++i)
                store16(tile + R::at(row, c * (int)sizeof(T) / 16 + i), uint4v{y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]});
        }
    }
};

// Sums of waves or parts p < n of one row, relative to the largest top: a part that
// saw nothing has the sum 0; one whose top is -inf and whose sum is not 0 has a NaN.
struct Joined {
    float top, sum;
    float4v o;
};
template <class GetStats, class GetSums>
__device__ __forceinline__ Joined joined(int n, const GetStats &stats, const GetSums &sums)
{
    Joined r = {-INFINITY, 0.0f, {}};
    for (int p = 0; p < n; ++p) {
        const float2 st = stats(p);
        r.top = st.y != 0.0f ? __builtin_fmaxf(r.top, st.x) : r.top;
    }
#pragma unroll 4
    for (int p = 0; p < n; ++p) {
        const float2 st = stats(p);
        const float4v x = sums(p);
        const float f = st.y == 0.0f ? 0.0f : (st.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.x - r.top));
        r.sum += f * st.y;
        r.o += f * x;
    }
    return r;
}

// Four channels of an output row from its maps' rows.
template <class T, class GetRow>
__device__ __forceinline__ void paged_out(const PagedArgs &a, int b, int hk, int x, int ch, const GetRow &row)
{
    const int g = x / a.len_q, i = x - g * a.len_q, h = hk * a.group + g;
    float y[4];
    const Joined r0 = row(x * a.pool.maps);
    const float i0 = r0.sum != 0.0f ? 1.0f / r0.sum : 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        y[j] = r0.o[j] * i0;
    if (a.pool.maps == 2) {
        const Joined r1 = row(x * 2 + 1);
        const float i1 = r1.sum != 0.0f ? 1.0f / r1.sum : 0.0f, lam = (float)((const T *)a.lam)[h];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            y[j] -= lam * (r1.o[j] * i1);
    }
    T *out = (T *)a.out + (((int64_t)b * a.len_q + i) * a.heads + h) * a.pool.dim_v;
    if (a.pool.dim_v % 4 == 0 && (uintptr_t)a.out % 16 == 0)
        store4<T, true>(out, ch, a.pool.dim_v, y);
    else
        store4<T, false>(out, ch, a.pool.dim_v, y);
}

// How the blocks of a head's tile of rows are shared among the sequences: `shares` blocks,
// so many to a sequence as its keys take in runs of one length, the shortest that the blocks
// suffice for; a sequence to a lane.  More than 64 sequences: as many to each.  (16 sequences of
// half to all of 16384 keys: 94 us for 97 with as many to each, before the values' fp16 scales.)
struct Shares {
    int n, first;  // of this lane's sequence (up to 64 sequences): blocks, and the first of them
    bool equal;
    int each;
    __device__ __forceinline__ explicit Shares(const PagedArgs &a)
    {
        const int B = a.pool.sequences, shares = B * a.parts;
        equal = B > 64 || a.parts == 1;
        each = a.parts;
        n = first = 0;
        if (equal)
            return;
        const int l = lane_id(), t = l < B ? (cached(a.pool, l) + 31) / 32 : 0;
        // blocks at runs of s tiles: the quotient rounded up, exactly
        auto blocks = [&](int s) {
            int k = (int)((float)t * (1.0f / (float)s));
            k += (int64_t)k * s < t;
            k += (int64_t)k * s < t;
            k -= (int64_t)(k - 1) * s >= t;
            k -= (int64_t)(k - 1) * s >= t;
            return l < B ? max(k, 1) : 0;
        };
        // Runs of all / (shares - B) tiles always suffice: each sequence has less than a block
        // more than its tiles over that.  Shorter ones than all / shares do not.  (Sums in 32
        // bits are off by a relative 2^-21 at the most.)
        const float all = lanes_sum<64>((float)t);
        const int least = kPagedLeast * kPagedWaves;
        int lo = max((int)uniform_float(all / (float)shares), least) - 1;
        int hi = max((int)uniform_float(__builtin_ceilf(all / (float)(shares - B) * (1.0f + 0x1p-20f))) + 1, lo + 1);
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (uniform_float(lanes_sum<64>((float)blocks(mid))) <= (float)shares)
                hi = mid;
            else
                lo = mid;
        }
        n = blocks(hi);
        int upto = n;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int x = __shfl_up(upto, s);
            upto += l >= s ? x : 0;
        }
        first = upto - n;
    }
    // the sequence of block r, its part and their number; -1: none
    __device__ __forceinline__ int find(int r, int &part, int &parts) const
    {
        if (equal) {
            const int b = r / each;
            part = r - b * each;
            parts = each;
            return b;
        }
        const uint64_t one = __ballot(r >= first && r < first + n);
        if (!one)
            return -1;
        const int b = __builtin_ctzll(one);
        part = r - uniform(__shfl(first, b));
        parts = uniform(__shfl(n, b));
        return b;
    }
};

// A block takes a part of the keys of a unit (32 rows of one key head of one
// sequence), and every wave a run of tiles of 32 keys of it.  A tile is brought from
// its pages to registers while the one before is worked on, turned into the
// queries' type on its way to LDS (e4m3 and int8 numbers are exact there), and
// read as operands from there: the values straight after the keys, in the same
// place.  The waves meet in LDS at the end.  Bound by the cache's bytes: 16 sequences of up to
// 16384 keys, 32 heads of 128 over 8, e4m3 numbers, 97 us with the join, 89 us at a large copy's
// rate; 8 x 4 tokens, 2 maps of 64, int8, up to 9000 keys, 24 us for 13, which is the start, the walk's
// first loads and the end of a walk of a few tiles.
template <class T, class S, int C, int PE>
__global__ __launch_bounds__(64 * kPagedWaves, (PagedSizes<T, C>::kWavesPerSimd)) void k_paged(PagedArgs a)
{
    using Z = PagedSizes<T, C>;
    using R = typename Z::R;
    // Numbers of 8 bits are exact in fp16, whose 11 bits leave next to nothing of a probability
    // beside a bf16 result.  It has no range for a probability times a scale, so that scales go
    // in relative to a power of two above the largest so far, and the sums follow when it grows
    // (what is below 2^-20 of the largest product loses precision, at most 2^-31 of it each).
    // Otherwise probabilities enter their product as two operands, so that the result alone is
    // rounded (with one, out is off by 1.3 to 1.6 times as much as by its own rounding; e4m3
    // with bf16 as two operands instead: 114 us for 94, 16 x 16384).
    constexpr bool kRelative = kScaled<S> && sizeof(T) == 2;
    constexpr bool kTwo = sizeof(T) == 2 && !(kScaled<S> && std::is_same<T, bf16>::value);
    typedef typename std::conditional<kRelative, f16, T>::type VT;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id();
    const float c = a.scale * kLog2e;
    const int stride = Z::wave_bytes(a.live);
    char *tile = lds + w * stride;
    float *scales = reinterpret_cast<float *>(lds + kPagedWaves * stride + w * Z::kScales);
    const uint32_t kr = lds_address(tile) + R::row_lane(), vc = lds_address(tile) + R::col_lane();
    const uint32_t items = (uint32_t)a.units * a.parts, heads = a.pool.kv_heads * a.tiles;
    const Shares shares(a);
    for (uint32_t n = blockIdx.x; n < items; n += gridDim.x) {
        const uint32_t share = uniform(n / heads), head = n - share * heads;
        int part, parts;
        const int b = uniform(shares.find(share, part, parts));
        if (b < 0)  // the same in the whole block
            continue;
        const int hk = uniform(head / a.tiles), rt = head - hk * a.tiles;
        const int nk = a.pool.pages ? uniform(cached(a.pool, b)) : 0;
        const int nq = uniform(a.q_len ? min(max(a.q_len[b], 0), a.len_q) : a.len_q);
        // this lane's row
        const int r = rt * 32 + (l & 31), x = r / a.pool.maps, m = r - x * a.pool.maps;
        const int g = x / a.len_q, i = x - g * a.len_q, h = hk * a.group + g;
        const bool in = r < a.rows && i < nq;
        const int limit = in ? max(min(nk, i + nk - nq + 1), 0) : 0;
        int wend = limit, wall = r < a.rows ? limit : nk;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            wend = max(wend, __shfl_xor(wend, s));
            wall = min(wall, __shfl_xor(wall, s));
        }
        wend = uniform(wend);
        wall = uniform(wall);
        int from, to;
        {
            const int trips = (wend + 31) / 32, runs = parts * kPagedWaves, per = trips / runs, more = trips - per * runs;
            const int run = part * kPagedWaves + w;  // runs differ by a tile at the most
            from = uniform(run * per + min(run, more));
            to = uniform(from + per + (run < more));
        }

        Staged<T, S, C, PE> ks;
        Staged<VT, S, C, PE> vs;
        int rid = -1, next = -1;          // rows of the tile under way, and of the one after
        float sk0 = 0.0f, sk1 = 0.0f, sv = 0.0f;
        auto find = [&](int t) {          // lane j: row of key j of tile t
            const int j = t * 32 + (l & 31);
            return j < wend ? cache_row(a.pool, a.by_page, b, hk, j) : -1;
        };
        auto fetch_keys = [&]() {
            ks.load((const S *)a.pool.k, rid, a.pool.maps * a.pool.dim);
            if constexpr (kScaled<S>) {
                const int64_t at = max(rid, 0);
                sk0 = rid < 0 ? 0.0f : a.pool.ks[at * a.pool.maps];
                sk1 = rid < 0 || a.pool.maps == 1 ? 0.0f : a.pool.ks[at * 2 + 1];
                sv = rid < 0 ? 0.0f : a.pool.vs[at];
            }
        };
        if (from < to) {
            rid = find(from);
            fetch_keys();
            if (from + 1 < to)
                next = find(from + 1);
            vs.load((const S *)a.pool.v, rid, a.pool.dim_v);
        }
        // the row as an operand, 0 outside its map's channels
        uint4v q[Z::CK];
        {
            constexpr int per = 16 / sizeof(T);
            const T *row = (const T *)a.q + b * a.qs[0] + i * a.qs[1] + h * a.qs[2] + m * a.qs[3];
#pragma unroll
            for (int s = 0; s < Z::CK; ++s) {
                const int ch = s * kChunk<T> + (l >> 5) * per - m * a.pool.dim;
                q[s] = uint4v{0, 0, 0, 0};
                if (a.q_wide) {
                    if (in && ch >= 0 && ch < a.pool.dim)
                        q[s] = load16(row + ch);
                } else {
                    T y[per];
#pragma unroll
                    for (int j = 0; j < per; ++j)
                        y[j] = in && ch + j >= 0 && ch + j < a.pool.dim ? row[ch + j] : (T)0.0f;
                    __builtin_memcpy(&q[s], y, 16);
                }
            }
        }
        f32x16 o[Z::TV] = {};
        float top = -INFINITY, sum = 0.0f;
        int unit_exp = -126;  // scales of values are in units of 2^unit_exp
        for (int t = from; t < to; ++t) {
            const uint32_t seen = (uint32_t)__ballot(rid >= 0);
            ks.put(tile);
            if constexpr (kRelative) {
                float most = sv;
                most = __builtin_fmaxf(most, lane_move<0xb1>(most));
                most = __builtin_fmaxf(most, lane_move<0x4e>(most));
                most = __builtin_fmaxf(most, lane_move<0x141>(most));
                most = __builtin_fmaxf(most, lane_move<0x140>(most));
                const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(most), __float_as_uint(most), false, false);
                most = __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
                // most < 2^e.  By the exponent's bits: a tile that has no scale, without a page or of zeros, is
                // at the lowest and leaves the unit as it is.
                const int e = min((int)((uint32_t)uniform(__float_as_int(most)) >> 23) - 126, 127);
                if (e > unit_exp) {
                    const float f = __builtin_ldexpf(1.0f, max(unit_exp - e, -200));
#pragma unroll
                    for (int v = 0; v < Z::TV; ++v)
                        o[v] *= f;
                    unit_exp = e;
                }
                sv = __builtin_ldexpf(sv, -unit_exp);
            }
            if constexpr (kScaled<S>) {
                if (l < 32) {
                    scales[l] = sk0;
                    scales[32 + l] = sk1;
                    scales[64 + l] = sv;
                }
            }
            wave_fence();
            const int after = rid = next;
            if (t + 1 < to) {
                fetch_keys();
                next = t + 2 < to ? find(t + 2) : -1;
            }
            f32x16 s = {};
#pragma unroll
            for (int k = 0; k < Z::CK; ++k)
                mma<T>(s, R::row_chunk(kr, 0, k), q[k]);
            if constexpr (kScaled<S>) {
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float4v f = *reinterpret_cast<const float4v *>(scales + m * 32 + 8 * y + 4 * (l >> 5));
#pragma unroll
                    for (int z = 0; z < 4; ++z)
                        s[4 * y + z] *= f[z];
                }
            }
            if (seen != ~0u || t * 32 + 32 > wall) {
                const uint32_t bits = (seen & low_bits(limit - t * 32)) >> (4 * (l >> 5));
#pragma unroll
                for (int y = 0; y < 16; ++y)
                    s[y] = bits >> (8 * (y >> 2) + (y & 3)) & 1 ? s[y] : -INFINITY;
            }
            float mx = s[0];
#pragma unroll
            for (int y = 1; y < 16; ++y)
                mx = __builtin_fmaxf(mx, s[y]);
            mx *= c;
            if (__any(mx > top + 8.0f)) {  // the maximum is followed only when it grew by more than 2^8
                const float up = __builtin_fmaxf(top, xor32_max(mx));
                const float f = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - up);
                top = up;
                sum *= f;
#pragma unroll
                for (int v = 0; v < Z::TV; ++v)
                    o[v] *= f;
            }
            const float base = top == -INFINITY ? 0.0f : top - kLift<VT>;
            float add = 0.0f;
#pragma unroll
            for (int y = 0; y < 16; ++y) {
                s[y] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y], c, -base));
                add += s[y];
            }
            sum += add;
            if constexpr (kScaled<S>) {
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float4v f = *reinterpret_cast<const float4v *>(scales + 64 + 8 * y + 4 * (l >> 5));
#pragma unroll
                    for (int z = 0; z < 4; ++z)
                        s[4 * y + z] *= f[z];
                }
            }
            uint4v p[Z::CP], low[Z::CP];
#pragma unroll
            for (int k = 0; k < Z::CP; ++k) {
                if constexpr (kTwo)
                    operands<VT>(s, k, p[k], low[k]);
                else
                    p[k] = operand<VT>(s, k);
            }
            wave_fence();  // the keys are read
            vs.put(tile);
            wave_fence();
            if (t + 1 < to)
                vs.load((const S *)a.pool.v, after, a.pool.dim_v);
#pragma unroll
            for (int k = 0; k < Z::CP; ++k)
#pragma unroll
                for (int v = 0; v < Z::TV; ++v) {
                    const uint4v vf = R::col_chunk(vc, 0, k, 32 * v);
                    mma<VT>(o[v], vf, p[k]);
                    if constexpr (kTwo)
                        mma<VT>(o[v], vf, low[k]);
                }
            wave_fence();  // the values are read
        }
        sum = xor32_add(sum);
        if constexpr (kRelative) {
            const float f = __builtin_ldexpf(1.0f, unit_exp);
#pragma unroll
            for (int v = 0; v < Z::TV; ++v)
                o[v] *= f;
        }
        // [row][channel] of this wave where its tile was, tops and sums where its scales were
        float *mine = reinterpret_cast<float *>(tile);
        if ((l & 31) < a.live) {
#pragma unroll
            for (int v = 0; v < Z::TV; ++v)
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    *reinterpret_cast<float4v *>(mine + (l & 31) * C + 32 * v + 8 * y + 4 * (l >> 5)) =
                        sum != 0.0f ? float4v{o[v][4 * y], o[v][4 * y + 1], o[v][4 * y + 2], o[v][4 * y + 3]} : float4v{};
            if (l < 32)
                *reinterpret_cast<float2 *>(scales + 2 * l) = make_float2(top, sum);
        }
        __syncthreads();
        auto row_at = [&](int row, int ch) {
            return joined(
                kPagedWaves,
                [&](int p) {
                    return *reinterpret_cast<const float2 *>(lds + kPagedWaves * stride + p * Z::kScales + row * 8);
                },
                [&](int p) {
                    return *reinterpret_cast<const float4v *>(reinterpret_cast<const float *>(lds + p * stride) + row * C + ch);
                });
        };
        const int rows = min(a.rows - rt * 32, 32);
        if (parts == 1) {
            const int outs = rows / a.pool.maps;
            for (int e = threadIdx.x; e < outs * (C / 4); e += 64 * kPagedWaves) {
                const int ch = e % (C / 4) * 4;
                if (ch < a.pool.dim_v)
                    paged_out<T>(a, b, hk, rt * 32 / a.pool.maps + e / (C / 4), ch,
                                 [&](int row) { return row_at(row - rt * 32, ch); });
            }
        } else {
            const int64_t at = (int64_t)n * a.live;
            for (int e = threadIdx.x; e < rows * (C / 4); e += 64 * kPagedWaves) {
                const int row = e / (C / 4), ch = e % (C / 4) * 4;
                const Joined j = row_at(row, ch);
                *reinterpret_cast<float4v *>(a.part + (at + row) * C + ch) = j.o;
                if (ch == 0)
                    *reinterpret_cast<float2 *>(a.part + (int64_t)items * a.live * C + (at + row) * 2) =
                        make_float2(j.top, j.sum);
            }
        }
        // for the join: the unit's first block and their number
        if (a.parts > 1 && part == 0 && threadIdx.x == 0)
            a.cuts[(uint32_t)b * heads + head] = make_int2(share, parts);
        __syncthreads();
    }
}

// Joins the parts of the units that have several: a block per output row, its threads in
// teams that take every so-manieth part of four channels each.  What bounds it is the loads'
// latency: four parts of both maps are under way together.
constexpr int kJoinThreads = 1024;  // the most

template <class T, int C>
__global__ __launch_bounds__(kJoinThreads) void k_paged_join(PagedArgs a)
{
    constexpr int QUADS = C / 4, MOST = kJoinThreads / QUADS, AHEAD = 4;
    __shared__ float2 s[2][MOST];
    __shared__ float4v so[2][MOST][QUADS];
    const int teams = blockDim.x / QUADS, team = threadIdx.x / QUADS, quad = threadIdx.x % QUADS, ch = quad * 4;
    const int maps = a.pool.maps;
    const float2 *stats = reinterpret_cast<const float2 *>(a.part + (int64_t)a.units * a.parts * a.live * C);
    const uint32_t per = a.live / maps, heads = a.pool.kv_heads * a.tiles;  // per: output rows of a unit
    const uint32_t rows = (uint32_t)a.units * per;
    for (uint32_t e = blockIdx.x; e < rows; e += gridDim.x) {
        const uint32_t unit = e / per, b = unit / heads, head = unit - b * heads;
        const int hk = head / a.tiles, rt = head - hk * a.tiles;
        const int x = rt * 32 / maps + (e - unit * per);
        const int2 cut = a.cuts[unit];
        const int from = cut.x, parts = cut.y;
        if (x * maps >= a.rows || parts == 1)  // the same in every thread
            continue;
        float top[2] = {-INFINITY, -INFINITY}, sum[2] = {};
        float4v o[2] = {};
        for (int p0 = team; p0 < parts; p0 += AHEAD * teams) {
            float2 st[AHEAD][2];
            float4v y[AHEAD][2];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int p = min(p0 + k * teams, parts - 1);
                const int64_t at = ((int64_t)(from + p) * heads + head) * a.live + x * maps - rt * 32;
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const int64_t row = at + (m < maps ? m : 0);
                    st[k][m] = stats[row];
                    y[k][m] = *reinterpret_cast<const float4v *>(a.part + row * C + ch);
                }
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    if (p0 + k * teams >= parts || st[k][m].y == 0.0f)  // saw nothing
                        continue;
                    // a top of -inf beside a sum that is not 0: a NaN
                    const float to = __builtin_fmaxf(top[m], st[k][m].x);
                    const float f0 = top[m] == -INFINITY ? (sum[m] == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(top[m] - to);
                    const float f1 = st[k][m].x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st[k][m].x - to);
                    o[m] = o[m] * f0 + y[k][m] * f1;
                    sum[m] = sum[m] * f0 + st[k][m].y * f1;
                    top[m] = to;
                }
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            if (quad == 0)
                s[m][team] = make_float2(top[m], sum[m]);
            so[m][team][quad] = o[m];
        }
        __syncthreads();
        if (team == 0 && ch < a.pool.dim_v)
            paged_out<T>(a, b, hk, x, ch, [&](int row) {
                const int m = row - x * maps;
                return joined(
                    min(teams, parts), [&](int p) { return s[m][p]; }, [&](int p) { return so[m][p][quad]; });
            });
    }
}

template <class T, class S, int C, int PE>
hipError_t paged_launch(const PagedArgs &a, hipStream_t s)
{
    using Z = PagedSizes<T, C>;
    hipError_t e = launch_lds<k_paged<T, S, C, PE>>(item_blocks((int64_t)a.units * a.parts), 64 * kPagedWaves,
                                                    Z::bytes(a.live), a, s);
    if (e != hipSuccess || a.parts == 1)
        return e;
    const unsigned rows = (unsigned)std::min<int64_t>((int64_t)a.units * (a.live / a.pool.maps), 1 << 23);
    // enough teams for a round or two of the loads
    const int64_t threads = (int64_t)C / 4 * std::max(a.parts / 4, 4);
    hipLaunchKernelGGL((k_paged_join<T, C>), dim3(rows), dim3(threads <= 256 ? 256 : kJoinThreads), 0, s, a);
    return hipGetLastError();
}

template <class T, class S, int PE>
hipError_t paged_class_launch(const PagedArgs &a, hipStream_t s)
{
    switch (paged_class(a.pool.maps * a.pool.dim, a.pool.dim_v)) {
    case 64: return paged_launch<T, S, 64, PE>(a, s);
    case 128: return paged_launch<T, S, 128, PE>(a, s);
    default: return paged_launch<T, S, 256, PE>(a, s);
    }
}

// piece: the elements that every row is whole pieces of: 16 (types of 8 bits), 8, or 0
template <class T, class S>
hipError_t paged_store(const PagedArgs &a, int piece, hipStream_t s)
{
    if constexpr (kScaled<S>) {
        if (piece == 16)
            return paged_class_launch<T, S, 16>(a, s);
    }
    return piece ? paged_class_launch<T, S, 8>(a, s) : paged_class_launch<T, S, 0>(a, s);
}

template <class T>
hipError_t paged_type(const PagedArgs &a, int store, int piece, hipStream_t s)
{
    if (store == PAM_STORE_E4M3)
        return paged_store<T, e4m3>(a, piece, s);
    return store == PAM_STORE_INT8 ? paged_store<T, int8>(a, piece, s) : paged_store<T, T>(a, piece, s);
}

}  // namespace

}  // namespace pam
