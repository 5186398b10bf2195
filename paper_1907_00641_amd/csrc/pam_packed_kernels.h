// Kernels of softmax attention over packed sequences for one element type
// (included by one source file per type, so that they compile side by side).
//
//   s = scale q k^T, p = softmax of s over the keys that are seen, out = p v;
//   D = <dout, out>, dp = dout v^T, ds = scale p (dp - D),
//   dq = ds k, dk = ds^T q, dv = p^T dout.
// A block of four waves takes 128 rows of one head of one sequence (queries; in
// the keys' gradient pass: keys), 32 per wave, and walks over tiles of the other
// axis that the block's loads bring to LDS a tile ahead, straight from memory.  The
// rows' operands stay in registers, and so do the probabilities: scores are formed
// transposed, which makes a lane hold one row, and their layout, rounded, is an
// operand of the next product (pam_attn_tiles.h).
// KS: teams of four waves in a block, which take every KS-th tile of the walk for the same
// rows and meet in LDS.  Two where the card has room for them: a wave alone on its SIMD
// computes its products and its softmax one after the other, two overlap, and the walk is
// half as long.
#pragma once

#include "pam_attn_common.h"
#include "pam_packed.h"

namespace pam {

namespace {

// Sizes of a class of head sizes, keys' and values' channels padded to C.
template <class T, int C>
struct PackedSizes {
    using R = Rows<T, C>;
    static constexpr int kKeys = R::kBytes <= 256 ? 64 : 32;  // keys per tile
    static constexpr int kQueries = R::kBytes <= 128 ? 64 : 32;  // queries per tile of the keys' pass
    static constexpr int CK = C / kChunk<T>, TV = C / 32, CP = 32 / kChunk<T>;
    // waves per SIMD that the registers are for
    static constexpr bool kSmall = sizeof(T) == 2 || C == 64;
    static constexpr int kWavesPerSimd = kSmall ? 2 : 1;
    static constexpr bool kTwoOperands = sizeof(T) == 2 && C == 64;  // dq's score gradients
    static constexpr int kKeyTile = 2 * R::size(kKeys);
    static constexpr int kQueryTile = 2 * R::size(kQueries) + 2 * kQueries * 4;  // queries, dout, two statistics
    static constexpr int kValues = R::size(kPackedRows);                         // the keys' pass: the block's values
    // LDS of a block of KS teams of four waves: two tiles for each; at the end, the sums of all
    // teams but the first
    static constexpr int rows_lds(int ks) { return std::max(2 * ks * kKeyTile, (ks - 1) * kPackedRows * (C * 4 + 8)); }
    static constexpr int keys_lds(int ks)
    {
        return std::max(2 * ks * kQueryTile + kValues, (ks - 1) * kPackedRows * 2 * C * 4);
    }
};

// Sums that two teams of waves hold, a register at a time through LDS: [wave][register / 4][lane].
template <int N>
__device__ __forceinline__ void leave_sums(char *lds, int wave, const f32x16 (&x)[N])
{
#pragma unroll
    for (int v = 0; v < N; ++v)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4v *>(lds + (((wave * N + v) * 4 + g) * 64 + lane_id()) * 16) =
                float4v{x[v][4 * g], x[v][4 * g + 1], x[v][4 * g + 2], x[v][4 * g + 3]};
}
// x = x f + theirs f2
template <int N>
__device__ __forceinline__ void take_sums(const char *lds, int wave, f32x16 (&x)[N], float f, float f2)
{
#pragma unroll
    for (int v = 0; v < N; ++v)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4v y = *reinterpret_cast<const float4v *>(lds + (((wave * N + v) * 4 + g) * 64 + lane_id()) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[v][4 * g + j] = x[v][4 * g + j] * f + y[j] * f2;
        }
}

// A sequence's rows.
struct Sequence {
    int q0, nq, k0, nk;
};
__device__ __forceinline__ void rows_of(const int32_t *start, int total, int b, int &from, int &n)
{
    from = 0;
    n = total;
    if (start) {
        from = min(max(start[b], 0), total);
        n = min(max(start[b + 1], from), total) - from;
    }
}

// tiles of sequence s, 0 past the last
__device__ __forceinline__ int tiles_of(const int32_t *start, int sequences, int total, int s)
{
    int from, n = 0;
    if (s < sequences)
        rows_of(start, total, s, from, n);
    return (n + kPackedRows - 1) / kPackedRows;
}

// Tiles before every sequence and, behind the last one, in all, for places of more than kScanned
// sequences; a block for the queries' and one for the keys'.  Sums stop at 2^30, past every place: only those of
// starts that fall come there.
constexpr int kPlacesThreads = 1024, kPlacesPer = 8;  // sequences of a thread and turn
__global__ __launch_bounds__(kPlacesThreads) void k_packed_places(PackedArgs a)
{
    __shared__ uint32_t wave[kPlacesThreads / 64];
    const bool key = blockIdx.x;
    const int32_t *start = key ? a.k_start : a.q_start;
    const int total = key ? a.keys : a.tokens, l = lane_id(), w = wave_id();
    uint32_t *upto = key ? a.k_places : a.q_places;
    auto add = [](uint32_t x, uint32_t y) { return min(x + y, 1u << 30); };
    uint32_t past = 0;
    for (int s0 = 0; s0 < a.sequences; s0 += kPlacesThreads * kPlacesPer) {
        const int s = s0 + threadIdx.x * kPlacesPer;
        uint32_t t[kPlacesPer], sum = 0;
#pragma unroll
        for (int j = 0; j < kPlacesPer; ++j) {
            t[j] = tiles_of(start, a.sequences, total, s + j);
            sum = add(sum, t[j]);
        }
        uint32_t before = sum;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
            const uint32_t y = __shfl_up(before, x);
            before = l >= x ? add(before, y) : before;
        }
        __syncthreads();  // the turn before is done with the waves' sums
        if (l == 63)
            wave[w] = before;
        const uint32_t lane = __shfl_up(before, 1);
        __syncthreads();
        before = past;
        for (int x = 0; x < kPlacesThreads / 64; ++x) {
            before = x < w ? add(before, wave[x]) : before;
            past = add(past, wave[x]);
        }
        before = l > 0 ? add(before, lane) : before;
#pragma unroll
        for (int j = 0; j < kPlacesPer; ++j) {
            if (s + j < a.sequences)
                upto[s + j] = before;
            before = add(before, t[j]);
        }
    }
    if (threadIdx.x == 0)
        upto[a.sequences] = past;
}

// Which tile a place holds.  Up to 64 sequences: the longest first (tiles in the order
// of how many their sequence has before them: a causal query tile walks over so many
// keys), a sequence to a lane; the number of tiles with `t` or more before them
// falls with t, which is found by halving.  More sequences: one after the other, up to
// kScanned of them in runs of 64 from the first on, and still more among `upto` (k_packed_places), which 64 lanes cut in 64 at
// a time.  Scanned, and with places (causal, 8 heads of 64, bf16, forward and backward): 128 sequences of 128 tokens 22 and 71 us
// for 27 and 78, 300 49 and 170 for 49 and 162, 512 89 and 342 for 75 and 289, 4096 2219 and 6175 for 698 and 2235. The
// search of all blocks grows with the square of the sequences where each starts at the first.
// RANK: as many tiles before it in its sequence, of `tiles`.
struct Place {
    int b = -1, rank = 0, tiles = 0;
    __device__ __forceinline__ Place(const int32_t *start, const uint32_t *upto, int sequences, int total, uint32_t slot)
    {
        const int l = lane_id();
        if (sequences == 1) {
            tiles = tiles_of(start, sequences, total, 0);
            rank = tiles - 1 - (int)slot;
            b = rank >= 0 ? 0 : -1;
        } else if (sequences <= 64) {
            const int t = tiles_of(start, sequences, total, l);
            // sums of at most 2^24 tiles are exact in 32 bits
            auto before = [&](int x) { return (uint32_t)uniform((int)lanes_sum<64>((float)max(t - x, 0))); };
            int most = t;
#pragma unroll
            for (int s = 1; s < 64; s <<= 1)
                most = max(most, __shfl_xor(most, s));
            most = uniform(most);
            if (slot >= before(0))
                return;
            int lo = 0, hi = most;
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (before(mid) > slot)
                    lo = mid;
                else
                    hi = mid;
            }
            const uint64_t has = __ballot(t > lo);
            const int at = (int)(slot - before(hi)), mine = __builtin_amdgcn_mbcnt_hi(
                (uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0));
            const uint64_t one = __ballot(t > lo && mine == at);
            if (!one)  // starts that fall: the sums need not be exact
                return;
            b = __builtin_ctzll(one);
            rank = lo;
            tiles = uniform(__shfl(t, b));
        } else if (!upto) {
            uint32_t past = 0;
            for (int s0 = 0; s0 < sequences; s0 += 64) {
                const int t = tiles_of(start, sequences, total, s0 + l);
                uint32_t to = t;
#pragma unroll
                for (int s = 1; s < 64; s <<= 1) {
                    const uint32_t x = __shfl_up(to, s);
                    to += l >= s ? x : 0;
                }
                const uint64_t reach = __ballot(past + to > slot);
                if (reach) {
                    const int at = __builtin_ctzll(reach);
                    b = s0 + at;
                    tiles = uniform(__shfl(t, at));
                    rank = uniform((int)(past + __shfl(to, at) - 1 - slot));
                    return;
                }
                past += uniform((int)__shfl(to, 63));
            }
        } else {
            if (slot >= (uint32_t)uniform((int)upto[sequences]))
                return;
            int lo = 0, n = sequences;  // upto[lo] <= slot < upto[lo + n]
            while (n > 1) {
                const int step = (n + 63) / 64, at = l * step;
                const int last = __popcll(__ballot(at < n && upto[lo + min(at, n - 1)] <= slot)) - 1;
                lo = uniform(lo + last * step);
                n = uniform(min(step, n - last * step));
            }
            b = lo;
            tiles = uniform(tiles_of(start, sequences, total, b));
            rank = uniform((int)upto[b]) + tiles - 1 - (int)slot;
        }
    }
};

// A work item: a part of the walk of one tile of one head.  Items come in the order of
// their places, all heads of a place behind each other, so that the longest units are
// the first and eight heads' units, dealt to the eight dies in turn, find their keys in
// their die's L2.  Where two blocks share a CU, the second ones of the first round are
// taken in reverse: the longest unit is paired with the shortest of the round.
struct PackedItem {
    uint32_t unit, slot;  // slot: of the parts' sums, the number of the part
    int part, parts, h;
    Place place;
    __device__ __forceinline__ static uint32_t order(const PackedPlan &p, uint32_t n)
    {
        return n >= p.fold && n < 2 * p.fold ? 3 * p.fold - 1 - n : n;
    }
    __device__ __forceinline__ PackedItem(const PackedPlan &p, const int32_t *start, const uint32_t *upto, int sequences,
                                          int total, uint32_t n)
        : PackedItem(p, start, upto, sequences, total, order(p, n), uniform((order(p, n) - p.full) / p.parts))
    {
    }
    __device__ __forceinline__ PackedItem(const PackedPlan &p, const int32_t *start, const uint32_t *upto, int sequences,
                                          int total, uint32_t m, uint32_t cut)
        : unit(m < p.full ? m : p.full + cut), slot(m - p.full), part(m < p.full ? 0 : m - p.full - cut * p.parts),
          parts(m < p.full ? 1 : p.parts), h(0), place(start, upto, sequences, total, uniform(unit / p.heads))
    {
        h = uniform(unit - unit / p.heads * p.heads);
    }
    // the walked tiles of this item, of `trips` of its unit
    __device__ __forceinline__ void range(int trips, int &from, int &to) const
    {
        const int per = trips / parts, more = trips - per * parts;
        from = uniform(part * per + min(part, more));
        to = uniform(from + per + (part < more));
    }
};

// Clears the rows of no sequence: those before the first, and from the last's end on.
template <int KS, class T>
__device__ __forceinline__ void clear_outside(T *rows, const int32_t *start, int sequences, int total, int64_t width)
{
    if (!start)
        return;
    int first, last, n;
    rows_of(start, total, 0, first, n);
    rows_of(start, total, sequences - 1, last, n);
    last += n;
    const int64_t head = first * width, all = head + (int64_t)(total - last) * width;
    for (int64_t e = (int64_t)blockIdx.x * (KS * kAttnThreads) + threadIdx.x; e < all;
         e += (int64_t)gridDim.x * (KS * kAttnThreads))
        rows[e < head ? e : e - head + last * width] = (T)0.0f;
}

// The lowest n of 64 bits.
__device__ __forceinline__ uint64_t low_bits64(int n) { return n >= 64 ? ~0ull : (1ull << max(n, 0)) - 1; }

// Scores of this lane's row to -inf where a bit is 0.  bits: of the tile's 32 rows.
__device__ __forceinline__ void hide_rows(f32x16 &s, uint32_t bits)
{
    bits >>= 4 * (lane_id() >> 5);
#pragma unroll
    for (int r = 0; r < 16; ++r)
        s[r] = bits >> (8 * (r >> 2) + (r & 3)) & 1 ? s[r] : -INFINITY;
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------

// One pass over the keys with the running maximum and sum of the softmax, 4 products of pairs and
// channels: bound by the matrix cores and, side by side with them, by the exponentials.  Measured, bf16:
// 16384 tokens, causal, 8 heads of 128 over 2 key heads 555 us (990 TFLOP/s; matrix cores busy
// 50 % of the time); 2 x 4800, 8 heads of 64, 132 us (39 % busy: 64 channels per exponential
// instead of 128).  64 keys per step halve what a step costs besides (three tiles ahead
// instead of one changed nothing).
// Maxima are followed only when they grow by more than 2^8 (then the sums are
// scaled): the probabilities are at most 2^8 then, and nothing is lost, since both
// sums carry the same factor.  Probabilities are rounded to the activations' type for
// their product; their sum is of the 32-bit values.
template <class T, int C, bool WIDE, int KS>
__global__ __launch_bounds__(KS *kAttnThreads, (PackedSizes<T, C>::kWavesPerSimd)) void k_packed_fwd(PackedArgs a)
{
    using S = PackedSizes<T, C>;
    using R = typename S::R;
    constexpr int KT = S::kKeys, N = KT / 32;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id() % kAttnWaves, ks = wave_id() / kAttnWaves;
    const float c = a.scale * kLog2e;
    clear_outside<KS>((T *)a.out, a.q_start, a.sequences, a.tokens, (int64_t)a.heads * a.dim_v);
    // the channels that no load writes (teams meet where they lie, and then take no further item:
    // a plan has two teams only with fewer than 1024 units)
    if (a.dim < C || a.dim_v < C) {
        for (int e = threadIdx.x; e < 2 * KS * S::kKeyTile / 16; e += KS * kAttnThreads)
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
        __syncthreads();
    }
    const uint32_t items = a.plan.items();
    for (uint32_t n = blockIdx.x; n < items; n += gridDim.x) {
        const PackedItem item(a.plan, a.q_start, a.q_places, a.sequences, a.tokens, n);
        if (item.place.b < 0)  // the same in the whole block
            continue;
        const int h = item.h, hk = uniform(h / a.group);
        int qb, nq, kb0, nk;
        rows_of(a.q_start, a.tokens, item.place.b, qb, nq);
        rows_of(a.k_start, a.keys, item.place.b, kb0, nk);
        const int q0 = item.place.rank * kPackedRows;
        const int i = q0 + 32 * w + (l & 31);  // this lane's query
        const bool in = i < nq;
        const int limit = in ? (a.causal ? min(nk, i + nk - nq + 1) : nk) : 0;
        // keys that a row of the block, and of the wave, sees at the most; and
        // that every row of the wave sees
        const int last = min(q0 + kPackedRows, nq) - 1, wlast = min(q0 + 32 * w + 31, nq - 1);
        const int end = a.causal ? min(nk, last + nk - nq + 1) : nk;
        const int wend = q0 + 32 * w < nq ? (a.causal ? min(nk, wlast + nk - nq + 1) : nk) : 0;
        const int wall = q0 + 32 * w + 31 < nq ? (a.causal ? min(nk, q0 + 32 * w + nk - nq + 1) : nk) : 0;
        int from, to;
        item.range(max(end + KT - 1, 0) / KT, from, to);
        const T *kp = uniform_ptr((const T *)a.k + (kb0 + (int64_t)(from + ks) * KT) * a.ks[0] + hk * a.ks[1]);
        const T *vp = uniform_ptr((const T *)a.v + (kb0 + (int64_t)(from + ks) * KT) * a.vs[0] + hk * a.vs[1]);
        char *mine = lds + ks * 2 * S::kKeyTile;  // this team's two tiles
        auto issue = [&](int t, int place) {      // tiles in order
            char *at = mine + place * S::kKeyTile;
            load_rows<T, C, 1, KT, kAttnWaves, WIDE>(at, kp, a.ks[0], 0, nk - 1 - t * KT, a.dim, w);
            load_rows<T, C, 1, KT, kAttnWaves, WIDE>(at + R::size(KT), vp, a.vs[0], 0, nk - 1 - t * KT, a.dim_v, w);
            kp = uniform_ptr(kp + KS * KT * a.ks[0]);
            vp = uniform_ptr(vp + KS * KT * a.vs[0]);
        };
        if (from + ks < to)
            issue(from + ks, 0);
        uint4v q[S::CK];
        const T *qrow = (const T *)a.q + (qb + (int64_t)i) * a.qs[0] + h * a.qs[1];
#pragma unroll
        for (int x = 0; x < S::CK; ++x)
            q[x] = memory_chunk<T, WIDE>(qrow, x, a.dim, in);
        f32x16 o[S::TV] = {};
        float top = -INFINITY, sum = 0.0f;
        for (int t0 = from, place = 0; t0 < to; t0 += KS, place ^= 1) {  // the teams' tiles of a turn
            const int t = t0 + ks, k0 = t * KT;
            char *kb = mine + place * S::kKeyTile, *vb = kb + R::size(KT);
            wait_loads();
            __syncthreads();  // the tiles are there for every wave, and those before done with
            if (t + KS < to)
                issue(t + KS, place ^ 1);
            if (min(t0 + KS, to) * KT > nk) {  // rows past the sequence: of keys, the scores are hidden
                if (t < to && k0 + KT > nk)
                    clear_rows<T, C, KT, kAttnWaves>(vb, (1ull << (nk - k0)) - 1, w);
                __syncthreads();
            }
            if (t >= to || k0 >= wend)
                continue;
            const uint32_t kr = lds_address(kb) + R::row_lane(), vc = lds_address(vb) + R::col_lane();
            f32x16 s[N] = {};
#pragma unroll
            for (int x = 0; x < S::CK; ++x)
#pragma unroll
                for (int y = 0; y < N; ++y)
                    mma<T>(s[y], R::row_chunk(kr, 32 * y, x), q[x]);
            if (k0 + KT > wall) {
#pragma unroll
                for (int y = 0; y < N; ++y)
                    hide_rows(s[y], low_bits(limit - k0 - 32 * y));
            }
            float mx = s[0][0];
#pragma unroll
            for (int y = 0; y < N; ++y)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    mx = __builtin_fmaxf(mx, s[y][r]);
            mx *= c;
            if (__any(mx > top + 8.0f)) {
                const float up = __builtin_fmaxf(top, xor32_max(mx));
                const float f = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - up);
                top = up;
                sum *= f;
#pragma unroll
                for (int v = 0; v < S::TV; ++v)
                    o[v] *= f;
            }
            const float base = top == -INFINITY ? 0.0f : top - kLift<T>;
            uint4v p[N][S::CP];
            float add = 0.0f;  // a step's sum first: shorter chains of rounded additions
#pragma unroll
            for (int y = 0; y < N; ++y) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[y][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[y][r], c, -base));
                    add += s[y][r];
                }
#pragma unroll
                for (int x = 0; x < S::CP; ++x)
                    p[y][x] = operand<T>(s[y], x);
            }
            sum += add;
#pragma unroll
            for (int y = 0; y < N; ++y)
#pragma unroll
                for (int x = 0; x < S::CP; ++x)
#pragma unroll
                    for (int v = 0; v < S::TV; ++v)
                        mma<T>(o[v], R::col_chunk(vc, 32 * y, x, 32 * v), p[y][x]);
        }
        __syncthreads();  // the next item's loads write where this one's were read
        sum = xor32_add(sum);
        if constexpr (KS == 2) {
            float2 *stats = reinterpret_cast<float2 *>(lds + kPackedRows * C * 4);
            if (ks == 1) {
                if (__any(sum == 0.0f)) {
#pragma unroll
                    for (int v = 0; v < S::TV; ++v)
                        o[v] = sum == 0.0f ? f32x16{} : o[v];
                }
                leave_sums(lds, w, o);
                if (l < 32)
                    stats[w * 32 + l] = make_float2(top, sum);
            }
            __syncthreads();
            if (ks == 0) {
                const float2 st = stats[w * 32 + (l & 31)];
                const float up = __builtin_fmaxf(sum != 0.0f ? top : -INFINITY, st.y != 0.0f ? st.x : -INFINITY);
                // a team whose top is -inf and whose sum is not 0 has a NaN in it; one whose sum is
                // 0 saw nothing, and what it holds need not be finite
                const float f = sum == 0.0f ? 0.0f : (top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - up));
                const float f2 = st.y == 0.0f ? 0.0f : (st.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.x - up));
                if (__any(sum == 0.0f)) {
#pragma unroll
                    for (int v = 0; v < S::TV; ++v)
                        o[v] = sum == 0.0f ? f32x16{} : o[v];
                }
                take_sums(lds, w, o, f, f2);
                sum = sum * f + st.y * f2;
                top = up;
            }
            __syncthreads();
            if (ks == 1)
                continue;
        }
        if (item.parts > 1) {  // unnormalised sums, tops and sums, for k_packed_join
            const int64_t at = ((int64_t)item.slot * kAttnWaves + w) * 32 + (l & 31);
#pragma unroll
            for (int v = 0; v < S::TV; ++v)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<float4v *>(a.part + at * C + 32 * v + 8 * g + 4 * (l >> 5)) =
                        sum != 0.0f ? float4v{o[v][4 * g], o[v][4 * g + 1], o[v][4 * g + 2], o[v][4 * g + 3]} : float4v{};
            if (l < 32)
                *reinterpret_cast<float2 *>(a.part + (int64_t)a.plan.cut() * a.plan.parts * kPackedRows * C + at * 2) =
                    make_float2(top, sum);
            continue;
        }
        if (!in)
            continue;
        // a query that saw nothing has 0 times its tiles' values, which need not be finite
        const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
        const int64_t row = ((int64_t)(qb + i) * a.heads + h) * a.dim_v;
#pragma unroll
        for (int v = 0; v < S::TV; ++v)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    y[j] = sum != 0.0f ? o[v][4 * g + j] * inv : 0.0f;
                const int ch = 32 * v + 8 * g + 4 * (l >> 5);
                store4<T, WIDE>((T *)a.out + row, ch, a.dim_v, y);
                if (a.so)
                    store4<float, WIDE>(a.so + row, ch, a.dim_v, y);
            }
        if (a.lse && l < 32)
            a.lse[(int64_t)h * a.tokens + qb + i] = lse_of<T>(top, sum);
    }
}

// Joins the parts of every unit, a thread per four channels of a row:
//   o = sum_p 2^(top_p - top) o_p / sum_p 2^(top_p - top) sum_p.
// Bound by memory: 2 x 4800 tokens, 8 heads of 64, three parts 8.6 us.
template <class T, int C, bool WIDE>
__global__ __launch_bounds__(kAttnThreads) void k_packed_join(PackedArgs a)
{
    constexpr int QUADS = C / 4, ROWS = kAttnThreads / QUADS, STEPS = kPackedRows / ROWS;
    const float *stats = a.part + (int64_t)a.plan.cut() * a.plan.parts * kPackedRows * C;
    const uint32_t blocks = a.plan.cut() * STEPS;
    for (uint32_t n = blockIdx.x; n < blocks; n += gridDim.x) {
        const uint32_t u = n / STEPS, unit = a.plan.full + u, slot = unit / a.plan.heads;
        const int h = unit - slot * a.plan.heads;
        const Place place(a.q_start, a.q_places, a.sequences, a.tokens, uniform(slot));
        if (place.b < 0)
            continue;
        int qb, nq;
        rows_of(a.q_start, a.tokens, place.b, qb, nq);
        const int row = (n - u * STEPS) * ROWS + threadIdx.x / QUADS, ch = threadIdx.x % QUADS * 4;
        const int i = place.rank * kPackedRows + row;
        if (i >= nq || ch >= a.dim_v)
            continue;
        auto at = [&](uint32_t p) { return ((int64_t)u * a.plan.parts + p) * kPackedRows + row; };
        float top = -INFINITY, sum = 0.0f;
        float4v o = {};
        for (uint32_t p = 0; p < a.plan.parts; ++p) {
            const float2 st = *reinterpret_cast<const float2 *>(stats + at(p) * 2);
            top = st.y != 0.0f ? __builtin_fmaxf(top, st.x) : top;
        }
#pragma unroll 4
        for (uint32_t p = 0; p < a.plan.parts; ++p) {
            const float2 st = *reinterpret_cast<const float2 *>(stats + at(p) * 2);
            const float4v x = *reinterpret_cast<const float4v *>(a.part + at(p) * C + ch);
            // a part whose top is -inf and whose sum is not 0 has a NaN in it
            const float f = st.y == 0.0f ? 0.0f : (st.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.x - top));
            sum += f * st.y;
            o += f * x;
        }
        const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
        const float y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
        const int64_t to = ((int64_t)(qb + i) * a.heads + h) * a.dim_v;
        store4<T, WIDE>((T *)a.out + to, ch, a.dim_v, y);
        if (a.so)
            store4<float, WIDE>(a.so + to, ch, a.dim_v, y);
        if (a.lse && ch == 0)
            a.lse[(int64_t)h * a.tokens + qb + i] = lse_of<T>(top, sum);
    }
}

// ---------------------------------------------------------------------------
// backward: queries
// ---------------------------------------------------------------------------

// D and dq: three products of pairs, bound by the matrix cores and the exponentials (bf16:
// 16384 tokens, causal, 8 heads of 128, 768 us, 1075 TFLOP/s, matrix cores busy 58 %; 2 x 4800, 8 of
// 64, 212 us).  D is taken from out in 32 bits: it is the difference of dp and D that
// counts, which may be far smaller than either.  A row's score gradients add up to 0, so that
// what their rounding leaves counts for more than in the other products, the more the fewer
// channels there are: with one operand dq was off by 1.45 (heads of 128) to 1.56 times (of 16) as
// much as by being rounded alone, with two by 1.01 to 1.04.  Heads of up to 64 take two (bf16, 8 of 64, 2 x
// 4800: 212 us for 165), larger ones one (16384 causal, of 128: 768 us; with two 988).
template <class T, int C, bool WIDE, int KS>
__global__ __launch_bounds__(KS *kAttnThreads, (PackedSizes<T, C>::kWavesPerSimd)) void k_packed_dq(PackedArgs a)
{
    using S = PackedSizes<T, C>;
    using R = typename S::R;
    constexpr int KT = S::kKeys;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id() % kAttnWaves, ks = wave_id() / kAttnWaves;
    const float c = a.scale * kLog2e;
    clear_outside<KS>((T *)a.gq, a.q_start, a.sequences, a.tokens, (int64_t)a.heads * a.dim);
    if (a.dim < C || a.dim_v < C) {
        for (int e = threadIdx.x; e < 2 * KS * S::kKeyTile / 16; e += KS * kAttnThreads)
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
        __syncthreads();
    }
    const uint32_t items = a.plan.items();
    for (uint32_t n = blockIdx.x; n < items; n += gridDim.x) {
        const PackedItem item(a.plan, a.q_start, a.q_places, a.sequences, a.tokens, n);
        if (item.place.b < 0)
            continue;
        const int h = item.h, hk = uniform(h / a.group);
        int qb, nq, kb0, nk;
        rows_of(a.q_start, a.tokens, item.place.b, qb, nq);
        rows_of(a.k_start, a.keys, item.place.b, kb0, nk);
        const int q0 = item.place.rank * kPackedRows;
        const int i = q0 + 32 * w + (l & 31);
        const bool in = i < nq;
        const int limit = in ? (a.causal ? min(nk, i + nk - nq + 1) : nk) : 0;
        const int last = min(q0 + kPackedRows, nq) - 1, wlast = min(q0 + 32 * w + 31, nq - 1);
        const int end = a.causal ? min(nk, last + nk - nq + 1) : nk;
        const int wend = q0 + 32 * w < nq ? (a.causal ? min(nk, wlast + nk - nq + 1) : nk) : 0;
        const int wall = q0 + 32 * w + 31 < nq ? (a.causal ? min(nk, q0 + 32 * w + nk - nq + 1) : nk) : 0;
        int from, to;
        item.range(max(end + KT - 1, 0) / KT, from, to);
        const T *kp = uniform_ptr((const T *)a.k + (kb0 + (int64_t)(from + ks) * KT) * a.ks[0] + hk * a.ks[1]);
        const T *vp = uniform_ptr((const T *)a.v + (kb0 + (int64_t)(from + ks) * KT) * a.vs[0] + hk * a.vs[1]);
        char *mine = lds + ks * 2 * S::kKeyTile;
        auto issue = [&](int t, int place) {
            char *at = mine + place * S::kKeyTile;
            load_rows<T, C, 1, KT, kAttnWaves, WIDE>(at, kp, a.ks[0], 0, nk - 1 - t * KT, a.dim, w);
            load_rows<T, C, 1, KT, kAttnWaves, WIDE>(at + R::size(KT), vp, a.vs[0], 0, nk - 1 - t * KT, a.dim_v, w);
            kp = uniform_ptr(kp + KS * KT * a.ks[0]);
            vp = uniform_ptr(vp + KS * KT * a.vs[0]);
        };
        if (from + ks < to)
            issue(from + ks, 0);
        const int64_t row = (int64_t)(qb + i) * a.heads + h;
        uint4v q[S::CK], g[S::CK];
        const T *qrow = (const T *)a.q + (qb + (int64_t)i) * a.qs[0] + h * a.qs[1];
        const T *grow = (const T *)a.dout + (qb + (int64_t)i) * a.dos[0] + h * a.dos[1];
        float D = 0.0f, lse = INFINITY;
#pragma unroll
        for (int x = 0; x < S::CK; ++x) {
            q[x] = memory_chunk<T, WIDE>(qrow, x, a.dim, in);
            g[x] = memory_chunk<T, WIDE>(grow, x, a.dim_v, in);
            D += piece_dot<T, WIDE>(g[x], a.so + row * a.dim_v, x, a.dim_v, in);
            if (x % 4 == 3)  // no more of o under way than the registers hold
                asm volatile("" : "+v"(D));
        }
        D = xor32_add(D);
        if (in) {  // a row that sees nothing has probabilities 0
            const float x = a.lse[(int64_t)h * a.tokens + qb + i];
            lse = x == -INFINITY ? INFINITY : x * kLog2e;
        }
        D = lse == INFINITY ? 0.0f : D;
        if (l < 32 && in && item.part == 0 && ks == 0) {
            float *st = a.stats + (int64_t)h * 2 * a.tokens + qb + i;
            st[0] = lse;
            st[a.tokens] = D;
        }
        f32x16 acc[S::TV] = {};
        Range range;
        for (int t0 = from, place = 0; t0 < to; t0 += KS, place ^= 1) {
            const int t = t0 + ks, k0 = t * KT;
            char *kb = mine + place * S::kKeyTile, *vb = kb + R::size(KT);
            wait_loads();
            __syncthreads();
            if (t + KS < to)
                issue(t + KS, place ^ 1);
            if (min(t0 + KS, to) * KT > nk) {
                if (t < to && k0 + KT > nk) {
                    const uint64_t seen = (1ull << (nk - k0)) - 1;
                    clear_rows<T, C, KT, kAttnWaves>(kb, seen, w);
                    clear_rows<T, C, KT, kAttnWaves>(vb, seen, w);
                }
                __syncthreads();
            }
            if (t >= to)
                continue;
            const uint32_t kr = lds_address(kb) + R::row_lane(), kc = lds_address(kb) + R::col_lane();
            const uint32_t vr = lds_address(vb) + R::row_lane();
#pragma unroll
            for (int kt = 0; kt < KT / 32; ++kt) {
                const int j0 = k0 + 32 * kt;
                if (j0 >= wend)
                    break;
                f32x16 s[1] = {}, dp = {};
#pragma unroll
                for (int x = 0; x < S::CK; ++x) {
                    mma<T>(s[0], R::row_chunk(kr, 32 * kt, x), q[x]);
                    mma<T>(dp, R::row_chunk(vr, 32 * kt, x), g[x]);
                }
                if (j0 + 32 > wall)
                    hide_rows(s[0], low_bits(limit - j0));
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[0][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][r], c, -lse)) * (dp[r] - D);
                if constexpr (std::is_same<T, f16>::value)
                    range.fit(s, [&](float f) {
#pragma unroll
                        for (int v = 0; v < S::TV; ++v)
                            acc[v] *= f;
                    });
#pragma unroll
                for (int x = 0; x < S::CP; ++x) {
                    if constexpr (S::kTwoOperands) {
                        uint4v ds, low;
                        operands<T>(s[0], x, ds, low);
#pragma unroll
                        for (int v = 0; v < S::TV; ++v) {
                            const uint4v kf = R::col_chunk(kc, 32 * kt, x, 32 * v);
                            mma<T>(acc[v], kf, ds);
                            mma<T>(acc[v], kf, low);
                        }
                    } else {
                        const uint4v ds = operand<T>(s[0], x);
#pragma unroll
                        for (int v = 0; v < S::TV; ++v)
                            mma<T>(acc[v], R::col_chunk(kc, 32 * kt, x, 32 * v), ds);
                    }
                }
            }
        }
        __syncthreads();
        float f = a.scale * range.down();
        if constexpr (KS == 2) {
            if (ks == 1) {
#pragma unroll
                for (int v = 0; v < S::TV; ++v)
                    acc[v] *= f;
                leave_sums(lds, w, acc);
            }
            __syncthreads();
            if (ks == 0)
                take_sums(lds, w, acc, f, 1.0f);
            f = 1.0f;
            __syncthreads();
            if (ks == 1)
                continue;
        }
        float *part = a.part + (((int64_t)item.slot * kAttnWaves + w) * 32 + (l & 31)) * C;
#pragma unroll
        for (int v = 0; v < S::TV; ++v)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                float x[4];  // a row that sees nothing: 0 times keys that need not be finite
#pragma unroll
                for (int z = 0; z < 4; ++z)
                    x[z] = lse == INFINITY ? 0.0f : acc[v][4 * y + z] * f;
                const int ch = 32 * v + 8 * y + 4 * (l >> 5);
                if (item.parts > 1)
                    store4<float, true>(part, ch, C, x);
                else if (in)
                    store4<T, WIDE>((T *)a.gq + row * a.dim, ch, a.dim, x);
            }
    }
}

// ---------------------------------------------------------------------------
// backward: keys and values
// ---------------------------------------------------------------------------

// dk and dv of 128 keys, over the queries of every head of the key head: four products of pairs,
// bound as dq's (bf16: 16384 tokens, causal, 8 heads of 128 over 2 key heads 1130 us, 975 TFLOP/s,
// matrix cores busy 47 %; 2 x 4800, 8 of 64, 265 us; 64 queries at once there, with 32 it was 279).  Scores
// are formed with queries as rows here: a lane holds one key.  A kernel of its own,
// apart from dq's: one pass would save two of the seven products, but either dq or
// dk and dv would have to be summed over blocks, by atomics in an order that changes
// from run to run, or by parts of 32 bits as large as the scores' rows over 128.
template <class T, int C, bool WIDE, int KS>
__global__ __launch_bounds__(KS *kAttnThreads, (PackedSizes<T, C>::kWavesPerSimd)) void k_packed_dkv(PackedArgs a)
{
    using S = PackedSizes<T, C>;
    using R = typename S::R;
    constexpr int QT = S::kQueries;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int l = lane_id(), w = wave_id() % kAttnWaves, ks = wave_id() / kAttnWaves;
    const float c = a.scale * kLog2e;
    clear_outside<KS>((T *)a.gk, a.k_start, a.sequences, a.keys, (int64_t)a.kv_heads * a.dim);
    clear_outside<KS>((T *)a.gv, a.k_start, a.sequences, a.keys, (int64_t)a.kv_heads * a.dim_v);
    if (a.dim < C || a.dim_v < C) {
        for (int e = threadIdx.x; e < (2 * KS * S::kQueryTile + S::kValues) / 16; e += KS * kAttnThreads)
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
        __syncthreads();
    }
    const uint32_t items = a.key_plan.items();
    for (uint32_t n = blockIdx.x; n < items; n += gridDim.x) {
        const PackedItem item(a.key_plan, a.k_start, a.k_places, a.sequences, a.keys, n);
        if (item.place.b < 0)
            continue;
        const int hk = item.h, h0 = hk * a.group, h1 = h0 + a.group;
        int qb, nq, kb0, nk;
        rows_of(a.q_start, a.tokens, item.place.b, qb, nq);
        rows_of(a.k_start, a.keys, item.place.b, kb0, nk);
        // the keys that most queries see are the first
        const int k0 = (item.place.tiles - 1 - item.place.rank) * kPackedRows;
        const int j = k0 + 32 * w + (l & 31);  // this lane's key
        const bool seen = j < nk;
        // the first query that sees this lane's key, and the first of the block's; queries
        // before those may see nothing at all
        const int off = a.causal ? nk - nq : (1 << 30);
        const int from = seen ? j - off : 0x7fffffff;
        const int lowest = k0 - off, first = max(lowest, 0) / QT * QT, wfirst = k0 + 32 * w - off;
        const bool wany = k0 + 32 * w < nk;
        uint4v kf[S::CK];
        const T *krow = (const T *)a.k + (kb0 + (int64_t)j) * a.ks[0] + hk * a.ks[1];
        // the wave's 32 rows of values stay in LDS: in registers too they did not fit 256
        char *vrows = lds + 2 * KS * S::kQueryTile + R::size(32) * w;  // (the teams write the same)
        const T *vrow = (const T *)a.v + (kb0 + (int64_t)j) * a.vs[0] + hk * a.vs[1];
#pragma unroll
        for (int x = 0; x < S::CK; ++x) {
            kf[x] = memory_chunk<T, WIDE>(krow, x, a.dim, seen);
            store16(vrows + R::at(l & 31, 2 * x + (l >> 5)), memory_chunk<T, WIDE>(vrow, x, a.dim_v, seen));
        }
        f32x16 gk[S::TV] = {}, gv[S::TV] = {};
        Range range;
        // fp16: probabilities, at most 1, go into the product 2^14 times larger (with
        // scores so small that what their sums would start from passes 32 bits there is
        // nothing to lift)
        const float lift = std::is_same<T, f16>::value && c > 0x1p-100f ? 14.0f : 0.0f;
        const float lifted = lift / c;  // what the scores' sums start from

        // tiles of all heads in one run, loads a tile ahead
        const int per = nq > first ? (nq - first + QT - 1) / QT : 0;
        int t0, t1;
        item.range(per * a.group, t0, t1);
        // head and first query of the next tile to load
        int nh = h0 + (per ? (t0 + ks) / per : 0), ni = first + (per ? (t0 + ks) % per : 0) * QT;
        nh = uniform(nh);
        ni = uniform(ni);
        const T *qp, *gp;
        const float *sp;
        auto head = [&](int h) {
            qp = uniform_ptr((const T *)a.q + (qb + (int64_t)ni) * a.qs[0] + h * a.qs[1]);
            gp = uniform_ptr((const T *)a.dout + (qb + (int64_t)ni) * a.dos[0] + h * a.dos[1]);
            sp = uniform_ptr(a.stats + (int64_t)h * 2 * a.tokens + qb + ni);
        };
        // the first query of the tile KS tiles on, and its head: a step may pass several heads
        auto step = [&](int &i, int &h) {
            i += KS * QT;
            while (i >= nq && h < h1) {  // nq > first: every head has a tile
                i -= per * QT;
                ++h;
            }
        };
        char *mine = lds + ks * 2 * S::kQueryTile;
        auto issue = [&](int buf) {
            char *to = mine + buf * S::kQueryTile;
            load_rows<T, C, 1, QT, kAttnWaves, WIDE>(to, qp, a.qs[0], 0, nq - 1 - ni, a.dim, w);
            load_rows<T, C, 1, QT, kAttnWaves, WIDE>(to + R::size(QT), gp, a.dos[0], 0, nq - 1 - ni, a.dim_v, w);
            // 2 statistics of a tile's queries, one by each of two waves
            const int y = again(l);
            if (w < 2 && y < QT)
                load_lds4(uniform_ptr(sp + w * (int64_t)a.tokens), 4u * (uint32_t)min(y, nq - 1 - ni),
                          lds_address(to + 2 * R::size(QT)) + w * (4 * QT));
            const int was = nh;
            step(ni, nh);
            if (nh != was) {
                if (nh < h1)
                    head(nh);
            } else {
                qp = uniform_ptr(qp + KS * QT * a.qs[0]);
                gp = uniform_ptr(gp + KS * QT * a.dos[0]);
                sp += KS * QT;
            }
        };
        int i0s[KS], ihs[KS];  // of every team's tile at hand
#pragma unroll
        for (int x = 0; x < KS; ++x) {
            ihs[x] = uniform(h0 + (per ? (t0 + x) / per : 0));
            i0s[x] = uniform(first + (per ? (t0 + x) % per : 0) * QT);
        }
        if (t0 + ks < t1) {
            head(nh);
            issue(0);
        }
        for (int tt = t0, buf = 0; tt < t1; tt += KS, buf ^= 1) {
            const int t = tt + ks;
            char *qb_ = mine + buf * S::kQueryTile, *gb = qb_ + R::size(QT);
            const float *st = reinterpret_cast<const float *>(gb + R::size(QT));
            wait_loads();
            __syncthreads();
            if (t + KS < t1)
                issue(buf ^ 1);
            // rows past the sequence, or before the first that sees a key of the block
            bool clear = false;
#pragma unroll
            for (int x = 0; x < KS; ++x)
                clear = clear || (tt + x < t1 && (i0s[x] + QT > nq || i0s[x] < lowest));
            const int i0 = KS == 2 && ks ? i0s[KS - 1] : i0s[0];
            if (clear) {  // the same in the whole block
                if (t < t1 && (i0 + QT > nq || i0 < lowest)) {
                    const uint64_t live = low_bits64(nq - i0) & ~low_bits64(lowest - i0);
                    clear_rows<T, C, QT, kAttnWaves>(qb_, live, w);
                    clear_rows<T, C, QT, kAttnWaves>(gb, live, w);
                }
                __syncthreads();
            }
#pragma unroll
            for (int x = 0; x < KS; ++x)
                step(i0s[x], ihs[x]);
            if (t >= t1 || !wany || i0 + QT <= wfirst)
                continue;
            const uint32_t qr = lds_address(qb_) + R::row_lane(), qc = lds_address(qb_) + R::col_lane();
            const uint32_t gr = lds_address(gb) + R::row_lane(), gc = lds_address(gb) + R::col_lane();
            const uint32_t vr = lds_address(vrows) + R::row_lane();
#pragma unroll
            for (int qt = 0; qt < QT / 32; ++qt) {
                const int i1 = i0 + 32 * qt;
                if (i1 >= nq || i1 + 32 <= wfirst)
                    continue;
                f32x16 s[1], dp = {};
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[0][r] = std::is_same<T, f16>::value ? lifted : 0.0f;
#pragma unroll
                for (int x = 0; x < S::CK; ++x) {
                    mma<T>(s[0], R::row_chunk(qr, 32 * qt, x), kf[x]);
                    mma<T>(dp, R::row_chunk(gr, 32 * qt, x), R::row_chunk(vr, 0, x));
                }
                if (k0 + 32 * w + 32 > nk || i1 < wfirst + 31 || i1 + 32 > nq)
                    hide_rows(s[0], low_bits(nq - i1) & ~low_bits(from > i1 ? from - i1 : 0));
                uint4v pf[S::CP], ds[S::CP];
                f32x16 p;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int at = 32 * qt + 8 * g + 4 * (l >> 5);
                    const float4v ls = *reinterpret_cast<const float4v *>(st + at);
                    const float4v d = *reinterpret_cast<const float4v *>(st + QT + at);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const int r = 4 * g + y;
                        p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][r], c, -ls[y]));
                        s[0][r] = p[r] * (dp[r] - d[y]);
                    }
                }
                if constexpr (std::is_same<T, f16>::value)
                    range.fit(s, [&](float f) {
#pragma unroll
                        for (int v = 0; v < S::TV; ++v)
                            gk[v] *= f;
                    });
#pragma unroll
                for (int x = 0; x < S::CP; ++x) {
                    pf[x] = operand<T>(p, x);
                    ds[x] = operand<T>(s[0], x);
                }
#pragma unroll
                for (int x = 0; x < S::CP; ++x)
#pragma unroll
                    for (int v = 0; v < S::TV; ++v) {
                        mma<T>(gv[v], R::col_chunk(gc, 32 * qt, x, 32 * v), pf[x]);
                        mma<T>(gk[v], R::col_chunk(qc, 32 * qt, x, 32 * v), ds[x]);
                    }
            }
        }
        __syncthreads();
        const float fv = __builtin_amdgcn_exp2f(-lift);
        float fk = a.scale * range.down() * fv;
        if constexpr (KS == 2) {
            char *lds_v = lds + kPackedRows * C * 4;
            if (ks == 1) {
#pragma unroll
                for (int v = 0; v < S::TV; ++v)
                    gk[v] *= fk;
                leave_sums(lds, w, gk);
                leave_sums(lds_v, w, gv);
            }
            __syncthreads();
            if (ks == 0) {
                take_sums(lds, w, gk, fk, 1.0f);
                take_sums(lds_v, w, gv, 1.0f, 1.0f);
            }
            fk = 1.0f;
            __syncthreads();
            if (ks == 1)
                continue;
        }
        if (!seen && item.parts == 1)
            continue;
        const int64_t row = (int64_t)(kb0 + j) * a.kv_heads + hk;
        float *part = a.key_part + (((int64_t)item.slot * kAttnWaves + w) * 32 + (l & 31)) * 2 * C;
        auto put = [&](T *to, float *to_part, const f32x16 &x, int v, int dim, float f) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float y[4];  // a key past the sequence has sums of 0 times what the queries hold
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
#pragma unroll
        for (int v = 0; v < S::TV; ++v) {
            put((T *)a.gk + row * a.dim, part, gk[v], v, a.dim, fk);
            put((T *)a.gv + row * a.dim_v, part + C, gv[v], v, a.dim_v, fv);
        }
    }
}

// Sums of the parts of both passes' units, in a fixed order: a thread per four channels.  Bound by
// memory: 16384 tokens, 8 heads of 128 over 2 key heads, parts of both 24 us.
template <class T, int C, bool WIDE>
__global__ __launch_bounds__(kAttnThreads) void k_packed_finish(PackedArgs a)
{
    // blocks of a unit: of queries, C channels a row; of keys, 2 C
    constexpr int SQ = kPackedRows * (C / 4) / kAttnThreads, SK = 2 * SQ;
    const uint32_t nq = a.plan.cut() * SQ, nk = a.key_plan.cut() * SK;
    for (uint32_t n = blockIdx.x; n < nq + nk; n += gridDim.x) {
        const bool key = n >= nq;
        const PackedPlan &p = key ? a.key_plan : a.plan;
        const uint32_t m = key ? n - nq : n, steps = key ? SK : SQ, width = key ? 2 * C : C;
        const uint32_t u = m / steps, unit = p.full + u, slot = unit / p.heads;
        const int h = unit - slot * p.heads;
        const int32_t *start = key ? a.k_start : a.q_start;
        const int total = key ? a.keys : a.tokens;
        const Place place(start, key ? a.k_places : a.q_places, a.sequences, total, uniform(slot));
        if (place.b < 0)
            continue;
        int base, len;
        rows_of(start, total, place.b, base, len);
        const uint32_t e = (m - u * steps) * kAttnThreads + threadIdx.x, row = e / (width / 4), ch = e % (width / 4) * 4;
        const int i = (key ? place.tiles - 1 - place.rank : place.rank) * kPackedRows + row;
        const bool value = ch >= C;
        const int cc = value ? ch - C : ch, dim = value ? a.dim_v : a.dim;
        if (i >= len || cc >= dim)
            continue;
        const float *from = (key ? a.key_part : a.part) + ((int64_t)u * p.parts * kPackedRows + row) * width + ch;
        float4v s = {};
#pragma unroll 4
        for (uint32_t q = 0; q < p.parts; ++q)
            s += *reinterpret_cast<const float4v *>(from + (int64_t)q * kPackedRows * width);
        const float y[4] = {s[0], s[1], s[2], s[3]};
        T *to = (T *)(key ? (value ? a.gv : a.gk) : a.gq);
        store4<T, WIDE>(to + ((int64_t)(base + i) * p.heads + h) * dim, cc, dim, y);
    }
}

template <class T, int C, bool WIDE, int KS>
hipError_t packed_fwd_teams(const PackedArgs &a, hipStream_t s)
{
    return launch_lds<k_packed_fwd<T, C, WIDE, KS>>(item_blocks(a.plan.items()), KS * kAttnThreads,
                                                   PackedSizes<T, C>::rows_lds(KS), a, s);
}
template <class T, int C, bool WIDE, int KS>
hipError_t packed_dq_teams(const PackedArgs &a, hipStream_t s)
{
    return launch_lds<k_packed_dq<T, C, WIDE, KS>>(item_blocks(a.plan.items()), KS * kAttnThreads,
                                                  PackedSizes<T, C>::rows_lds(KS), a, s);
}
template <class T, int C, bool WIDE, int KS>
hipError_t packed_dkv_teams(const PackedArgs &a, hipStream_t s)
{
    return launch_lds<k_packed_dkv<T, C, WIDE, KS>>(item_blocks(a.key_plan.items()), KS * kAttnThreads,
                                                   PackedSizes<T, C>::keys_lds(KS), a, s);
}

// two teams where the plan says so, and the registers are for two waves per SIMD
template <class T, int C, bool WIDE>
hipError_t packed_fwd_launch(const PackedArgs &a, hipStream_t s)
{
    hipError_t e = hipErrorInvalidValue;
    if constexpr (PackedSizes<T, C>::kSmall) {
        e = a.plan.teams == 2 ? packed_fwd_teams<T, C, WIDE, 2>(a, s) : packed_fwd_teams<T, C, WIDE, 1>(a, s);
    } else {
        e = packed_fwd_teams<T, C, WIDE, 1>(a, s);
    }
    if (e != hipSuccess || a.plan.cut() == 0)
        return e;
    const int64_t blocks = (int64_t)a.plan.cut() * (kPackedRows * (C / 4) / kAttnThreads);
    hipLaunchKernelGGL((k_packed_join<T, C, WIDE>), dim3(item_blocks(blocks)), dim3(kAttnThreads), 0, s, a);
    return hipGetLastError();
}

template <class T, int C, bool WIDE>
hipError_t packed_bwd_launch(const PackedArgs &a, hipStream_t s)
{
    hipError_t e = hipSuccess;
    if constexpr (PackedSizes<T, C>::kSmall) {
        if (a.plan.units())
            e = a.plan.teams == 2 ? packed_dq_teams<T, C, WIDE, 2>(a, s) : packed_dq_teams<T, C, WIDE, 1>(a, s);
        if (e == hipSuccess && a.key_plan.units())
            e = a.key_plan.teams == 2 ? packed_dkv_teams<T, C, WIDE, 2>(a, s) : packed_dkv_teams<T, C, WIDE, 1>(a, s);
    } else {
        if (a.plan.units())
            e = packed_dq_teams<T, C, WIDE, 1>(a, s);
        if (e == hipSuccess && a.key_plan.units())
            e = packed_dkv_teams<T, C, WIDE, 1>(a, s);
    }
    constexpr int SQ = kPackedRows * (C / 4) / kAttnThreads;
    const int64_t blocks = (int64_t)a.plan.cut() * SQ + (int64_t)a.key_plan.cut() * 2 * SQ;
    if (e != hipSuccess || blocks == 0)
        return e;
    hipLaunchKernelGGL((k_packed_finish<T, C, WIDE>), dim3(item_blocks(blocks)), dim3(kAttnThreads), 0, s, a);
    return hipGetLastError();
}

// more than kScanned sequences: the tiles before each, for the queries, and (both) for the keys
inline hipError_t packed_places(const PackedArgs &a, bool both, hipStream_t s)
{
    if (!a.q_places)
        return hipSuccess;
    hipLaunchKernelGGL(k_packed_places, dim3(both ? 2 : 1), dim3(kPlacesThreads), 0, s, a);
    return hipGetLastError();
}

template <class T>
hipError_t packed_fwd(const PackedArgs &a, hipStream_t s)
{
    const hipError_t e = packed_places(a, false, s);
    if (e != hipSuccess)
        return e;
    if (packed_class(a.dim, a.dim_v) == 64)
        return a.wide ? packed_fwd_launch<T, 64, true>(a, s) : packed_fwd_launch<T, 64, false>(a, s);
    return a.wide ? packed_fwd_launch<T, 128, true>(a, s) : packed_fwd_launch<T, 128, false>(a, s);
}

template <class T>
hipError_t packed_bwd(const PackedArgs &a, hipStream_t s)
{
    const hipError_t e = packed_places(a, true, s);
    if (e != hipSuccess)
        return e;
    if (packed_class(a.dim, a.dim_v) == 64)
        return a.wide ? packed_bwd_launch<T, 64, true>(a, s) : packed_bwd_launch<T, 64, false>(a, s);
    return a.wide ? packed_bwd_launch<T, 128, true>(a, s) : packed_bwd_launch<T, 128, false>(a, s);
}

}  // namespace

}  // namespace pam
