// Norms of the heads of queries and keys with the rotation in the same pass
// (gfx950), and their gradients.
//
//   n = x r,  r = 1 / sqrt(mean x^2 + eps)  (layer: of x - mean x),  y = n w,
//   (a, b) -> (a c - b s, a s + b c) over the first 2 pairs channels of y;
// backward, with dy the upstream gradient turned back and dn = dy w:
//   dx = r (dn - n mean(dn n))  (layer: less r mean dn),  dw = sum dy n.
// A head's row stays in the registers of a group of lanes, both channels of a
// pair in one lane, so that the norm is a sum over lanes and the rotation needs
// none.  Nothing is kept for the backward pass, which forms n again.  Both are
// bound by memory.
#include "pam_rows.h"

#include <algorithm>
#include <type_traits>

namespace pam {

namespace {

constexpr int kThreads = 256;
constexpr int kSumThreads = 1024;
constexpr int kSumSlots = 16;  // slots of a vector that a block of the summing kernel takes

struct HeadNormArgs {
    const void *q, *k;
    const float *w_q, *w_k;
    const float2 *table;
    const int32_t *pos;
    void *q_out, *k_out;         // backward: grad_q, grad_k
    const void *gq, *gk;         // backward: of the outputs
    float *gw_q, *gw_k, *part;
    int64_t qs[3], ks[3];
    int64_t start, entries;
    int32_t batch, length, heads, kv_heads, dim, pairs;
    int32_t group;               // lanes per row, a power of two
    int32_t chunks_q, chunks_k;  // blocks per vector of weights of q, of k
    Divisor by_length, by_heads, by_kv_heads;
    bool layer, per_head;
    float eps;
};

// Sum over an aligned group of lanes, left in every lane.  `group` is the same
// in every lane; called in wave-uniform control flow.
__device__ __forceinline__ float group_sum(float x, int group)
{
    if (group >= 2)
        x += lane_move<0xb1>(x);
    if (group >= 4)
        x += lane_move<0x4e>(x);
    if (group >= 8)
        x += lane_move<0x141>(x);
    if (group >= 16)
        x += lane_move<0x140>(x);
    if (group >= 32)
        x = xor16_add(x);
    if (group >= 64)
        x = xor32_add(x);
    return x;
}

// What a lane holds of a row: 2 V channels, V from c0 and V from c1 on.  Halves:
// the pairs (i, pairs + i) of V consecutive i, or 2 V of the channels behind the
// rotated ones; interleaved: 2 V consecutive channels.  WIDE: every V channels are
// there whole or not at all, and read in one or two accesses.
template <class T, int V, bool INTERLEAVED, bool WIDE>
struct Lane {
    int c0, c1, n0, n1, pair0, turns;  // channels that there are; the first pair; pairs that are turned
    __device__ __forceinline__ Lane(const HeadNormArgs &a, int j)
    {
        const int nt = (a.pairs + V - 1) / V;
        if (INTERLEAVED) {
            c0 = 2 * V * j;
            c1 = c0 + V;
            n0 = min(max(a.dim - c0, 0), V);
            n1 = min(max(a.dim - c1, 0), V);
            pair0 = V * j;
            turns = min(max(a.pairs - pair0, 0), V);
        } else if (j < nt) {
            c0 = V * j;
            c1 = a.pairs + c0;
            turns = n0 = n1 = min(a.pairs - c0, V);
            pair0 = c0;
        } else {
            c0 = 2 * a.pairs + 2 * V * (j - nt);
            c1 = c0 + V;
            n0 = min(max(a.dim - c0, 0), V);
            n1 = min(max(a.dim - c1, 0), V);
            pair0 = turns = 0;
        }
    }
    // V elements in accesses of up to 16 bytes
    template <class X>
    struct Wide {
        typedef X Vec __attribute__((ext_vector_type(V), aligned(sizeof(X) * V > 16 ? 16 : sizeof(X) * V)));
    };
    template <class X>
    __device__ __forceinline__ static void get(const X *p, int n, bool ok, float (&x)[V])
    {
        if constexpr (WIDE) {
            typename Wide<X>::Vec y = {};
            if (ok && n > 0)
                y = *reinterpret_cast<const typename Wide<X>::Vec *>(p);
#pragma unroll
            for (int j = 0; j < V; ++j)
                x[j] = (float)y[j];
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                x[j] = ok && j < n ? (float)p[j] : 0.0f;
        }
    }
    // this lane's channels of a row, c0's first; 0 where there are none
    template <class X>
    __device__ __forceinline__ void load(const X *row, bool ok, float (&x)[2][V]) const
    {
        get(row + c0, n0, ok, x[0]);
        get(row + c1, n1, ok, x[1]);
    }
    __device__ __forceinline__ void store(T *row, const float (&x)[2][V]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            T *p = row + (i ? c1 : c0);
            const int n = i ? n1 : n0;
            if constexpr (WIDE) {
                typename Wide<T>::Vec y;
#pragma unroll
                for (int j = 0; j < V; ++j)
                    y[j] = rounded<T>(x[i][j]);
                if (n > 0)
                    *reinterpret_cast<typename Wide<T>::Vec *>(p) = y;
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (j < n)
                        p[j] = rounded<T>(x[i][j]);
            }
        }
    }
    // weights of this lane's channels
    __device__ __forceinline__ void weights(const float *w, float (&x)[2][V]) const
    {
        if (w) {
            load(w, true, x);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                x[0][j] = x[1][j] = 1.0f;
        }
    }
    // cosines and sines of this lane's turned pairs of a token
    __device__ __forceinline__ void angles(const HeadNormArgs &a, int64_t tok, int l, float (&c)[V], float (&s)[V]) const
    {
        const int64_t at = a.pos ? (int64_t)a.pos[tok] : a.start + l;
        const bool in = at >= 0 && at < a.entries;
        const float2 *row = a.table + (in ? at : 0) * a.pairs + pair0;
        const float *p = reinterpret_cast<const float *>(row);
        const float nan = __builtin_nanf("");
        if constexpr (WIDE) {
            float4v y[V / 2] = {};
            if (turns > 0) {
#pragma unroll
                for (int j = 0; j < V / 2; ++j)
                    y[j] = *reinterpret_cast<const float4v *>(p + 4 * j);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                c[j] = in ? y[j / 2][2 * (j % 2)] : nan;
                s[j] = in ? y[j / 2][2 * (j % 2) + 1] : nan;
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                c[j] = j >= turns ? 1.0f : (in ? p[2 * j] : nan);
                s[j] = j >= turns ? 0.0f : (in ? p[2 * j + 1] : nan);
            }
        }
    }
    // the rotation by the angle, or (sign -1) back; one rounding per product and
    // one per sum, whatever the width
    __device__ __forceinline__ void turn(float (&x)[2][V], const float (&c)[V], const float (&s)[V], float sign) const
    {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float &p = INTERLEAVED ? x[2 * j / V][2 * j % V] : x[0][j];
            float &r = INTERLEAVED ? x[2 * j / V][2 * j % V + 1] : x[1][j];
            const bool turned = WIDE ? turns > 0 : j < turns;
            const float sj = sign * s[j], u = p, v = r;
            p = turned ? __builtin_fmaf(-v, sj, u * c[j]) : u;
            r = turned ? __builtin_fmaf(v, c[j], u * sj) : v;
        }
    }
    // a row's normalised values and their factor r; what is no channel stays 0
    __device__ __forceinline__ float normalise(const HeadNormArgs &a, float (&x)[2][V]) const
    {
        const float inv = 1.0f / (float)a.dim;
        if (a.layer) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j)
                sum += x[0][j] + x[1][j];
            const float mean = group_sum(sum, a.group) * inv;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[0][j] = (WIDE ? n0 > 0 : j < n0) ? x[0][j] - mean : 0.0f;
                x[1][j] = (WIDE ? n1 > 0 : j < n1) ? x[1][j] - mean : 0.0f;
            }
        }
        float sq = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j)
            sq = __builtin_fmaf(x[0][j], x[0][j], __builtin_fmaf(x[1][j], x[1][j], sq));
        const float r = 1.0f / sqrtf(__builtin_fmaf(group_sum(sq, a.group), inv, a.eps));
#pragma unroll
        for (int j = 0; j < V; ++j) {
            x[0][j] *= r;
            x[1][j] *= r;
        }
        return r;
    }
};

// The vectors of weights: one of q and one of k, or one per head; a vector's
// rows are dealt to its blocks in turn.  Blocks of q's vectors come first.
struct Vector {
    int first, chunks;   // blocks
    bool key;
    int head;            // -1: all
    __device__ __forceinline__ Vector(const HeadNormArgs &a, int block)
    {
        const int nq = a.per_head ? a.heads : 1, of_q = nq * a.chunks_q;
        key = block >= of_q;
        chunks = key ? a.chunks_k : a.chunks_q;
        const int at = (key ? block - of_q : block) / chunks;
        first = (key ? of_q : 0) + at * chunks;
        head = a.per_head ? at : -1;
    }
};

// Rows of a block's vector: which token and head, and where the row lies.
template <class T>
struct VectorRows {
    const T *base;
    int64_t st[3];
    int of;            // heads of a token among the rows
    int head, heads;
    uint32_t rows;
    Divisor by_of, by_length;
    int length;
    __device__ __forceinline__ VectorRows(const HeadNormArgs &a, const Vector &vec)
        : base(vec.key ? (const T *)a.k : (const T *)a.q), head(vec.head), heads(vec.key ? a.kv_heads : a.heads),
          by_length(a.by_length), length(a.length)
    {
        by_of.m = vec.key ? a.by_kv_heads.m : a.by_heads.m;
        by_of.s = vec.key ? a.by_kv_heads.s : a.by_heads.s;
#pragma unroll
        for (int i = 0; i < 3; ++i)
            st[i] = vec.key ? a.ks[i] : a.qs[i];
        of = head < 0 ? heads : 1;
        rows = (uint32_t)a.batch * a.length * of;
    }
    // row e: its token, its place in its sequence, its elements, and where it is in contiguous arrays
    __device__ __forceinline__ const T *at(uint32_t e, uint32_t &tok, uint32_t &l, int64_t &dense) const
    {
        tok = head < 0 ? by_of(e) : e;
        const uint32_t h = head < 0 ? e - tok * of : (uint32_t)head, b = by_length(tok);
        l = tok - b * length;
        dense = (int64_t)tok * heads + h;
        return base + b * st[0] + l * st[1] + h * st[2];
    }
};

// Forward: a row read and written once (2 x 4800 tokens, 16 and 16 heads of 64, bf16 20 us; 16384, 32
// and 8 of 128, fp16 84 us, 4.0 TB/s).  A block's rows share a vector of weights, which its lanes keep; the next
// row's loads are under way while a row is worked on.
template <class T, int V, bool INTERLEAVED, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_head_norm_fwd(HeadNormArgs a)
{
    using L = Lane<T, V, INTERLEAVED, WIDE>;
    const int per = kThreads / a.group, j = threadIdx.x & (a.group - 1), g = threadIdx.x / a.group;
    const L lane(a, j);
    const Vector vec(a, blockIdx.x);
    const VectorRows<T> in(a, vec);
    const uint32_t step = vec.chunks * per;
    T *to = vec.key ? (T *)a.k_out : (T *)a.q_out;
    const float *wv = vec.key ? a.w_k : a.w_q;
    struct Row {
        float x[2][V], c[V], s[V];
        int64_t at;
        bool live;
    };
    auto fetch = [&](uint32_t e) {
        Row r;
        uint32_t tok, l;
        r.live = e < in.rows;
        const T *from = in.at(min(e, in.rows - 1), tok, l, r.at);
        lane.load(from, r.live, r.x);
        lane.angles(a, tok, l, r.c, r.s);
        return r;
    };
    float w[2][V];
    uint32_t e0 = (blockIdx.x - vec.first) * per;
    if (e0 >= in.rows)
        return;
    Row row = fetch(e0 + g);
    lane.weights(wv && vec.head >= 0 ? wv + (int64_t)vec.head * a.dim : wv, w);
    for (; e0 < in.rows; e0 += step) {
        Row next = row;
        if (e0 + step < in.rows)
            next = fetch(e0 + step + g);
        lane.normalise(a, row.x);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            row.x[0][i] *= w[0][i];
            row.x[1][i] *= w[1][i];
        }
        lane.turn(row.x, row.c, row.s, 1.0f);
        if (row.live)
            lane.store(to + row.at * a.dim, row.x);
        row = next;
    }
}

// Backward: row and gradient read, the row's gradient written (the same calls 27 and 116 us, 4.3
// TB/s).  A block's rows share a vector of weights, whose gradient its lanes
// sum over them; the block's groups are added in LDS, the blocks by a second
// kernel, both in a fixed order.
template <class T, int V, bool INTERLEAVED, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_head_norm_bwd(HeadNormArgs a)
{
    using L = Lane<T, V, INTERLEAVED, WIDE>;
    __shared__ float sums[kThreads * 2 * V];
    const int per = kThreads / a.group, j = threadIdx.x & (a.group - 1), g = threadIdx.x / a.group;
    const L lane(a, j);
    const Vector vec(a, blockIdx.x);
    const VectorRows<T> in(a, vec);
    const float *wv = vec.key ? a.w_k : a.w_q;
    float w[2][V], dw[2][V] = {};
    lane.weights(wv && vec.head >= 0 ? wv + (int64_t)vec.head * a.dim : wv, w);
    const float inv = 1.0f / (float)a.dim;
    for (uint32_t e0 = (blockIdx.x - vec.first) * per; e0 < in.rows; e0 += vec.chunks * per) {
        const bool live = e0 + g < in.rows;
        uint32_t tok, l;
        int64_t at;
        const T *from = in.at(min(e0 + g, in.rows - 1), tok, l, at);
        at *= a.dim;
        float x[2][V], y[2][V], c[V], s[V];
        lane.load(from, live, x);
        lane.load((const T *)(vec.key ? a.gk : a.gq) + at, live, y);
        lane.angles(a, tok, l, c, s);
        const float r = lane.normalise(a, x);
        lane.turn(y, c, s, -1.0f);
        float dot = 0.0f, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if (live)  // a row that is not there: x r may be NaN with eps 0
                    dw[i][k] = __builtin_fmaf(y[i][k], x[i][k], dw[i][k]);
                y[i][k] *= w[i][k];
                dot = __builtin_fmaf(y[i][k], x[i][k], dot);
                sum += y[i][k];
            }
        dot = group_sum(dot, a.group) * inv;
        const float mean = a.layer ? group_sum(sum, a.group) * inv : 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k)
                y[i][k] = (__builtin_fmaf(-x[i][k], dot, y[i][k]) - mean) * r;
        if (live)
            lane.store((T *)(vec.key ? a.k_out : a.q_out) + at, y);
    }
    if (!(vec.key ? a.gw_k : a.gw_q))
        return;
    // slot j 2 V + i V + k of group g
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < V; ++k)
            sums[threadIdx.x * 2 * V + i * V + k] = dw[i][k];
    __syncthreads();
    const int slots = a.group * 2 * V;
    for (int t = threadIdx.x; t < slots; t += kThreads) {
        float sum = 0.0f;
        for (int i = 0; i < per; ++i)
            sum += sums[i * slots + t];
        a.part[(int64_t)blockIdx.x * slots + t] = sum;
    }
}

// Sums of the blocks' parts, a block per kSumSlots slots of a vector (the same calls 4 and 5.5 us).
template <class T, int V, bool INTERLEAVED, bool WIDE>
__global__ __launch_bounds__(kSumThreads) void k_head_norm_sum(HeadNormArgs a)
{
    constexpr int kTeams = kSumThreads / kSumSlots;
    __shared__ float s[kTeams][kSumSlots + 1];
    const int slots = a.group * 2 * V, per = (slots + kSumSlots - 1) / kSumSlots;
    const int v = blockIdx.x / per, slot = (blockIdx.x - v * per) * kSumSlots + threadIdx.x % kSumSlots;
    const int nq = a.per_head ? a.heads : 1;
    const bool key = v >= nq;
    const int chunks = key ? a.chunks_k : a.chunks_q, first = key ? nq * a.chunks_q + (v - nq) * chunks : v * chunks;
    float *out = key ? a.gw_k : a.gw_q;
    if (!out)
        return;
    float sum = 0.0f;
#pragma unroll 4
    for (int b = threadIdx.x / kSumSlots; b < chunks; b += kTeams)
        sum += slot < slots ? a.part[(int64_t)(first + b) * slots + slot] : 0.0f;
    s[threadIdx.x / kSumSlots][threadIdx.x % kSumSlots] = sum;
    for (int n = kTeams / 2; n > 0; n /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < n * kSumSlots)
            s[threadIdx.x / kSumSlots][threadIdx.x % kSumSlots] += s[threadIdx.x / kSumSlots + n][threadIdx.x % kSumSlots];
    }
    if (threadIdx.x >= kSumSlots || slot >= slots)
        return;
    const Lane<T, V, INTERLEAVED, WIDE> lane(a, slot / (2 * V));
    const int in = slot % (2 * V), i = in / V, k = in % V;
    if (k < (i ? lane.n1 : lane.n0))
        out[(a.per_head ? (int64_t)(key ? v - nq : v) * a.dim : 0) + (i ? lane.c1 : lane.c0) + k] = s[0][threadIdx.x];
}

// How a call's rows go to lanes: V channels twice per lane, `group` lanes.
struct Shape {
    int v, group, chunks_q, chunks_k;
    bool wide;
    int64_t blocks(const pam_head_norm_desc_t &d) const
    {
        return d.w_per_head ? (int64_t)d.heads * chunks_q + (int64_t)d.kv_heads * chunks_k
                            : chunks_q + (d.kv_heads ? chunks_k : 0);
    }
};

int lanes_of(const pam_head_norm_desc_t &d, int v)
{
    const int n = (d.flags & PAM_ROTARY_INTERLEAVED)
                      ? (d.dim + 2 * v - 1) / (2 * v)
                      : (d.pairs + v - 1) / v + (d.dim - 2 * d.pairs + 2 * v - 1) / (2 * v);
    int g = 1;
    while (g < n)
        g *= 2;
    return g;
}

// Blocks of a pass where there are rows for that, and the turns of its rows that a block
// takes at least.
constexpr int kFwdBlocks = 2048, kFwdTurns = 2, kBwdBlocks = 1024, kBwdTurns = 8;

Shape shape_of(const pam_head_norm_desc_t &d, bool backward, int v, bool wide)
{
    Shape s{v, lanes_of(d, v), 1, 1, wide};
    const int64_t tokens = (int64_t)d.batch * d.length, per = kThreads / s.group;
    const int64_t blocks = backward ? kBwdBlocks : kFwdBlocks, turns = backward ? kBwdTurns : kFwdTurns;
    auto chunks = [&](int64_t rows, int64_t share) {
        return (int)std::max<int64_t>({1, std::min<int64_t>(share, rows / (per * turns))});
    };
    const int64_t all = d.heads + d.kv_heads;
    if (d.w_per_head) {
        s.chunks_q = s.chunks_k = chunks(tokens, std::max<int64_t>(1, blocks / all));
    } else {
        s.chunks_q = chunks(tokens * d.heads, std::max<int64_t>(1, blocks * (int64_t)d.heads / all));
        s.chunks_k = chunks(tokens * d.kv_heads, std::max<int64_t>(1, blocks * (int64_t)d.kv_heads / all));
    }
    if (!backward && (tokens * all) / per < blocks) {  // few rows: a turn each, in blocks of their own
        auto turn = [&](int64_t rows) { return (int)std::max<int64_t>(1, (rows + per - 1) / per); };
        s.chunks_q = turn(d.w_per_head ? tokens : tokens * d.heads);
        s.chunks_k = turn(d.w_per_head ? tokens : tokens * d.kv_heads);
    }
    return s;
}

// The widest groups of channels, of 8 or 4, that divide a row's parts and the
// place of every row; else 8, one by one.
Shape shape_of(const pam_head_norm_desc_t &d, bool backward, uint64_t places, const float *w_q, const float *w_k,
               const float *table)
{
    const int es = d.dtype == PAM_F32 ? 4 : 2;
    uint64_t all = (uint64_t)(d.pairs | d.dim) | places / es;
    for (int i = 0; i < 3; ++i)
        all |= (uint64_t)d.q_stride[i] | (d.kv_heads ? (uint64_t)d.k_stride[i] : 0);
    const uint64_t vectors = (uintptr_t)w_q | (uintptr_t)w_k | (uintptr_t)table;
    if (vectors % 16 == 0 && places % es == 0) {
        // f32: eight are two accesses of 16 bytes, which every place has to be a multiple of
        if (all % 8 == 0)
            return shape_of(d, backward, 8, true);
        if (all % 4 == 0 && lanes_of(d, 4) <= 64)
            return shape_of(d, backward, 4, true);
    }
    return shape_of(d, backward, 8, false);
}

HeadNormArgs args_of(const pam_head_norm_desc_t &d, const Shape &s, const void *q, const void *k, const float *w_q,
                     const float *w_k, const float *table, const int32_t *pos)
{
    HeadNormArgs a{};
    a.q = q;
    a.k = k;
    a.w_q = w_q;
    a.w_k = w_k;
    a.table = (const float2 *)table;
    a.pos = pos;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = d.q_stride[i];
        a.ks[i] = d.k_stride[i];
    }
    a.start = d.start;
    a.entries = d.entries;
    a.batch = d.batch;
    a.length = d.length;
    a.heads = d.heads;
    a.kv_heads = d.kv_heads;
    a.dim = d.dim;
    a.pairs = d.pairs;
    a.group = s.group;
    a.chunks_q = s.chunks_q;
    a.chunks_k = s.chunks_k;
    a.layer = d.norm == PAM_NORM_LAYER;
    a.per_head = d.w_per_head != 0;
    a.eps = d.eps;
    a.by_length = Divisor::of(std::max(d.length, 1));
    a.by_heads = Divisor::of(d.heads);
    a.by_kv_heads = Divisor::of(std::max(d.kv_heads, 1));
    return a;
}

template <class T, int V, bool INTERLEAVED, bool WIDE>
hipError_t launch_as(const HeadNormArgs &a, const Shape &sh, unsigned blocks, bool backward, hipStream_t s)
{
    if (!backward) {
        hipLaunchKernelGGL((k_head_norm_fwd<T, V, INTERLEAVED, WIDE>), dim3(blocks), dim3(kThreads), 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((k_head_norm_bwd<T, V, INTERLEAVED, WIDE>), dim3(blocks), dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !(a.gw_q || a.gw_k))
        return e;
    const int64_t vectors = a.per_head ? a.heads + a.kv_heads : 1 + (a.kv_heads > 0);
    const int64_t per = (sh.group * 2 * V + kSumSlots - 1) / kSumSlots;
    hipLaunchKernelGGL((k_head_norm_sum<T, V, INTERLEAVED, WIDE>), dim3((unsigned)(vectors * per)), dim3(kSumThreads), 0,
                       s, a);
    return hipGetLastError();
}

template <class T>
hipError_t launch_type(const HeadNormArgs &a, const Shape &sh, bool interleaved, unsigned blocks, bool backward,
                       hipStream_t s)
{
    if (!sh.wide)
        return interleaved ? launch_as<T, 8, true, false>(a, sh, blocks, backward, s)
                           : launch_as<T, 8, false, false>(a, sh, blocks, backward, s);
    if (sh.v == 8)
        return interleaved ? launch_as<T, 8, true, true>(a, sh, blocks, backward, s)
                           : launch_as<T, 8, false, true>(a, sh, blocks, backward, s);
    return interleaved ? launch_as<T, 4, true, true>(a, sh, blocks, backward, s)
                       : launch_as<T, 4, false, true>(a, sh, blocks, backward, s);
}

hipError_t launch_any(int32_t dtype, const HeadNormArgs &a, const Shape &sh, bool interleaved, unsigned blocks, bool backward,
                      hipStream_t s)
{
    if (dtype == PAM_F32)
        return launch_type<float>(a, sh, interleaved, blocks, backward, s);
    return dtype == PAM_F16 ? launch_type<f16>(a, sh, interleaved, blocks, backward, s)
                            : launch_type<bf16>(a, sh, interleaved, blocks, backward, s);
}

}  // namespace

hipError_t launch_head_norm_fwd(const pam_head_norm_desc_t &d, const void *q, const void *k, const float *w_q,
                                const float *w_k, const float *table, const int32_t *pos, void *q_out, void *k_out,
                                hipStream_t s)
{
    const Shape sh = shape_of(d, false, (uintptr_t)q | (uintptr_t)k | (uintptr_t)q_out | (uintptr_t)k_out, w_q, w_k, table);
    HeadNormArgs a = args_of(d, sh, q, k, w_q, w_k, table, pos);
    a.q_out = q_out;
    a.k_out = k_out;
    return launch_any(d.dtype, a, sh, d.flags & PAM_ROTARY_INTERLEAVED, (unsigned)sh.blocks(d), false, s);
}

// by the descriptor alone: the largest of what the widths take
size_t head_norm_bwd_workspace(const pam_head_norm_desc_t &d)
{
    int64_t most = 0;
    for (int v = 4; v <= 8; v += 4) {
        if (lanes_of(d, v) > 64)
            continue;
        const Shape s = shape_of(d, true, v, true);
        most = std::max(most, s.blocks(d) * s.group * 2 * v);
    }
    return (size_t)most * sizeof(float);
}

hipError_t launch_head_norm_bwd(const pam_head_norm_desc_t &d, const void *q, const void *k, const float *w_q,
                                const float *w_k, const float *table, const int32_t *pos, const void *gq_out,
                                const void *gk_out, void *gq, void *gk, float *gw_q, float *gw_k, void *workspace,
                                hipStream_t s)
{
    const Shape sh = shape_of(d, true, (uintptr_t)q | (uintptr_t)k | (uintptr_t)gq_out | (uintptr_t)gk_out | (uintptr_t)gq |
                                     (uintptr_t)gk,
                              w_q, w_k, table);
    HeadNormArgs a = args_of(d, sh, q, k, w_q, w_k, table, pos);
    a.q_out = gq;
    a.k_out = gk;
    a.gq = gq_out;
    a.gk = gk_out;
    a.gw_q = gw_q;
    a.gw_k = gw_k;
    a.part = (float *)workspace;
    return launch_any(d.dtype, a, sh, d.flags & PAM_ROTARY_INTERLEAVED, (unsigned)sh.blocks(d), true, s);
}

}  // namespace pam
