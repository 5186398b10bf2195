// The norms before and after a block with its gate, residual scale and
// dropout, and dropout alone (gfx950).
//
//   r = x + m scale gate (N(z) w_post + b_post),  h = N(r) w_pre + b_pre,
// m the factors of dropout.  A row stays in the registers of the lanes that
// hold it from its one load to its one store: the sums of its norms are sums
// over lanes.  The backward pass forms r again from x and z, so it reads what
// the forward pass read and no statistic is kept.
#include "pam_rows.h"

#include <algorithm>
#include <initializer_list>
#include <type_traits>

namespace pam {

namespace {

struct NormArgs {
    const void *x, *z, *gate, *grad_r, *grad_h;
    const float *w_post, *b_post, *scale, *w_pre, *b_pre;
    void *r, *h, *grad_x, *grad_z;
    float *part;  // per chunk: sums of gate t zn, gate t, dh rn, dh, and the gate's gradient
    void *grad_gate;
    int64_t rows, gate_rows, groups, xs, zs;
    int32_t channels, chunks, per_group;  // per_group: chunks per gate row, 0: a chunk holds whole gate rows
    float eps;
    Dropout drop;
    bool dropping, layer;
};

// A team of G lanes (of W waves, if W > 1) holds a row, 8 NV channels in
// every lane: VEC, runs of eight channels per lane, read and written 16 bytes
// at a time; else consecutive lanes hold consecutive channels.
template <class T, int G, int NV, int W, bool VEC>
struct Team {
    static constexpr int kLanes = G * W;
    static constexpr int kThreads = W > 4 ? 64 * W : 256;
    static constexpr int kTeams = kThreads / kLanes;
    int lane, team, C;

    __device__ __forceinline__ explicit Team(int channels)
        : lane(threadIdx.x % kLanes), team(threadIdx.x / kLanes), C(channels)
    {
    }
    __device__ __forceinline__ int col(int v, int j) const
    {
        return VEC ? (v * kLanes + lane) * 8 + j : (v * 8 + j) * kLanes + lane;
    }
    template <class E>
    __device__ __forceinline__ void load(const E *p, float (&x)[NV][8], float rest, bool ok = true) const
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (VEC) {
                if (ok && col(v, 0) < C) {
                    load8(p + col(v, 0), x[v]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        x[v][j] = rest;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[v][j] = ok && col(v, j) < C ? (float)p[col(v, j)] : rest;
            }
        }
    }
    // a vector of channels fp32 values: one, or `rest` everywhere
    __device__ __forceinline__ void param(const float *p, float (&x)[NV][8], float rest) const
    {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[v][j] = p && col(v, j) < C ? p[col(v, j)] : rest;
    }
    template <class E>
    __device__ __forceinline__ void store(E *p, const float (&x)[NV][8]) const
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (VEC) {
                if (col(v, 0) < C)
                    store8(p + col(v, 0), x[v]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col(v, j) < C)
                        p[col(v, j)] = (E)x[v][j];
            }
        }
    }
    // Sum over the team, in every lane.  All threads of the block take part.
    __device__ __forceinline__ float sum(float x, float *lds, int &turn) const
    {
        x = lanes_sum<G>(x);
        if constexpr (W > 1) {
            // two sets of places in turn: a set is written again only after
            // the barrier that follows its reading
            float *at = lds + turn * W;
            turn ^= 1;
            if ((threadIdx.x & 63) == 0)
                at[threadIdx.x >> 6] = x;
            __syncthreads();
            x = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w)
                x += at[w];
        }
        return x;
    }
    // Factors of dropout of row `row`.  Eight channels of a lane are the eight
    // of one counter where the rows are whole counters.
    __device__ __forceinline__ void factors(const Dropout &d, int64_t row, float (&m)[NV][8]) const
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (VEC) {
                const uint4v w = philox(d, (uint64_t)(row * C + col(v, 0)) >> 3);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    m[v][j] = kept(d, w, j) ? d.keep : 0.0f;
            } else {
#pragma unroll 1
                for (int j = 0; j < 8; ++j) {
                    const uint64_t e = (uint64_t)(row * C + col(v, j));
                    const uint4v w = philox(d, e >> 3);
                    const int i = (int)(e & 7);
                    const uint32_t lo = (i & 2) ? w[1] : w[0], hi = (i & 2) ? w[3] : w[2];
                    const uint32_t u = ((i & 4) ? hi : lo) >> (16 * (i & 1)) & 0xffffu;
                    const float f = u >= d.limit ? d.keep : 0.0f;
#pragma unroll
                    for (int k = 0; k < 8; ++k)  // no index into registers that is not constant
                        m[v][k] = k == j ? f : m[v][k];
                }
            }
        }
    }
    __device__ __forceinline__ bool holds(int v, int j) const { return col(v, VEC ? 0 : j) < C; }
};

// t to N(t) in place (0 outside the row); returns the reciprocal deviation.
// The mean is taken out before the squares are summed.
template <class TM, int NV>
__device__ __forceinline__ float normalise(const TM &tm, bool layer, float (&t)[NV][8], float eps, float inv_c,
                                           float *lds, int &turn)
{
    if (layer) {
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                s += t[v][j];
        const float mean = tm.sum(s, lds, turn) * inv_c;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                t[v][j] = tm.holds(v, j) ? t[v][j] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            s += t[v][j] * t[v][j];
    const float rd = 1.0f / __builtin_sqrtf(tm.sum(s, lds, turn) * inv_c + eps);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            t[v][j] *= rd;
    return rd;
}

// gradient of t from that of n = N(t): dn to (dn - n mean(dn n) - [mean dn]) rd
template <class TM, int NV>
__device__ __forceinline__ void normalise_grad(const TM &tm, bool layer, float (&dn)[NV][8], const float (&n)[NV][8],
                                               float rd, float inv_c, float *lds, int &turn)
{
    float s = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s += dn[v][j] * n[v][j];
            s1 += dn[v][j];
        }
    const float a = tm.sum(s, lds, turn) * inv_c;
    float b = 0.0f;
    if (layer)
        b = tm.sum(s1, lds, turn) * inv_c;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            dn[v][j] = (dn[v][j] - n[v][j] * a - b) * rd;
}

template <class T, int G, int NV, int W, bool VEC>
__global__ __launch_bounds__((W > 4 ? 64 * W : 256)) void k_norm_fwd(NormArgs a)
{
    using TM = Team<T, G, NV, W, VEC>;
    __shared__ float lds[2 * W];
    const TM tm(a.channels);
    const float inv_c = 1.0f / (float)a.channels;
    int turn = 0;
    float wq[NV][8], bq[NV][8], sc[NV][8], wp[NV][8], bp[NV][8];
    tm.param(a.w_post, wq, 1.0f);
    tm.param(a.b_post, bq, 0.0f);
    tm.param(a.scale, sc, 1.0f);
    tm.param(a.w_pre, wp, 1.0f);
    tm.param(a.b_pre, bp, 0.0f);
    for (int64_t r0 = (int64_t)blockIdx.x * TM::kTeams; r0 < a.rows; r0 += (int64_t)gridDim.x * TM::kTeams) {
        const int64_t row = r0 + tm.team;
        const bool ok = row < a.rows;
        float x[NV][8];
        tm.load((const T *)a.x + row * a.xs, x, 0.0f, ok);
        if (a.z) {
            float u[NV][8], m[NV][8];
            tm.load((const T *)a.z + row * a.zs, u, 0.0f, ok);
            if (a.gate)
                tm.load((const T *)a.gate + (ok ? row / a.gate_rows : 0) * a.channels, m, 0.0f, ok);
            normalise(tm, a.layer, u, a.eps, inv_c, lds, turn);
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    u[v][j] = (u[v][j] * wq[v][j] + bq[v][j]) * sc[v][j];
                    if (a.gate)
                        u[v][j] *= m[v][j];
                }
            if (a.dropping) {
                tm.factors(a.drop, row, m);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        u[v][j] = m[v][j] != 0.0f ? u[v][j] * m[v][j] : 0.0f;
            }
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[v][j] = tm.holds(v, j) ? x[v][j] + u[v][j] : 0.0f;
            if (ok)
                tm.store((T *)a.r + row * a.channels, x);
        }
        if (a.h) {
            normalise(tm, a.layer, x, a.eps, inv_c, lds, turn);
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[v][j] = x[v][j] * wp[v][j] + bp[v][j];
            if (ok)
                tm.store((T *)a.h + row * a.channels, x);
        }
    }
}

// Backward.  With t = m dr (dr the gradient of r) and zn = N(z), the sums over
// the rows that the vectors' gradients need are
//   A1 = sum gate t zn, A0 = sum gate t, P1 = sum dh rn, P0 = sum dh:
//   grad_w_post = scale A1, grad_b_post = scale A0, grad_scale = w_post A1 + b_post A0,
//   grad_w_pre = P1, grad_b_pre = P0,
// and a gate row's gradient is scale (w_post T1 + b_post T0) with T1 = sum t zn,
// T0 = sum t over its rows.  A block takes a chunk of rows, adds up in
// registers, and writes one row of partial sums; a second kernel adds those
// up in a fixed order.  Few gate rows are cut into several chunks each
// (per_group), many are dealt whole to the chunks' teams, which then write
// their gradients themselves.
template <class T, int G, int NV, int W, bool VEC>
__global__ __launch_bounds__((W > 4 ? 64 * W : 256)) void k_norm_bwd(NormArgs a)
{
    using TM = Team<T, G, NV, W, VEC>;
    __shared__ float lds[2 * W];
    __shared__ float cols[TM::kTeams > 1 ? TM::kTeams * TM::kLanes * 8 * NV : 1];
    const TM tm(a.channels);
    const float inv_c = 1.0f / (float)a.channels;
    int turn = 0;
    float wq[NV][8], bq[NV][8], sc[NV][8], wp[NV][8];
    tm.param(a.w_post, wq, 1.0f);
    tm.param(a.b_post, bq, 0.0f);
    tm.param(a.scale, sc, 1.0f);
    tm.param(a.w_pre, wp, 1.0f);
    float A1[NV][8] = {}, A0[NV][8] = {}, P1[NV][8] = {}, P0[NV][8] = {}, DG[NV][8] = {};

    int64_t first, last, outer, inner, step;  // rows of this block; trips
    if (a.per_group) {
        const int64_t g = blockIdx.x / a.per_group, s = blockIdx.x - g * a.per_group;
        const int64_t len = (a.gate_rows + a.per_group - 1) / a.per_group;
        first = g * a.gate_rows + min(s * len, a.gate_rows);
        last = g * a.gate_rows + min((s + 1) * len, a.gate_rows);
        outer = 1;
        inner = (last - first + TM::kTeams - 1) / TM::kTeams;
        step = TM::kTeams;
        first += tm.team;
    } else {
        const int64_t per = (a.groups + a.chunks - 1) / a.chunks;
        const int64_t g0 = min(blockIdx.x * per, a.groups), g1 = min((blockIdx.x + 1) * per, a.groups);
        outer = (g1 - g0 + TM::kTeams - 1) / TM::kTeams;
        inner = a.gate_rows;
        first = (g0 + tm.team) * a.gate_rows;
        last = g1 * a.gate_rows;
        step = 1;
    }
    for (int64_t o = 0; o < outer; ++o) {
        float T1[NV][8] = {}, T0[NV][8] = {}, gate[NV][8];
        const bool some = first < last;
        if (a.gate) {
            tm.load((const T *)a.gate + (some ? first / a.gate_rows : 0) * a.channels, gate, 0.0f, some);
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    gate[v][j] = 1.0f;
        }
        for (int64_t i = 0; i < inner; ++i) {
            const int64_t row = first + i * step;
            const bool ok = row < last;
            float x[NV][8], n[NV][8], m[NV][8], d[NV][8];
            tm.load((const T *)a.x + row * a.xs, x, 0.0f, ok);
            float rz = 0.0f;
            if (a.z)
                tm.load((const T *)a.z + row * a.zs, n, 0.0f, ok);
            if (a.grad_h)
                tm.load((const T *)a.grad_h + row * a.channels, d, 0.0f, ok);
            if (a.z) {
                rz = normalise(tm, a.layer, n, a.eps, inv_c, lds, turn);
                if (a.dropping) {
                    tm.factors(a.drop, row, m);
                } else {
#pragma unroll
                    for (int v = 0; v < NV; ++v)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            m[v][j] = 1.0f;
                }
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float u = (n[v][j] * wq[v][j] + bq[v][j]) * sc[v][j] * gate[v][j];
                        x[v][j] = tm.holds(v, j) && m[v][j] != 0.0f ? x[v][j] + u * m[v][j] : x[v][j];
                    }
            }
            if (a.grad_h) {
                const float rr = normalise(tm, a.layer, x, a.eps, inv_c, lds, turn);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (ok) {
                            P1[v][j] += d[v][j] * x[v][j];
                            P0[v][j] += d[v][j];
                        }
                        d[v][j] *= wp[v][j];
                    }
                normalise_grad(tm, a.layer, d, x, rr, inv_c, lds, turn);
            } else {
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        d[v][j] = 0.0f;
            }
            if (a.grad_r) {
                tm.load((const T *)a.grad_r + row * a.channels, x, 0.0f, ok);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        d[v][j] += x[v][j];
            }
            if (a.grad_x && ok)
                tm.store((T *)a.grad_x + row * a.channels, d);
            if (a.z) {
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float t = tm.holds(v, j) && m[v][j] != 0.0f ? d[v][j] * m[v][j] : 0.0f;
                        if (ok) {
                            T1[v][j] += t * n[v][j];
                            T0[v][j] += t;
                        }
                        d[v][j] = t * gate[v][j] * sc[v][j] * wq[v][j];
                    }
                normalise_grad(tm, a.layer, d, n, rz, inv_c, lds, turn);
                if (a.grad_z && ok)
                    tm.store((T *)a.grad_z + row * a.channels, d);
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                A1[v][j] += gate[v][j] * T1[v][j];
                A0[v][j] += gate[v][j] * T0[v][j];
                DG[v][j] = sc[v][j] * (wq[v][j] * T1[v][j] + bq[v][j] * T0[v][j]);
            }
        if (!a.per_group) {
            if (a.grad_gate && some)
                tm.store((T *)a.grad_gate + first / a.gate_rows * a.channels, DG);
            first += TM::kTeams * a.gate_rows;
        }
    }
    // partial sums of the chunk, the teams' added up in order
    float *part = a.part + (int64_t)blockIdx.x * 5 * a.channels;
    auto flush = [&](const float (&s)[NV][8], int k) {
        if constexpr (TM::kTeams > 1) {
            constexpr int P = TM::kLanes * 8 * NV;
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    cols[tm.team * P + tm.col(v, j)] = s[v][j];
            __syncthreads();
            for (int c = threadIdx.x; c < a.channels; c += TM::kThreads) {
                float y = 0.0f;
                for (int q = 0; q < TM::kTeams; ++q)
                    y += cols[q * P + c];
                part[k * a.channels + c] = y;
            }
        } else {
            tm.store(part + k * a.channels, s);
        }
    };
    if (a.z) {
        flush(A1, 0);
        flush(A0, 1);
    }
    if (a.grad_h) {
        flush(P1, 2);
        flush(P0, 3);
    }
    if (a.grad_gate && a.per_group)
        flush(DG, 4);
}

// Sums of the partial rows: 32 columns per block, 32 rows of threads that
// take every 32nd partial row each, then those 32 added in order.
// blockIdx.y: 0 the post-norm's sums, 1 the pre-norm's, 2 + g gate row g.
template <class T>
__global__ __launch_bounds__(1024) void k_norm_sums(NormArgs a, float *gw_post, float *gb_post, float *gscale,
                                                    float *gw_pre, float *gb_pre)
{
    __shared__ float rows[2][32][33];
    const int cx = threadIdx.x & 31, j = threadIdx.x >> 5, C = a.channels;
    const int c = blockIdx.x * 32 + cx;
    const int what = blockIdx.y;
    const int64_t from = what < 2 ? 0 : (int64_t)(what - 2) * a.per_group;
    const int64_t to = what < 2 ? a.chunks : from + a.per_group;
    const int k0 = what == 0 ? 0 : (what == 1 ? 2 : 4), k1 = what < 2 ? k0 + 1 : k0;
    float s0 = 0.0f, s1 = 0.0f;
    if (c < C)
        for (int64_t p = from + j; p < to; p += 32) {
            s0 += a.part[(p * 5 + k0) * C + c];
            s1 += a.part[(p * 5 + k1) * C + c];
        }
    rows[0][j][cx] = s0;
    rows[1][j][cx] = s1;
    __syncthreads();
    if (j != 0 || c >= C)
        return;
    s0 = s1 = 0.0f;
    for (int q = 0; q < 32; ++q) {
        s0 += rows[0][q][cx];
        s1 += rows[1][q][cx];
    }
    const float w = a.w_post ? a.w_post[c] : 1.0f, b = a.b_post ? a.b_post[c] : 0.0f, sc = a.scale ? a.scale[c] : 1.0f;
    if (what == 0) {
        if (gw_post)
            gw_post[c] = sc * s0;
        if (gb_post)
            gb_post[c] = sc * s1;
        if (gscale)
            gscale[c] = w * s0 + b * s1;
    } else if (what == 1) {
        if (gw_pre)
            gw_pre[c] = s0;
        if (gb_pre)
            gb_pre[c] = s1;
    } else {
        ((T *)a.grad_gate)[(int64_t)(what - 2) * C + c] = (T)s0;
    }
}

template <class T, bool VEC>
__global__ __launch_bounds__(256) void k_dropout(const T *x, T *y, int64_t n, Dropout d)
{
    const int64_t groups = (n + 7) / 8;
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += (int64_t)gridDim.x * 256) {
        const uint4v w = philox(d, (uint64_t)g);
        if (VEC && g * 8 + 8 <= n) {
            float v[8];
            load8(x + g * 8, v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = kept(d, w, j) ? v[j] * d.keep : 0.0f;
            store8(y + g * 8, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (g * 8 + j < n)
                    y[g * 8 + j] = kept(d, w, j) ? (T)((float)x[g * 8 + j] * d.keep) : (T)0.0f;
        }
    }
}

Dropout dropout_of(double p, uint64_t seed, uint64_t offset)
{
    Dropout d;
    d.k0 = (uint32_t)seed;
    d.k1 = (uint32_t)(seed >> 32);
    d.o0 = (uint32_t)offset;
    d.o1 = (uint32_t)(offset >> 32);
    d.limit = (uint32_t)__builtin_rint(p * 65536.0);
    d.keep = d.limit < 65536u ? (float)(65536.0 / (65536.0 - d.limit)) : 0.0f;
    return d;
}

// The team for rows of c channels.  16-byte accesses: the smallest that holds
// a row, groups of 8 to 64 lanes with eight channels each, then sixteen per
// lane, then 4 and 8 waves.  Others (an odd number of channels, odd strides or
// addresses) have three sizes, and read as many lines as whole waves do.
template <class F>
auto with_shape(int c, bool vec, const F &f)
{
#define PAM_TEAM(G, NV, W, VEC)                                                                   \
    f(std::integral_constant<int, G>(), std::integral_constant<int, NV>(), std::integral_constant<int, W>(),      \
      std::integral_constant<bool, VEC>())
    if (!vec)
        return c <= 512 ? PAM_TEAM(64, 1, 1, false) : (c <= 2048 ? PAM_TEAM(64, 1, 4, false) : PAM_TEAM(64, 2, 8, false));
    if (c <= 64)
        return PAM_TEAM(8, 1, 1, true);
    if (c <= 128)
        return PAM_TEAM(16, 1, 1, true);
    if (c <= 256)
        return PAM_TEAM(32, 1, 1, true);
    if (c <= 512)
        return PAM_TEAM(64, 1, 1, true);
    if (c <= 1024)
        return PAM_TEAM(64, 2, 1, true);
    if (c <= 2048)
        return PAM_TEAM(64, 1, 4, true);
    if (c <= 4096)
        return PAM_TEAM(64, 2, 4, true);
    return PAM_TEAM(64, 2, 8, true);
#undef PAM_TEAM
}
int teams_of(int c, bool vec)
{
    return with_shape(c, vec, [](auto g, auto, auto w, auto) { return (w > 4 ? 64 * w : 256) / (g * w); });
}

struct Chunks {
    int32_t chunks, per_group;
};
Chunks chunks_of(const pam_norm_desc_t &d, bool gated, bool vec)
{
    // about four blocks per CU, none without a row for each of its teams
    const int64_t most = 1024, teams = teams_of(d.channels, vec);
    const int64_t groups = gated ? d.rows / std::max<int64_t>(d.gate_rows, 1) : 1;
    const int64_t gate_rows = gated ? d.gate_rows : d.rows;
    if (groups > most)
        return {(int32_t)std::min<int64_t>(most, (groups + teams - 1) / teams), 0};
    int64_t per = std::max<int64_t>(1, most / std::max<int64_t>(groups, 1));
    per = std::max<int64_t>(1, std::min<int64_t>(per, (gate_rows + teams - 1) / teams));
    return {(int32_t)(per * std::max<int64_t>(groups, 1)), (int32_t)per};
}

template <class T>
void launch_norm_t(const NormArgs &a, bool vec, bool bwd, hipStream_t s)
{
    with_shape(a.channels, vec, [&](auto g, auto nv, auto w, auto wide) {
        using TM = Team<T, g, nv, w, wide>;
        if (bwd) {
            hipLaunchKernelGGL((k_norm_bwd<T, g, nv, w, wide>), dim3(a.chunks), dim3(TM::kThreads), 0, s, a);
        } else {
            const unsigned blocks = (unsigned)std::min<int64_t>((a.rows + TM::kTeams - 1) / TM::kTeams, 4096);
            hipLaunchKernelGGL((k_norm_fwd<T, g, nv, w, wide>), dim3(blocks), dim3(TM::kThreads), 0, s, a);
        }
    });
}

void launch_norm(const pam_norm_desc_t &d, const NormArgs &a, bool vec, bool bwd, hipStream_t s)
{
    if (d.dtype == PAM_F32)
        launch_norm_t<float>(a, vec, bwd, s);
    else if (d.dtype == PAM_F16)
        launch_norm_t<f16>(a, vec, bwd, s);
    else
        launch_norm_t<bf16>(a, vec, bwd, s);
}

// 16-byte accesses: rows of whole groups of eight channels, every one at a
// multiple of 16 bytes
bool rows_wide(const pam_norm_desc_t &d, std::initializer_list<const void *> ptrs)
{
    const int v = d.dtype == PAM_F32 ? 4 : 8;
    if (d.channels % 8 || d.x_stride % v || d.z_stride % v)
        return false;
    for (const void *p : ptrs)
        if ((uintptr_t)p % 16)
            return false;
    return true;
}

NormArgs norm_args(const pam_norm_desc_t &d, const void *x, const void *z, const float *w_post, const float *b_post,
                   const void *gate, const float *scale, const float *w_pre)
{
    NormArgs a{};
    a.x = x;
    a.z = z;
    a.gate = gate;
    a.w_post = w_post;
    a.b_post = b_post;
    a.scale = scale;
    a.w_pre = w_pre;
    a.rows = d.rows;
    a.gate_rows = gate ? d.gate_rows : d.rows;
    a.groups = a.gate_rows ? d.rows / a.gate_rows : 0;
    a.xs = d.x_stride;
    a.zs = d.z_stride;
    a.channels = d.channels;
    a.eps = d.eps;
    a.dropping = d.p > 0.0;
    a.layer = d.norm == PAM_NORM_LAYER;
    a.drop = dropout_of(d.p, d.seed, d.offset);
    return a;
}

}  // namespace

hipError_t launch_norm_fwd(const pam_norm_desc_t &d, const void *x, const void *z, const float *w_post,
                           const float *b_post, const void *gate, const float *scale, const float *w_pre,
                           const float *b_pre, void *r, void *h, hipStream_t s)
{
    if (d.rows == 0)
        return hipSuccess;
    NormArgs a = norm_args(d, x, z, w_post, b_post, gate, scale, w_pre);
    a.b_pre = b_pre;
    a.r = r;
    a.h = h;
    launch_norm(d, a, rows_wide(d, {x, z, gate, r, h}), false, s);
    return hipGetLastError();
}

size_t norm_bwd_workspace(const pam_norm_desc_t &d)
{
    // with and without a gate, with wide accesses and without: whichever needs most
    int64_t n = 0;
    for (int how = 0; how < 4; ++how)
        n = std::max<int64_t>(n, chunks_of(d, how & 1, how & 2).chunks);
    return (size_t)n * 5 * d.channels * sizeof(float);
}

hipError_t launch_norm_bwd(const pam_norm_desc_t &d, const void *x, const void *z, const float *w_post,
                           const float *b_post, const void *gate, const float *scale, const float *w_pre,
                           const void *grad_r, const void *grad_h, void *grad_x, void *grad_z, float *gw_post,
                           float *gb_post, void *grad_gate, float *gscale, float *gw_pre, float *gb_pre,
                           void *workspace, hipStream_t s)
{
    NormArgs a = norm_args(d, x, z, w_post, b_post, gate, scale, w_pre);
    a.grad_r = grad_r;
    a.grad_h = grad_h;
    a.grad_x = grad_x;
    a.grad_z = grad_z;
    a.grad_gate = grad_gate;
    a.part = (float *)workspace;
    const bool vec = rows_wide(d, {x, z, gate, grad_r, grad_h, grad_x, grad_z, grad_gate});
    const Chunks ch = chunks_of(d, gate != nullptr, vec);
    a.chunks = ch.chunks;
    a.per_group = ch.per_group;
    if (d.rows)
        launch_norm(d, a, vec, true, s);
    else
        a.chunks = 0;  // sums of no rows
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    const bool by_group = grad_gate && a.per_group && d.rows;
    const dim3 grid((d.channels + 31) / 32, 2 + (by_group ? (unsigned)a.groups : 0));
    // sums that were not written are not read: no output asks for them
    if (!z && d.rows)
        gw_post = gb_post = gscale = nullptr;
    if (!grad_h && d.rows)
        gw_pre = gb_pre = nullptr;
    if (!gw_post && !gb_post && !gscale && !gw_pre && !gb_pre && !by_group)
        return hipSuccess;
    if (d.dtype == PAM_F32)
        hipLaunchKernelGGL(k_norm_sums<float>, grid, dim3(1024), 0, s, a, gw_post, gb_post, gscale, gw_pre, gb_pre);
    else if (d.dtype == PAM_F16)
        hipLaunchKernelGGL(k_norm_sums<f16>, grid, dim3(1024), 0, s, a, gw_post, gb_post, gscale, gw_pre, gb_pre);
    else
        hipLaunchKernelGGL(k_norm_sums<bf16>, grid, dim3(1024), 0, s, a, gw_post, gb_post, gscale, gw_pre, gb_pre);
    return hipGetLastError();
}

hipError_t launch_dropout(const void *x, int64_t n, int32_t dtype, double p, uint64_t seed, uint64_t offset, void *y,
                          hipStream_t s)
{
    if (n == 0)
        return hipSuccess;
    const Dropout d = dropout_of(p, seed, offset);
    const bool vec = ((uintptr_t)x | (uintptr_t)y) % 16 == 0;
    const unsigned blocks = (unsigned)std::min<int64_t>(((n + 7) / 8 + 255) / 256, 1 << 20);
    auto go = [&](auto t) {
        using T = decltype(t);
        if (vec)
            hipLaunchKernelGGL((k_dropout<T, true>), dim3(blocks), dim3(256), 0, s, (const T *)x, (T *)y, n, d);
        else
            hipLaunchKernelGGL((k_dropout<T, false>), dim3(blocks), dim3(256), 0, s, (const T *)x, (T *)y, n, d);
    };
    if (dtype == PAM_F32)
        go(0.0f);
    else if (dtype == PAM_F16)
        go((f16)0.0f);
    else
        go((bf16)0.0f);
    return hipGetLastError();
}

}  // namespace pam
