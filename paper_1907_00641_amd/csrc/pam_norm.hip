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

// Eight consecutive channels of a row as they lie in memory, so that the rows
// ahead wait in few registers.
template <class T>
struct Raw {
    static constexpr int kPieces = sizeof(T) / 2;  // of 16 bytes
    uint4v p[kPieces];
    __device__ __forceinline__ void unpack(float (&x)[8]) const
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t y = p[j / 4][j % 4];
                x[j] = __uint_as_float(y);
            }
        } else {
            typedef T T8 __attribute__((ext_vector_type(8)));
            const T8 y = __builtin_bit_cast(T8, p[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = (float)y[j];
        }
    }
};

// A team of G lanes (of W waves, if W > 1) holds a row, eight consecutive
// channels in every lane, read and written 16 bytes at a time; WIDE: at multiples
// of 16 bytes and in whole eights, else wherever the row starts, and the row's last
// few one by one.  A block has one team or more.
template <class T, int G, int W, bool WIDE>
struct Team {
    static constexpr int kLanes = G * W;
    static constexpr int kThreads = W > 4 ? 64 * W : 256;
    static constexpr int kTeams = kThreads / kLanes;
    int lane, team, C, c0;

    __device__ __forceinline__ explicit Team(int channels)
        : lane(threadIdx.x % kLanes), team(threadIdx.x / kLanes), C(channels), c0(threadIdx.x % kLanes * 8)
    {
    }
    __device__ __forceinline__ bool holds(int j) const { return WIDE ? c0 < C : c0 + j < C; }
    // this lane's channels of the row at p; 0 past the row, or if not `ok`
    __device__ __forceinline__ Raw<T> load(const T *p, bool ok) const
    {
        Raw<T> r{};
        if constexpr (WIDE) {
            if (ok && c0 < C) {
#pragma unroll
                for (int i = 0; i < Raw<T>::kPieces; ++i)
                    r.p[i] = load16((const char *)(p + c0) + 16 * i);
            }
        } else {
            if (ok && c0 + 8 <= C) {
                __builtin_memcpy(&r, p + c0, sizeof r);
            } else if (ok && c0 < C) {
                T x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[j] = c0 + j < C ? p[c0 + j] : (T)0.0f;
                __builtin_memcpy(&r, x, sizeof r);
            }
        }
        return r;
    }
    // A vector of fp32 values, one for each channel, laid out in LDS for the block's
    // teams (`rest` everywhere if there is none); read back 8 at a time, in two
    // halves without bank conflicts.
    struct Vector {
        float4v half[2][kLanes];
    };
    __device__ __forceinline__ static float at(const float *p, int c, int C, float rest)
    {
        return p && c < C ? p[c] : rest;
    }
    template <class F>
    __device__ __forceinline__ static void lay(Vector &v, const F &f)
    {
        for (int c = threadIdx.x; c < kLanes * 8; c += kThreads)
            ((float *)&v.half[(c >> 2) & 1][c >> 3])[c & 3] = f(c);
    }
    __device__ __forceinline__ void take(const Vector &v, float (&x)[8]) const
    {
        int l = lane;
        asm volatile("" : "+v"(l));  // read again for every row, rather than kept in registers
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[j] = v.half[j >> 2][l][j & 3];
    }
    template <class E>
    __device__ __forceinline__ void store(E *p, const float (&x)[8]) const
    {
        if (WIDE ? c0 < C : c0 + 8 <= C) {
            if constexpr (WIDE) {
                store8(p + c0, x);
            } else {
                E y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    y[j] = (E)x[j];
                __builtin_memcpy(p + c0, y, sizeof y);
            }
        } else if (!WIDE) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j < C)
                    p[c0 + j] = (E)x[j];
        }
    }
    // Sum over the team, in every lane.  All threads of the block take part.
    __device__ __forceinline__ float sum(float x, float *lds, int &turn) const
    {
        x = lanes_sum<G>(x);
        if constexpr (W > 1) {
            // two sets of places in turn: a set is written again only after
            // the barrier that follows its reading
            float *at = lds + turn * (kThreads / 64);
            turn ^= 1;
            if ((threadIdx.x & 63) == 0)
                at[threadIdx.x >> 6] = x;
            __syncthreads();
            x = lanes_sum<W>(at[team * W + lane % W]);
        }
        return x;
    }
    // Which of this lane's channels of row `row` dropout keeps, as bits.  Eight
    // elements take the numbers of one counter; a row that does not start with one
    // has eight of the sixteen of two.
    __device__ __forceinline__ uint32_t kept_bits(const Dropout &d, int64_t row) const
    {
        const uint64_t e = (uint64_t)row * C + c0;
        uint32_t bits = bits_of(d, philox(d, e >> 3));
        if (!WIDE && (e & 7))
            bits = (bits | bits_of(d, philox(d, (e >> 3) + 1)) << 8) >> (e & 7);
        return bits;
    }
    __device__ __forceinline__ static uint32_t bits_of(const Dropout &d, const uint4v &w)
    {
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            bits |= kept(d, w, j) ? 1u << j : 0u;
        return bits;
    }
};

// t to N(t) in place (0 outside the row); returns the reciprocal deviation.
// The mean is taken out before the squares are summed.  `ok` false: the team has no
// row, t is 0 and stays 0, also with eps 0, since the vectors' sums run over it.
template <class TM>
__device__ __forceinline__ float normalise(const TM &tm, bool ok, bool layer, float (&t)[8], float eps, float inv_c,
                                           float *lds, int &turn)
{
    if (layer) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            s += t[j];
        const float mean = tm.sum(s, lds, turn) * inv_c;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            t[j] = tm.holds(j) ? t[j] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        s += t[j] * t[j];
    const float deviation = __builtin_sqrtf(tm.sum(s, lds, turn) * inv_c + eps);
    const float rd = ok ? 1.0f / deviation : 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        t[j] *= rd;
    return rd;
}

// gradient of t from that of n = N(t): dn to (dn - n mean(dn n) - [mean dn]) rd
template <class TM>
__device__ __forceinline__ void normalise_grad(const TM &tm, bool layer, float (&dn)[8], const float (&n)[8], float rd,
                                               float inv_c, float *lds, int &turn)
{
    float s = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        s += dn[j] * n[j];
        s1 += dn[j];
    }
    const float a = tm.sum(s, lds, turn) * inv_c;
    float b = 0.0f;
    if (layer)
        b = tm.sum(s1, lds, turn) * inv_c;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        dn[j] = (dn[j] - n[j] * a - b) * rd;
}

// Forward.  Bound by memory: it reads x and z and writes r and h once, and each
// row is loaded while the one before it is at work (against loading it when it is
// needed: 64 us for 97).  The vectors stay in registers; read from LDS for every
// row they cost 72 us for 64.  bf16 76800 x 512, all outputs, dropout: 66 us,
// 4.8 TB/s, the rate of a large copy.
template <class T, int G, int W, bool WIDE>
__global__ __launch_bounds__((W > 4 ? 64 * W : 256)) void k_norm_fwd(NormArgs a)
{
    using TM = Team<T, G, W, WIDE>;
    __shared__ float lds[2 * (TM::kThreads / 64)];
    const TM tm(a.channels);
    const float inv_c = 1.0f / (float)a.channels;
    int turn = 0;
    // scale w_post, scale b_post, w_pre, b_pre
    float k1[8], k0[8], wp[8], bp[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = tm.c0 + j, C = a.channels;
        k1[j] = TM::at(a.scale, c, C, 1.0f) * TM::at(a.w_post, c, C, 1.0f);
        k0[j] = TM::at(a.scale, c, C, 1.0f) * TM::at(a.b_post, c, C, 0.0f);
        wp[j] = TM::at(a.w_pre, c, C, 1.0f);
        bp[j] = TM::at(a.b_pre, c, C, 0.0f);
    }
    const int64_t step = (int64_t)gridDim.x * TM::kTeams;
    int64_t r0 = (int64_t)blockIdx.x * TM::kTeams;
    Raw<T> nx, nz, ng;
    auto fetch = [&](int64_t row) {
        const bool ok = row < a.rows;
        nx = tm.load((const T *)a.x + row * a.xs, ok);
        if (a.z) {
            nz = tm.load((const T *)a.z + row * a.zs, ok);
            if (a.gate)
                ng = tm.load((const T *)a.gate + (ok ? quotient(row, a.gate_rows) : 0) * a.channels, ok);
        }
    };
    fetch(r0 + tm.team);
    for (; r0 < a.rows; r0 += step) {
        const int64_t row = r0 + tm.team;
        const bool ok = row < a.rows;
        float x[8], u[8], g[8];
        nx.unpack(x);
        if (a.z) {
            nz.unpack(u);
            if (a.gate)
                ng.unpack(g);
        }
        fetch(row + step);
        if (a.z) {
            const uint32_t bits = a.dropping ? tm.kept_bits(a.drop, row) : 255u;
            normalise(tm, ok, a.layer, u, a.eps, inv_c, lds, turn);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float y = u[j] * k1[j] + k0[j];
                if (a.gate)
                    y *= g[j];
                y *= a.drop.keep;
                x[j] = (bits >> j & 1) && tm.holds(j) ? x[j] + y : x[j];
            }
            if (ok)
                tm.store((T *)a.r + row * a.channels, x);
        }
        if (a.h) {
            normalise(tm, ok, a.layer, x, a.eps, inv_c, lds, turn);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = x[j] * wp[j] + bp[j];
            if (ok)
                tm.store((T *)a.h + row * a.channels, x);
        }
    }
}

// Backward.  With t = m dr (dr the gradient of r, m the factors of dropout) and
// zn = N(z), the sums over the rows that the vectors' gradients need are
//   A1 = sum gate t zn, A0 = sum gate t, P1 = sum dh rn, P0 = sum dh:
//   grad_w_post = scale A1, grad_b_post = scale A0, grad_scale = w_post A1 + b_post A0,
//   grad_w_pre = P1, grad_b_pre = P0,
// and a gate row's gradient is scale (w_post T1 + b_post T0) with T1 = sum t zn,
// T0 = sum t over its rows.  A block takes a chunk of rows, adds up in
// registers, and writes one row of partial sums; a second kernel adds those
// up in a fixed order.  Few gate rows (WHOLE false) are cut into per_group chunks
// each; many are dealt whole to the chunks' teams, which then write their
// gradients themselves.
template <class T, int G, int W, bool WIDE, bool WHOLE>
__global__ __launch_bounds__((W > 4 ? 64 * W : 256)) void k_norm_bwd(NormArgs a)
{
    using TM = Team<T, G, W, WIDE>;
    __shared__ float lds[2 * (TM::kThreads / 64)];
    __shared__ float cols[TM::kTeams > 1 ? TM::kTeams * TM::kLanes * 8 : 1];
    const TM tm(a.channels);
    const float inv_c = 1.0f / (float)a.channels;
    int turn = 0;
    __shared__ typename TM::Vector k1, k0, wp;  // scale w_post, scale b_post, w_pre
    const int C = a.channels;
    TM::lay(k1, [&](int c) { return TM::at(a.scale, c, C, 1.0f) * TM::at(a.w_post, c, C, 1.0f); });
    TM::lay(k0, [&](int c) { return TM::at(a.scale, c, C, 1.0f) * TM::at(a.b_post, c, C, 0.0f); });
    TM::lay(wp, [&](int c) { return TM::at(a.w_pre, c, C, 1.0f); });
    __syncthreads();
    float A1[8] = {}, A0[8] = {}, P1[8] = {}, P0[8] = {}, T1[8] = {}, T0[8] = {};

    int64_t first, last, outer, inner, step;  // rows of this block; trips
    if constexpr (WHOLE) {
        const int64_t per = (a.groups + a.chunks - 1) / a.chunks;
        const int64_t g0 = min(blockIdx.x * per, a.groups), g1 = min((blockIdx.x + 1) * per, a.groups);
        outer = (g1 - g0 + TM::kTeams - 1) / TM::kTeams;
        inner = a.gate_rows;
        first = (g0 + tm.team) * a.gate_rows;
        last = g1 * a.gate_rows;
        step = 1;
    } else {
        const int64_t g = blockIdx.x / a.per_group, s = blockIdx.x - g * a.per_group;
        const int64_t len = (a.gate_rows + a.per_group - 1) / a.per_group;
        first = g * a.gate_rows + min(s * len, a.gate_rows);
        last = g * a.gate_rows + min((s + 1) * len, a.gate_rows);
        outer = 1;
        inner = (last - first + TM::kTeams - 1) / TM::kTeams;
        step = TM::kTeams;
        first += tm.team;
    }
    // The next row's loads are under way while a row is at work, but in the
    // largest blocks, which have no registers left for it.
    constexpr bool AHEAD = W < 16;
    Raw<T> nx, nz, nh, nr;
    auto fetch = [&](int64_t row, bool ok) {
        nx = tm.load((const T *)a.x + row * a.xs, ok);
        if (a.z)
            nz = tm.load((const T *)a.z + row * a.zs, ok);
        if (a.grad_h)
            nh = tm.load((const T *)a.grad_h + row * a.channels, ok);
        if (a.grad_r)
            nr = tm.load((const T *)a.grad_r + row * a.channels, ok);
    };
    // [w_post, b_post, scale of T1 and T0] as a gate row's gradient
    auto gate_grad = [&](float (&y)[8]) {
        float m[8], b[8];
        tm.take(k1, m);
        tm.take(k0, b);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            y[j] = m[j] * T1[j] + b[j] * T0[j];
    };
    for (int64_t o = 0; o < outer; ++o) {
        const bool some = first < last;
        Raw<T> gates;
        if (a.gate)
            gates = tm.load((const T *)a.gate + (some ? quotient(first, a.gate_rows) : 0) * a.channels, some);
        auto times_gate = [&](float (&y)[8]) {
            if (a.gate) {
                float g[8];
                gates.unpack(g);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    y[j] *= g[j];
            }
        };
        if constexpr (AHEAD)
            fetch(first, some);
        for (int64_t i = 0; i < inner; ++i) {
            const int64_t row = first + i * step;
            const bool ok = row < last;
            float x[8], n[8], d[8], r[8];
            if constexpr (!AHEAD)
                fetch(row, ok);
            nx.unpack(x);
            if (a.z)
                nz.unpack(n);
            if (a.grad_h)
                nh.unpack(d);
            const Raw<T> up = nr;
            if constexpr (AHEAD)
                fetch(row + step, row + step < last && i + 1 < inner);
            float rz = 0.0f;
            uint32_t bits = 0;
            if (a.z) {
                bits = !ok ? 0u : (a.dropping ? tm.kept_bits(a.drop, row) : 255u);
                rz = normalise(tm, ok, a.layer, n, a.eps, inv_c, lds, turn);
                float y[8], b[8];
                tm.take(k1, y);
                tm.take(k0, b);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    y[j] = n[j] * y[j] + b[j];
                times_gate(y);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    bits = tm.holds(j) ? bits : bits & ~(1u << j);
                    x[j] = (bits >> j & 1) ? x[j] + y[j] * a.drop.keep : x[j];
                }
            }
            if (a.grad_h) {
                const float rr = normalise(tm, ok, a.layer, x, a.eps, inv_c, lds, turn);
                float m[8];
                tm.take(wp, m);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    P1[j] += d[j] * x[j];  // both are 0 past the last row
                    P0[j] += d[j];
                    d[j] *= m[j];
                }
                normalise_grad(tm, a.layer, d, x, rr, inv_c, lds, turn);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    d[j] = 0.0f;
            }
            if (a.grad_r) {
                up.unpack(r);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    d[j] += r[j];
            }
            if (a.grad_x && ok)
                tm.store((T *)a.grad_x + row * a.channels, d);
            if (a.z) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float t = (bits >> j & 1) ? d[j] * a.drop.keep : 0.0f;
                    T1[j] += t * n[j];
                    T0[j] += t;
                    d[j] = t;
                }
                times_gate(d);
                float m[8];
                tm.take(k1, m);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    d[j] *= m[j];
                normalise_grad(tm, a.layer, d, n, rz, inv_c, lds, turn);
                if (a.grad_z && ok)
                    tm.store((T *)a.grad_z + row * a.channels, d);
            }
        }
        if constexpr (WHOLE) {
            if (a.grad_gate && some) {
                float y[8];
                gate_grad(y);
                tm.store((T *)a.grad_gate + quotient(first, a.gate_rows) * a.channels, y);
            }
            first += TM::kTeams * a.gate_rows;
        }
        float S1[8], S0[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            S1[j] = T1[j];
            S0[j] = T0[j];
            if constexpr (WHOLE)
                T1[j] = T0[j] = 0.0f;
        }
        times_gate(S1);
        times_gate(S0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            A1[j] += S1[j];
            A0[j] += S0[j];
        }
    }
    // partial sums of the chunk, the teams' added up in order
    float *part = a.part + (int64_t)blockIdx.x * 5 * a.channels;
    auto flush = [&](const float (&s)[8], int k) {
        if constexpr (TM::kTeams > 1) {
            constexpr int P = TM::kLanes * 8;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j)
                cols[tm.team * P + tm.c0 + j] = s[j];
            __syncthreads();
            for (int c = threadIdx.x; c < a.channels; c += TM::kThreads) {
                float y = 0.0f;
                for (int q = 0; q < TM::kTeams; ++q)
                    y += cols[q * P + c];
                part[k * a.channels + c] = y;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (tm.c0 + j < a.channels)
                    part[k * a.channels + tm.c0 + j] = s[j];
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
    if (!WHOLE && a.grad_gate) {
        float y[8];
        gate_grad(y);
        flush(y, 4);
    }
}

// Sums of the partial rows: 16 columns per block, 64 rows of threads that take
// every 64th partial row each, then those added in order.  blockIdx.y: 0 the
// post-norm's sums, 1 the pre-norm's, 2 + g gate row g.
template <class T>
__global__ __launch_bounds__(1024) void k_norm_sums(NormArgs a, float *gw_post, float *gb_post, float *gscale,
                                                    float *gw_pre, float *gb_pre)
{
    constexpr int COLS = 16, ROWS = 1024 / COLS;
    __shared__ float rows[2][ROWS][COLS + 1];
    const int cx = threadIdx.x % COLS, j = threadIdx.x / COLS, C = a.channels;
    const int c = blockIdx.x * COLS + cx;
    const int what = blockIdx.y;
    const int64_t from = what < 2 ? 0 : (int64_t)(what - 2) * a.per_group;
    const int64_t to = what < 2 ? a.chunks : from + a.per_group;
    const int k0 = what == 0 ? 0 : (what == 1 ? 2 : 4), k1 = what < 2 ? k0 + 1 : k0;
    float s0 = 0.0f, s1 = 0.0f;
    if (c < C) {
#pragma unroll 4
        for (int64_t p = from + j; p < to; p += ROWS) {
            s0 += a.part[(p * 5 + k0) * C + c];
            s1 += a.part[(p * 5 + k1) * C + c];
        }
    }
    rows[0][j][cx] = s0;
    rows[1][j][cx] = s1;
    __syncthreads();
    if (j >= 2)
        return;
    float s = 0.0f;
    for (int q = 0; q < ROWS; ++q)
        s += rows[j][q][cx];
    rows[j][0][cx] = s;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // j = 0 and 1 are lanes of one wave
    __builtin_amdgcn_wave_barrier();
    if (j != 0 || c >= C)
        return;
    s0 = rows[0][0][cx];
    s1 = rows[1][0][cx];
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

// A thread takes the eight elements that one counter's numbers decide on, so its
// ten rounds are shared by eight and the result does not depend on the launch.
// Bound by memory: 39 M elements, bf16 24 us, 6.6 TB/s; fp32 53 us, 5.9.
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
                v[j] = kept(d, w, j) ? (float)rounded<T>(v[j] * d.keep) : 0.0f;
            store8(y + g * 8, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (g * 8 + j < n)
                    y[g * 8 + j] = kept(d, w, j) ? rounded<T>((float)x[g * 8 + j] * d.keep) : (T)0.0f;
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

// The smallest team that holds a row of c channels: groups of 8 to 64 lanes, then
// 2 to 16 waves.  Rows that start anywhere take a wave at least.
template <class F>
auto with_team(int c, bool wide, const F &f)
{
#define PAM_TEAM(G, W, WIDE)                                                                      \
    f(std::integral_constant<int, G>(), std::integral_constant<int, W>(), std::integral_constant<bool, WIDE>())
    if (wide && c <= 64)
        return PAM_TEAM(8, 1, true);
    if (wide && c <= 128)
        return PAM_TEAM(16, 1, true);
    if (wide && c <= 256)
        return PAM_TEAM(32, 1, true);
    if (c <= 512)
        return wide ? PAM_TEAM(64, 1, true) : PAM_TEAM(64, 1, false);
    if (c <= 1024)
        return wide ? PAM_TEAM(64, 2, true) : PAM_TEAM(64, 2, false);
    if (c <= 2048)
        return wide ? PAM_TEAM(64, 4, true) : PAM_TEAM(64, 4, false);
    if (c <= 4096)
        return wide ? PAM_TEAM(64, 8, true) : PAM_TEAM(64, 8, false);
    return wide ? PAM_TEAM(64, 16, true) : PAM_TEAM(64, 16, false);
#undef PAM_TEAM
}
// teams of a block, and blocks that the card holds with four waves per SIMD, as the forward pass has
int teams_of(int c, bool wide)
{
    return with_team(c, wide, [](auto g, auto w, auto) { return (w > 4 ? 64 * w : 256) / (g * w); });
}
int blocks_at_once(int c) { return c <= 2048 ? 1024 : (c <= 4096 ? 512 : 256); }
// Blocks of the backward pass that the card holds: by its registers three waves
// per SIMD, two of fp32 or where the teams write the gate's gradient.  One such
// round, against 1024 blocks: 99 us for 109 us (bf16 76800 x 512, 768 blocks),
// 84 for 92 (fp32 38400 x 512, 512 blocks).
int chunks_at_once(int32_t dtype, int c, bool whole)
{
    return c > 2048 ? 256 : (dtype == PAM_F32 || whole ? 512 : 768);
}

struct Chunks {
    int32_t chunks, per_group;
};
Chunks chunks_of(const pam_norm_desc_t &d, bool gated, bool wide)
{
    // one round of blocks, none without a row for each of its teams
    int64_t most = chunks_at_once(d.dtype, d.channels, false);
    const int64_t teams = teams_of(d.channels, wide);
    const int64_t groups = gated ? d.rows / std::max<int64_t>(d.gate_rows, 1) : 1;
    const int64_t gate_rows = gated ? d.gate_rows : d.rows;
    if (groups > most) {
        most = chunks_at_once(d.dtype, d.channels, true);
        return {(int32_t)std::min<int64_t>(most, (groups + teams - 1) / teams), 0};
    }
    int64_t per = std::max<int64_t>(1, most / std::max<int64_t>(groups, 1));
    per = std::max<int64_t>(1, std::min<int64_t>(per, (gate_rows + teams - 1) / teams));
    return {(int32_t)(per * std::max<int64_t>(groups, 1)), (int32_t)per};
}

template <class T>
void launch_norm_t(const NormArgs &a, bool wide, bool bwd, hipStream_t s)
{
    with_team(a.channels, wide, [&](auto g, auto w, auto wd) {
        using TM = Team<T, g, w, wd>;
        if (bwd && a.per_group) {
            hipLaunchKernelGGL((k_norm_bwd<T, g, w, wd, false>), dim3(a.chunks), dim3(TM::kThreads), 0, s, a);
        } else if (bwd) {
            hipLaunchKernelGGL((k_norm_bwd<T, g, w, wd, true>), dim3(a.chunks), dim3(TM::kThreads), 0, s, a);
        } else {
            const unsigned blocks =
                (unsigned)std::min<int64_t>((a.rows + TM::kTeams - 1) / TM::kTeams, blocks_at_once(a.channels));
            hipLaunchKernelGGL((k_norm_fwd<T, g, w, wd>), dim3(blocks), dim3(TM::kThreads), 0, s, a);
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
    const dim3 grid((d.channels + 15) / 16, 2 + (by_group ? (unsigned)a.groups : 0));
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
