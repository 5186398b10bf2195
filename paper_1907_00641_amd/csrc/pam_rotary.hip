// Rotary positions (gfx950): the table of cosines and sines, and the rotation
// of queries and keys in one launch.
#include "pam_rows.h"

#include <algorithm>

namespace pam {

namespace {

constexpr int kThreads = 256;
constexpr int kHeadsPerThread = 4;  // heads that one thread turns with the cosines and sines it has loaded

__global__ __launch_bounds__(kThreads) void k_rotary_table(const double *__restrict__ freq,
                                                           const float *__restrict__ coord,
                                                           const int32_t *__restrict__ axis, int64_t count, int pairs,
                                                           int axes, double magnitude, float2 *__restrict__ table)
{
    // the product and its reduction to one turn in 64 bits: in 32 an angle of
    // 10^5 is off by 4e-3
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < count; e += (int64_t)gridDim.x * kThreads) {
        const int64_t t = e / pairs;
        const int i = (int)(e - t * pairs);
        int ax = axis ? axis[i] : 0;
        ax = (ax < 0 || ax >= axes) ? 0 : ax;
        const double pos = coord ? (double)coord[t * axes + ax] : (double)t;
        double s, c;
        sincos(pos * freq[i], &s, &c);
        table[e] = make_float2((float)(c * magnitude), (float)(s * magnitude));
    }
}

struct RotaryArgs {
    const void *q, *k;
    const float2 *table;
    const int32_t *pos;
    void *q_out, *k_out;
    int64_t qs[3], ks[3];
    int64_t start, entries;
    int32_t batch, length, heads, kv_heads, dim, pairs;
    int32_t units, head_slots;  // work items per head; threads over the heads of a token
    float sign;
};

// A thread takes one unit of a head, V pairs of channels to turn or V (2 V
// interleaved) channels to copy, for kHeadsPerThread heads of one token: the
// table is read once for those, and all their loads are under way before the
// first is used.  Units run fastest over the threads, then heads, so that a
// wave reads and writes whole rows.  The products are fused with the sums by hand,
// which gives the same bits at every width.  Bound by memory:
// fp16 16384 tokens, 32 + 8 heads of 128, 71 us, 4.7 TB/s, the rate of a large copy;
// bf16, heads of 80 with 20 pairs, in accesses of 4 channels, 40 us, 5.2 TB/s (one
// channel at a time: 94 us).
template <class T, int V, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void k_rotary(RotaryArgs a)
{
    const int64_t per_token = (int64_t)a.units * a.head_slots;
    const int64_t total = per_token * a.batch * a.length;
    const int heads = a.heads + a.kv_heads;
    const int turn_units = a.pairs / V;
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < total; e += (int64_t)gridDim.x * kThreads) {
        const int64_t tok = quotient(e, per_token);
        const int rest = (int)(e - tok * per_token);
        const int slot = rest / a.units, u = rest - slot * a.units;
        const int b = (int)quotient(tok, a.length), l = (int)(tok - (int64_t)b * a.length);
        const bool turn = u < turn_units;
        float c[V], s[V];
        if (turn) {
            const int64_t at = a.pos ? (int64_t)a.pos[tok] : a.start + l;
            const bool in = at >= 0 && at < a.entries;
            const float2 *row = a.table + (in ? at : 0) * a.pairs + u * V;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float2 cs = row[j];
                c[j] = in ? cs.x : __builtin_nanf("");
                s[j] = in ? a.sign * cs.y : __builtin_nanf("");
            }
        }
        // first and second group of V channels of this unit; a copied unit
        // has the first only
        int c0, c1;
        if (turn) {
            c0 = INTERLEAVED ? 2 * u * V : u * V;
            c1 = INTERLEAVED ? c0 + V : a.pairs + u * V;
        } else {
            c0 = 2 * a.pairs + (u - turn_units) * V;
            c1 = c0;
        }
        T x0[kHeadsPerThread][V], x1[kHeadsPerThread][V];
#pragma unroll
        for (int k = 0; k < kHeadsPerThread; ++k) {
            const int h = slot + k * a.head_slots;
            if (h < heads) {
                const T *row = h < a.heads ? (const T *)a.q + b * a.qs[0] + l * a.qs[1] + h * a.qs[2]
                                           : (const T *)a.k + b * a.ks[0] + l * a.ks[1] + (h - a.heads) * a.ks[2];
                __builtin_memcpy(x0[k], __builtin_assume_aligned(row + c0, sizeof(T) * V > 16 ? 16 : sizeof(T) * V),
                                 sizeof(T) * V);
                if (turn)
                    __builtin_memcpy(x1[k],
                                     __builtin_assume_aligned(row + c1, sizeof(T) * V > 16 ? 16 : sizeof(T) * V),
                                     sizeof(T) * V);
            }
        }
#pragma unroll
        for (int k = 0; k < kHeadsPerThread; ++k) {
            const int h = slot + k * a.head_slots;
            if (h >= heads)
                continue;
            T *row = h < a.heads ? (T *)a.q_out + (tok * a.heads + h) * a.dim
                                 : (T *)a.k_out + (tok * a.kv_heads + (h - a.heads)) * a.dim;
            if (turn) {
                T y[2 * V];
                if constexpr (INTERLEAVED) {
                    T x[2 * V];
                    __builtin_memcpy(x, x0[k], sizeof(T) * V);
                    __builtin_memcpy(x + V, x1[k], sizeof(T) * V);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float p = (float)x[2 * j], r = (float)x[2 * j + 1];
                        y[2 * j] = rounded<T>(__builtin_fmaf(-r, s[j], p * c[j]));
                        y[2 * j + 1] = rounded<T>(__builtin_fmaf(r, c[j], p * s[j]));
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float p = (float)x0[k][j], r = (float)x1[k][j];
                        y[j] = rounded<T>(__builtin_fmaf(-r, s[j], p * c[j]));
                        y[V + j] = rounded<T>(__builtin_fmaf(r, c[j], p * s[j]));
                    }
                }
                __builtin_memcpy(__builtin_assume_aligned(row + c0, sizeof(T) * V > 16 ? 16 : sizeof(T) * V), y,
                                 sizeof(T) * V);
                __builtin_memcpy(__builtin_assume_aligned(row + c1, sizeof(T) * V > 16 ? 16 : sizeof(T) * V), y + V,
                                 sizeof(T) * V);
            } else {
                __builtin_memcpy(__builtin_assume_aligned(row + c0, sizeof(T) * V > 16 ? 16 : sizeof(T) * V), x0[k],
                                 sizeof(T) * V);
            }
        }
    }
}

template <class T, int V>
void launch_rotary_v(const RotaryArgs &a, bool interleaved, unsigned blocks, hipStream_t s)
{
    if (interleaved)
        hipLaunchKernelGGL((k_rotary<T, V, true>), dim3(blocks), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((k_rotary<T, V, false>), dim3(blocks), dim3(kThreads), 0, s, a);
}

// v: channels per access
template <class T>
void launch_rotary_t(RotaryArgs &a, int v, bool interleaved, hipStream_t s)
{
    a.units = a.pairs / v + (a.dim - 2 * a.pairs) / v;
    const int heads = a.heads + a.kv_heads;
    a.head_slots = (heads + kHeadsPerThread - 1) / kHeadsPerThread;
    const int64_t total = (int64_t)a.units * a.head_slots * a.batch * a.length;
    const unsigned blocks = (unsigned)std::min<int64_t>((total + kThreads - 1) / kThreads, 1 << 20);
    if constexpr (sizeof(T) == 2) {
        if (v == 8)
            return launch_rotary_v<T, 8>(a, interleaved, blocks, s);
    }
    if (v == 4)
        launch_rotary_v<T, 4>(a, interleaved, blocks, s);
    else if (v == 2)
        launch_rotary_v<T, 2>(a, interleaved, blocks, s);
    else
        launch_rotary_v<T, 1>(a, interleaved, blocks, s);
}

}  // namespace

hipError_t launch_rotary_table(const double *freq, const float *coord, const int32_t *axis, int64_t entries,
                               int32_t pairs, int32_t axes, double magnitude, float *table, hipStream_t s)
{
    const int64_t count = entries * pairs;
    if (count <= 0)
        return hipSuccess;
    hipLaunchKernelGGL(k_rotary_table, dim3((unsigned)std::min<int64_t>((count + kThreads - 1) / kThreads, 1 << 16)),
                       dim3(kThreads), 0, s, freq, coord, axis, count, pairs, axes, magnitude, (float2 *)table);
    return hipGetLastError();
}

hipError_t launch_rotary(const pam_rotary_desc_t &d, const void *q, const void *k, const float *table,
                         const int32_t *pos, void *q_out, void *k_out, hipStream_t s)
{
    if (d.batch == 0 || d.length == 0)
        return hipSuccess;
    RotaryArgs a;
    a.q = q;
    a.k = k;
    a.table = (const float2 *)table;
    a.pos = pos;
    a.q_out = q_out;
    a.k_out = k_out;
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
    a.sign = (d.flags & PAM_ROTARY_INVERSE) ? -1.0f : 1.0f;
    // the widest accesses, up to 16 bytes, that divide every group of channels
    // and the place of every row
    const int es = d.dtype == PAM_F32 ? 4 : 2;
    uint64_t all = (uint64_t)(d.pairs | d.dim | 16 / es);
    for (int i = 0; i < 3; ++i)
        all |= (uint64_t)d.q_stride[i] | (d.kv_heads ? (uint64_t)d.k_stride[i] : 0);
    all |= ((uintptr_t)q | (uintptr_t)q_out | (uintptr_t)k | (uintptr_t)k_out) / es;
    const int v = (int)(all & -all);
    const bool inter = d.flags & PAM_ROTARY_INTERLEAVED;
    if (d.dtype == PAM_F32)
        launch_rotary_t<float>(a, v, inter, s);
    else if (d.dtype == PAM_F16)
        launch_rotary_t<f16>(a, v, inter, s);
    else
        launch_rotary_t<bf16>(a, v, inter, s);
    return hipGetLastError();
}

}  // namespace pam
