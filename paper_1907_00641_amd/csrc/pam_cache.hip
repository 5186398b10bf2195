// Writing a paged cache and reading it back (gfx950).  A row (one head's keys of
// one map, or its values, of one token) is taken by a group of lanes, eight
// channels each; both directions are bound by memory.
#include "pam_store.h"

#include <algorithm>
#include <type_traits>

namespace pam {

namespace {

constexpr int kThreads = 256;

struct CacheArgs {
    Pool pool;
    void *k, *v;  // new rows, or what is read
    const int32_t *starts, *new_len;
    int64_t ks[4], vs[3];  // new rows: sequence, token, head, map
    int64_t rows;          // of all sequences
    int32_t length;        // rows of a sequence (write: without starts)
    int32_t group;         // lanes per row, a power of two
    uint32_t kinds;        // rows of a token and head: the maps' keys, the values
};

// largest over an aligned group of lanes (a power of two up to 32), left in every lane
__device__ __forceinline__ float group_max(float x, int group)
{
    if (group >= 2)
        x = __builtin_fmaxf(x, lane_move<0xb1>(x));
    if (group >= 4)
        x = __builtin_fmaxf(x, lane_move<0x4e>(x));
    if (group >= 8)
        x = __builtin_fmaxf(x, lane_move<0x141>(x));
    if (group >= 16)
        x = __builtin_fmaxf(x, lane_move<0x140>(x));
    if (group >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return x;
}

// Which row of which head a group takes: the rows of a token and head behind each
// other, then the heads.
struct Unit {
    int64_t row;
    int head, kind, dim;
    bool value;
    __device__ __forceinline__ Unit(const CacheArgs &a, uint64_t u)
    {
        const uint32_t per = a.kinds * a.pool.kv_heads;
        row = (int64_t)(u >> 32 ? u / per : (uint32_t)u / per);
        const uint32_t rest = (uint32_t)(u - (uint64_t)row * per);
        head = rest / a.kinds;
        kind = rest - head * a.kinds;
        value = kind == a.pool.maps;
        dim = value ? a.pool.dim_v : a.pool.dim;
    }
};

// Eight elements of a row as numbers; the first n of them where rows are not wide.
template <class T, bool WIDE>
__device__ __forceinline__ void get8(const T *p, int n, float (&x)[8])
{
    Stored8<T> r{};
    if constexpr (WIDE) {
        if (n > 0)
            r = load_stored(p);
    } else {
        r = load_stored_some(p, n);
    }
    unpack<T>(r, x);
}

// New rows to their pages.  The scale of a row is taken from its lanes' largest
// magnitude; the maximum passes over NaN, so that a row with one is found by the
// products with 0, which are 0 for finite numbers alone.
template <class T, class S, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_cache_write(CacheArgs a)
{
    const int per = kThreads / a.group, c = (threadIdx.x & (a.group - 1)) * 8;
    const uint64_t units = (uint64_t)a.rows * a.pool.kv_heads * a.kinds;
    for (uint64_t u0 = (uint64_t)blockIdx.x * per; u0 < units; u0 += (uint64_t)gridDim.x * per) {
        const uint64_t u = u0 + threadIdx.x / a.group;
        const Unit x(a, u < units ? u : units - 1);
        int b, i, n;
        if (a.starts) {  // the last sequence that starts at this row or before
            int lo = 0, hi = a.pool.sequences;
            while (hi - lo > 1) {
                const int mid = lo + (hi - lo) / 2;
                if (a.starts[mid] <= x.row)
                    lo = mid;
                else
                    hi = mid;
            }
            b = lo;
            const int64_t from = min(max((int64_t)a.starts[b], (int64_t)0), a.rows);
            n = (int)(min(max((int64_t)a.starts[b + 1], from), a.rows) - from);
            i = (int)(x.row - from);
        } else {
            b = (int)quotient(x.row, a.length);
            i = (int)(x.row - (int64_t)b * a.length);
            n = a.new_len ? min(max(a.new_len[b], 0), a.length) : a.length;
        }
        const int p = cached(a.pool, b) - n + i;
        const int at = u < units && i >= 0 && i < n && p >= 0 ? cache_row(a.pool, b, x.head, p) : -1;
        const int m = at < 0 ? 0 : max(min(x.dim - c, 8), 0);
        // with starts, rows are the tokens of one sequence
        const int64_t rb = a.starts ? 0 : b, ri = a.starts ? x.row : i;
        const T *from = x.value ? (const T *)a.v + rb * a.vs[0] + ri * a.vs[1] + x.head * a.vs[2]
                                : (const T *)a.k + rb * a.ks[0] + ri * a.ks[1] + x.head * a.ks[2] + x.kind * a.ks[3];
        float y[8];
        get8<T, WIDE>(from + c, m, y);
        if constexpr (kScaled<S>) {
            float top = 0.0f, none = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                top = __builtin_fmaxf(top, __builtin_fabsf(y[j]));
                none = __builtin_fmaf(y[j], 0.0f, none);
            }
            // -1: some number of the row is not finite
            top = group_max(top, a.group);
            const bool bad = group_max(none == 0.0f ? 0.0f : 1.0f, a.group) != 0.0f;
            const float scale = bad ? __builtin_nanf("") : __builtin_fmaxf(top / kTop<S>, 0x1p-126f);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                y[j] = bad ? 0.0f : __builtin_fminf(__builtin_fmaxf(y[j] / scale, -kTop<S>), kTop<S>);
            if (at >= 0 && c == 0)
                *(x.value ? a.pool.vs + at : a.pool.ks + (int64_t)at * a.pool.maps + x.kind) = scale;
        }
        S *to = (x.value ? (S *)a.pool.v + (int64_t)at * a.pool.dim_v
                         : (S *)a.pool.k + ((int64_t)at * a.pool.maps + x.kind) * a.pool.dim) + c;
        const Stored8<S> r = pack<S>(y);
        if constexpr (WIDE) {
            if (m > 0)
                put_stored(to, r);
        } else {
            put_stored_some(to, r, m);
        }
    }
}

// The first `length` positions of every sequence, 0 where there is no token.
template <class T, class S, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_cache_read(CacheArgs a)
{
    const int per = kThreads / a.group, c = (threadIdx.x & (a.group - 1)) * 8;
    const uint64_t units = (uint64_t)a.rows * a.pool.kv_heads * a.kinds;
    for (uint64_t u = (uint64_t)blockIdx.x * per + threadIdx.x / a.group; u < units; u += (uint64_t)gridDim.x * per) {
        const Unit x(a, u);
        T *to = x.value ? (T *)a.v : (T *)a.k;
        if (!to)
            continue;
        const int b = (int)quotient(x.row, a.length), p = (int)(x.row - (int64_t)b * a.length);
        const int at = p < cached(a.pool, b) ? cache_row(a.pool, b, x.head, p) : -1;
        const int m = max(min(x.dim - c, 8), 0), got = at < 0 ? 0 : m;
        float y[8];
        get8<S, WIDE>((x.value ? (const S *)a.pool.v + (int64_t)at * a.pool.dim_v
                               : (const S *)a.pool.k + ((int64_t)at * a.pool.maps + x.kind) * a.pool.dim) + c,
                      got, y);
        if constexpr (kScaled<S>) {
            const float scale = at < 0 ? 0.0f : (x.value ? a.pool.vs[at] : a.pool.ks[(int64_t)at * a.pool.maps + x.kind]);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                y[j] *= scale;
        }
        to += (x.value ? (x.row * a.pool.kv_heads + x.head) * a.pool.dim_v
                       : ((x.row * a.pool.kv_heads + x.head) * a.pool.maps + x.kind) * a.pool.dim) + c;
        const Stored8<T> r = pack<T>(y);
        if constexpr (WIDE) {
            if (m > 0)
                put_stored(to, r);
        } else {
            put_stored_some(to, r, m);
        }
    }
}

// eight elements at a time: rows are whole eights, and every place a multiple of
// 16 bytes, or of 8 for stored types of 8 bits
bool wide_of(const pam_cache_desc_t &d, const void *k, const void *v, const int64_t *ks, const int64_t *vs)
{
    uint64_t all = (uint64_t)d.dim | (uint64_t)d.dim_v;
    for (int i = 0; ks && i < 4; ++i)
        all |= (uint64_t)ks[i];
    for (int i = 0; vs && i < 3; ++i)
        all |= (uint64_t)vs[i];
    return all % 8 == 0 && ((uintptr_t)k | (uintptr_t)v) % 16 == 0;
}

CacheArgs args_of(const pam_cache_desc_t &d, const Pool &pool)
{
    CacheArgs a{};
    a.pool = pool;
    a.kinds = (uint32_t)d.maps + 1;
    a.group = 1;
    while (a.group * 8 < std::max(d.dim, d.dim_v))
        a.group *= 2;
    return a;
}

unsigned blocks_of(const CacheArgs &a)
{
    const int64_t per = kThreads / a.group;
    return (unsigned)std::min<int64_t>((a.rows * a.pool.kv_heads * a.kinds + per - 1) / per, 1 << 20);
}

template <class T, class S>
void launch_pair(const CacheArgs &a, bool write, bool wide, hipStream_t s)
{
    const dim3 grid(blocks_of(a)), block(kThreads);
    if (write && wide)
        hipLaunchKernelGGL((k_cache_write<T, S, true>), grid, block, 0, s, a);
    else if (write)
        hipLaunchKernelGGL((k_cache_write<T, S, false>), grid, block, 0, s, a);
    else if (wide)
        hipLaunchKernelGGL((k_cache_read<T, S, true>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_cache_read<T, S, false>), grid, block, 0, s, a);
}

template <class T>
void launch_type(const pam_cache_desc_t &d, const CacheArgs &a, bool write, bool wide, hipStream_t s)
{
    if (d.store == PAM_STORE_E4M3)
        launch_pair<T, e4m3>(a, write, wide, s);
    else if (d.store == PAM_STORE_INT8)
        launch_pair<T, int8>(a, write, wide, s);
    else
        launch_pair<T, T>(a, write, wide, s);
}

hipError_t launch_any(const pam_cache_desc_t &d, const CacheArgs &a, bool write, bool wide, hipStream_t s)
{
    if (d.dtype == PAM_F32)
        launch_type<float>(d, a, write, wide, s);
    else if (d.dtype == PAM_F16)
        launch_type<f16>(d, a, write, wide, s);
    else
        launch_type<bf16>(d, a, write, wide, s);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const pam_cache_desc_t &d, const pam_cache_rows_t &rows, const Pool &pool, const void *k,
                              const void *v, const int32_t *starts, const int32_t *new_len, hipStream_t s)
{
    CacheArgs a = args_of(d, pool);
    a.k = const_cast<void *>(k);
    a.v = const_cast<void *>(v);
    a.starts = starts;
    a.new_len = new_len;
    for (int i = 0; i < 4; ++i)
        a.ks[i] = rows.k_stride[i];
    for (int i = 0; i < 3; ++i)
        a.vs[i] = rows.v_stride[i];
    a.rows = rows.rows;
    a.length = rows.length;
    return launch_any(d, a, true, wide_of(d, k, v, rows.k_stride, rows.v_stride), s);
}

hipError_t launch_cache_read(const pam_cache_desc_t &d, int32_t length, const Pool &pool, void *k, void *v,
                             hipStream_t s)
{
    CacheArgs a = args_of(d, pool);
    a.k = k;
    a.v = v;
    a.rows = (int64_t)d.sequences * length;
    a.length = length;
    return launch_any(d, a, false, wide_of(d, k, v, nullptr, nullptr), s);
}

}  // namespace pam
