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
    uint32_t rows;         // tokens of all sequences
    int32_t length;        // of them in a sequence (write: without starts)
    int32_t group[2];      // lanes per row of keys, of values: powers of two
    Divisor by_length, by_heads[2], by_page;  // heads: of keys, times the maps
    Divisor by_block[2];                      // kBlockTokens times that
};

// Writing takes so many tokens of a head behind each other, whose rows are neighbours in
// their page: a wave then writes a kilobyte in one place.  (In the order of the new rows,
// which is that of reading, 2 x 8192 tokens, 8 heads of 2 x 64, bf16 to e4m3, took 39 us.)
constexpr int kBlockTokens = 16;

// largest over an aligned group of lanes (a power of two up to 32), left in every lane
__device__ __forceinline__ uint32_t group_max(uint32_t x, int group)
{
    auto move = [](uint32_t y, auto ctrl) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)y, decltype(ctrl)::value, 0xf, 0xf, false);
    };
    if (group >= 2)
        x = max(x, move(x, std::integral_constant<int, 0xb1>()));
    if (group >= 4)
        x = max(x, move(x, std::integral_constant<int, 0x4e>()));
    if (group >= 8)
        x = max(x, move(x, std::integral_constant<int, 0x141>()));
    if (group >= 16)
        x = max(x, move(x, std::integral_constant<int, 0x140>()));
    if (group >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = max((uint32_t)r[0], (uint32_t)r[1]);
    }
    return x;
}

// Which row a group takes: blocks with blockIdx.y 0 take keys, others values; the maps of
// a head behind each other, then the heads of a token.
struct Unit {
    uint32_t row;  // token
    int head, map;
    __device__ __forceinline__ Unit(const CacheArgs &a, uint32_t u)
    {
        const bool value = blockIdx.y;
        const int maps = value ? 1 : a.pool.maps;
        row = a.by_heads[value](u);
        const int rest = (int)(u - row * (a.pool.kv_heads * maps));
        head = maps == 2 ? rest >> 1 : rest;
        map = maps == 2 ? rest & 1 : 0;
    }
    __device__ __forceinline__ static Unit of_blocks(const CacheArgs &a, uint32_t u)
    {
        const bool value = blockIdx.y;
        const int maps = value ? 1 : a.pool.maps;
        Unit x;
        const uint32_t block = a.by_block[value](u);
        uint32_t rest = u - block * (a.pool.kv_heads * maps * kBlockTokens);
        x.map = maps == 2 ? rest & 1 : 0;
        rest = maps == 2 ? rest >> 1 : rest;
        x.head = rest / kBlockTokens;
        x.row = block * kBlockTokens + rest % kBlockTokens;
        return x;
    }
    __device__ __forceinline__ Unit() {}
};
// where the rows of a kind are in the pool, from the number of a token of a head
template <class S>
__device__ __forceinline__ S *stored_row(const Pool &p, bool value, int64_t at, int map)
{
    return value ? (S *)p.v + at * p.dim_v : (S *)p.k + (at * p.maps + map) * p.dim;
}
__device__ __forceinline__ float *scale_of(const Pool &p, bool value, int64_t at, int map)
{
    return value ? p.vs + at : p.ks + at * p.maps + map;
}
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

// E elements of a row as they lie in memory, 0 from n on.  PE elements are read at once
// where rows are whole pieces of them; PE 0: eight, one by one.
template <class T, int PE>
struct Piece {
    static constexpr int E = PE ? PE : 8, kWords = E * sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T *p, int n)
    {
        if constexpr (PE != 0) {
            typedef uint32_t Words __attribute__((ext_vector_type(kWords), aligned(16)));
            Words y = {};
            if (n > 0)
                y = *reinterpret_cast<const Words *>(p);
#pragma unroll
            for (int i = 0; i < kWords; ++i)
                w[i] = y[i];
        } else {
            const Stored8<T> y = load_stored_some(p, n);
#pragma unroll
            for (int i = 0; i < kWords; ++i)
                w[i] = y.w[i];
        }
    }
    // The largest magnitude as the bits of an fp32 number.  Taken as integers: those of
    // infinities and NaN are the largest.
    __device__ __forceinline__ uint32_t top() const
    {
        if constexpr (sizeof(T) == 4) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < kWords; ++i)
                m = max(m, w[i] & 0x7fffffffu);
            return m;
        } else {
            typedef uint16_t Two __attribute__((ext_vector_type(2)));
            Two m = {};
#pragma unroll
            for (int i = 0; i < kWords; ++i)
                m = __builtin_elementwise_max(m, __builtin_bit_cast(Two, w[i] & 0x7fff7fffu));
            const uint16_t x = max(m[0], m[1]);
            return __float_as_uint((float)__builtin_bit_cast(T, x));
        }
    }
    __device__ __forceinline__ void numbers(float (&x)[E]) const
    {
        T y[E];
        __builtin_memcpy(y, w, sizeof(y));
#pragma unroll
        for (int j = 0; j < E; ++j)
            x[j] = (float)y[j];
    }
};

// Numbers of a row with this scale, quotients correctly rounded to 32 bits: from the
// correctly rounded reciprocal y of the scale, q = x y, and q + (x - q scale) y is
// (Markstein 1990) where nothing underflows; the division itself where it could.
template <class S, int E>
__device__ __forceinline__ void quotients(float (&x)[E], float scale)
{
    if (__any(scale < 0x1p-60f)) {
#pragma unroll
        for (int j = 0; j < E; ++j)
            x[j] /= scale;
    } else {
        const float y = 1.0f / scale;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float q = x[j] * y;
            x[j] = __builtin_fmaf(__builtin_fmaf(-q, scale, x[j]), y, q);
        }
    }
#pragma unroll
    for (int j = 0; j < E; ++j)
        x[j] = __builtin_amdgcn_fmed3f(x[j], -kTop<S>, kTop<S>);
}

// Rows of a group and turn, so that their loads are under way together.
constexpr int kTurnRows = 2;

// New rows to their pages.  Bound by instructions before memory, which is why a lane takes
// sixteen channels where it can: 2 x 8192 tokens, 8 heads of 2 x 64, bf16 to e4m3, eight: 39 us,
// sixteen 22 us (17 us at a large copy's rate).
template <class T, class S, int PE>
__global__ __launch_bounds__(kThreads) void k_cache_write(CacheArgs a)
{
    using P = Piece<T, PE>;
    constexpr int E = P::E;
    const bool value = blockIdx.y;
    const int group = a.group[value], per = kThreads / group, c = (threadIdx.x & (group - 1)) * E;
    const int dim = value ? a.pool.dim_v : a.pool.dim;
    const uint32_t blocks = (a.rows + kBlockTokens - 1) / kBlockTokens;
    const uint32_t units = blocks * kBlockTokens * a.pool.kv_heads * (value ? 1 : a.pool.maps);
    for (uint32_t u0 = blockIdx.x * per * kTurnRows; u0 < units; u0 += gridDim.x * per * kTurnRows) {
        P y[kTurnRows];
        int at[kTurnRows], map[kTurnRows], m[kTurnRows];
#pragma unroll
        for (int k = 0; k < kTurnRows; ++k) {
            const uint32_t u = u0 + k * per + threadIdx.x / group;
            const Unit x = Unit::of_blocks(a, min(u, units - 1));
            int b = 0, i = 0, n = 0;
            if (x.row >= a.rows) {  // the last block of tokens
            } else if (a.starts) {  // the last sequence that starts at this row or before
                int lo = 0, hi = a.pool.sequences;
                while (hi - lo > 1) {
                    const int mid = lo + (hi - lo) / 2;
                    if (a.starts[mid] <= (int64_t)x.row)
                        lo = mid;
                    else
                        hi = mid;
                }
                b = lo;
                const int64_t from = min(max((int64_t)a.starts[b], (int64_t)0), (int64_t)a.rows);
                n = (int)(min(max((int64_t)a.starts[b + 1], from), (int64_t)a.rows) - from);
                i = (int)(x.row - from);
            } else {
                b = (int)a.by_length(x.row);
                i = (int)(x.row - b * (uint32_t)a.length);
                n = a.new_len ? min(max(a.new_len[b], 0), a.length) : a.length;
            }
            // from the length as it is: of one past the table, only what the table reaches is written
            const uint32_t p = (uint32_t)max(a.pool.k_len[b], 0) - (uint32_t)n + (uint32_t)i;
            const bool live = u < units && i >= 0 && i < n && p < (uint32_t)a.pool.width * (uint32_t)a.pool.page;
            at[k] = live ? cache_row(a.pool, a.by_page, b, x.head, (int)p) : -1;
            map[k] = x.map;
            m[k] = live ? max(min(dim - c, E), 0) : 0;
            // with starts, rows are the tokens of one sequence
            const int64_t rb = a.starts ? 0 : b, ri = a.starts ? (int64_t)x.row : i;
            const T *from = value ? (const T *)a.v + rb * a.vs[0] + ri * a.vs[1] + x.head * a.vs[2]
                                  : (const T *)a.k + rb * a.ks[0] + ri * a.ks[1] + x.head * a.ks[2] + x.map * a.ks[3];
            y[k].load(from + c, m[k]);
        }
#pragma unroll
        for (int k = 0; k < kTurnRows; ++k) {
            S *to = stored_row<S>(a.pool, value, at[k], map[k]) + c;
            if constexpr (kScaled<S>) {
                const float top = __uint_as_float(group_max(y[k].top(), group));
                const bool bad = !(top < INFINITY);
                const float scale = bad ? 1.0f : __builtin_fmaxf(top / kTop<S>, 0x1p-126f);
                float x[E];
                y[k].numbers(x);
                quotients<S>(x, scale);
                if (at[k] < 0 || m[k] == 0)
                    continue;
                if (c == 0)
                    *scale_of(a.pool, value, at[k], map[k]) = bad ? __builtin_nanf("") : scale;
#pragma unroll
                for (int i = 0; i < E / 8; ++i) {
                    float z[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        z[j] = bad ? 0.0f : x[8 * i + j];
                    const Stored8<S> r = pack<S>(z);
                    if constexpr (PE != 0)
                        put_stored(to + 8 * i, r);
                    else
                        put_stored_some(to, r, m[k]);
                }
            } else {
                if (at[k] < 0 || m[k] == 0)
                    continue;
#pragma unroll
                for (int i = 0; i < E / 8; ++i) {
                    Stored8<S> r;
                    __builtin_memcpy(r.w, y[k].w + i * Stored8<S>::kWords, sizeof(r.w));
                    if constexpr (PE != 0)
                        put_stored(to + 8 * i, r);
                    else
                        put_stored_some(to, r, m[k]);
                }
            }
        }
    }
}

// The first `length` positions of every sequence, 0 where there is no token.  Bound by
// memory (the same cache 19 us).
template <class T, class S, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_cache_read(CacheArgs a)
{
    const bool value = blockIdx.y;
    T *const to = value ? (T *)a.v : (T *)a.k;
    if (!to)
        return;
    const int group = a.group[value], per = kThreads / group, c = (threadIdx.x & (group - 1)) * 8;
    const int dim = value ? a.pool.dim_v : a.pool.dim, m = max(min(dim - c, 8), 0);
    const uint32_t units = a.rows * a.pool.kv_heads * (value ? 1 : a.pool.maps);
    for (uint32_t u0 = blockIdx.x * per * kTurnRows; u0 < units; u0 += gridDim.x * per * kTurnRows) {
        float y[kTurnRows][8], scale[kTurnRows];
#pragma unroll
        for (int k = 0; k < kTurnRows; ++k) {
            const uint32_t u = u0 + k * per + threadIdx.x / group;
            const Unit x(a, min(u, units - 1));
            const int b = (int)a.by_length(x.row), p = (int)(x.row - b * (uint32_t)a.length);
            const int at = p < cached(a.pool, b) ? cache_row(a.pool, a.by_page, b, x.head, p) : -1;
            get8<S, WIDE>(stored_row<const S>(a.pool, value, at, x.map) + c, at < 0 ? 0 : m, y[k]);
            if constexpr (kScaled<S>)
                scale[k] = at < 0 ? 0.0f : *scale_of(a.pool, value, at, x.map);
        }
#pragma unroll
        for (int k = 0; k < kTurnRows; ++k) {
            const uint32_t u = u0 + k * per + threadIdx.x / group;
            if (u >= units || m == 0)
                continue;
            if constexpr (kScaled<S>) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    y[k][j] *= scale[k];
            }
            // units come in the order of the rows that are read
            T *row = to + (int64_t)u * dim + c;
            const Stored8<T> r = pack<T>(y[k]);
            if constexpr (WIDE)
                put_stored(row, r);
            else
                put_stored_some(row, r, m);
        }
    }
}

// Eight elements at a time, or `piece`: rows are whole pieces, and every place a multiple of
// 16 bytes, or of 8 for stored types of 8 bits.
bool wide_of(int piece, const pam_cache_desc_t &d, const void *k, const void *v, const int64_t *ks, const int64_t *vs)
{
    uint64_t all = (uint64_t)d.dim | (uint64_t)d.dim_v;
    for (int i = 0; ks && i < 4; ++i)
        all |= (uint64_t)ks[i];
    for (int i = 0; vs && i < 3; ++i)
        all |= (uint64_t)vs[i];
    return all % piece == 0 && ((uintptr_t)k | (uintptr_t)v) % 16 == 0;
}

CacheArgs args_of(const pam_cache_desc_t &d, const Pool &pool, int64_t rows, int32_t length, int piece)
{
    CacheArgs a{};
    a.pool = pool;
    a.rows = (uint32_t)rows;
    a.length = length;
    for (int v = 0; v < 2; ++v) {
        a.group[v] = 1;
        while (a.group[v] * (piece ? piece : 8) < (v ? d.dim_v : d.dim))
            a.group[v] *= 2;
        a.by_heads[v] = Divisor::of(d.kv_heads * (int64_t)(v ? 1 : d.maps));
        a.by_block[v] = Divisor::of(d.kv_heads * (int64_t)(v ? 1 : d.maps) * kBlockTokens);
    }
    a.by_length = Divisor::of(std::max(length, 1));
    a.by_page = Divisor::of(d.page_size);
    return a;
}

dim3 grid_of(const CacheArgs &a)
{
    int64_t blocks = 1;
    for (int v = 0; v < 2; ++v) {
        const int64_t per = (int64_t)kThreads / a.group[v] * kTurnRows;
        blocks = std::max(blocks, (((int64_t)a.rows + kBlockTokens - 1) / kBlockTokens * kBlockTokens * a.pool.kv_heads * (v ? 1 : a.pool.maps) + per - 1) / per);
    }
    return dim3((unsigned)std::min<int64_t>(blocks, 1 << 20), 2);
}

template <class T, class S>
void launch_pair(const CacheArgs &a, bool write, int piece, hipStream_t s)
{
    const dim3 grid = grid_of(a), block(kThreads);
    if (write && piece == 16)
        hipLaunchKernelGGL((k_cache_write<T, S, 16>), grid, block, 0, s, a);
    else if (write && piece == 8)
        hipLaunchKernelGGL((k_cache_write<T, S, 8>), grid, block, 0, s, a);
    else if (write)
        hipLaunchKernelGGL((k_cache_write<T, S, 0>), grid, block, 0, s, a);
    else if (piece)
        hipLaunchKernelGGL((k_cache_read<T, S, true>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_cache_read<T, S, false>), grid, block, 0, s, a);
}

template <class T>
void launch_type(const pam_cache_desc_t &d, const CacheArgs &a, bool write, int piece, hipStream_t s)
{
    if (d.store == PAM_STORE_E4M3)
        launch_pair<T, e4m3>(a, write, piece, s);
    else if (d.store == PAM_STORE_INT8)
        launch_pair<T, int8>(a, write, piece, s);
    else
        launch_pair<T, T>(a, write, piece, s);
}

hipError_t launch_any(const pam_cache_desc_t &d, const CacheArgs &a, bool write, int piece, hipStream_t s)
{
    if (d.dtype == PAM_F32)
        launch_type<float>(d, a, write, piece, s);
    else if (d.dtype == PAM_F16)
        launch_type<f16>(d, a, write, piece, s);
    else
        launch_type<bf16>(d, a, write, piece, s);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const pam_cache_desc_t &d, const pam_cache_rows_t &rows, const Pool &pool, const void *k,
                              const void *v, const int32_t *starts, const int32_t *new_len, hipStream_t s)
{
    const int64_t *ks = rows.k_stride, *vs = rows.v_stride;
    const int piece = wide_of(16, d, k, v, ks, vs) ? 16 : (wide_of(8, d, k, v, ks, vs) ? 8 : 0);
    CacheArgs a = args_of(d, pool, rows.rows, rows.length, piece);
    a.k = const_cast<void *>(k);
    a.v = const_cast<void *>(v);
    a.starts = starts;
    a.new_len = new_len;
    for (int i = 0; i < 4; ++i)
        a.ks[i] = ks[i];
    for (int i = 0; i < 3; ++i)
        a.vs[i] = vs[i];
    return launch_any(d, a, true, piece, s);
}

hipError_t launch_cache_read(const pam_cache_desc_t &d, int32_t length, const Pool &pool, void *k, void *v,
                             hipStream_t s)
{
    const int piece = wide_of(8, d, k, v, nullptr, nullptr) ? 8 : 0;
    CacheArgs a = args_of(d, pool, (int64_t)d.sequences * length, length, piece);
    a.k = k;
    a.v = v;
    return launch_any(d, a, false, piece, s);
}

}  // namespace pam
