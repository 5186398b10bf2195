// Rows of a paged cache (gfx950): stored types, eight elements at a time, and
// where a token's rows lie.
#pragma once

#include "pam_rows.h"

namespace pam {

// numbers of 8 bits
struct e4m3 {
    uint8_t bits;
};
typedef int8_t int8;

template <class S>
constexpr bool kScaled = sizeof(S) == 1;
// the number that a row's largest magnitude is stored as
template <class S>
constexpr float kTop = std::is_same<S, e4m3>::value ? 448.0f : 127.0f;

// Eight stored elements as they lie in memory.
template <class S>
struct Stored8 {
    static constexpr int kWords = 2 * sizeof(S);
    uint32_t w[kWords];
};

// eight elements at p, which is a multiple of their size up to 16 bytes
template <class S>
__device__ __forceinline__ Stored8<S> load_stored(const S *p)
{
    Stored8<S> r;
    __builtin_memcpy(r.w, __builtin_assume_aligned(p, sizeof(S) == 1 ? 8 : 16), 8 * sizeof(S));
    return r;
}
// the first n of eight elements at p, one by one; the others are 0
template <class S>
__device__ __forceinline__ Stored8<S> load_stored_some(const S *p, int n)
{
    S x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        x[j] = j < n ? p[j] : S{};
    Stored8<S> r;
    __builtin_memcpy(r.w, x, sizeof(x));
    return r;
}
template <class S>
__device__ __forceinline__ void put_stored(S *p, const Stored8<S> &r)
{
    __builtin_memcpy(__builtin_assume_aligned(p, sizeof(S) == 1 ? 8 : 16), r.w, 8 * sizeof(S));
}
template <class S>
__device__ __forceinline__ void put_stored_some(S *p, const Stored8<S> &r, int n)
{
    S x[8];
    __builtin_memcpy(x, r.w, sizeof(x));
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n)
            p[j] = x[j];
}

// as numbers
template <class S>
__device__ __forceinline__ void unpack(const Stored8<S> &r, float (&x)[8])
{
    if constexpr (std::is_same<S, e4m3>::value) {
        typedef float float2v __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2v y = j & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(r.w[j / 2], true)
                                    : __builtin_amdgcn_cvt_pk_f32_fp8(r.w[j / 2], false);
            x[2 * j] = y[0];
            x[2 * j + 1] = y[1];
        }
    } else {
        S y[8];
        __builtin_memcpy(y, r.w, sizeof(y));
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[j] = (float)y[j];
    }
}

// Four stored numbers of 8 bits, which lie in a word, as T: exact.
template <class T, class S>
__device__ __forceinline__ void widen(uint32_t w, uint32_t (&to)[sizeof(T)])
{
    if constexpr (std::is_same<S, e4m3>::value && std::is_same<T, bf16>::value) {
        to[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
        to[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
    } else if constexpr (std::is_same<S, e4m3>::value && std::is_same<T, f16>::value) {
        to[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
        to[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
    } else {
        typedef T T4 __attribute__((ext_vector_type(4)));
        float x[4];
        if constexpr (std::is_same<S, e4m3>::value) {
            const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            x[0] = a[0];
            x[1] = a[1];
            x[2] = b[0];
            x[3] = b[1];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[j] = (float)(int8)(w >> (8 * j));
        }
        const T4 y = {(T)x[0], (T)x[1], (T)x[2], (T)x[3]};
        __builtin_memcpy(to, &y, sizeof(y));
    }
}

// Numbers as stored: to nearest, ties to even.  Those of 8 bits are in
// [-kTop, kTop].
template <class S>
__device__ __forceinline__ Stored8<S> pack(const float (&x)[8])
{
    Stored8<S> r;
    if constexpr (std::is_same<S, e4m3>::value) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * j], x[4 * j + 1], 0, false);
            r.w[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * j + 2], x[4 * j + 3], w, true);
        }
    } else if constexpr (std::is_same<S, int8>::value) {
        int8 y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            y[j] = (int8)(int)__builtin_rintf(x[j]);
        __builtin_memcpy(r.w, y, sizeof(y));
    } else {
        S y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            y[j] = rounded<S>(x[j]);
        __builtin_memcpy(r.w, y, sizeof(y));
    }
    return r;
}

// tokens of sequence b
__device__ __forceinline__ int cached(const Pool &c, int b)
{
    return min(max(c.k_len[b], 0), (int)((uint32_t)c.width * (uint32_t)c.page));
}

// Number of the row of head h of the token at position p (in [0, width page)) of
// sequence b, counted in tokens of a head; negative: there is no such page.
// by_page: of the page's size.
__device__ __forceinline__ int cache_row(const Pool &c, const Divisor &by_page, int b, int h, int p)
{
    const int w = (int)by_page((uint32_t)p), at = c.table[(int64_t)b * c.width + w];
    return at >= 0 && at < c.pages ? (at * c.kv_heads + h) * c.page + (p - w * c.page) : -1;
}

}  // namespace pam
