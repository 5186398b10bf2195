// Device code shared by the operators around the attention layer: element
// types, wide loads and stores of eight elements, sums over lanes, the
// counter-based generator of dropout.
#pragma once

#include "pam_internal.h"

namespace pam {

typedef _Float16 f16;
typedef __bf16 bf16;

typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));

// 16 bytes at p (16-byte aligned)
__device__ __forceinline__ uint4v load16(const void *p) { return *reinterpret_cast<const uint4v *>(p); }
__device__ __forceinline__ void store16(void *p, uint4v x) { *reinterpret_cast<uint4v *>(p) = x; }

// eight elements at p (16-byte aligned) as floats
template <class T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
        const float4v a = *reinterpret_cast<const float4v *>(p), b = *reinterpret_cast<const float4v *>(p + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = a[j];
            x[4 + j] = b[j];
        }
    } else {
        typedef T T8 __attribute__((ext_vector_type(8)));
        const T8 a = *reinterpret_cast<const T8 *>(p);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[j] = (float)a[j];
    }
}

template <class T>
__device__ __forceinline__ void store8(T *p, const float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
        float4v a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = x[j];
            b[j] = x[4 + j];
        }
        *reinterpret_cast<float4v *>(p) = a;
        *reinterpret_cast<float4v *>(p + 4) = b;
    } else {
        typedef T T8 __attribute__((ext_vector_type(8)));
        T8 a;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            a[j] = (T)x[j];  // to nearest, ties to even
        *reinterpret_cast<T8 *>(p) = a;
    }
}

// Lane moves within rows of 16 lanes; the lanes 16 and 32 away by exchanging
// halves of a register pair.  Every lane of the wave takes part.
template <int CTRL>
__device__ __forceinline__ float lane_move(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float xor16_add(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float xor32_add(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float xor32_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Sum over an aligned group of G lanes (a power of two), left in every lane.
// Call in wave-uniform control flow.
template <int G>
__device__ __forceinline__ float lanes_sum(float x)
{
    if constexpr (G >= 2)
        x += lane_move<0xb1>(x);   // lane ^ 1
    if constexpr (G >= 4)
        x += lane_move<0x4e>(x);   // lane ^ 2
    if constexpr (G >= 8)
        x += lane_move<0x141>(x);  // 7 - lane within 8
    if constexpr (G >= 16)
        x += lane_move<0x140>(x);  // 15 - lane within 16
    if constexpr (G >= 32)
        x = xor16_add(x);
    if constexpr (G >= 64)
        x = xor32_add(x);
    return x;
}

// x, an fp32 result, as T.  The compiler may fuse the operation that gave x with
// the rounding to fp16, and does so for some widths of access only; out of its
// sight, the bits do not depend on the width.
template <class T>
__device__ __forceinline__ T rounded(float x)
{
    asm("" : "+v"(x));
    return (T)x;
}

// Division of numbers below 2^31 by one that the host knows, 1 <= d < 2^31, as a product (the
// round-up method of Granlund and Montgomery 1994): with s = ceil(log2 d) and
// m = floor(2^32 (2^s - d) / d) + 1, n / d = (n + floor(n m / 2^32)) / 2^s.
struct Divisor {
    uint32_t m, s;
    __host__ static Divisor of(int64_t d)
    {
        uint32_t s = 0;
        while (((int64_t)1 << s) < d)
            ++s;
        return {(uint32_t)(((((uint64_t)1 << s) - (uint64_t)d) << 32) / (uint64_t)d + 1), s};
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (__umulhi(n, m) + n) >> s; }
};

// a / b of numbers that are not negative, in 32 bits where they fit
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b)
{
    return ((a | b) >> 32) ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// Philox4x32-10 (Salmon, Moraes, Dror and Shaw 2011, "Parallel random
// numbers: as easy as 1, 2, 3"): ten rounds of two 32 x 32 -> 64 bit products,
// the key stepped by Weyl constants.
struct Dropout {
    uint32_t k0, k1;    // key: the seed
    uint32_t o0, o1;    // upper half of the counter: the offset
    uint32_t limit;     // drop where the 16-bit number is below: rint(65536 p)
    float keep;         // factor of what is kept
};

__device__ __forceinline__ uint4v philox(const Dropout &d, uint64_t block)
{
    uint32_t a = (uint32_t)block, b = (uint32_t)(block >> 32), c = d.o0, e = d.o1, k0 = d.k0, k1 = d.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t x = (uint64_t)a * 0xD2511F53u, y = (uint64_t)c * 0xCD9E8D57u;
        a = (uint32_t)(y >> 32) ^ b ^ k0;
        b = (uint32_t)y;
        c = (uint32_t)(x >> 32) ^ e ^ k1;
        e = (uint32_t)x;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return uint4v{a, b, c, e};
}

// whether element j (0..7) of a block's eight is kept
__device__ __forceinline__ bool kept(const Dropout &d, const uint4v &w, int j)
{
    return ((w[j >> 1] >> (16 * (j & 1))) & 0xffffu) >= d.limit;
}

}  // namespace pam
