// What the attention kernels share: the range of fp16, fences of a wave, launches
// with much LDS.
#pragma once

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "pam_attn_tiles.h"

namespace pam {

namespace {

constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = 4;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// fp16 has 2^-14 as its smallest full-precision value: its probabilities are
// taken 2^7 larger, which gives small ones 7 bits of room, and are at most 2^15.
template <class T>
constexpr float kLift = std::is_same<T, f16>::value ? 7.0f : 0.0f;

// Score gradients have no such bound.  In fp16 a lane (a query, or a key)
// multiplies its own by a power of two that puts the first tile's largest at
// 2^7 .. 2^8, and takes a smaller one, scaling what it has summed, if a later
// tile would pass 2^15.
struct Range {
    float up = 0.0f;  // 0: not chosen yet
    // x: this lane's results of a tile; both lanes of a column agree
    template <int N, class F>
    __device__ __forceinline__ void fit(f32x16 (&x)[N], const F &scale_sums)
    {
        float mx = 0.0f;
#pragma unroll
        for (int m = 0; m < N; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                mx = __builtin_fmaxf(mx, __builtin_fabsf(x[m][r]));
        mx = xor32_max(mx);
        const bool change = up == 0.0f ? mx > 0.0f : mx * up > 32768.0f;
        if (__any(change)) {
            const float to = change ? __builtin_ldexpf(1.0f, min(8 - __builtin_amdgcn_frexp_expf(mx), 100)) : up;
            scale_sums(up == 0.0f ? 1.0f : to / up);
            up = to;
        }
#pragma unroll
        for (int m = 0; m < N; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                x[m][r] *= up;
    }
    __device__ __forceinline__ float down() const { return up == 0.0f ? 1.0f : 1.0f / up; }
};

// Orders a wave's own LDS accesses: its lanes exchange data through LDS.  They are
// waited for, since the loads that write LDS directly keep no order with them.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt 0, others not waited for
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A value that is the same in every lane, in a scalar register: divisions are
// vector code, and what is computed from their results would stay there.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uniform_float(float x)
{
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}

// The lowest n of 32 bits.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : (1u << max(n, 0)) - 1; }

// a row's logarithm of its sum, from the running maximum in base 2
template <class T>
__device__ __forceinline__ float lse_of(float top, float sum)
{
    return sum != 0.0f ? (top - kLift<T> + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

// blocks of a launch: fewer than 2^32 work items, the rest in turns
inline unsigned item_blocks(int64_t items) { return (unsigned)std::min<int64_t>(items, 1 << 23); }

// `done`: devices that know of the kernel's LDS beyond 64 KB
template <class A, class K>
hipError_t launch_lds(K kernel, unsigned blocks, unsigned threads, int lds, const A &a, hipStream_t s,
                      std::atomic<uint64_t> &done)
{
    if (lds > (64 << 10)) {
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
        if (e == hipSuccess && !(done.load(std::memory_order_relaxed) & bit)) {
            e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            if (e == hipSuccess)
                done.fetch_or(bit, std::memory_order_relaxed);
        }
        if (e != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), lds, s, a);
    return hipGetLastError();
}
template <auto K, class A>
hipError_t launch_lds(unsigned blocks, unsigned threads, int lds, const A &a, hipStream_t s)
{
    static std::atomic<uint64_t> done{0};
    return launch_lds(K, blocks, threads, lds, a, s, done);
}

inline unsigned sum_blocks(int64_t sums)
{
    return (unsigned)std::min<int64_t>((sums + kAttnThreads - 1) / kAttnThreads, 8192);
}

}  // namespace

}  // namespace pam
