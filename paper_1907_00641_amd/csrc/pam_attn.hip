// Differential attention (gfx950): out = (P0 - lambda P1) v and its gradients.
#include "pam_attn.h"

#include <algorithm>

namespace pam {

namespace {

constexpr int kWaves = 4;
constexpr int kRowThreads = 64 * kWaves;

__device__ __forceinline__ float wave_max(float x)
{
    for (int s = 1; s < 64; s <<= 1)
        x = __builtin_fmaxf(x, __shfl_xor(x, s));
    return x;
}

// Orders a wave's own LDS accesses (its lanes exchange data through LDS).
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ bool sees(const AttnArgs &a, int b, int i, int j, int nq, int nk)
{
    if (i >= nq || j >= nk || (a.causal && j > i + nk - nq))
        return false;
    return !a.key_mask || a.key_mask[(int64_t)b * a.len_k + j];
}

// A wave per query row; lanes take keys for the scores, channels for the sums.
template <class T>
__global__ __launch_bounds__(kRowThreads) void k_attn_row_fwd(AttnArgs a)
{
    __shared__ float sq[kWaves][2][PAM_ATTN_MAX_DIM], sp[kWaves][2][64];
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
    const int64_t rows = (int64_t)a.batch * a.heads * a.len_q;
    for (int64_t r0 = (int64_t)blockIdx.x * kWaves; r0 < rows; r0 += (int64_t)gridDim.x * kWaves) {
        const int64_t r = r0 + w;
        if (r >= rows)
            break;
        const int i = (int)(r % a.len_q), h = (int)(r / a.len_q % a.heads), b = (int)(r / a.len_q / a.heads);
        const int hk = h / a.group, nq = q_len_of(a, b), nk = k_len_of(a, b);
        const float lam = (float)((const T *)a.lam)[h];
        const T *q = (const T *)a.q + b * a.qs[0] + i * a.qs[1] + h * a.qs[2];
        wave_fence();
        for (int x = l; x < a.dim; x += 64)
            for (int m = 0; m < 2; ++m)
                sq[w][m][x] = (float)q[m * a.qs[3] + x] * a.scale;
        wave_fence();
        float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0, 0}, o[2][4] = {};
        const int end = i < nq ? (a.causal ? min(nk, i + nk - nq + 1) : nk) : 0;
        for (int j0 = 0; j0 < end; j0 += 64) {
            const int j = j0 + l;
            const bool see = j < end && sees(a, b, i, j, nq, nk);
            float s[2] = {-INFINITY, -INFINITY};
            if (see) {
                const T *k = (const T *)a.k + b * a.ks[0] + j * a.ks[1] + hk * a.ks[2];
                for (int m = 0; m < 2; ++m) {
                    s[m] = 0.0f;
                    for (int x = 0; x < a.dim; ++x)
                        s[m] += sq[w][m][x] * (float)k[m * a.ks[3] + x];
                }
            }
            const unsigned long long any = __ballot(see);
            if (!any)
                continue;
            for (int m = 0; m < 2; ++m) {
                const float t = __builtin_fmaxf(top[m], wave_max(s[m]));
                const float f = top[m] == -INFINITY ? 0.0f : __expf(top[m] - t);
                top[m] = t;
                const float p = see ? __expf(s[m] - t) : 0.0f;
                sum[m] = sum[m] * f + lanes_sum<64>(p);
                for (int c = 0; c < 4; ++c)
                    o[m][c] *= f;
                sp[w][m][l] = p;
            }
            wave_fence();
            for (int t = 0; t < 64; ++t) {
                if (!(any >> t & 1))
                    continue;
                const T *v = (const T *)a.v + b * a.vs[0] + (j0 + t) * a.vs[1] + hk * a.vs[2];
                for (int c = 0; c < 4; ++c)
                    if (c * 64 + l < a.dim_v) {
                        const float vv = (float)v[c * 64 + l];
                        o[0][c] += sp[w][0][t] * vv;
                        o[1][c] += sp[w][1][t] * vv;
                    }
            }
            wave_fence();
        }
        const float i0 = sum[0] != 0.0f ? 1.0f / sum[0] : 0.0f, i1 = sum[1] != 0.0f ? 1.0f / sum[1] : 0.0f;
        const int64_t row = ((int64_t)b * a.len_q + i) * a.heads + h;
        for (int c = 0; c < 4; ++c)
            if (c * 64 + l < a.dim_v) {
                const float o0 = o[0][c] * i0, o1 = o[1][c] * i1;
                const int64_t at = row * a.dim_v + c * 64 + l;
                ((T *)a.out)[at] = (T)(o0 - lam * o1);
                if (a.so) {
                    ((T *)a.so)[at] = (T)o0;
                    ((T *)a.so)[a.so_map + at] = (T)o1;
                }
            }
        if (a.lse && l < 2)
            a.lse[l * a.lse_map + r] = sum[l] != 0.0f ? top[l] + __logf(sum[l]) : -INFINITY;
    }
}

// D^m = <grad_out, o^m>, a wave per row
template <class T>
__global__ __launch_bounds__(kRowThreads) void k_attn_row_dsum(AttnArgs a)
{
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
    const int64_t rows = (int64_t)a.batch * a.heads * a.len_q;
    for (int64_t r0 = (int64_t)blockIdx.x * kWaves; r0 < rows; r0 += (int64_t)gridDim.x * kWaves) {
        const int64_t r = r0 + w;
        if (r >= rows)
            break;
        const int i = (int)(r % a.len_q), h = (int)(r / a.len_q % a.heads), b = (int)(r / a.len_q / a.heads);
        const int64_t row = ((int64_t)b * a.len_q + i) * a.heads + h;
        const T *g = (const T *)a.dout + b * a.dos[0] + i * a.dos[1] + h * a.dos[2];
        float s0 = 0.0f, s1 = 0.0f;
        if (i < q_len_of(a, b))
            for (int c = l; c < a.dim_v; c += 64) {
                s0 += (float)g[c] * (float)((const T *)a.so)[row * a.dim_v + c];
                s1 += (float)g[c] * (float)((const T *)a.so)[a.so_map + row * a.dim_v + c];
            }
        s0 = lanes_sum<64>(s0);
        s1 = lanes_sum<64>(s1);
        if (l == 0) {
            a.dsum[r] = s0;
            a.dsum[a.lse_map + r] = s1;
        }
    }
}

// p and ds of both maps for one pair; q and k rows, dout and v rows in memory
template <class T>
__device__ __forceinline__ void pair_terms(const AttnArgs &a, const T *q, const T *k, const T *g, const T *v,
                                           float lam, const float lse[2], const float D[2], float p[2], float ds[2],
                                           float &dp)
{
    dp = 0.0f;
    for (int c = 0; c < a.dim_v; ++c)
        dp += (float)g[c] * (float)v[c];
    for (int m = 0; m < 2; ++m) {
        float s = 0.0f;
        for (int x = 0; x < a.dim; ++x)
            s += (float)q[m * a.qs[3] + x] * (float)k[m * a.ks[3] + x];
        p[m] = __expf(s * a.scale - lse[m]);
        ds[m] = p[m] * (dp - D[m]) * a.scale * (m ? -lam : 1.0f);
    }
}

template <class T>
__global__ __launch_bounds__(kRowThreads) void k_attn_row_dq(AttnArgs a)
{
    __shared__ float sp[kWaves][2][64];
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
    const int64_t rows = (int64_t)a.batch * a.heads * a.len_q;
    for (int64_t r0 = (int64_t)blockIdx.x * kWaves; r0 < rows; r0 += (int64_t)gridDim.x * kWaves) {
        const int64_t r = r0 + w;
        if (r >= rows)
            break;
        const int i = (int)(r % a.len_q), h = (int)(r / a.len_q % a.heads), b = (int)(r / a.len_q / a.heads);
        const int hk = h / a.group, nq = q_len_of(a, b), nk = k_len_of(a, b);
        const float lam = (float)((const T *)a.lam)[h];
        const T *q = (const T *)a.q + b * a.qs[0] + i * a.qs[1] + h * a.qs[2];
        const T *g = (const T *)a.dout + b * a.dos[0] + i * a.dos[1] + h * a.dos[2];
        const float lse[2] = {a.lse[r], a.lse[a.lse_map + r]}, D[2] = {a.dsum[r], a.dsum[a.lse_map + r]};
        float acc[2][2] = {}, dlam = 0.0f;
        const int end = i < nq ? (a.causal ? min(nk, i + nk - nq + 1) : nk) : 0;
        for (int j0 = 0; j0 < end; j0 += 64) {
            const int j = j0 + l;
            const bool see = j < end && sees(a, b, i, j, nq, nk);
            float p[2], ds[2] = {0, 0}, dp;
            if (see) {
                pair_terms(a, q, (const T *)a.k + b * a.ks[0] + j * a.ks[1] + hk * a.ks[2], g,
                           (const T *)a.v + b * a.vs[0] + j * a.vs[1] + hk * a.vs[2], lam, lse, D, p, ds, dp);
                dlam += p[1] * dp;
            }
            sp[w][0][l] = ds[0];
            sp[w][1][l] = ds[1];
            const unsigned long long any = __ballot(see);
            wave_fence();
            for (int t = 0; t < 64; ++t) {
                if (!(any >> t & 1))
                    continue;
                const T *k = (const T *)a.k + b * a.ks[0] + (j0 + t) * a.ks[1] + hk * a.ks[2];
                for (int m = 0; m < 2; ++m)
                    for (int c = 0; c < 2; ++c)
                        if (c * 64 + l < a.dim)
                            acc[m][c] += sp[w][m][t] * (float)k[m * a.ks[3] + c * 64 + l];
            }
            wave_fence();
        }
        const int64_t row = ((int64_t)b * a.len_q + i) * a.heads + h;
        for (int m = 0; m < 2; ++m)
            for (int c = 0; c < 2; ++c)
                if (c * 64 + l < a.dim)
                    ((T *)a.gq)[(row * 2 + m) * a.dim + c * 64 + l] = (T)acc[m][c];
        dlam = lanes_sum<64>(dlam);
        if (l == 0)
            a.dlam[r] = dlam;
    }
}

template <class T>
__global__ __launch_bounds__(kRowThreads) void k_attn_row_dkv(AttnArgs a)
{
    __shared__ float sp[kWaves][3][64];
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
    const int64_t rows = (int64_t)a.batch * a.kv_heads * a.len_k;
    for (int64_t r0 = (int64_t)blockIdx.x * kWaves; r0 < rows; r0 += (int64_t)gridDim.x * kWaves) {
        const int64_t r = r0 + w;
        if (r >= rows)
            break;
        const int j = (int)(r % a.len_k), hk = (int)(r / a.len_k % a.kv_heads), b = (int)(r / a.len_k / a.kv_heads);
        const int nq = q_len_of(a, b), nk = k_len_of(a, b);
        const T *k = (const T *)a.k + b * a.ks[0] + j * a.ks[1] + hk * a.ks[2];
        const T *v = (const T *)a.v + b * a.vs[0] + j * a.vs[1] + hk * a.vs[2];
        float gk[2][2] = {}, gv[4] = {};
        for (int h = hk * a.group; h < (hk + 1) * a.group; ++h) {
            const float lam = (float)((const T *)a.lam)[h];
            for (int i0 = 0; i0 < nq; i0 += 64) {
                const int i = i0 + l;
                const bool see = i < nq && sees(a, b, i, j, nq, nk);
                float p[2] = {0, 0}, ds[2] = {0, 0}, dp;
                if (see) {
                    const int64_t at = ((int64_t)b * a.heads + h) * a.len_q + i;
                    const float lse[2] = {a.lse[at], a.lse[a.lse_map + at]},
                                D[2] = {a.dsum[at], a.dsum[a.lse_map + at]};
                    pair_terms(a, (const T *)a.q + b * a.qs[0] + i * a.qs[1] + h * a.qs[2], k,
                               (const T *)a.dout + b * a.dos[0] + i * a.dos[1] + h * a.dos[2], v, lam, lse, D, p, ds,
                               dp);
                }
                sp[w][0][l] = ds[0];
                sp[w][1][l] = ds[1];
                sp[w][2][l] = p[0] - lam * p[1];
                const unsigned long long any = __ballot(see);
                wave_fence();
                for (int t = 0; t < 64; ++t) {
                    if (!(any >> t & 1))
                        continue;
                    const T *q = (const T *)a.q + b * a.qs[0] + (i0 + t) * a.qs[1] + h * a.qs[2];
                    const T *g = (const T *)a.dout + b * a.dos[0] + (i0 + t) * a.dos[1] + h * a.dos[2];
                    for (int m = 0; m < 2; ++m)
                        for (int c = 0; c < 2; ++c)
                            if (c * 64 + l < a.dim)
                                gk[m][c] += sp[w][m][t] * (float)q[m * a.qs[3] + c * 64 + l];
                    for (int c = 0; c < 4; ++c)
                        if (c * 64 + l < a.dim_v)
                            gv[c] += sp[w][2][t] * (float)g[c * 64 + l];
                }
                wave_fence();
            }
        }
        const int64_t row = ((int64_t)b * a.len_k + j) * a.kv_heads + hk;
        for (int m = 0; m < 2; ++m)
            for (int c = 0; c < 2; ++c)
                if (c * 64 + l < a.dim)
                    ((T *)a.gk)[(row * 2 + m) * a.dim + c * 64 + l] = (T)gk[m][c];
        for (int c = 0; c < 4; ++c)
            if (c * 64 + l < a.dim_v)
                ((T *)a.gv)[row * a.dim_v + c * 64 + l] = (T)gv[c];
    }
}

// grad_lambda[h] = -sum over the sequences and queries, in a fixed order
template <class T>
__global__ __launch_bounds__(1024) void k_attn_dlam(AttnArgs a)
{
    __shared__ float s[16];
    const int h = blockIdx.x;
    float y = 0.0f;
    for (int b = 0; b < a.batch; ++b)
        for (int i = threadIdx.x; i < a.len_q; i += 1024)
            y += a.dlam[((int64_t)b * a.heads + h) * a.len_q + i];
    y = lanes_sum<64>(y);
    if ((threadIdx.x & 63) == 0)
        s[threadIdx.x >> 6] = y;
    __syncthreads();
    if (threadIdx.x == 0) {
        y = 0.0f;
        for (int w = 0; w < 16; ++w)
            y += s[w];
        ((T *)a.glam)[h] = (T)-y;
    }
}

unsigned row_blocks(int64_t rows) { return (unsigned)std::min<int64_t>((rows + kWaves - 1) / kWaves, 1 << 20); }

template <class T>
hipError_t fwd_t(const AttnArgs &a, hipStream_t s)
{
    const int64_t rows = (int64_t)a.batch * a.heads * a.len_q;
    if (rows == 0)
        return hipSuccess;
    hipLaunchKernelGGL(k_attn_row_fwd<T>, dim3(row_blocks(rows)), dim3(kRowThreads), 0, s, a);
    return hipGetLastError();
}

template <class T>
hipError_t bwd_t(const AttnArgs &a, hipStream_t s)
{
    const int64_t rows = (int64_t)a.batch * a.heads * a.len_q, keys = (int64_t)a.batch * a.kv_heads * a.len_k;
    if (rows) {
        hipLaunchKernelGGL(k_attn_row_dsum<T>, dim3(row_blocks(rows)), dim3(kRowThreads), 0, s, a);
        hipLaunchKernelGGL(k_attn_row_dq<T>, dim3(row_blocks(rows)), dim3(kRowThreads), 0, s, a);
    }
    if (keys)
        hipLaunchKernelGGL(k_attn_row_dkv<T>, dim3(row_blocks(keys)), dim3(kRowThreads), 0, s, a);
    hipLaunchKernelGGL(k_attn_dlam<T>, dim3(a.heads), dim3(1024), 0, s, a);
    return hipGetLastError();
}

AttnArgs attn_args(const pam_diff_attn_desc_t &d, const void *q, const void *k, const void *v, const void *lam,
                   const int32_t *q_len, const int32_t *k_len, const uint8_t *key_mask)
{
    AttnArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.lam = lam;
    a.q_len = q_len;
    a.k_len = k_len;
    a.key_mask = key_mask;
    for (int i = 0; i < 4; ++i) {
        a.qs[i] = d.q_stride[i];
        a.ks[i] = d.k_stride[i];
    }
    for (int i = 0; i < 3; ++i)
        a.vs[i] = d.v_stride[i];
    a.batch = d.batch;
    a.heads = d.heads;
    a.kv_heads = d.kv_heads;
    a.group = d.heads / d.kv_heads;
    a.dim = d.dim;
    a.dim_v = d.dim_v;
    a.len_q = d.len_q;
    a.len_k = d.len_k;
    a.causal = (d.flags & PAM_ATTN_CAUSAL) != 0;
    a.scale = d.scale;
    a.lse_map = (int64_t)d.batch * d.heads * d.len_q;
    a.so_map = a.lse_map * d.dim_v;
    return a;
}

}  // namespace

size_t attn_fwd_workspace(const pam_diff_attn_desc_t &) { return 0; }

size_t attn_bwd_workspace(const pam_diff_attn_desc_t &d)
{
    return 3 * sizeof(float) * (size_t)d.batch * d.heads * d.len_q;
}

hipError_t launch_attn_fwd(const pam_diff_attn_desc_t &d, const void *q, const void *k, const void *v,
                           const void *lam, const int32_t *q_len, const int32_t *k_len, const uint8_t *key_mask,
                           void *out, void *so, float *lse, void *workspace, hipStream_t s)
{
    AttnArgs a = attn_args(d, q, k, v, lam, q_len, k_len, key_mask);
    a.out = out;
    a.so = so;
    a.lse = lse;
    if (d.dtype == PAM_F32)
        return fwd_t<float>(a, s);
    return d.dtype == PAM_F16 ? fwd_t<f16>(a, s) : fwd_t<bf16>(a, s);
}

hipError_t launch_attn_bwd(const pam_diff_attn_desc_t &d, const void *q, const void *k, const void *v,
                           const void *lam, const int32_t *q_len, const int32_t *k_len, const uint8_t *key_mask,
                           const void *so, const float *lse, const void *dout, const int64_t *dos, void *gq, void *gk,
                           void *gv, void *glam, void *workspace, hipStream_t s)
{
    AttnArgs a = attn_args(d, q, k, v, lam, q_len, k_len, key_mask);
    a.so = const_cast<void *>(so);
    a.lse = const_cast<float *>(lse);
    a.dout = dout;
    for (int i = 0; i < 3; ++i)
        a.dos[i] = dos[i];
    a.gq = gq;
    a.gk = gk;
    a.gv = gv;
    a.glam = glam;
    a.dsum = (float *)workspace;
    a.dlam = a.dsum + 2 * a.lse_map;
    if (d.dtype == PAM_F32)
        return bwd_t<float>(a, s);
    return d.dtype == PAM_F16 ? bwd_t<f16>(a, s) : bwd_t<bf16>(a, s);
}

}  // namespace pam
