// Tiles of the differential attention's matrix-core kernels (gfx950).
//
// Everything is built from 32 x 32 products with 32-bit sums
// (v_mfma_f32_32x32x16 of fp16 / bf16, v_mfma_f32_32x32x2 of fp32).  Lane l of
// a wave holds, of the result, column l % 32 and the sixteen rows
// 8 (r / 4) + 4 (l / 32) + r % 4.  A "chunk" is 16 bytes of an operand per lane:
// 16 (fp32: 8) values of the contracted axis, of which lane half h = l / 32
// holds one half.  Which eight of sixteen it holds is free as long as both
// operands agree, and is chosen so that
//   - where channels are contracted (scores, grad_out v^T) a lane reads 16
//     consecutive bytes of its row;
//   - where rows are contracted (P^T v, ds^T q, ...) a lane half holds the
//     rows 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3 of sixteen, which are the
//     rows of its registers of a 32 x 32 result: probabilities go from one
//     product to the next in the registers that they are computed in.
#pragma once

#include "pam_attn.h"

namespace pam {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));

#define PAM_LDS __attribute__((address_space(3)))
#define PAM_GLOBAL __attribute__((address_space(1)))

__device__ __forceinline__ int lane_id() { return threadIdx.x & 63; }
// the wave's number within its block, in a scalar register
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
__device__ __forceinline__ int result_row(int r) { return 8 * (r >> 2) + 4 * (lane_id() >> 5) + (r & 3); }

// channels (or rows) of a chunk
template <class T>
constexpr int kChunk = sizeof(T) == 4 ? 8 : 16;

// acc += a b over one chunk
template <class T>
__device__ __forceinline__ void mma(f32x16 &acc, uint4v a, uint4v b)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]), acc, 0, 0, 0);
    } else if constexpr (std::is_same<T, f16>::value) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc,
                                                     0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b),
                                                      acc, 0, 0, 0);
    }
}

// Chunk s of sixteen results as an operand, rounded to the operand's type (to
// nearest, ties to even): the matrix unit takes no wider one.  Each rounding
// is off by at most u = 2^-8 (bf16), 2^-11 (fp16) of its value.
template <class T>
__device__ __forceinline__ uint4v operand(const f32x16 &p, int s)
{
    if constexpr (sizeof(T) == 4) {
        uint4v r;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            r[j] = __float_as_uint(p[4 * s + j]);
        return r;
    } else {
        typedef T T8 __attribute__((ext_vector_type(8)));
        T8 r;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            r[j] = (T)p[8 * s + j];
        return __builtin_bit_cast(uint4v, r);
    }
}

// Rows of NC channels in LDS, without padding, since the loads that write LDS
// directly fill it in order.  The 16-byte pieces of a row are permuted by an
// exclusive or with an even number that depends on the row, so that eight
// lanes that read one piece of eight rows, and sixteen that read two pieces of
// four rows, meet every bank once.
template <class T, int NC>
struct Rows {
    static constexpr int kBytes = NC * sizeof(T);  // per row
    static constexpr int kPieces = kBytes / 16;
    static_assert(kPieces >= 8, "rows of 128 bytes at least");
    __device__ __forceinline__ static int turn(int row)
    {
        return kPieces == 8 ? (row & 6) : ((row & 7) << 1);
    }
    // chunk s of channels of row (row0 + lane % 32)
    __device__ __forceinline__ static uint4v row_chunk(const char *lds, int row0, int s)
    {
        const int l = lane_id(), row = l & 31;
        return load16(lds + (row0 + row) * kBytes + (((2 * s + (l >> 5)) ^ turn(row)) << 4));
    }
    // chunk s of the rows from row0 on, column c0 + lane % 32 (c0 a multiple of 32)
    __device__ __forceinline__ static uint4v col_chunk(const char *lds, int row0, int s, int c0)
    {
        const int l = lane_id(), h = l >> 5;
        if constexpr (sizeof(T) == 4) {
            uint4v r;
            const int piece = (c0 >> 2) + ((l & 31) >> 2);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = 4 * h + j;
                r[j] = *reinterpret_cast<const uint32_t *>(lds + (row0 + 8 * s + row) * kBytes +
                                                           ((piece ^ turn(row)) << 4) + ((l & 3) << 2));
            }
            return r;
        } else {
            // the transposing read: of sixteen lanes, lane 4 r + c gives the
            // address of four columns of row r, lane i gets column i of the four rows
            const int row = 4 * h + ((l & 15) >> 2);
            const int piece = ((2 * ((l >> 4) & 1) + ((l & 3) >> 1)) ^ turn(row)) ^ (c0 >> 3);
            const char *p = lds + (row0 + 16 * s + row) * kBytes + (piece << 4) + ((l & 1) << 3);
            const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PAM_LDS short4v *)p);
            const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PAM_LDS short4v *)(p + 8 * kBytes));
            const uint2v x = __builtin_bit_cast(uint2v, a), y = __builtin_bit_cast(uint2v, b);
            return uint4v{x[0], x[1], y[0], y[1]};
        }
    }
};

// Brings ROWS rows of PARTS parts (maps) of up to NC / PARTS channels from
// memory to LDS.  Rows past `last` repeat row `last` (they are cleared, or
// their products thrown away, by the caller); channels past `dim` of a part are
// not written: the caller has cleared the buffer once.
//   WIDE: 16 bytes per lane straight to LDS, nothing waits here.  All rows and
//   parts start at multiples of 16 bytes, dim is whole pieces, no stride is
//   negative, and a tile's offsets in bytes fit 32 bits.
//   else: element by element through registers.
template <class T, int NC, int PARTS, int ROWS, int WAVES, bool WIDE>
__device__ __forceinline__ void load_rows(char *lds, const T *from, int64_t row_stride, int64_t part_stride, int last,
                                          int dim)
{
    using R = Rows<T, NC>;
    constexpr int per = 16 / sizeof(T), kPart = R::kPieces / PARTS;
    if constexpr (WIDE) {
        constexpr int kLoads = ROWS * R::kBytes / 1024, kStep = WAVES * 64 / R::kPieces;  // rows between a wave's loads
        static_assert(kLoads % WAVES == 0, "whole loads per wave");
        const int w = wave_id(), at = w * 64 + lane_id();
        const int row0 = at / R::kPieces;
#pragma unroll
        for (int n = 0; n < kLoads / WAVES; ++n) {
            const int row = row0 + n * kStep;
            const int piece = (at % R::kPieces) ^ R::turn(kStep % 8 == 0 ? row0 : row);
            const int part = piece / kPart, ch = (piece % kPart) * per;
            const uint32_t off = (uint32_t)(min(row, last) * (int)row_stride + part * (int)part_stride + ch);
            if (ch < dim)
                __builtin_amdgcn_global_load_lds(
                    (const PAM_GLOBAL void *)((const char *)from + (uint32_t)(off * sizeof(T))),
                    (PAM_LDS void *)(lds + (n * WAVES + w) * 1024), 16, 0, 0);
        }
    } else {
        for (int e = threadIdx.x; e < ROWS * PARTS * dim; e += 64 * WAVES) {
            const int c = e % dim, part = e / dim % PARTS, row = e / dim / PARTS;
            const int ch = part * (NC / PARTS) + c;
            const int piece = (ch / per) ^ R::turn(row);
            *reinterpret_cast<T *>(lds + row * R::kBytes + piece * 16 + (ch % per) * sizeof(T)) =
                from[min(row, last) * row_stride + part * part_stride + c];
        }
    }
}

// Clears the rows whose bit is 0 in `seen` (row r: bit r).
template <class T, int NC, int ROWS, int WAVES>
__device__ __forceinline__ void clear_rows(char *lds, uint64_t seen)
{
    using R = Rows<T, NC>;
    for (int e = threadIdx.x; e < ROWS * R::kPieces; e += 64 * WAVES)
        if (!(seen >> (e / R::kPieces) & 1))
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
}

// A row as an operand, straight from memory: chunk s of channels of `row` for
// this lane, 0 past dim; `ok` false: 0 (nothing is read).
template <class T, bool WIDE>
__device__ __forceinline__ uint4v memory_chunk(const T *row, int s, int dim, bool ok)
{
    constexpr int per = 16 / sizeof(T);
    const int c = s * kChunk<T> + (lane_id() >> 5) * per;
    uint4v r = {0, 0, 0, 0};
    if constexpr (WIDE) {
        if (ok && c < dim)
            r = load16(row + c);
    } else {
        T x[per];
#pragma unroll
        for (int j = 0; j < per; ++j)
            x[j] = ok && c + j < dim ? row[c + j] : (T)0.0f;
        __builtin_memcpy(&r, x, 16);
    }
    return r;
}

// the values of a chunk piece held by a lane
template <class T>
__device__ __forceinline__ float piece_dot(uint4v a, uint4v b)
{
    float s = 0.0f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            s += __uint_as_float(a[j]) * __uint_as_float(b[j]);
    } else {
        typedef T T8 __attribute__((ext_vector_type(8)));
        const T8 x = __builtin_bit_cast(T8, a), y = __builtin_bit_cast(T8, b);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            s += (float)x[j] * (float)y[j];
    }
    return s;
}

// Four consecutive channels (registers 4 g .. 4 g + 3 of a result whose rows
// are channels) to a row of an array, each times f.
template <class T, bool WIDE>
__device__ __forceinline__ void store4(T *row, int c, int dim, const float (&x)[4])
{
    if (WIDE) {
        if (c < dim) {
            if constexpr (sizeof(T) == 4) {
                *reinterpret_cast<float4v *>(row + c) = float4v{x[0], x[1], x[2], x[3]};
            } else {
                typedef T T4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<T4 *>(row + c) = T4{(T)x[0], (T)x[1], (T)x[2], (T)x[3]};
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < dim)
                row[c + j] = (T)x[j];
    }
}

// all loads to LDS of this wave have arrived
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // vmcnt 0, others not waited for

}  // namespace pam
