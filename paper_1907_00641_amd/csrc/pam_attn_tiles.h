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

__device__ __forceinline__ int lane_id() { return threadIdx.x & 63; }
// address of LDS memory
__device__ __forceinline__ uint32_t lds_address(const char *p) { return (uint32_t)(uintptr_t)(const PAM_LDS char *)p; }
template <class X>
__device__ __forceinline__ PAM_LDS X *lds_at(uint32_t address)
{
    return (PAM_LDS X *)(uintptr_t)address;
}
// the wave's number within its block, in a scalar register
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
__device__ __forceinline__ int result_row(int r) { return 8 * (r >> 2) + 4 * (lane_id() >> 5) + (r & 3); }

// x, of which the compiler cannot tell that it is the same in every turn of a
// loop: what is derived from it is computed again there instead of being kept in
// registers, or spilled, across the loop.
__device__ __forceinline__ int again(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

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

// The same in two operands, the rounded value and what the rounding left, rounded: together
// off by u^2, which is no more than the 32-bit sums are.
template <class T>
__device__ __forceinline__ void operands(const f32x16 &p, int s, uint4v &high, uint4v &low)
{
    static_assert(sizeof(T) == 2, "fp32 is exact");
    typedef T T8 __attribute__((ext_vector_type(8)));
    T8 h, l;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        h[j] = (T)p[8 * s + j];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        l[j] = (T)(p[8 * s + j] - (float)h[j]);
    high = __builtin_bit_cast(uint4v, h);
    low = __builtin_bit_cast(uint4v, l);
}

// Rows of NC channels in LDS.  The loads that write LDS directly fill 1024
// bytes in order, so rows cannot be padded: the 16-byte pieces of a row are
// permuted by an exclusive or with a number that depends on the row.  LDS serves
// 256 bytes of different banks at a time.  The numbers are such that
//   - sixteen lanes that read one piece each of sixteen rows (row_chunk),
//   - 32 that read four pieces of four rows (the transposing read), and
//   - fp32: 64 that read eight pieces of two rows four apart (col_chunk)
// meet every bank once: 4.1, 2.3 and 1 cycles (measured: 8.1 and 4.1 with four
// numbers and 128 bytes left free after every fourth row of 256).
template <class T, int NC>
struct Rows {
    static constexpr int kBytes = NC * sizeof(T);  // per row
    static constexpr int kPieces = kBytes / 16;
    static_assert(kPieces >= (sizeof(T) == 4 ? 16 : 8), "rows of 128 bytes (fp32: 256) at least");
    static constexpr int size(int rows) { return rows * kBytes; }
    __device__ __forceinline__ static int turn(int row)
    {
        if constexpr (sizeof(T) == 4)
            return ((row & 4) << 1) | ((row & 3) << 1) | ((row >> 3) & 1);
        else if constexpr (kPieces == 8)
            return ((row & 2) << 1) | ((row >> 2) & 3);
        else
            return ((row & 3) << 2) | ((row >> 2) & 3);
    }
    __device__ __forceinline__ static int at(int row) { return row * kBytes; }
    __device__ __forceinline__ static int at(int row, int piece) { return at(row) + ((piece ^ turn(row)) << 4); }
    // A lane's place in a tile, to be added to the tile's address once, and the
    // chunks that follow from the sum (tiles start at multiples of 256 bytes):
    // chunk s of channels of row (row0 + lane % 32)
    __device__ __forceinline__ static uint32_t row_lane() { return at(lane_id() & 31, lane_id() >> 5); }
    __device__ __forceinline__ static uint4v row_chunk(uint32_t tile_lane, int row0, int s)
    {
        return *lds_at<uint4v>((tile_lane ^ ((2 * s & 15) << 4)) + at(row0) + ((2 * s >> 4) << 8));
    }
    // chunk s of the rows from row0 on, column c0 + lane % 32 (c0 a multiple of 32)
    __device__ __forceinline__ static uint32_t col_lane()
    {
        const int l = lane_id(), h = l >> 5;
        if constexpr (sizeof(T) == 4)
            return at(4 * h, (l & 31) >> 2) + ((l & 3) << 2);
        else  // the transposing read: of sixteen lanes, lane 4 r + c gives the address of four columns of row r,
              // and lane i gets column i of the four rows
            return at(4 * h + ((l & 15) >> 2), 2 * ((l >> 4) & 1) + ((l & 3) >> 1)) + ((l & 1) << 3);
    }
    __device__ __forceinline__ static uint4v col_chunk(uint32_t tile_lane, int row0, int s, int c0)
    {
        if constexpr (sizeof(T) == 4) {
            uint4v r;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                r[j] = *lds_at<uint32_t>((tile_lane ^ (j << 5) ^ ((s & 1) << 4) ^ ((c0 & 32) << 2)) + j * kBytes +
                                         at(row0 + 8 * s) + ((c0 >> 6) << 8));
            return r;
        } else {
            const uint32_t p = tile_lane ^ ((c0 & 96) << 1), far = at(row0 + 16 * s) + ((c0 >> 7) << 8);
            const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<short4v>(p + far));
            const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<short4v>((p ^ 32) + far + at(8)));
            const uint2v x = __builtin_bit_cast(uint2v, a), y = __builtin_bit_cast(uint2v, b);
            return uint4v{x[0], x[1], y[0], y[1]};
        }
    }
};

// A pointer that is the same in every lane, in scalar registers.
template <class P>
__device__ __forceinline__ P *uniform_ptr(P *p)
{
    const uint64_t x = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (P *)((uint64_t)hi << 32 | lo);
}

// 16 (4) bytes per lane from `base` + off straight to LDS, at `to` + 16 (4) times the
// lane.  Written as assembly without outputs: the compiler, which sees that such a
// load writes LDS but not where, waits for all of them before it reads any other
// part of LDS, and the tile ahead would be waited for in the middle of the one at
// hand.  wait_loads and a barrier stand between a tile's loads and its reads.
__device__ __forceinline__ void load_lds16(const void *base, uint32_t off, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(off), "s"(base)
                 : "memory");
}
__device__ __forceinline__ void load_lds4(const void *base, uint32_t off, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(off), "s"(base)
                 : "memory");
}

// Brings, by WAVES waves (1: each wave for itself), ROWS rows of PARTS parts (maps) of up to NC / PARTS channels from
// memory to LDS.  Rows past `last` repeat row `last` (they are cleared, or
// their products thrown away, by the caller); channels past `dim` of a part are
// not written: the caller has cleared the buffer once.
//   WIDE: 16 bytes per lane straight to LDS, nothing waits here.  All rows and
//   parts start at multiples of 16 bytes, dim is whole pieces, no stride is
//   negative, and a tile's offsets in bytes fit 32 bits.
//   else: element by element through registers.
//   Blocks whose waves work in teams of WAVES give the wave's number in its team.
template <class T, int NC, int PARTS, int ROWS, int WAVES, bool WIDE>
__device__ __forceinline__ void load_rows(char *lds, const T *from, int64_t row_stride, int64_t part_stride, int last,
                                          int dim, int wave)
{
    using R = Rows<T, NC>;
    constexpr int per = 16 / sizeof(T), kPart = R::kPieces / PARTS;
    if constexpr (WIDE) {
        constexpr int kLoads = ROWS * R::kBytes / 1024, kStep = WAVES * 64 / R::kPieces;  // rows between a wave's loads
        static_assert(kLoads % WAVES == 0, "whole loads per wave");
        const int w = WAVES == 1 ? 0 : wave;
        const uint32_t at = w * 64 + again(lane_id());
        const int row0 = at / R::kPieces;
#pragma unroll
        for (int n = 0; n < kLoads / WAVES; ++n) {
            const int row = row0 + n * kStep;
            const uint32_t piece = (at % R::kPieces) ^ R::turn(kStep % 16 == 0 ? row0 : row);
            const int part = piece / kPart, ch = (piece % kPart) * per;
            const uint32_t off = (uint32_t)(min(row, last) * (int)row_stride + part * (int)part_stride + ch);
            if (ch < dim)
                load_lds16(from, (uint32_t)(off * sizeof(T)),
                           lds_address(lds) + R::at((n * WAVES + w) * 64 / R::kPieces));
        }
    } else {
        for (int e = again((WAVES == 1 ? 0 : wave * 64) + lane_id()); e < ROWS * PARTS * dim; e += 64 * WAVES) {
            const int c = e % dim, part = e / dim % PARTS, row = e / dim / PARTS;
            const int ch = part * (NC / PARTS) + c;
            *reinterpret_cast<T *>(lds + R::at(row, ch / per) + (ch % per) * sizeof(T)) =
                from[min(row, last) * row_stride + part * part_stride + c];
        }
    }
}

template <class T, int NC, int PARTS, int ROWS, int WAVES, bool WIDE>
__device__ __forceinline__ void load_rows(char *lds, const T *from, int64_t row_stride, int64_t part_stride, int last,
                                          int dim)
{
    load_rows<T, NC, PARTS, ROWS, WAVES, WIDE>(lds, from, row_stride, part_stride, last, dim, wave_id());
}

// Clears the rows whose bit is 0 in `seen` (row r: bit r).
template <class T, int NC, int ROWS, int WAVES>
__device__ __forceinline__ void clear_rows(char *lds, uint64_t seen, int wave)
{
    using R = Rows<T, NC>;
    for (int e = again((WAVES == 1 ? 0 : wave * 64) + lane_id()); e < ROWS * R::kPieces; e += 64 * WAVES)
        if (!(seen >> (e / R::kPieces) & 1))
            store16(lds + e * 16, uint4v{0, 0, 0, 0});
}
template <class T, int NC, int ROWS, int WAVES>
__device__ __forceinline__ void clear_rows(char *lds, uint64_t seen)
{
    clear_rows<T, NC, ROWS, WAVES>(lds, seen, wave_id());
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

// Sum of the products of what memory_chunk gives of a row, its chunk s, with the
// same channels of a row of 32-bit values.
template <class T, bool WIDE>
__device__ __forceinline__ float piece_dot(uint4v a, const float *row, int s, int dim, bool ok)
{
    constexpr int per = 16 / sizeof(T);
    typedef T Tp __attribute__((ext_vector_type(per)));
    const int c = s * kChunk<T> + (lane_id() >> 5) * per;
    const Tp x = __builtin_bit_cast(Tp, a);
    float y[per] = {}, sum = 0.0f;
    if constexpr (WIDE) {
        if (ok && c < dim) {
#pragma unroll
            for (int j = 0; j < per; j += 4) {
                const float4v z = *reinterpret_cast<const float4v *>(row + c + j);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[j + i] = z[i];
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < per; ++j)
            y[j] = ok && c + j < dim ? row[c + j] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < per; ++j)
        sum += (float)x[j] * y[j];
    return sum;
}

// Four consecutive channels (registers 4 g .. 4 g + 3 of a result whose rows
// are channels) to a row of an array.
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
