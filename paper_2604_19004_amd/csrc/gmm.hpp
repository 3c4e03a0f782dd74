// Tiles of out(m, n) = sum over c of L(m, c) * R(n, c) on the matrix cores, with operands stored along c ("row": a row of memory is
// a row of the operand) or across it ("col": a row of memory is one c).
//
// LDS holds a step of 128 bytes of c of each operand.  A row tile is [rows][8 pieces of 16 bytes], a col tile [c][pieces]; the
// piece's place inside its line is XORed with bits of the line's number, so that the 16 lines that a wave reads at once lie on
// different banks.  Tiles come straight from memory to LDS where every piece is aligned (a lane names the 16 bytes it wants, its
// place in LDS is fixed by its number, so the XOR is applied to the source), otherwise through registers by unaligned loads.
//
// A 16 x 16 result tile of v_mfma_16x16 has its columns' operand first, so that a lane holds 4 columns of one row; the lines of R that
// four such tiles read are interleaved in fours, so that a lane holds 16 consecutive columns and writes 32 or 64 bytes side by side.
#pragma once

#include "routed.hpp"

namespace ocean {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int LINE = 128;                                   // bytes of c in a step
template <class T> constexpr int STEP = LINE / (int)sizeof(T);   // elements of c in a step
template <class T> constexpr int PIECE = 16 / (int)sizeof(T);    // elements of 16 bytes

__device__ const uint4 g_zero_piece = {0u, 0u, 0u, 0u};     // what stands for pieces behind the end of c

// acc += A * B for 64 bytes of c of 16 lines each: a lane has 16 bytes of line lane % 16, piece lane / 16.
__device__ __forceinline__ void mma(f32x4 &acc, bf16x8 a, bf16x8 b) { acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0); }
__device__ __forceinline__ void mma(f32x4 &acc, f16x8 a, f16x8 b) { acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, acc, 0, 0, 0); }
// (single precision: c in another order, the same one for both operands)
__device__ __forceinline__ void mma(f32x4 &acc, f32x4 a, f32x4 b)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], acc, 0, 0, 0);
}
template <class T> struct FragOf;
template <> struct FragOf<float> { using type = f32x4; };
template <> struct FragOf<bf16_t> { using type = bf16x8; };
template <> struct FragOf<f16_t> { using type = f16x8; };
template <class T> using Frag = typename FragOf<T>::type;

// Which line of an operand lane r (0 .. 15) of 16 x 16 tile j reads: in order, or four tiles interleaved in fours.
template <bool INTER> __device__ __forceinline__ int tile_line(int j, int r)
{
    return INTER ? (j / 4) * 64 + (r / 4) * 16 + (j % 4) * 4 + r % 4 : j * 16 + r;
}
// The XOR of a row tile's line: the bits in which the 16 lines that are read at once differ, but the lowest (two lines of 128
// bytes lie side by side in the 64 banks).
template <bool INTER> __device__ __forceinline__ int row_xor(int line)
{
    return INTER ? ((line >> 1) & 1) | ((line >> 4) & 3) << 1 : (line >> 1) & 7;
}
// The XOR of a col tile's line c: 16-bit types read c = 8 g + 0 .. 3 (and + 4) at once, single precision c = 4 g + j.
template <class T> __device__ __forceinline__ int col_xor(int c)
{
    return sizeof(T) == 2 ? (c & 3) | ((c >> 3) & 3) << 2 : ((c >> 2) & 3) << 2;
}

// One operand's tile of B lines (row) or B columns (col), moved by THREADS threads.
template <class T, bool COL, bool INTER, int B, int THREADS>
struct Tile {
    static constexpr int BYTES = B * LINE;
    static constexpr int LOADS = BYTES / 16 / THREADS;       // pieces a thread moves
    static constexpr int PIECES = COL ? B / PIECE<T> : 8;    // pieces in a line
    static_assert(BYTES % (16 * THREADS) == 0, "whole pieces a thread");

    __device__ static int line_of(int i) { return (i * THREADS + (int)threadIdx.x) / PIECES; }
    __device__ static int piece_of(int i)
    {
        const int q = i * THREADS + (int)threadIdx.x, line = q / PIECES;
        return (q % PIECES) ^ (COL ? col_xor<T>(line) : row_xor<INTER>(line));
    }
    // 64 bytes of c (half: 0 or 1) of 16x16 tile j, as mma takes them.
    __device__ static Frag<T> read(const char *lds, int first, int j, int half)
    {
        const int lane = lane_id(), r = lane % 16, g = lane / 16;
        if constexpr (!COL) {
            const int line = first + tile_line<INTER>(j, r);
            return *reinterpret_cast<const Frag<T> *>(lds + line * LINE + (((half * 4 + g) ^ row_xor<INTER>(line)) * 16));
        } else if constexpr (sizeof(T) == 2) {
            // each lane names 4 columns of one c; a group of 16 lanes gets its 4 x 16 block transposed
            const int col = first + tile_line<INTER>(j, (r % 4) * 4);
            s16x8 v;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = half * 32 + g * 8 + h * 4 + r / 4;
                const int at = c * (PIECES * 16) + (((col / 8) ^ col_xor<T>(c)) * 16) + (col % 8) * 2;
                const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(lds + at));
#pragma unroll
                for (int i = 0; i < 4; ++i) v[h * 4 + i] = x[i];
            }
            return __builtin_bit_cast(Frag<T>, v);
        } else {
            const int col = first + tile_line<INTER>(j, r);
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = half * 16 + g * 4 + i;
                v[i] = *reinterpret_cast<const float *>(lds + c * (PIECES * 16) + (((col / 4) ^ col_xor<T>(c)) * 16) + (col % 4) * 4);
            }
            return v;
        }
    }
};

// 16 bytes from memory straight to LDS; the wave's 1024 bytes begin at `lds` (the same number in every lane).
__device__ __forceinline__ void load_to_lds(const void *src, char *lds)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src, (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}
// Up to a piece from any address of the element type; what lies behind `valid` elements is not read and 0.
template <class T> __device__ __forceinline__ uint4 load_piece(const T *p, int valid)
{
    typedef uint32_t any_u32x4 __attribute__((ext_vector_type(4), aligned(2)));
    if (valid >= PIECE<T>) return __builtin_bit_cast(uint4, (u32x4)*reinterpret_cast<const any_u32x4 *>(p));
    Vec<T, PIECE<T>> e = {};
#pragma unroll
    for (int i = 0; i < PIECE<T>; ++i)
        if (i < valid) e.e[i] = p[i];
    return __builtin_bit_cast(uint4, e);
}

}  // namespace ocean
