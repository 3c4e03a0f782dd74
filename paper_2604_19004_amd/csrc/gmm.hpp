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

#include <algorithm>

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

namespace {

struct GmmArgs {
    const void *l, *r;
    void *out;
    int64_t ldl, ldr, ldo;
    int64_t stride;            // elements from a group's matrix (R, or with ragged c the output) to the next's
    const int64_t *ptr;        // groups + 1 offsets into `rows`
    int64_t groups, rows;      // rows: slots; the ragged dimension
    int64_t m, n, c;           // sizes of the dimensions that are not ragged
    int64_t c_part;            // (GM_SHRINK) a multiple of the step
    const int32_t *index;      // row of x of each slot, or null
    int64_t index_rows;
    int index_on_r;            // (GM_DEPTH) x is the right operand
    // adapters: rows in the order of their adapters
    const int32_t *slot_id;    // adapter of each slot, -1: none
    const int64_t *adapter_ptr;
    int64_t adapters;
    const void *h;             // [rows][parts * rank up to whole pieces]: x * A^T with the scale over row_scale, in the operands' type
    const float *row_scale;
    const void *b;
    int64_t ldb, stride_b;
    const int32_t *ranks;
    int rank, rank_up;
};

// What is ragged, and what becomes of a tile.
enum GmmMode {
    GM_ROWS,     // groups of rows, each with its own R
    GM_DEPTH,    // groups along c, each with its own output
    GM_SHRINK,   // as GM_ROWS, c cut into stretches of `c_part`: the sums of each, [stretch][rows][ldo], in 32 bits
    GM_EXPAND    // one R for all rows; after c, the products of h with the rows' adapters' b; rows are stored where they came from
};

__device__ __forceinline__ void group_range(const GmmArgs &a, int64_t e, int64_t &lo, int64_t &hi)
{
    lo = min(max(a.ptr[e], (int64_t)0), a.rows);
    hi = min(max(a.ptr[e + 1], lo), a.rows);
}

// Which group and which of its tiles of `size` rows tile number `t` is; false: there are fewer.  Every wave for itself.  `used` receives the
// tiles there are where it is false.
__device__ __forceinline__ bool find_tile(const GmmArgs &a, int64_t t, int size, int64_t &group, int64_t &lo, int64_t &hi, int64_t &used)
{
    uint32_t before = 0;
    for (int64_t e0 = 0; e0 < a.groups; e0 += WAVE) {
        const int64_t e = e0 + lane_id();
        int64_t l = 0, h = 0;
        if (e < a.groups) group_range(a, e, l, h);
        const uint32_t tiles = (uint32_t)((h - l + size - 1) / size), incl = wave_inclusive_scan_u32(tiles);
        const unsigned long long past = __ballot(before + incl > t);
        if (past) {
            const int k = __ffsll(past) - 1;
            group = e0 + k;
            const uint32_t first = wave_read_lane_u32(before + incl - tiles, k);
            lo = wave_first(__shfl(l, k, WAVE)) + (int64_t)((uint32_t)t - first) * size;
            hi = wave_first(__shfl(h, k, WAVE));
            return true;
        }
        before += wave_read_lane_u32(incl, WAVE - 1);
    }
    used = before;
    return false;
}

// Work item of a workgroup: workgroups go to the 8 dies in turn, each die with its own L2, so each die gets a contiguous stretch.
__device__ __forceinline__ int64_t by_die(int64_t block, int64_t blocks) { return (block & 7) * (blocks >> 3) + (block >> 3); }

// m-tiles by n-tiles in bands of `band` m-tiles, so that workgroups that run together share lines of both operands.
__device__ __forceinline__ void banded(int64_t item, int64_t mt, int64_t nt, int band, int64_t &m, int64_t &n)
{
    const int64_t per = band * nt, b = item / per, in = item - b * per, height = min((int64_t)band, mt - b * band);
    m = b * band + in % height;
    n = in / height;
}

template <class T, bool LCOL, bool RCOL, int BM, int BN, int WAVES_M, int WAVES_N, bool ASYNC, GmmMode MODE, class O = T>
__global__ void __launch_bounds__(WAVES_M * WAVES_N * WAVE, 2) k_gmm(GmmArgs a, int64_t mt, int64_t nt)
{
    constexpr int THREADS = WAVES_M * WAVES_N * WAVE, WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 16, TN = WN / 16;
    static_assert(WN % 64 == 0, "four interleaved tiles");
    using TL = Tile<T, LCOL, false, BM, THREADS>;
    using TR = Tile<T, RCOL, true, BN, THREADS>;
    constexpr int BUFFER = TL::BYTES + TR::BYTES;
    constexpr bool DEPTH = MODE == GM_DEPTH;
    __shared__ __align__(16) char lds[2 * BUFFER];

    int64_t mi, ni, group = 0, lo = 0, hi = 0, c_lo = 0, c_hi = a.c;
    int64_t item = by_die(blockIdx.x, gridDim.x), stretch = 0;
    if constexpr (MODE == GM_EXPAND) {
        if (item >= mt * nt) return;
        banded(item, mt, nt, 4, mi, ni);
        lo = mi * BM;
        hi = a.rows;
    } else if constexpr (DEPTH) {
        group = item / (mt * nt);
        if (group >= a.groups) return;
        banded(item - group * mt * nt, mt, nt, 4, mi, ni);
        group_range(a, group, c_lo, c_hi);
        lo = mi * BM;
        hi = a.m;
    } else {
        if constexpr (MODE == GM_SHRINK) {
            stretch = item / (mt * nt);
            item -= stretch * mt * nt;
            c_lo = stretch * a.c_part;
            if (c_lo >= a.c) return;
            c_hi = min(c_lo + a.c_part, a.c);
        }
        if (item >= mt * nt) return;
        banded(item, mt, nt, 4, mi, ni);
        int64_t used;
        if (!find_tile(a, mi, BM, group, lo, hi, used)) {   // no rows left: clear those of no group
            if constexpr (MODE == GM_SHRINK) return;
            const int64_t first = min(max(a.ptr[0], (int64_t)0), a.rows), last = min(max(a.ptr[a.groups], first), a.rows);
            const int64_t outside = a.rows - (last - first), width = min((int64_t)BN, a.n - ni * BN);
            for (int64_t i = (mi - used) * BM; i < outside; i += (mt - used) * BM) {
                const int64_t count = min((int64_t)BM, outside - i) * width;
                for (int64_t k = threadIdx.x; k < count; k += THREADS) {
                    const int64_t row = i + k / width;
                    static_cast<O *>(a.out)[(row < first ? row : row - first + last) * a.ldo + ni * BN + k % width] = (O)0.0f;
                }
            }
            return;
        }
    }
    const int64_t n0 = ni * BN, m0 = lo;
    const T *lbase = static_cast<const T *>(a.l), *rbase = static_cast<const T *>(a.r) + (DEPTH ? 0 : group * a.stride);
    O *out = static_cast<O *>(a.out) + (DEPTH ? group * a.stride : stretch * a.rows * a.ldo);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int wm = (wave / WAVES_N) * WM, wn = (wave % WAVES_N) * WN;
    const int64_t depth = c_hi - c_lo, steps = (depth + STEP<T> - 1) / STEP<T>;

    // Where each piece of this thread begins in memory, at step 0.  Lines behind the end are those of the last line: what
    // comes of them is not stored.  With ragged c the line of memory is found step by step.
    const T *lp[TL::LOADS], *rp[TR::LOADS];
#pragma unroll
    for (int i = 0; i < TL::LOADS; ++i) {
        const int line = TL::line_of(i), piece = TL::piece_of(i);
        if constexpr (!LCOL) {
            int64_t row = min(m0 + line, hi - 1);
            if (!DEPTH && a.index) {
                row = a.index[row];
                if ((uint64_t)row >= (uint64_t)a.index_rows) row = 0;   // (its result is replaced by 0)
            }
            lp[i] = lbase + row * a.ldl + c_lo + piece * PIECE<T>;
        } else {
            const int64_t col = min(m0 + piece * PIECE<T>, ASYNC ? a.m - PIECE<T> : a.m);
            lp[i] = lbase + (c_lo + line) * a.ldl + col;
        }
    }
#pragma unroll
    for (int i = 0; i < TR::LOADS; ++i) {
        const int line = TR::line_of(i), piece = TR::piece_of(i);
        if constexpr (!RCOL) {
            rp[i] = rbase + min(n0 + line, a.n - 1) * a.ldr + c_lo + piece * PIECE<T>;
        } else {
            const int64_t col = min(n0 + piece * PIECE<T>, ASYNC ? a.n - PIECE<T> : a.n);
            rp[i] = rbase + (c_lo + line) * a.ldr + col;
        }
    }

    // The pointer of piece i of step t, and how many of its elements there are (0 or less: none, the pointer may not be read).
    auto piece_l = [&](int i, int64_t t, int &valid) -> const T * {
        const int line = TL::line_of(i), piece = TL::piece_of(i);
        if constexpr (!LCOL) {
            valid = (int)min((int64_t)PIECE<T>, depth - t * STEP<T> - piece * PIECE<T>);
            return lp[i] + t * STEP<T>;
        } else {
            const int64_t c = t * STEP<T> + line;
            valid = c < depth ? (int)min((int64_t)PIECE<T>, a.m - (m0 + piece * PIECE<T>)) : 0;
            if (ASYNC && c < depth) valid = PIECE<T>;
            if (DEPTH && a.index && !a.index_on_r && c < depth) {
                const int64_t row = a.index[c_lo + c];
                if ((uint64_t)row >= (uint64_t)a.index_rows) { valid = 0; return lp[i]; }
                return lp[i] + (row - c_lo - line) * a.ldl;
            }
            return lp[i] + t * STEP<T> * a.ldl;
        }
    };
    auto piece_r = [&](int i, int64_t t, int &valid) -> const T * {
        const int line = TR::line_of(i), piece = TR::piece_of(i);
        if constexpr (!RCOL) {
            valid = (int)min((int64_t)PIECE<T>, depth - t * STEP<T> - piece * PIECE<T>);
            return rp[i] + t * STEP<T>;
        } else {
            const int64_t c = t * STEP<T> + line;
            valid = c < depth ? (int)min((int64_t)PIECE<T>, a.n - (n0 + piece * PIECE<T>)) : 0;
            if (ASYNC && c < depth) valid = PIECE<T>;
            if (DEPTH && a.index && a.index_on_r && c < depth) {
                const int64_t row = a.index[c_lo + c];
                if ((uint64_t)row >= (uint64_t)a.index_rows) { valid = 0; return rp[i]; }
                return rp[i] + (row - c_lo - line) * a.ldr;
            }
            return rp[i] + t * STEP<T> * a.ldr;
        }
    };

    uint4 kept_l[ASYNC ? 1 : TL::LOADS], kept_r[ASYNC ? 1 : TR::LOADS];
    auto fetch = [&](int64_t t, int buffer) {
        char *to = lds + buffer * BUFFER;
#pragma unroll
        for (int i = 0; i < TL::LOADS; ++i) {
            int valid;
            const T *p = piece_l(i, t, valid);
            if constexpr (ASYNC) load_to_lds(valid > 0 ? static_cast<const void *>(p) : &g_zero_piece, to + (i * THREADS + wave * WAVE) * 16);
            else kept_l[i] = load_piece(p, valid);
        }
#pragma unroll
        for (int i = 0; i < TR::LOADS; ++i) {
            int valid;
            const T *p = piece_r(i, t, valid);
            if constexpr (ASYNC) load_to_lds(valid > 0 ? static_cast<const void *>(p) : &g_zero_piece, to + TL::BYTES + (i * THREADS + wave * WAVE) * 16);
            else kept_r[i] = load_piece(p, valid);
        }
    };
    auto stash = [&](int buffer) {
        if constexpr (!ASYNC) {
            char *to = lds + buffer * BUFFER;
#pragma unroll
            for (int i = 0; i < TL::LOADS; ++i) *reinterpret_cast<uint4 *>(to + (i * THREADS + threadIdx.x) * 16) = kept_l[i];
#pragma unroll
            for (int i = 0; i < TR::LOADS; ++i) *reinterpret_cast<uint4 *>(to + TL::BYTES + (i * THREADS + threadIdx.x) * 16) = kept_r[i];
        }
    };

    f32x4 acc[TM][TN] = {};
    if (steps > 0) {
        fetch(0, 0);
        stash(0);
    }
    for (int64_t t = 0; t < steps; ++t) {
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): this wave's part of the step is in LDS
        __syncthreads();                      // everyone's is, and nobody reads the other buffer any more
        const int buffer = (int)(t & 1);
        if (t + 1 < steps) fetch(t + 1, buffer ^ 1);
        const char *from = lds + buffer * BUFFER;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            Frag<T> fr[TN], fl[TM];
#pragma unroll
            for (int j = 0; j < TN; ++j) fr[j] = TR::read(from + TL::BYTES, wn, j, half);
#pragma unroll
            for (int i = 0; i < TM; ++i) fl[i] = TL::read(from, wm, i, half);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) mma(acc[i][j], fr[j], fl[i]);
        }
        if (t + 1 < steps) stash(buffer ^ 1);
    }

    const int lane = lane_id(), r = lane % 16, g = lane / 16;
    if constexpr (MODE == GM_EXPAND) {
        // The adapters of the tile's rows, one after the other: 128 bytes of h and b a step, h's parts side by side and b's line again
        // for each.  A row takes only its own adapter's products (not 0 times the others', which may be infinite or NaN).
        const int64_t end = min(m0 + BM, hi);
        constexpr int PARTS = sizeof(T) == 2 ? 2 : 1;
        const int wide_h = PARTS * a.rank_up;
        for (int64_t s = m0; s < end;) {
            const int64_t e = wave_first(a.slot_id[s]);
            if (e < 0 || e >= a.adapters) break;   // (rows without an adapter come last)
            const int64_t e_end = wave_first(a.adapter_ptr[e + 1]);
            const int rank = a.ranks ? min(max(a.ranks[e], 0), a.rank) : a.rank;
            const T *b = static_cast<const T *>(a.b) + e * a.stride_b, *h = static_cast<const T *>(a.h);
            for (int p0 = 0; p0 < wide_h && rank > 0; p0 += STEP<T>) {
                uint4 xl[TL::LOADS], xr[TR::LOADS];
#pragma unroll
                for (int i = 0; i < TL::LOADS; ++i) {
                    const int p = p0 + TL::piece_of(i) * PIECE<T>;
                    const int64_t line = min(m0 + TL::line_of(i), end - 1);
                    xl[i] = load_piece(h + line * wide_h + p, p < wide_h ? PIECE<T> : 0);
                }
#pragma unroll
                for (int i = 0; i < TR::LOADS; ++i) {
                    const int p = p0 + TR::piece_of(i) * PIECE<T>, q = p % a.rank_up;
                    const int64_t line = min(n0 + TR::line_of(i), a.n - 1);
                    xr[i] = load_piece(b + line * a.ldb + q, p < wide_h ? rank - q : 0);
                }
                __syncthreads();
#pragma unroll
                for (int i = 0; i < TL::LOADS; ++i) *reinterpret_cast<uint4 *>(lds + (i * THREADS + threadIdx.x) * 16) = xl[i];
#pragma unroll
                for (int i = 0; i < TR::LOADS; ++i) *reinterpret_cast<uint4 *>(lds + TL::BYTES + (i * THREADS + threadIdx.x) * 16) = xr[i];
                __syncthreads();
                Frag<T> fr[2][TN];
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int j = 0; j < TN; ++j) fr[half][j] = TR::read(lds + TL::BYTES, wn, j, half);
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const int64_t row = m0 + wm + i * 16 + r;
                    const bool mine = row >= s && row < e_end;
                    if (!__any(mine)) continue;
                    f32x4 sum[TN] = {};
                    const float back = mine ? a.row_scale[row] : 0.0f;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const Frag<T> fl = TL::read(lds, wm, i, half);
#pragma unroll
                        for (int j = 0; j < TN; ++j) mma(sum[j], fr[half][j], fl);
                    }
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[i][j][k] = mine ? acc[i][j][k] + back * sum[j][k] : acc[i][j][k];
                }
            }
            s = e_end > s ? e_end : s + 1;
        }
    }

    constexpr int OP = PIECE<O>;
    const bool wide = a.ldo % OP == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t row = m0 + wm + i * 16 + r;
        if (row >= hi) continue;
        bool zero = false;
        int64_t at = row;
        if (!DEPTH && a.index) {
            const int64_t x_row = a.index[row];
            zero = (uint64_t)x_row >= (uint64_t)a.index_rows;
            if (MODE == GM_EXPAND) {
                if (zero) continue;
                at = x_row;
            }
        }
#pragma unroll
        for (int b = 0; b < TN / 4; ++b) {
            const int64_t col = n0 + wn + b * 64 + g * 16;
            O v[16];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) v[j * 4 + k] = (O)(zero ? 0.0f : acc[i][b * 4 + j][k]);
            O *p = out + at * a.ldo + col;
#pragma unroll
            for (int j = 0; j < 16; j += OP) {
                if (wide && col + j + OP <= a.n) {
                    Vec<O, OP> o;
#pragma unroll
                    for (int k = 0; k < OP; ++k) o.e[k] = v[j + k];
                    *reinterpret_cast<Vec<O, OP> *>(p + j) = o;
                } else {
#pragma unroll
                    for (int k = 0; k < OP; ++k)
                        if (col + j + k < a.n) p[j + k] = v[j + k];
                }
            }
        }
    }
}

inline int64_t up8(int64_t n) { return (n + 7) & ~(int64_t)7; }

template <class T, bool LCOL, bool RCOL, int BM, int BN, int WAVES_M, int WAVES_N, bool ASYNC, GmmMode MODE, class O = T>
hipError_t launch_gmm(const GmmArgs &a, hipStream_t s)
{
    const int64_t nt = (a.n + BN - 1) / BN;
    const int64_t mt = MODE == GM_DEPTH ? (a.m + BM - 1) / BM : MODE == GM_EXPAND ? (a.rows + BM - 1) / BM : a.rows / BM + std::min(a.groups, a.rows) + 1;
    const int64_t blocks = up8(mt * nt * (MODE == GM_DEPTH ? a.groups : MODE == GM_SHRINK ? (a.c + a.c_part - 1) / a.c_part : 1));
    constexpr int threads = WAVES_M * WAVES_N * WAVE;
    if (blocks * threads >= (1ll << 32)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((k_gmm<T, LCOL, RCOL, BM, BN, WAVES_M, WAVES_N, ASYNC, MODE, O>), dim3((uint32_t)blocks), dim3(threads), 0, s, a, mt, nt);
    return hipGetLastError();
}

bool pieces_aligned(const void *p, int64_t ld, int64_t stride, int size)
{
    const int e = 16 / size;
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % e == 0 && stride % e == 0;
}

}  // namespace

}  // namespace ocean
