// Tiles of out(m, n) = sum over c of L(m, c) * R(n, c) on the matrix cores, with operands stored along c ("row": a row of memory is
// a row of the operand) or across it ("col": a row of memory is one c).
//
// LDS holds a step of 128 bytes of c of each operand.  A row tile is [rows][8 pieces of 16 bytes], a col tile [c][pieces]; the
// piece's place inside its line is XORed with bits of the line's number, so that the 16 lines that a wave reads at once lie on
// different banks.  Tiles come straight from memory to LDS where every piece is aligned (a lane names the 16 bytes it wants, its
// place in LDS is fixed by its number, so the XOR is applied to the source), otherwise through registers by unaligned loads.
//
// A 16 x 16 result tile of v_mfma_16x16 has its columns' operand first, so that a lane holds 4 columns of one row; the lines of R that
// four such tiles read are interleaved in fours, so that a lane holds 16 consecutive columns, whole pieces of a result's line (not in a col tile:
// the transposing read would use half of each piece).
#pragma once

#include <algorithm>
#include <type_traits>

#include "routed.hpp"

namespace ocean {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int LINE = 128;                                   // bytes of c in a step of most kernels
template <class T> constexpr int STEP = LINE / (int)sizeof(T);   // elements of c in it
template <class T> constexpr int PIECE = 16 / (int)sizeof(T);    // elements of 16 bytes

__device__ const uint4 g_zero_piece = {0u, 0u, 0u, 0u};     // what stands for pieces behind the end of c

// acc += A * B for 64 bytes of c of 16 lines each: a lane has 16 bytes of line lane % 16, piece lane / 16.  In as many parts as the type
// takes matrix instructions (single precision: c in another order, the same one for both operands), so that a caller can put other
// products between two of the same sum.
template <class T> constexpr int MMA_PARTS = sizeof(T) == 4 ? 4 : 1;
__device__ __forceinline__ void mma_part(f32x4 &acc, bf16x8 a, bf16x8 b, int) { acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0); }
__device__ __forceinline__ void mma_part(f32x4 &acc, f16x8 a, f16x8 b, int) { acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, acc, 0, 0, 0); }
__device__ __forceinline__ void mma_part(f32x4 &acc, f32x4 a, f32x4 b, int p) { acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[p], b[p], acc, 0, 0, 0); }
template <class T> struct FragOf;
template <> struct FragOf<float> { using type = f32x4; };
template <> struct FragOf<bf16_t> { using type = bf16x8; };
template <> struct FragOf<f16_t> { using type = f16x8; };
template <class T> using Frag = typename FragOf<T>::type;
template <class T, int M, int N> __device__ __forceinline__ void mma(f32x4 (&acc)[M][N], const Frag<T> (&columns)[N], const Frag<T> (&rows)[M])
{
#pragma unroll
    for (int p = 0; p < MMA_PARTS<T>; ++p)
#pragma unroll
        for (int i = 0; i < M; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) mma_part(acc[i][j], columns[j], rows[i], p);
}

// Which line of an operand lane r (0 .. 15) of 16 x 16 tile j reads: in order, or four tiles interleaved in fours.
template <bool INTER> __device__ __forceinline__ int tile_line(int j, int r)
{
    return INTER ? (j / 4) * 64 + (r / 4) * 16 + (j % 4) * 4 + r % 4 : j * 16 + r;
}
// The XOR of a row tile's line of PIECES pieces (2 lines of 128 or 4 of 64 bytes lie side by side in the 64 banks).  A 16-byte read of a
// wave takes four turns, the first of lanes 0 - 3, 12 - 15 and 20 - 27, the second of 4 - 11, 16 - 19 and 28 - 31, and so on: with lane %
// 16 the line and lane / 16 the piece, the 16 of a turn fall on 16 places (no conflict is counted).
template <bool INTER, int PIECES> __device__ __forceinline__ int row_xor(int line)
{
    if (PIECES == 4) {
        const int q = (INTER ? line >> 4 : line >> 2) & 3;
        return ((q ^ q << 1) & 2) | q >> 1;
    }
    return INTER ? ((line >> 1) & 1) | ((line >> 4) & 3) << 1 : (line >> 1) & 7;
}
// The XOR of a col tile's line c of PIECES pieces: 16-bit types read two pieces each of c = 8 g + 0 .. 3 (and + 4), two g at once, single
// precision four pieces of c = 4 g + j, all g at once.  (Lines of 8 pieces lie two by two on the banks.)
template <class T, int PIECES> __device__ __forceinline__ int col_xor(int c)
{
    if (sizeof(T) == 4) return ((c >> 2) & 3) << 2;
    return PIECES == 8 ? ((c >> 1) & 1) << 1 | ((c >> 3) & 1) << 2 : (c & 3) << 1 | ((c >> 3) & 1) << 3;
}

// Transposing reads of LDS: each lane names 4 16-bit numbers at `at` + OFFSET, and a group of 16 lanes gets its block of 4 x 16 turned round; the
// same at OFFSET + NEXT into the upper half of the fragment.  Of N addresses at once, and waited for here: the compiler, which cannot
// tell the buffers of a pipeline apart, puts a wait for all loads on their way to LDS in front of the builtin (64 us instead of 35 for two
// products with 4096 x 8192 weights across c, a row each).
__device__ __forceinline__ uint32_t lds_address(const char *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p; }
template <int OFFSET, int NEXT, int N> __device__ __forceinline__ void read_transposed(const uint32_t (&at)[N], s16x8 (&out)[N])
{
    static_assert(N == 1 || N == 2 || N % 4 == 0, "one, two, fours or eights");
    s16x4 v[2 * N];
    if constexpr (N == 1) {
        asm volatile("ds_read_b64_tr_b16 %0, %2 offset:%3\n\tds_read_b64_tr_b16 %1, %2 offset:%4\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]) : "v"(at[0]), "n"(OFFSET), "n"(OFFSET + NEXT) : "memory");
    } else if constexpr (N == 2) {
        asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
                     "ds_read_b64_tr_b16 %2, %5 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%7\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]) : "v"(at[0]), "v"(at[1]), "n"(OFFSET), "n"(OFFSET + NEXT) : "memory");
    } else if constexpr (N % 8 == 0) {
#pragma unroll
        for (int k = 0; k < 2 * N; k += 16)
            asm volatile("ds_read_b64_tr_b16 %0, %16 offset:%24\n\tds_read_b64_tr_b16 %1, %16 offset:%25\n\t"
                         "ds_read_b64_tr_b16 %2, %17 offset:%24\n\tds_read_b64_tr_b16 %3, %17 offset:%25\n\t"
                         "ds_read_b64_tr_b16 %4, %18 offset:%24\n\tds_read_b64_tr_b16 %5, %18 offset:%25\n\t"
                         "ds_read_b64_tr_b16 %6, %19 offset:%24\n\tds_read_b64_tr_b16 %7, %19 offset:%25\n\t"
                         "ds_read_b64_tr_b16 %8, %20 offset:%24\n\tds_read_b64_tr_b16 %9, %20 offset:%25\n\t"
                         "ds_read_b64_tr_b16 %10, %21 offset:%24\n\tds_read_b64_tr_b16 %11, %21 offset:%25\n\t"
                         "ds_read_b64_tr_b16 %12, %22 offset:%24\n\tds_read_b64_tr_b16 %13, %22 offset:%25\n\t"
                         "ds_read_b64_tr_b16 %14, %23 offset:%24\n\tds_read_b64_tr_b16 %15, %23 offset:%25\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(v[k + 0]), "=&v"(v[k + 1]), "=&v"(v[k + 2]), "=&v"(v[k + 3]), "=&v"(v[k + 4]), "=&v"(v[k + 5]), "=&v"(v[k + 6]), "=&v"(v[k + 7]), "=&v"(v[k + 8]), "=&v"(v[k + 9]), "=&v"(v[k + 10]), "=&v"(v[k + 11]), "=&v"(v[k + 12]), "=&v"(v[k + 13]), "=&v"(v[k + 14]), "=&v"(v[k + 15])
                         : "v"(at[k / 2 + 0]), "v"(at[k / 2 + 1]), "v"(at[k / 2 + 2]), "v"(at[k / 2 + 3]), "v"(at[k / 2 + 4]), "v"(at[k / 2 + 5]), "v"(at[k / 2 + 6]), "v"(at[k / 2 + 7]), "n"(OFFSET), "n"(OFFSET + NEXT) : "memory");
    } else {
#pragma unroll
        for (int k = 0; k < 2 * N; k += 8)
            asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
                         "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
                         "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
                         "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(v[k + 0]), "=&v"(v[k + 1]), "=&v"(v[k + 2]), "=&v"(v[k + 3]), "=&v"(v[k + 4]), "=&v"(v[k + 5]), "=&v"(v[k + 6]), "=&v"(v[k + 7])
                         : "v"(at[k / 2 + 0]), "v"(at[k / 2 + 1]), "v"(at[k / 2 + 2]), "v"(at[k / 2 + 3]), "n"(OFFSET), "n"(OFFSET + NEXT) : "memory");
    }
#pragma unroll
    for (int k = 0; k < N; ++k) out[k] = __builtin_shufflevector(v[2 * k], v[2 * k + 1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// One operand's tile of B lines (row) or B columns (col), DEPTH bytes of c, moved by THREADS threads.
template <class T, bool COL, bool INTER, int B, int THREADS, int DEPTH>
struct Tile {
    static constexpr int BYTES = B * DEPTH, LINE_C = DEPTH / (int)sizeof(T);
    static constexpr int LOADS = BYTES / 16 / THREADS;       // pieces a thread moves
    static constexpr int PIECES = COL ? B / PIECE<T> : DEPTH / 16;    // pieces in a line
    static_assert(BYTES % (16 * THREADS) == 0, "whole pieces a thread");

    // The line and the piece of it that thread `tid` moves as its i-th.
    __device__ static int line_of(int tid, int i) { return (i * THREADS + tid) / PIECES; }
    __device__ static int piece_of(int tid, int i)
    {
        const int q = i * THREADS + tid, line = q / PIECES;
        return (q % PIECES) ^ (COL ? col_xor<T, PIECES>(line) : row_xor<INTER, PIECES>(line));
    }
    // Where this lane reads tile 0 of the lines from `first` on (a multiple of the lines that the wave reads), in bytes.  The bits that the XOR takes and
    // those that the tile's number j and the half add are different ones, so all other places follow from this one by constants.
    __device__ static uint32_t place(int first)
    {
        const int lane = lane_id(), r = lane % 16, g = lane / 16;
        if constexpr (!COL) {
            const int line = first + tile_line<INTER>(0, r);
            return line * DEPTH + (g ^ row_xor<INTER, PIECES>(line)) * 16;
        } else if constexpr (sizeof(T) == 2) {
            // each lane names 4 columns of one c; a group of 16 lanes gets its 4 x 16 block transposed
            const int col = first + tile_line<INTER>(0, (r % 4) * 4), c = g * 8 + r / 4;
            return c * (PIECES * 16) + ((col / 8) ^ col_xor<T, PIECES>(c)) * 16 + (col % 8) * 2;
        } else {
            const int col = first + tile_line<INTER>(0, r), c = g * 4;
            return c * (PIECES * 16) + ((col / 4) ^ col_xor<T, PIECES>(c)) * 16 + (col % 4) * 4;
        }
    }
    // 64 bytes of c (the HALF-th of DEPTH) of 16 x 16 tiles 0 .. N - 1, as mma takes them.
    template <int HALF, int N> __device__ static void read(const char *lds, uint32_t place, Frag<T> (&out)[N])
    {
        if constexpr (!COL) {
#pragma unroll
            for (int j = 0; j < N; ++j) out[j] = *reinterpret_cast<const Frag<T> *>(lds + (place ^ (HALF * 64)) + tile_line<INTER>(j, 0) * DEPTH);
        } else if constexpr (sizeof(T) == 2) {
            uint32_t at[N];
            s16x8 v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) at[j] = lds_address(lds) + (place ^ (tile_line<INTER>(j, 0) * 2));
            read_transposed<HALF * 32 * PIECES * 16, 4 * PIECES * 16>(at, v);
#pragma unroll
            for (int j = 0; j < N; ++j) out[j] = __builtin_bit_cast(Frag<T>, v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    out[j][i] = *reinterpret_cast<const float *>(lds + (place ^ (tile_line<INTER>(j, 0) * 4)) + (HALF * 16 + i) * (PIECES * 16));
        }
    }
};

// 16 bytes from memory straight to LDS; the wave's 1024 bytes begin at `lds` (the same number in every lane).
__device__ __forceinline__ void load_to_lds(const void *src, char *lds)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src, (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}
// A piece from any even address.
__device__ __forceinline__ uint4 load_any(const char *p)
{
    typedef uint32_t any_u32x4 __attribute__((ext_vector_type(4), aligned(2)));
    return __builtin_bit_cast(uint4, (u32x4)*reinterpret_cast<const any_u32x4 *>(p));
}
// Up to a piece from any address of the element type; what lies behind `valid` elements is not read and 0.
template <class T> __device__ __forceinline__ uint4 load_piece(const T *p, int valid)
{
    if (valid >= PIECE<T>) return load_any(reinterpret_cast<const char *>(p));
    Vec<T, PIECE<T>> e = {};
#pragma unroll
    for (int i = 0; i < PIECE<T>; ++i)
        if (i < valid) e.e[i] = p[i];
    return __builtin_bit_cast(uint4, e);
}

// A piece of a 16-bit type with zeros in place of infinities and NaN.  (Pieces of numbers below 2 are seen to have none by one bit of each.)
template <class T> __device__ __forceinline__ uint4 finite_piece(uint4 v)
{
    static_assert(sizeof(T) == 2, "two numbers a word");
    constexpr uint32_t EXPONENT = std::is_same<T, bf16_t>::value ? 0x7f80u : 0x7c00u;
    if ((v.x | v.y | v.z | v.w) & 0x40004000u) {
        uint32_t *w[4] = {&v.x, &v.y, &v.z, &v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if ((*w[i] & EXPONENT) == EXPONENT) *w[i] &= 0xffff0000u;
            if ((*w[i] >> 16 & EXPONENT) == EXPONENT) *w[i] &= 0xffffu;
        }
    }
    return v;
}

// A piece to any address of the element type; past the cache or not.
template <bool PAST, class T> __device__ __forceinline__ void store_any(T *p, const Vec<T, PIECE<T>> &v)
{
    typedef uint32_t any_u32x4 __attribute__((ext_vector_type(4), aligned(2)));
    if constexpr (PAST) __builtin_nontemporal_store((any_u32x4)__builtin_bit_cast(u32x4, v), reinterpret_cast<any_u32x4 *>(p));
    else *reinterpret_cast<any_u32x4 *>(p) = __builtin_bit_cast(u32x4, v);
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

__device__ __forceinline__ void group_range(const GmmArgs &a, int e, int &lo, int &hi)
{
    const int64_t l = min(max(a.ptr[e], (int64_t)0), a.rows);   // (rows are below 2^31)
    lo = (int)l;
    hi = (int)min(max(a.ptr[e + 1], l), a.rows);
}

// Which group and which of its tiles of `size` rows tile number `t` is, and how many tiles there are; false: fewer than that.
// item_of(tiles) says the number where it depends on how many there are.  Every wave for itself.
template <class F>
__device__ __forceinline__ bool find_tile(const GmmArgs &a, int size, F item_of, int &group, int &lo, int &hi)
{
    const int groups = (int)a.groups;
    auto load = [&](int e0, int &l, int &h) -> uint32_t {   // tiles of group e0 + lane
        l = h = 0;
        if (e0 + lane_id() < groups) group_range(a, e0 + lane_id(), l, h);
        return wave_inclusive_scan_u32(((uint32_t)(h - l) + (uint32_t)size - 1) / (uint32_t)size);
    };
    int l, h;
    uint32_t tiles = 0, incl = 0;
    for (int e0 = 0; e0 < groups; e0 += WAVE) {
        incl = load(e0, l, h);
        tiles += wave_read_lane_u32(incl, WAVE - 1);
    }
    const int t = item_of((int)tiles);
    if (t < 0 || (uint32_t)t >= tiles) return false;
    uint32_t before = 0;
    for (int e0 = 0; e0 < groups; e0 += WAVE) {
        if (groups > WAVE) incl = load(e0, l, h);   // (else it is at hand)
        const unsigned long long past = __ballot(before + incl > (uint32_t)t);
        if (past) {
            const int k = __ffsll(past) - 1;
            group = e0 + k;
            const uint32_t first = before + (k > 0 ? wave_read_lane_u32(incl, k - 1) : 0u);
            lo = (int)wave_read_lane_u32((uint32_t)l, k) + (int)(((uint32_t)t - first) * (uint32_t)size);
            hi = (int)wave_read_lane_u32((uint32_t)h, k);
            return true;
        }
        before += wave_read_lane_u32(incl, WAVE - 1);
    }
    return false;
}

// Clears a stretch of columns of the rows that belong to no group; the part-th of `parts` workgroups that do so.
template <class O>
__device__ __forceinline__ void clear_outside(const GmmArgs &a, int64_t col, int64_t width, int64_t part, int64_t parts)
{
    const int64_t first = min(max(a.ptr[0], (int64_t)0), a.rows), last = min(max(a.ptr[a.groups], first), a.rows);
    const int64_t count = (a.rows - (last - first)) * width;
    for (int64_t i = part * blockDim.x + threadIdx.x; i < count; i += parts * blockDim.x) {
        const int64_t row = i / width;
        static_cast<O *>(a.out)[(row < first ? row : row - first + last) * a.ldo + col + i % width] = (O)0.0f;
    }
}

// The number-th item of this workgroup's die: workgroups go to the 8 dies in turn, each die with its own L2, so each die gets a
// contiguous stretch of the items.  -1: there is none; so it is for all blocks from the next multiple of 8 on where the number is blockIdx.x / 8.
__device__ __forceinline__ int by_die(int number, int items)
{
    const int per = (items + 7) >> 3, item = (int)(blockIdx.x & 7) * per + number;
    return number < per && item < items ? item : -1;
}

// m-tiles by n-tiles in bands of `band` m-tiles, so that workgroups that run together share lines of both operands (32568 rows of 4096 by eight
// 8192 x 4096 2.24 ms in bands of 2, 2.12 in those of 4, 2.10 in those of 8, when results still left in half lines).
__device__ __forceinline__ void banded(int item, int mt, int nt, int band, int &m, int &n)
{
    const int per = band * nt, b = item / per, in = item - b * per, height = min(band, mt - b * band);
    m = b * band + in % height;
    n = in / height;
}

// Where a thread's pieces of one operand begin in memory: a base that is the same for the workgroup, and for each piece the bytes from
// there, 32 bits where pieces go straight to LDS (the address then takes no vector instruction, see offsets_fit).
template <class T, class TI, bool COL, bool ASYNC>
struct Feed {
    using Off = std::conditional_t<ASYNC, uint32_t, int64_t>;
    const T *base;
    int64_t ld, advance;       // elements from a line to the next, from a step to the next
    Off off[TI::LOADS];
    int room;                  // (col) columns from the first on

    // (row) line l is row row_of(l) behind `at`
    template <class F> __device__ __forceinline__ void lines(int tid, const T *at, int64_t ld_, F row_of)
    {
        base = at, ld = ld_, advance = TI::LINE_C, room = 0;
#pragma unroll
        for (int i = 0; i < TI::LOADS; ++i) off[i] = (Off)((row_of(TI::line_of(tid, i)) * ld + TI::piece_of(tid, i) * PIECE<T>) * (int64_t)sizeof(T));
    }
    // (col) columns col0 .. of `cols`, lines from c0 on; by_number: the line is given with each piece (row()).  Columns behind the end:
    // the last piece's where pieces are whole, what comes of them is not stored
    __device__ __forceinline__ void columns(int tid, const T *at, int64_t ld_, int64_t col0, int64_t cols, int64_t c0, bool by_number)
    {
        base = at + (by_number ? 0 : c0 * ld_) + col0, ld = ld_, advance = TI::LINE_C * ld_;
        room = (int)min(cols - col0, (int64_t)1 << 30);
#pragma unroll
        for (int i = 0; i < TI::LOADS; ++i) {
            const int col = ASYNC ? min(TI::piece_of(tid, i) * PIECE<T>, room - PIECE<T>) : TI::piece_of(tid, i) * PIECE<T>;
            off[i] = (Off)(((by_number ? 0 : TI::line_of(tid, i) * ld) + col) * (int64_t)sizeof(T));
        }
    }
    __device__ __forceinline__ const char *step(int t) const { return reinterpret_cast<const char *>(base + t * advance); }
    __device__ __forceinline__ const char *row(int i, int64_t number) const { return reinterpret_cast<const char *>(base + number * ld) + off[i]; }
    // Elements of piece i that there are where the step has `left` c (0 or less: none).
    __device__ __forceinline__ int valid(int tid, int i, int left) const
    {
        if (!COL) return min(PIECE<T>, left - TI::piece_of(tid, i) * PIECE<T>);
        return TI::line_of(tid, i) >= left ? 0 : ASYNC ? PIECE<T> : min(PIECE<T>, room - TI::piece_of(tid, i) * PIECE<T>);
    }
    // Whether all pieces of a step with `left` c are whole.
    __device__ __forceinline__ bool whole(int left) const { return left == TI::LINE_C && (!COL || room >= TI::PIECES * PIECE<T>); }
    __device__ __forceinline__ const void *numbered(int tid, int i, int left, int32_t number, uint32_t rows) const
    {
        return valid(tid, i, left) > 0 && (uint32_t)number < rows ? static_cast<const void *>(row(i, number)) : &g_zero_piece;
    }
};

// One workgroup a tile, STAGES steps of both operands in LDS.  Large tiles are bound by the matrix cores, and those by what the card may draw: 32568 rows
// of 4096 by eight 8192 x 4096 in bfloat16 take 1.9 to 2.0 ms, 1100 TFLOP/s (with zeros for numbers 1300; a library's largest product 1320), no bank conflict
// counted.  Small ones are bound by the weights' bytes: two rows by two 8192 x 4096, 27 us or 5.1 TB/s.
template <class T, bool LCOL, bool RCOL, int BM, int BN, int WAVES_M, int WAVES_N, bool ASYNC, int STAGES, GmmMode MODE, class O = T>
__global__ void __launch_bounds__(WAVES_M * WAVES_N * WAVE, 2) k_gmm(GmmArgs a, int mt, int nt)
{
    constexpr int THREADS = WAVES_M * WAVES_N * WAVE, WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 16, TN = WN / 16;
    static_assert(RCOL || WN % 64 == 0, "four interleaved tiles");
    constexpr int BYTES = LINE, STEP_C = BYTES / (int)sizeof(T), HALVES = 2;
    using TL = Tile<T, LCOL, false, BM, THREADS, BYTES>;
    using TR = Tile<T, RCOL, !RCOL, BN, THREADS, BYTES>;
    constexpr int BUFFER = TL::BYTES + TR::BYTES;
    constexpr bool DEPTH = MODE == GM_DEPTH;
    static_assert(STAGES >= 2 && (ASYNC || STAGES == 2), "through registers: one step ahead");
    __shared__ __align__(16) char lds[STAGES * BUFFER];

    // The tile of the number-th work item of this workgroup's die.
    struct Work { int group, m0, hi, n0, c_lo, c_hi, stretch; };
    int tiles = 0;   // (GM_ROWS, GM_SHRINK) those that the groups make; mt is the most they may make
    auto locate = [&](int number, Work &w) -> bool {
        int mi, ni, lo = 0;
        w = Work{0, 0, (int)a.rows, 0, 0, (int)a.c, 0};
        if constexpr (MODE == GM_EXPAND) {
            const int item = by_die(number, mt * nt);
            if (item < 0) return false;
            banded(item, mt, nt, 8, mi, ni);
            lo = mi * BM;
        } else if constexpr (DEPTH) {
            // (each die has a stretch of every group's tiles, another one of each: a group's tiles take as long as it is deep)
            const int per = (mt * nt + 7) >> 3;
            w.group = number / per;
            const int item = (((int)blockIdx.x + w.group) & 7) * per + number - w.group * per;
            if (w.group >= a.groups || item >= mt * nt) return false;
            banded(item, mt, nt, 8, mi, ni);
            group_range(a, w.group, w.c_lo, w.c_hi);
            lo = mi * BM;
            w.hi = (int)a.m;
        } else {
            auto item_of = [&](int n) -> int {
                tiles = n;
                const int stretches = MODE == GM_SHRINK ? (int)((a.c + a.c_part - 1) / a.c_part) : 1;
                int item = by_die(number, n * nt * stretches);
                if (item < 0) return -1;
                if constexpr (MODE == GM_SHRINK) {
                    w.stretch = item / (n * nt);
                    item -= w.stretch * n * nt;
                }
                banded(item, n, nt, 8, mi, ni);
                return mi;
            };
            if (!find_tile(a, BM, item_of, w.group, lo, w.hi)) return false;
            if constexpr (MODE == GM_SHRINK) {
                w.c_lo = w.stretch * (int)a.c_part;
                w.c_hi = (int)min(w.c_lo + a.c_part, a.c);
            }
        }
        w.m0 = lo;
        w.n0 = ni * BN;
        return true;
    };
    // (GM_EXPAND) the adapters of the tile's rows, which are in their order, and where their rows begin.
    __shared__ int s_adapter[MODE == GM_EXPAND ? BM : 1], s_rank[MODE == GM_EXPAND ? BM : 1], s_begin[MODE == GM_EXPAND ? BM + 1 : 1];
    __shared__ int s_wave[8], s_adapters;
    Work w;
    if (!locate(blockIdx.x >> 3, w)) {
        if constexpr (MODE == GM_ROWS) {   // (some have no tile: see grid_of)
            const int from = (tiles * nt + 7) / 8 * 8, part = (int)blockIdx.x - from;
            if (part >= 0) clear_outside<O>(a, 0, a.n, part, (int)gridDim.x - from);
        }
        return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int wm = (wave / WAVES_N) * WM, wn = (wave % WAVES_N) * WN;
    const int tid = threadIdx.x;
    // What of x's rows this workgroup reads: those of its slots, or (GM_DEPTH) one for each c.
    const bool numbered = DEPTH && a.index != nullptr;
    const uint32_t x_rows = (uint32_t)a.index_rows;   // (below 2^31, and a negative number is not)
    Feed<T, TL, LCOL, ASYNC> feed_l;
    Feed<T, TR, RCOL, ASYNC> feed_r;
    const int depth = w.c_hi - w.c_lo, steps = (depth + STEP_C - 1) / STEP_C;
    {
        const T *rbase = static_cast<const T *>(a.r) + (DEPTH ? 0 : (int64_t)w.group * a.stride);
        if constexpr (LCOL) {
            feed_l.columns(tid, static_cast<const T *>(a.l), a.ldl, w.m0, a.m, w.c_lo, numbered && !a.index_on_r);
        } else {
            const bool gather = !DEPTH && a.index;
            feed_l.lines(tid, static_cast<const T *>(a.l) + (int64_t)(gather ? 0 : w.m0) * a.ldl + w.c_lo, a.ldl, [&](int line) -> int64_t {
                const int at = min(line, w.hi - 1 - w.m0);   // (what comes of lines behind the end is not stored)
                if (!gather) return at;
                const int64_t row = a.index[w.m0 + at];
                return (uint64_t)row < (uint64_t)a.index_rows ? row : 0;   // (its result is replaced by 0)
            });
        }
        if constexpr (RCOL) feed_r.columns(tid, rbase, a.ldr, w.n0, a.n, w.c_lo, numbered && a.index_on_r);
        else feed_r.lines(tid, rbase + (int64_t)w.n0 * a.ldr + w.c_lo, a.ldr, [&](int line) -> int64_t { return min(line, (int)a.n - 1 - w.n0); });
    }

    // (GM_DEPTH with row numbers: those of the step that is fetched next, loaded before the pieces of the step before it, since loads come
    // back in order and waiting for the numbers would otherwise mean waiting for all pieces under way)
    constexpr int NUMBERS = DEPTH ? (TL::LOADS > TR::LOADS ? TL::LOADS : TR::LOADS) : 1;
    constexpr bool SQUARE = BM == BN;   // (a thread's pieces of both operands are of the same lines)
    int32_t number[NUMBERS], other[SQUARE ? 1 : NUMBERS];   // for the lines of x, and for those of the operand that is in order
    auto load_numbers = [&](int t) {
        if constexpr (DEPTH) {
            if (!numbered) return;
            auto load = [&](auto tile, int32_t *to) {
                using TI = decltype(tile);
#pragma unroll
                for (int i = 0; i < TI::LOADS; ++i) to[i] = a.index[(int64_t)w.c_lo + min(t * STEP_C + TI::line_of(tid, i), depth - 1)];
            };
            if (a.index_on_r) {
                load(TR{}, number);
                if constexpr (!SQUARE) load(TL{}, other);
            } else {
                load(TL{}, number);
                if constexpr (!SQUARE) load(TR{}, other);
            }
        }
    };
    // A line whose number is outside is zeros in x, and in the other operand too, where an infinite or NaN number would not become 0 by a product
    // with 0.  Whether the wave has pieces of such lines, in the step fetched last and, a bit up for each, in those before it: they are cleared in LDS, by
    // the numbers read again (both gradients of 32 groups, 2048 x 1400, without such lines 478 us, unlooked-at 475, and with a choice at each load 508).
    uint32_t holes = 0;
    auto note_holes = [&] {
        if constexpr (DEPTH) {
            if (!numbered) return;
            bool outside = false;
#pragma unroll
            for (int i = 0; i < NUMBERS; ++i)
                if (SQUARE || i < (a.index_on_r ? TL::LOADS : TR::LOADS)) outside |= (uint32_t)(SQUARE ? number[i] : other[i]) >= x_rows;
            holes = holes << 1 | (__any(outside) ? 1u : 0u);
        }
    };
    // Step t's, which was fetched `ago` steps before the last one.
    auto fill_holes = [&](int t, int ago, char *buffer) {
        if constexpr (DEPTH) {
            if (!(holes >> ago & 1u)) return;
            auto fill = [&](auto tile, char *to) {
                using TI = decltype(tile);
#pragma unroll
                for (int i = 0; i < TI::LOADS; ++i)
                    if ((uint32_t)a.index[(int64_t)w.c_lo + min(t * STEP_C + TI::line_of(tid, i), depth - 1)] >= x_rows)
                        *reinterpret_cast<uint4 *>(to + (i * THREADS + tid) * 16) = make_uint4(0, 0, 0, 0);
            };
            if (a.index_on_r) fill(TL{}, buffer);
            else fill(TR{}, buffer + TL::BYTES);
            __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
        }
    };

    uint4 kept_l[ASYNC ? 1 : TL::LOADS], kept_r[ASYNC ? 1 : TR::LOADS];
    // Workgroups begin at different steps and go round: at the same one, the lines that they read all begin in the same few memory channels
    // where lines are a multiple of some KB long (32 products with 2048 x 2048 weights, 64 rows each: 53 us, from one step on 94).
    const int turn = DEPTH || steps == 0 ? 0 : (w.n0 / BN + w.group * 5) % steps;
    auto fetch = [&](int t, int buffer) {
        t += turn;
        if (t >= steps) t -= steps;
        char *to = lds + buffer * BUFFER;
        const int left = min(STEP_C, depth - t * STEP_C);   // c of this step
        if constexpr (ASYNC) {
            int32_t now[NUMBERS];
#pragma unroll
            for (int i = 0; i < NUMBERS; ++i) now[i] = number[i];
            note_holes();
            if constexpr (DEPTH) load_numbers(t + 1);
            asm volatile("" ::: "memory");
            char *to_wave = to + wave * (WAVE * 16);
            auto move = [&](auto &feed, auto tile, char *dst, bool by_number) {
                using TI = decltype(tile);
                if (DEPTH && by_number) {
#pragma unroll
                    for (int i = 0; i < TI::LOADS; ++i) load_to_lds(feed.numbered(tid, i, left, now[i], x_rows), dst + i * THREADS * 16);
                } else if (left == STEP_C) {
                    const char *base = feed.step(t);
#pragma unroll
                    for (int i = 0; i < TI::LOADS; ++i) load_to_lds(base + feed.off[i], dst + i * THREADS * 16);
                } else {
#pragma unroll
                    for (int i = 0; i < TI::LOADS; ++i)
                        load_to_lds(feed.valid(tid, i, left) > 0 ? static_cast<const void *>(feed.step(t) + feed.off[i]) : &g_zero_piece, dst + i * THREADS * 16);
                }
            };
            move(feed_l, TL{}, to_wave, numbered && !a.index_on_r);
            move(feed_r, TR{}, to_wave + TL::BYTES, numbered && a.index_on_r);
        } else {
            auto move = [&](auto &feed, auto tile, uint4 *dst, bool by_number) {
                using TI = decltype(tile);
                if (!(DEPTH && by_number) && feed.whole(left)) {   // (the same for all: no lane looks at its pieces' ends)
                    const char *base = feed.step(t);
#pragma unroll
                    for (int i = 0; i < TI::LOADS; ++i) dst[i] = load_any(base + feed.off[i]);
                    return;
                }
#pragma unroll
                for (int i = 0; i < TI::LOADS; ++i) {
                    int valid = feed.valid(tid, i, left);
                    const char *from = feed.step(t) + feed.off[i];
                    if (DEPTH && by_number) {
                        from = feed.row(i, number[i]);
                        if ((uint32_t)number[i] >= x_rows) valid = 0;
                    }
                    dst[i] = load_piece(reinterpret_cast<const T *>(from), valid);
                }
            };
            move(feed_l, TL{}, kept_l, numbered && !a.index_on_r);
            move(feed_r, TR{}, kept_r, numbered && a.index_on_r);
            note_holes();
            if constexpr (DEPTH) load_numbers(t + 1);
        }
    };
    auto stash = [&](int t) {
        if constexpr (!ASYNC) {
            char *to = lds + (t & 1) * BUFFER;
#pragma unroll
            for (int i = 0; i < TL::LOADS; ++i) *reinterpret_cast<uint4 *>(to + (i * THREADS + tid) * 16) = kept_l[i];
#pragma unroll
            for (int i = 0; i < TR::LOADS; ++i) *reinterpret_cast<uint4 *>(to + TL::BYTES + (i * THREADS + tid) * 16) = kept_r[i];
            if constexpr (DEPTH) fill_holes(t, 0, to);
        }
    };

    const int lane = lane_id(), r = lane % 16, g = lane / 16;
    const uint32_t at_l = TL::place(wm), at_r = TR::place(wn);
    // Results pass through LDS, a region for each wave, and a row's go out side by side, whole lines of memory at a time (65536 rows of 256 by eight 4096 x
    // 256 218 us and, w across c, 231; straight from the lanes that hold them, 16 or 8 bytes here and the rest of the line later, 370 and 550).
    auto store = [&](const f32x4 (&acc)[TM][TN]) {
        constexpr int RUN = RCOL ? 1 : 4;         // tiles whose columns a lane has side by side
        constexpr int E = PIECE<O>, ROW = WN * (int)sizeof(O), PIECES = ROW / 16, ROWS = WAVE / PIECES;
        // (256 of the largest tiles are as much as the dies' caches hold: past them, so that the operands' lines stay; 32768 rows, 32 groups, 2048 x 1400,
        // both gradients 461 us, else 500)
        constexpr bool PAST = BM * BN >= 256 * 256;
        static_assert(BM * BN * sizeof(O) <= sizeof(lds) && PIECES >= 8, "room for the results");
        char *mine = lds + wave * (WM * ROW);
        auto place = [&](int row, int col) { return mine + row * ROW + ((col / E ^ (row & 7)) * 16 + col % E * (int)sizeof(O)); };
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int row = i * 16 + r;
            const bool zero = MODE == GM_ROWS && a.index && (uint64_t)(int64_t)a.index[min(w.m0 + wm + row, w.hi - 1)] >= (uint64_t)a.index_rows;
#pragma unroll
            for (int b = 0; b < TN / RUN; ++b) {
                constexpr int OP = RUN * 4 < E ? RUN * 4 : E;
                const int col = b * RUN * 16 + g * RUN * 4;
#pragma unroll
                for (int k0 = 0; k0 < RUN * 4; k0 += OP) {
                    Vec<O, OP> o;
#pragma unroll
                    for (int k = 0; k < OP; ++k) o.e[k] = (O)(zero ? 0.0f : acc[i][b * RUN + (k0 + k) / 4][(k0 + k) % 4]);
                    *reinterpret_cast<Vec<O, OP> *>(place(row, col + k0)) = o;
                }
            }
        }
        wave_sync();
        O *out = static_cast<O *>(a.out) + (DEPTH ? (int64_t)w.group * a.stride : (int64_t)w.stretch * a.rows * a.ldo);
        const int piece = lane % PIECES, col = w.n0 + wn + piece * E, valid = (int)min(a.n - col, (int64_t)E);
#pragma unroll 4
        for (int i = 0; i < WM / ROWS; ++i) {
            const int row = i * ROWS + lane / PIECES, slot = w.m0 + wm + row;
            const auto o = *reinterpret_cast<const Vec<O, E> *>(place(row, piece * E));
            if (slot >= w.hi) continue;
            int64_t at = slot;
            if constexpr (MODE == GM_EXPAND) at = a.index[slot];
            O *p = out + at * a.ldo + col;
            if (valid == E) {
                store_any<PAST>(p, o);
            } else {
#pragma unroll
                for (int k = 0; k < E; ++k)
                    if (k < valid) p[k] = o.e[k];
            }
        }
    };

    if (steps > 0) load_numbers(0);
    if constexpr (MODE == GM_EXPAND) {
        const int slot = w.m0 + tid;
        const bool has = tid < BM && slot < w.hi && (uint32_t)a.slot_id[min(slot, w.hi - 1)] < (uint32_t)a.adapters;
        const int id = has ? a.slot_id[slot] : -1;
        const bool starts = has && (tid == 0 || a.slot_id[slot - 1] != id);
        const unsigned long long b = __ballot(starts), hb = __ballot(has);
        if (lane == 0) s_wave[wave] = __popcll(b) | __popcll(hb) << 16;
        __syncthreads();
        int before = 0, total = 0;
        for (int i = 0; i < WAVES_M * WAVES_N; ++i) {
            if (i < wave) before += s_wave[i];
            total += s_wave[i];
        }
        const int at = (before & 0xffff) + __popcll(b & ((1ull << lane) - 1));
        if (starts) {
            s_adapter[at] = id;
            s_begin[at] = slot;
            s_rank[at] = a.ranks ? a.ranks[id] : 0;
        }
        if (tid == 0) {
            s_adapters = total & 0xffff;
            s_begin[total & 0xffff] = w.m0 + (total >> 16);
        }
        __syncthreads();
    }
    f32x4 acc[TM][TN] = {};
    // Single precision: the sums of eight steps (256 c) are put aside, so that the roundings of a long sum grow with the root of a 256th of its terms (c =
    // 4096: a quarter of those of one running sum).  Results of 16 bits are rounded far above them.
    constexpr bool ASIDE = sizeof(T) == 4;
    f32x4 sums[ASIDE ? TM : 1][ASIDE ? TN : 1] = {};
    auto put_aside = [&] {
        if constexpr (ASIDE) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    sums[i][j] += acc[i][j];
                    acc[i][j] = f32x4{};
                }
        }
    };
    auto multiply = [&](int buffer) {
        const char *from = lds + buffer * BUFFER;
        auto part = [&](auto half) {
            Frag<T> fr[TN], fl[TM];
            TR::template read<decltype(half)::value>(from + TL::BYTES, at_r, fr);
            TL::template read<decltype(half)::value>(from, at_l, fl);
            mma<T>(acc, fr, fl);
        };
        part(std::integral_constant<int, 0>{});
        part(std::integral_constant<int, 1>{});
    };
    if constexpr (ASYNC) {
#pragma unroll
        for (int t = 0; t < STAGES - 1; ++t)
            if (t < steps) fetch(t, t);
        int buffer = 0;
        for (int t = 0; t < steps; ++t) {
            // This wave's part of the step is in LDS (loads come back in order: all but those of later steps), and what it read of the
            // step before has come; then everyone's is, and nobody reads the buffer of the step before any more.
            constexpr int LATER = (STAGES - 2) * (TL::LOADS + TR::LOADS);
            static_assert(LATER < 64, "what the counter holds");
            asm volatile("" ::: "memory");
            if (t + STAGES - 2 < steps) __builtin_amdgcn_s_waitcnt(0x0070 | (LATER & 15) | (LATER >> 4) << 14);
            else __builtin_amdgcn_s_waitcnt(0x0070);
            if constexpr (DEPTH) fill_holes(t, min(STAGES - 2, steps - 1 - t), lds + buffer * BUFFER);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (t + STAGES - 1 < steps) fetch(t + STAGES - 1, buffer == 0 ? STAGES - 1 : buffer - 1);   // (in place of the step before)
            multiply(buffer);
            if (ASIDE && t % 8 == 7) put_aside();
            buffer = buffer + 1 == STAGES ? 0 : buffer + 1;
        }
    } else {
        // Through registers, one step ahead (two were no faster).
        if (steps > 0) {
            fetch(0, 0);
            stash(0);
        }
        for (int t = 0; t < steps; ++t) {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): what this wave wrote is in LDS, what it read has come
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (t + 1 < steps) fetch(t + 1, 0);
            multiply(t & 1);
            if (ASIDE && t % 8 == 7) put_aside();
            if (t + 1 < steps) stash(t + 1);
        }
    }
    if constexpr (ASIDE) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] += sums[i][j];
    }

    if constexpr (MODE == GM_EXPAND) {
        // The adapters of the tile's rows: 64 bytes of h and b at a time (a unit), as many units a step as the tile has halves, h's parts side
        // by side and b's line again for each; with h's second part without its infinities and NaN, whose products are those with the first (the
        // second may be 0 or of the other sign).  A row takes only its own adapter's products (not 0 times the others', which may be infinite or NaN).
        constexpr int PARTS = sizeof(T) == 2 ? 2 : 1, UNIT = 64 / (int)sizeof(T);
        constexpr bool AHEAD = BM * BN <= 128 * 128;   // the next step's loads are under way meanwhile (larger tiles leave no registers)
        const int wide_h = PARTS * a.rank_up, each = (wide_h + UNIT - 1) / UNIT, units = s_adapters * each;
        const T *h = static_cast<const T *>(a.h);
        const int end = min(w.m0 + BM, w.hi);
        uint4 xl[TL::LOADS], xr[TR::LOADS];
        uint32_t seconds = 0;   // which of xr's pieces meet h's second part
        struct Unit { const T *b; int p, rank, last; };   // where its columns of h begin, those of b that there are; `last` of h's behind p
        auto unit = [&](int u) -> Unit {
            const int j = __builtin_amdgcn_readfirstlane(u / each), e = __builtin_amdgcn_readfirstlane(s_adapter[min(j, BM - 1)]);
            const int rank = a.ranks ? min(max(__builtin_amdgcn_readfirstlane(s_rank[min(j, BM - 1)]), 0), a.rank) : a.rank, p = (u - j * each) * UNIT;
            return u < units ? Unit{static_cast<const T *>(a.b) + e * a.stride_b, p, rank, wide_h - p} : Unit{static_cast<const T *>(a.b), 0, 0, 0};
        };
        auto load = [&](int u0) {
            const Unit u[2] = {unit(u0), unit(u0 + 1)};
            seconds = 0;
#pragma unroll
            for (int i = 0; i < TL::LOADS; ++i) {
                const int q = TL::piece_of(tid, i), in = q % 4 * PIECE<T>;
                const bool second = q >= 4;
                xl[i] = load_piece(h + (int64_t)min(w.m0 + TL::line_of(tid, i), end - 1) * wide_h + (second ? u[1].p : u[0].p) + in,
                                   in < (second ? u[1].last : u[0].last) ? PIECE<T> : 0);
            }
#pragma unroll
            for (int i = 0; i < TR::LOADS; ++i) {
                const int q = TR::piece_of(tid, i), in = q % 4 * PIECE<T>;
                const bool second = q >= 4;
                const int p = (second ? u[1].p : u[0].p) + in, at = p >= a.rank_up ? p - a.rank_up : p;
                xr[i] = load_piece((second ? u[1].b : u[0].b) + min(w.n0 + TR::line_of(tid, i), (int)a.n - 1) * a.ldb + at,
                                   in < (second ? u[1].last : u[0].last) ? (second ? u[1].rank : u[0].rank) - at : 0);
                if (PARTS == 2) seconds |= (uint32_t)(p >= a.rank_up) << i;
            }
        };
        if (AHEAD && units > 0) load(0);
        for (int u0 = 0; u0 < units; u0 += HALVES) {
            if (!AHEAD) load(u0);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < TL::LOADS; ++i) *reinterpret_cast<uint4 *>(lds + (i * THREADS + tid) * 16) = xl[i];
#pragma unroll
            for (int i = 0; i < TR::LOADS; ++i) {
                if constexpr (PARTS == 2)   // (here, where all loads have come: 6000 rows, 4096 columns, rank 64 247.7 us, 250.5 with a wait for each, 247.2 without)
                    if (seconds >> i & 1) xr[i] = finite_piece<T>(xr[i]);
                *reinterpret_cast<uint4 *>(lds + TL::BYTES + (i * THREADS + tid) * 16) = xr[i];
            }
            if (AHEAD && u0 + HALVES < units) load(u0 + HALVES);
            __syncthreads();
            auto part = [&](auto half_) {
                constexpr int half = decltype(half_)::value;
                if (u0 + half >= units) return;
                const int from = s_begin[(u0 + half) / each], to = s_begin[(u0 + half) / each + 1];
                Frag<T> fr[TN], fl[TM];
                TR::template read<half>(lds + TL::BYTES, at_r, fr);
                TL::template read<half>(lds, at_l, fl);
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const int row = w.m0 + wm + i * 16 + r;
                    const bool mine = row >= from && row < to;
                    if (!__any(mine)) continue;
                    const float back = mine ? a.row_scale[row] : 0.0f;
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        f32x4 sum = {};
#pragma unroll
                        for (int p = 0; p < MMA_PARTS<T>; ++p) mma_part(sum, fr[j], fl[i], p);
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[i][j][k] = mine ? acc[i][j][k] + back * sum[k] : acc[i][j][k];
                    }
                }
            };
            part(std::integral_constant<int, 0>{});
            part(std::integral_constant<int, 1>{});
        }
    }

    store(acc);
}

inline int64_t up8(int64_t n) { return (n + 7) & ~(int64_t)7; }

// Tiles of bm x bn, down and across, and the workgroups that they take.  (Ragged groups: a group's last tile may hold a single row, and the
// others of `rows` are whole.)
struct Grid { int64_t mt, nt, blocks; };
template <GmmMode MODE> Grid grid_of(const GmmArgs &a, int64_t bm, int64_t bn)
{
    Grid g;
    g.nt = (a.n + bn - 1) / bn;
    g.mt = MODE == GM_DEPTH ? (a.m + bm - 1) / bm : MODE == GM_EXPAND ? (a.rows + bm - 1) / bm : a.rows / bm + std::min(a.groups, a.rows);
    // (GM_ROWS: the last 8 at least have no tile and clear the rows of no group)
    g.blocks = (MODE == GM_ROWS ? 8 : 0) + (MODE == GM_DEPTH ? up8(g.mt * g.nt) * a.groups : up8(g.mt * g.nt * (MODE == GM_SHRINK ? (a.c + a.c_part - 1) / a.c_part : 1)));
    return g;
}
// Whether one launch has them: it has fewer than 2^32 threads.
template <GmmMode MODE> bool launches(const GmmArgs &a, int64_t bm, int64_t bn, int threads) { return grid_of<MODE>(a, bm, bn).blocks * threads < (1ll << 32); }
// Whether any tile does that launch_tiles may take.  (Where a smaller one does, one of these does.)
template <class T, GmmMode MODE> bool some_tile_launches(const GmmArgs &a, bool aligned)
{
    return launches<MODE>(a, 128, 128, 256) || (sizeof(T) == 2 && aligned && launches<MODE>(a, 256, 256, 512));
}

template <class T, bool LCOL, bool RCOL, int BM, int BN, int WAVES_M, int WAVES_N, bool ASYNC, int STAGES, GmmMode MODE, class O = T>
hipError_t launch_gmm(const GmmArgs &a, hipStream_t s)
{
    const Grid g = grid_of<MODE>(a, BM, BN);
    constexpr int threads = WAVES_M * WAVES_N * WAVE;
    if (g.blocks * threads >= (1ll << 32)) return TOO_MANY_TILES;
    hipLaunchKernelGGL((k_gmm<T, LCOL, RCOL, BM, BN, WAVES_M, WAVES_N, ASYNC, STAGES, MODE, O>), dim3((uint32_t)g.blocks), dim3(threads), 0, s, a, (int)g.mt, (int)g.nt);
    return hipGetLastError();
}

// Which tile: the one whose rounds over the chip's 256 compute units take the least.  A round is one tile of 256 x 256 or 128 x 256 a unit, or two
// of the others; what a round takes, or half of one (a tile a unit), in units of half a round of the largest: measured at c = 4096 in bfloat16 as
// 117 us for 256 tiles of 256 x 256, 68 of 128 x 256, 66 for 512 of 128 x 128 and 52 for 256, 40 and 32 of 64 x 128, 29 and 26 of 64 x 64.
inline double rounds(double tiles, double half, double full)
{
    const double whole = (double)(int64_t)(tiles / 512), rest = tiles - whole * 512;
    return whole * full + (rest > 256 ? full : rest > 0 ? half : 0.0);
}
// (a last round of few tiles is shorter, the others' power goes to them: 1152 tiles 228 us, a round of 256 57)
inline double large_rounds(double tiles)
{
    const double whole = (double)(int64_t)(tiles / 256), rest = tiles - whole * 256;
    return whole * 2.0 + (rest > 0 ? 1.5 + rest / 512 : 0.0);
}
// m_tiles(lines): about how many tiles of that many lines there are.
template <class T, bool LCOL, bool RCOL, GmmMode MODE, class F> hipError_t launch_tiles(const GmmArgs &a, F m_tiles, bool aligned, hipStream_t s)
{
    auto tiles = [&](int64_t bm, int64_t bn) { return (double)m_tiles(bm) * (double)((a.n + bn - 1) / bn); };
    // (adapters: 128 x 256 instead of 128 x 128, since each of a tile's columns goes through the adapters of its rows: 6000 rows of 4096, 4096 columns, rank
    // 64, 245 us and 271)
    constexpr bool WIDE = MODE == GM_EXPAND && sizeof(T) == 2;
    // (gradients of weights in a single round wait for the deepest group: 8 uneven groups, 32768 rows, 2048 x 1024, in 256 tiles of 256 x 256 264
    // us, in 1024 of 128 x 128 170; with even ones some 130 and 165)
    const double alone = MODE == GM_DEPTH && a.groups > 1 && tiles(256, 256) <= 256 ? 1.6 : 1.0;
    // (more tiles than a launch has: never)
    auto unless = [&](int64_t bm, int64_t bn, int threads, double time) { return launches<MODE>(a, bm, bn, threads) ? time : 1e300; };
    const double large = unless(256, 256, 512, large_rounds(tiles(256, 256)) * alone),
                 middle = WIDE ? unless(128, 256, 512, (double)(int64_t)((tiles(128, 256) + 255) / 256) * 1.16) : unless(128, 128, 256, rounds(tiles(128, 128), 0.89, 1.13)),
                 low = unless(64, 128, 256, rounds(tiles(64, 128), 0.55, 0.69)), small = unless(64, 64, 256, rounds(tiles(64, 64), 0.44, 0.50));
    if (!aligned) {   // (through registers: 8356 rows of 4517 by four 832 x 4517, 462 tiles of 128 x 128, 121 us and 169 in those of 64 x 64)
        if (tiles(128, 128) >= 256 || small == 1e300) return launch_gmm<T, LCOL, RCOL, 128, 128, 2, 2, false, 2, MODE>(a, s);
        return launch_gmm<T, LCOL, RCOL, 64, 64, 4, 1, false, 2, MODE>(a, s);
    }
    if constexpr (sizeof(T) == 2) {
        // (gradients of weights: waves of 64 x 128 are 3 % faster there than of 128 x 64)
        constexpr int DOWN = MODE == GM_DEPTH ? 4 : 2;
        if (large <= std::min(std::min(middle, low), small)) return launch_gmm<T, LCOL, RCOL, 256, 256, DOWN, 8 / DOWN, true, 2, MODE>(a, s);
    }
    if (middle <= std::min(low, small)) {
        if constexpr (WIDE) return launch_gmm<T, LCOL, RCOL, 128, 256, 2, 4, true, 3, MODE>(a, s);
        else return launch_gmm<T, LCOL, RCOL, 128, 128, 2, 2, true, 2, MODE>(a, s);
    }
    if (low <= small) return launch_gmm<T, LCOL, RCOL, 64, 128, 2, 2, true, 3, MODE>(a, s);
    return launch_gmm<T, LCOL, RCOL, 64, 64, 4, 1, true, 4, MODE>(a, s);
}

// Whether the places of an operand's pieces fit the 32-bit offsets of Feed: `lines` lines of `ld` elements from its base.
bool offsets_fit(int64_t lines, int64_t ld, int size) { return lines * ld * size < (1ll << 32) - 65536; }

bool pieces_aligned(const void *p, int64_t ld, int64_t stride, int size)
{
    const int e = 16 / size;
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % e == 0 && stride % e == 0;
}

}  // namespace

}  // namespace ocean
