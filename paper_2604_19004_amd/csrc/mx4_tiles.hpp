// What the products with matrices in four bits share: the matrices' places, the rows of a tile, and how results leave.
#pragma once

#include "few.hpp"
#include "mx4.hpp"

namespace ocean {

namespace {

// The matrices: outer products' columns are their rows (or, across, their numbers).
struct Mx4Args {
    const uint8_t *codes, *scales;
    int64_t ld_codes, stride_codes, ld_scales, stride_scales;   // bytes
    int blocks;                                                 // of a row
};
inline Mx4Args mx4_args(const ocean_mx4 &w) { return Mx4Args{w.codes, w.scales, w.ld_codes, w.stride_codes, w.ld_scales, w.stride_scales, (int)mx4_blocks(w.inner)}; }

// `there ? a : b` of addresses by masks, in which the compiler cannot see a branch.  (It made one of the plain choice where a workgroup's first step is the end of
// the lines, and there used a piece's offset, in lanes whose piece exists, from a register that it had only written in the others.)
__device__ __forceinline__ const void *either(bool there, const void *a, const void *b)
{
    uint32_t mask = there ? ~0u : 0u;
    asm volatile("" : "+v"(mask));
    const uint64_t m = (uint64_t)mask << 32 | mask, x = reinterpret_cast<uint64_t>(a), y = reinterpret_cast<uint64_t>(b);
    return reinterpret_cast<const void *>(y ^ ((x ^ y) & m));
}

// Which tile a workgroup has, of those that groups of rows make (mt: the most there may be); false: none, and it has cleared its share of the
// rows of no group.
struct RowsTile { int group, m0, hi, n0; };
template <class O> __device__ __forceinline__ bool rows_tile(const GmmArgs &a, int bm, int bn, int nt, RowsTile &w)
{
    int tiles = 0, mi, ni = 0;
    auto item_of = [&](int n) -> int {
        tiles = n;
        const int item = by_die((int)(blockIdx.x >> 3), n * nt);
        if (item < 0) return -1;
        banded(item, n, nt, 8, mi, ni);
        return mi;
    };
    if (!find_tile(a, bm, item_of, w.group, w.m0, w.hi)) {
        const int from = (tiles * nt + 7) / 8 * 8, part = (int)blockIdx.x - from;
        if (part >= 0) clear_outside<O>(a, 0, a.n, part, (int)gridDim.x - from);
        return false;
    }
    w.n0 = ni * bn;
    return true;
}

// The row of x behind line `line` of a tile; lines behind the group's end and numbers outside x stand for some row of x (what comes of them is not
// stored, or replaced by 0).
__device__ __forceinline__ int64_t tile_row(const GmmArgs &a, const RowsTile &w, int line)
{
    const int slot = w.m0 + min(line, w.hi - 1 - w.m0);
    if (!a.index) return slot;
    const int64_t row = a.index[slot];
    return (uint64_t)row < (uint64_t)a.index_rows ? row : 0;
}

// Results pass through LDS, a region for each wave, and leave in whole lines of memory (the largest tiles' past the cache).  INTER: a lane has 16
// columns of a row side by side, else 4.
template <class O, int BM, int BN, int WAVES_M, int WAVES_N, bool INTER, size_t LDS>
__device__ __forceinline__ void store_tile(const GmmArgs &a, const RowsTile &w, const f32x4 (&acc)[BM / WAVES_M / 16][BN / WAVES_N / 16], char *lds)
{
    constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 16, TN = WN / 16, RUN = INTER ? 4 : 1;
    constexpr int E = PIECE<O>, ROW = WN * (int)sizeof(O), PIECES = ROW / 16, ROWS = WAVE / PIECES;
    constexpr bool PAST = BM * BN >= 256 * 256;
    static_assert(BM * BN * sizeof(O) <= LDS && PIECES >= 8, "room for the results");
    const int lane = lane_id(), r = lane % 16, g = lane / 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int wm = (wave / WAVES_N) * WM, wn = (wave % WAVES_N) * WN;
    char *mine = lds + wave * (WM * ROW);
    auto place = [&](int row, int col) { return mine + row * ROW + ((col / E ^ (row & 7)) * 16 + col % E * (int)sizeof(O)); };
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int row = i * 16 + r;
        const bool zero = a.index && (uint64_t)(int64_t)a.index[min(w.m0 + wm + row, w.hi - 1)] >= (uint64_t)a.index_rows;
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
    const int piece = lane % PIECES, col = w.n0 + wn + piece * E, valid = (int)min(a.n - col, (int64_t)E);
#pragma unroll 4
    for (int i = 0; i < WM / ROWS; ++i) {
        const int row = i * ROWS + lane / PIECES, slot = w.m0 + wm + row;
        const auto o = *reinterpret_cast<const Vec<O, E> *>(place(row, piece * E));
        if (slot >= w.hi) continue;
        O *p = static_cast<O *>(a.out) + (int64_t)slot * a.ldo + col;
        if (valid == E) {
            store_any<PAST>(p, o);
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (k < valid) p[k] = o.e[k];
        }
    }
}

// The tile of few rows that workgroup (x, y) of k_few... has, as in k_few; the rows' numbers in s_row (-1: zeros).
template <class O, int COLS> __device__ __forceinline__ bool few_rows_tile(const GmmArgs &a, RowsTile &w, int &rows, int64_t *s_row)
{
    constexpr int FEW_ROWS = 64;
    int tiles = 0;
    w.n0 = (int)blockIdx.x * COLS;
    auto item_of = [&](int n) { tiles = n; return (int)blockIdx.y; };
    if (!find_tile(a, FEW_ROWS, item_of, w.group, w.m0, w.hi)) {
        clear_outside<O>(a, w.n0, min((int64_t)COLS, a.n - w.n0), (int)blockIdx.y - tiles, (int)gridDim.y - tiles);
        return false;
    }
    rows = min(FEW_ROWS, w.hi - w.m0);
    if ((int)threadIdx.x < rows) {
        const int64_t row = a.index ? a.index[w.m0 + threadIdx.x] : w.m0 + threadIdx.x;
        s_row[threadIdx.x] = (uint64_t)row < (uint64_t)a.index_rows ? row : -1;
    }
    __syncthreads();
    return true;
}
inline dim3 few_grid(const GmmArgs &a, int cols)
{
    return dim3((uint32_t)((a.n + cols - 1) / cols), (uint32_t)(a.rows / 64 + std::min(a.groups, a.rows)) + 1);
}

}  // namespace

}  // namespace ocean
