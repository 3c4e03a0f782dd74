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

// BYTES bytes a lane straight to LDS, where the wave's lie side by side from `lds` on.
template <int BYTES> __device__ __forceinline__ void memory_to_lds(Memory m, uint32_t offset, uint32_t step, char *lds)
{
    auto *to = (__attribute__((address_space(3))) void *)lds;
    if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(m, to, 16, offset, step, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(m, to, 4, offset, step, 0, 0);
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

// Few rows: workgroup (x, y) has columns 16 TN x .. of the y-th tile of up to 64 rows of a group, as in k_few.  Its waves take every WAVES-th 128 numbers
// of c, a block of 32 of a line a lane, and their sums meet in LDS.
constexpr int FEW_ROWS = 64;
template <class O, int COLS> __device__ __forceinline__ bool few_rows_tile(const GmmArgs &a, RowsTile &w)
{
    int tiles = 0;
    w.n0 = (int)blockIdx.x * COLS;
    auto item_of = [&](int n) { tiles = n; return (int)blockIdx.y; };
    if (find_tile(a, FEW_ROWS, item_of, w.group, w.m0, w.hi)) return true;
    clear_outside<O>(a, w.n0, min((int64_t)COLS, a.n - w.n0), (int)blockIdx.y - tiles, (int)gridDim.y - tiles);
    return false;
}

// A block of each of TN lines of a matrix, and its scale.
template <int TN> struct Mx4Blocks {
    uint4 v[TN];
    uint32_t s[TN];
    __device__ __forceinline__ void load(const uint8_t *const (&codes)[TN], const uint8_t *const (&scales)[TN], int block)
    {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            v[j] = *reinterpret_cast<const uint4 *>(codes[j] + (int64_t)block * 16);
            s[j] = scales[j][block];
        }
    }
    // only the first `valid` numbers
    __device__ __forceinline__ void end(int valid)
    {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            v[j] = make_uint4(mx4_first(v[j].x, valid), mx4_first(v[j].y, valid - 8), mx4_first(v[j].z, valid - 16), mx4_first(v[j].w, valid - 24));
            s[j] = valid > 0 ? s[j] : 127u;
        }
    }
};

// The walk of a wave over its steps of 128 numbers, U at a time, the matrix's blocks of the next ones under way meanwhile: first(t) loads those of step t
// into `next` ahead of everything else, x(u, t) what they meet, use(u, t, end) multiplies; `end`: the step may reach behind the lines' end, and is then
// told what is there by its blocks.
template <int U, int WAVES, class Blocks, class LoadW, class LoadX, class Use>
__device__ __forceinline__ void few_walk(Blocks (&now)[U], int wave, int steps, LoadW load_w, LoadX load_x, Use use)
{
    int t = wave;
    for (; t + U * WAVES < steps; t += U * WAVES) {   // (all of these lie before the end)
        Blocks next[U];
        load_x(t, false);
#pragma unroll
        for (int u = 0; u < U; ++u) load_w(next[u], t + (U + u) * WAVES);
        use(now, t, false);
#pragma unroll
        for (int u = 0; u < U; ++u) now[u] = next[u];
    }
    if (t < steps) {
        load_x(t, true);
        use(now, t, true);
    }
}

// The waves' sums meet, 16 rows at a time; store(row, column, sum) is called once for each of the tile's.
template <int TM, int TN, int WAVES, class Store>
__device__ __forceinline__ void few_meet(const f32x4 (&acc)[TM][TN], int rows, int64_t n0, int64_t n, float *lds, Store store)
{
    constexpr int COLS = TN * 16, LD = COLS + 4, THREADS = WAVES * WAVE;
    const int lane = lane_id(), r = lane % 16, g = lane / 16, wave = threadIdx.x / WAVE;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        if (i > 0) __syncthreads();
#pragma unroll
        for (int j = 0; j < TN; ++j) *reinterpret_cast<f32x4 *>(lds + (wave * 16 + r) * LD + j * 16 + g * 4) = acc[i][j];
        __syncthreads();
        for (int k = threadIdx.x; k < 16 * COLS; k += THREADS) {
            const int row = k / COLS, col = k % COLS;
            if (i * 16 + row >= rows || n0 + col >= n) continue;
            float v = 0.0f;
#pragma unroll
            for (int s = 0; s < WAVES; ++s) v += lds[(s * 16 + row) * LD + col];
            store(i * 16 + row, n0 + col, v);
        }
    }
}
constexpr int few_lds(int tn, int waves) { return waves * 16 * (tn * 16 + 4); }   // floats
inline dim3 few_grid(const GmmArgs &a, int cols)
{
    return dim3((uint32_t)((a.n + cols - 1) / cols), (uint32_t)(a.rows / FEW_ROWS + std::min(a.groups, a.rows)) + 1);
}

// Columns of a workgroup, in sixteens.
inline int few_columns(const GmmArgs &a)
{
    const int64_t tiles = std::min(a.groups, a.rows);
    return tiles * ((a.n + 63) / 64) >= 512 ? 4 : tiles * ((a.n + 31) / 32) >= 512 ? 2 : 1;
}
inline bool few(const GmmArgs &a)
{
    const int64_t groups = std::min(a.groups, a.rows);
    return groups > 0 && a.rows <= groups * 48 && a.n <= (1 << 20) && a.rows / FEW_ROWS + groups < 65535;
}

}  // namespace

}  // namespace ocean
