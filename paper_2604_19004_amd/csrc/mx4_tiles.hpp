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
// columns of a row side by side, else 4.  settle: of which columns NaN are looked at once more, and what stands in their place (NoSettle: none).
struct NoSettle {};
template <class O, int BM, int BN, int WAVES_M, int WAVES_N, bool INTER, size_t LDS, class Settle = NoSettle>
__device__ __forceinline__ void store_tile(const GmmArgs &a, const RowsTile &w, const f32x4 (&acc)[BM / WAVES_M / 16][BN / WAVES_N / 16], char *lds, Settle settle = {})
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
    bool nan = false;   // (a result of this lane)
#pragma unroll 4
    for (int i = 0; i < WM / ROWS; ++i) {
        const int row = i * ROWS + lane / PIECES, slot = w.m0 + wm + row;
        const auto o = *reinterpret_cast<const Vec<O, E> *>(place(row, piece * E));
        if (slot >= w.hi) continue;
        if constexpr (!std::is_same<Settle, NoSettle>::value) {
#pragma unroll
            for (int k = 0; k < E; ++k) nan |= o.e[k] != o.e[k];
        }
        O *p = static_cast<O *>(a.out) + (int64_t)slot * a.ldo + col;
        if (valid == E) {
            store_any<PAST>(p, o);
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (k < valid) p[k] = o.e[k];
        }
    }
    if constexpr (!std::is_same<Settle, NoSettle>::value) {
        if (__any(nan)) {
            const uint32_t blocks = settle.template of_wave<WN>(w.n0 + wn);
#pragma unroll 1
            for (int k = 0; k < (nan ? min(valid, E) : 0); ++k) {   // (each lane goes through what it has stored itself)
                if (!settle.of_column(col + k, w.n0 + wn, blocks)) continue;
#pragma unroll 1
                for (int slot = w.m0 + wm + lane / PIECES; slot < min(w.m0 + wm + WM, w.hi); slot += ROWS) {
                    O *p = static_cast<O *>(a.out) + (int64_t)slot * a.ldo + col + k;
                    if (*p != *p) *p = (O)settle.result(slot, col + k);
                }
            }
        }
    }
}

// Few rows: workgroup (x, y) has columns 16 TN x .. of the y-th tile of up to ROWS rows of a group, as in k_few.  Its waves take every WAVES-th 128 numbers
// of c, a block of 32 of a line a lane, and their sums meet in LDS.
template <class O, int ROWS, int COLS> __device__ __forceinline__ bool few_rows_tile(const GmmArgs &a, RowsTile &w)
{
    int tiles = 0;
    w.n0 = (int)blockIdx.x * COLS;
    auto item_of = [&](int n) { tiles = n; return (int)blockIdx.y; };
    if (find_tile(a, ROWS, item_of, w.group, w.m0, w.hi)) return true;
    clear_outside<O>(a, w.n0, min((int64_t)COLS, a.n - w.n0), (int)blockIdx.y - tiles, (int)gridDim.y - tiles);
    return false;
}

// U steps of 128 numbers of N lines: a block a lane and step (of 16 lanes' the group-th), and a word with the scales of a step's four blocks.
template <int N, int U> struct Mx4Batch {
    uint4 v[U][N];
    uint32_t s[N][U];
    // steps t .. t + U - 1 (blocks behind the end: the last one)
    __device__ __forceinline__ void load(const uint8_t *const (&codes)[N], int t, int group, int blocks)
    {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < N; ++j) v[u][j] = *reinterpret_cast<const uint4 *>(codes[j] + (int64_t)min((t + u) * 4 + group, blocks - 1) * 16);
    }
    // scales[j]: where line j's words of the steps are (t a multiple of U: nothing is read behind a row's 16 bytes)
    template <class P> __device__ __forceinline__ void load_scales(const P *const (&scales)[N])
    {
        using Words = std::conditional_t<U == 4, uint4, std::conditional_t<U == 2, uint2, uint32_t>>;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const Words w = *reinterpret_cast<const Words *>(scales[j]);
            __builtin_memcpy(s[j], &w, sizeof w);
        }
    }
    // only the first `valid` numbers of step u
    __device__ __forceinline__ void end(int u, int valid)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            uint4 &w = v[u][j];
            w = make_uint4(mx4_first(w.x, valid), mx4_first(w.y, valid - 8), mx4_first(w.z, valid - 16), mx4_first(w.w, valid - 24));
            s[j][u] = valid > 0 ? s[j][u] : 0x7f7f7f7fu;
        }
    }
    __device__ __forceinline__ uint32_t scale(int u, int j, int group) const { return s[j][u] >> 8 * group & 255u; }
};

// Few rows: the workgroup's 16 TN lines of the matrix go by in passes of four steps a wave.  Codes come straight into registers, 256 bytes of a line a wave.
// Scales pass through LDS: read where they are needed, 8 bytes of a line here and 8 there, their lines of memory were fetched into the compute unit again and
// again (96 rows of 16 experts, 4096 x 4096, rows in four bits: 45 us, and with all scales 1, 28).
template <int TN, int WAVES> struct FewScales {
    static constexpr int BYTES = WAVES * 16, PITCH = BYTES + 16, PIECES = TN * 16 * WAVES;   // of a line in a pass; in LDS, where 16 lines lie on different banks
    static_assert(PIECES <= WAVES * WAVE, "a piece a thread");
    const uint8_t *from;
    int left;            // bytes from there to the line's end (of up to 16 more there is memory)
    uint4 piece;
    __device__ __forceinline__ FewScales(const uint8_t *scales, int64_t ld, int64_t n0, int64_t n, int blocks) : piece(make_uint4(0, 0, 0, 0))
    {
        const int tid = threadIdx.x, at = tid % WAVES * 16;
        from = scales + min(n0 + tid / WAVES, n - 1) * ld + at;
        left = tid < PIECES ? blocks - at : 0;
        load();
    }
    __device__ __forceinline__ void load()
    {
        if (left > 0) piece = *reinterpret_cast<const uint4 *>(from);
    }
    __device__ __forceinline__ void store(uint8_t *lds) const
    {
        const int tid = threadIdx.x;
        if (tid < PIECES) *reinterpret_cast<uint4 *>(lds + tid / WAVES * PITCH + tid % WAVES * 16) = piece;
    }
    __device__ __forceinline__ void next()
    {
        from += BYTES, left -= BYTES;
        load();
    }
};

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
inline dim3 few_grid(const GmmArgs &a, int rows, int cols)
{
    return dim3((uint32_t)((a.n + cols - 1) / cols), (uint32_t)(a.rows / rows + std::min(a.groups, a.rows)) + 1);
}
// Columns of a workgroup of few rows, and its waves: calls launch(TN, WAVES) as constants.  64 columns where that leaves two workgroups a compute unit, else 32; eight
// waves to a long line where there are fewer workgroups than that all the same, else four (rows of bfloat16, us with four and eight: one group of 8 rows, 8192 x 4096,
// 14.4 and 11.4, one row, 28000 x 8192, 34 and 29; two groups of one row, 4096 x 8192, 11.6 and 12.5, sixteen of four, 4096 x 4096, 31 and 35).
inline int64_t few_columns(const GmmArgs &a, int cols) { return std::min(a.groups, a.rows) * ((a.n + cols - 1) / cols); }
inline bool fills_chip(const GmmArgs &a) { return few_columns(a, 64) >= 512; }
template <class Launch> hipError_t with_columns_and_waves(const GmmArgs &a, Launch launch)
{
    using std::integral_constant;
    if (fills_chip(a)) return launch(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    if (a.c < 4096 || few_columns(a, 32) >= 512) return launch(integral_constant<int, 2>{}, integral_constant<int, 4>{});
    return launch(integral_constant<int, 2>{}, integral_constant<int, 8>{});
}

// Which tiles: those that take the least by what was measured at c = 4096, us for n of them: of 64 x 64 one a compute unit, or so much for all and each; of
// 128 x 128 by rounds of two a compute unit, of 256 x 256 of one, and for a last round that is half full or less.
struct TileTimes { double small, small_all, small_each, middle, middle_half, large, large_least; };
inline double small_time(const TileTimes &t, double n) { return n <= 256 ? t.small : t.small_all + t.small_each * n; }
inline double middle_time(const TileTimes &t, double n)
{
    const double whole = (double)(int64_t)(n / 512), rest = n - whole * 512;
    return whole * t.middle + (rest > 256 ? t.middle : rest > 0 ? t.middle_half : 0.0);
}
inline double large_time(const TileTimes &t, double n)
{
    const double whole = (double)(int64_t)(n / 256), rest = n - whole * 256;
    return whole * t.large + (rest > 0 ? t.large_least + (t.large - t.large_least) * rest / 256 : 0.0);
}
// The tile's lines (256 only if `large`), among those that one launch has; 0: none does.
inline int pick_lines(const GmmArgs &a, const TileTimes &t, bool large)
{
    const int64_t groups = std::min(a.groups, a.rows);
    // (a group's last tile is half full on the average)
    auto tiles = [&](int64_t b) { return (double)std::max(groups, a.rows / b + groups / 2) * (double)((a.n + b - 1) / b); };
    double best = 1e300;
    int lines = 0;
    auto offer = [&](int b, int threads, double time) {
        if (time < best && launches<GM_ROWS>(a, b, b, threads)) best = time, lines = b;
    };
    offer(64, 256, small_time(t, tiles(64)));
    offer(128, 256, middle_time(t, tiles(128)));
    if (large) offer(256, 512, large_time(t, tiles(256)));
    return lines;
}

}  // namespace

}  // namespace ocean
