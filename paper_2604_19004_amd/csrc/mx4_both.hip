// Products of ragged groups of rows with their group's matrix, both in four bits, on the scaled matrix instructions: 16 x 16 results from 128 numbers
// of c, each lane with one block of a line and its scale.
#include "mx4_tiles.hpp"

namespace ocean {

// (codes as bytes: a tile's step of 128 bytes is 256 numbers of c, a fragment of 16 bytes one block)
template <> struct FragOf<uint8_t> { using type = u32x4; };

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int STEP_BLOCKS = LINE / 16, HALF_BLOCKS = STEP_BLOCKS / 2;   // blocks of a line in a step, in a matrix instruction

__device__ __forceinline__ void mma_mx4(f32x4 &acc, u32x4 a, uint32_t scale_a, u32x4 b, uint32_t scale_b)
{
    const i32x8 wa = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, wb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, acc, 4, 4, 0, (int)scale_a, 0, (int)scale_b);   // (4: e2m1; the scales' lowest bytes)
}

__device__ __forceinline__ u32x4 first_codes(u32x4 v, int valid)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = mx4_first(v[j], valid - j * 8);
    return v;
}

// 4 bytes from memory straight to LDS; the wave's 256 bytes begin at `lds`.
__device__ __forceinline__ void load_word_to_lds(const void *src, char *lds)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src, (__attribute__((address_space(3))) void *)lds, 4, 0, 0);
}

template <class O, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES>
__global__ void __launch_bounds__(WAVES_M * WAVES_N * WAVE, 2) k_gmm_mx4_mx4(GmmArgs a, Mx4Args x, Mx4Args m, int nt)
{
    constexpr int THREADS = WAVES_M * WAVES_N * WAVE, WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 16, TN = WN / 16;
    using TL = Tile<uint8_t, false, false, BM, THREADS, LINE>;
    using TR = Tile<uint8_t, false, true, BN, THREADS, LINE>;
    constexpr int LINES = BM + BN, WORDS = 2 * LINES, SCALE_LOADS = WORDS / THREADS, CODES = TL::BYTES + TR::BYTES, BUFFER = CODES + WORDS * 4;
    static_assert(WORDS % THREADS == 0, "whole words of scales a thread");
    __shared__ __align__(16) char lds[STAGES * BUFFER];
    RowsTile w;
    if (!rows_tile<O>(a, BM, BN, nt, w)) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), lane = lane_id(), r = lane % 16, g = lane / 16;
    const int wm = (wave / WAVES_N) * WM, wn = (wave % WAVES_N) * WN;
    const int depth = m.blocks * 16, steps = (m.blocks + STEP_BLOCKS - 1) / STEP_BLOCKS;   // bytes of a line
    const uint8_t *w_codes = m.codes + w.group * m.stride_codes, *w_scales = m.scales + w.group * m.stride_scales;

    Feed<uint8_t, TL, false, true> feed_l;
    Feed<uint8_t, TR, false, true> feed_r;
    const int64_t base = a.index ? 0 : w.m0;
    feed_l.lines(tid, x.codes + base * x.ld_codes, x.ld_codes, [&](int line) { return tile_row(a, w, line) - base; });
    feed_r.lines(tid, w_codes + (int64_t)w.n0 * m.ld_codes, m.ld_codes, [&](int line) -> int64_t { return min(line, (int)a.n - 1 - w.n0); });
    // Scales lie in LDS as [half of the step][line of x, then of the matrix], a word of four blocks each.
    const uint8_t *scale[SCALE_LOADS];
#pragma unroll
    for (int i = 0; i < SCALE_LOADS; ++i) {
        const int q = i * THREADS + tid, half = q / LINES, line = q % LINES;
        scale[i] = (line < BM ? x.scales + tile_row(a, w, line) * x.ld_scales : w_scales + min(w.n0 + line - BM, (int)a.n - 1) * m.ld_scales) + half * 4;
    }
    // (the order of the steps is that of k_gmm_mx4)
    const int whole = m.blocks / STEP_BLOCKS, turn = whole == 0 ? 0 : (w.n0 / BN + w.group * 5) % whole;
    auto at = [&](int t) { return t == whole ? t : t + turn >= whole ? t + turn - whole : t + turn; };
    auto fetch = [&](int t_, int buffer) {
        const int t = at(t_), left = min(LINE, depth - t * LINE);
        char *to = lds + buffer * BUFFER, *to_wave = to + wave * (WAVE * 16);
        auto move = [&](auto &feed, auto tile, char *dst) {
            using TI = decltype(tile);
            const char *from = feed.step(t);
#pragma unroll
            for (int i = 0; i < TI::LOADS; ++i) {
                if (left == LINE) load_to_lds(from + feed.off[i], dst + i * THREADS * 16);
                else load_to_lds(either(feed.valid(tid, i, left) > 0, from + feed.off[i], &g_zero_piece), dst + i * THREADS * 16);
            }
        };
        move(feed_l, TL{}, to_wave);
        move(feed_r, TR{}, to_wave + TL::BYTES);
#pragma unroll
        for (int i = 0; i < SCALE_LOADS; ++i) {
            const int half = (i * THREADS + tid) / LINES;
            const bool there = t * STEP_BLOCKS + half * HALF_BLOCKS < m.blocks;
            load_word_to_lds(either(there, scale[i] + t * STEP_BLOCKS, &g_zero_piece), to + CODES + (i * THREADS + wave * WAVE) * 4);
        }
    };

    const uint32_t at_l = TL::place(wm), at_r = TR::place(wn);
    f32x4 acc[TM][TN] = {};
    auto multiply = [&](int t_, int buffer) {
        const char *from = lds + buffer * BUFFER;
        const uint32_t *scales = reinterpret_cast<const uint32_t *>(from + CODES);
        const int t = at(t_);
        auto half = [&](auto h_) {
            constexpr int h = decltype(h_)::value;
            u32x4 fr[TN], fl[TM];
            uint32_t sr[TN], sl[TM];
            TR::template read<h>(from + TL::BYTES, at_r, fr);
            TL::template read<h>(from, at_l, fl);
#pragma unroll
            for (int j = 0; j < TN; ++j) sr[j] = scales[h * LINES + BM + wn + tile_line<true>(j, r)] >> (8 * g);
#pragma unroll
            for (int i = 0; i < TM; ++i) sl[i] = scales[h * LINES + wm + tile_line<false>(i, r)] >> (8 * g);
            const int left = (int)a.c - (t * STEP_BLOCKS + h * HALF_BLOCKS) * MX4_BLOCK;
            if (left < HALF_BLOCKS * MX4_BLOCK) {   // (the end of the lines: codes behind it count as 0, and scales as 1)
                const int valid = left - g * MX4_BLOCK;
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    fl[i] = first_codes(fl[i], valid);
                    sl[i] = valid > 0 ? sl[i] : 127u;
                }
#pragma unroll
                for (int j = 0; j < TN; ++j) sr[j] = valid > 0 ? sr[j] : 127u;
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) mma_mx4(acc[i][j], fr[j], sr[j], fl[i], sl[i]);
        };
        half(std::integral_constant<int, 0>{});
        half(std::integral_constant<int, 1>{});
    };
#pragma unroll
    for (int t = 0; t < STAGES - 1; ++t)
        if (t < steps) fetch(t, t);
    int buffer = 0;
    for (int t = 0; t < steps; ++t) {
        // This wave's part of the step is in LDS (loads come back in order: all but those of later steps), and what it read of the step before has
        // come; then everyone's is, and nobody reads the buffer of the step before any more.
        constexpr int LATER = (STAGES - 2) * (TL::LOADS + TR::LOADS + SCALE_LOADS);
        static_assert(LATER < 64, "what the counter holds");
        asm volatile("" ::: "memory");
        if (t + STAGES - 2 < steps) __builtin_amdgcn_s_waitcnt(0x0070 | (LATER & 15) | (LATER >> 4) << 14);
        else __builtin_amdgcn_s_waitcnt(0x0070);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + STAGES - 1 < steps) fetch(t + STAGES - 1, buffer == 0 ? STAGES - 1 : buffer - 1);   // (in place of the step before)
        multiply(t, buffer);
        buffer = buffer + 1 == STAGES ? 0 : buffer + 1;
    }
    store_tile<O, BM, BN, WAVES_M, WAVES_N, true, sizeof(lds)>(a, w, acc, lds);
}

// Few rows: the matrix is read once, straight into registers, each wave every WAVES-th 128 numbers of its lines, a block and its scale a lane.
template <class O, int TN, int WAVES>
__global__ void __launch_bounds__(WAVES * WAVE, 2) k_few_mx4_mx4(GmmArgs a, Mx4Args x, Mx4Args m)
{
    __shared__ __align__(16) float s_sums[WAVES * 64 * (TN * 16 + 4)];
    __shared__ int64_t s_row[64];
    RowsTile w;
    int rows;
    if (!few_rows_tile<O, TN * 16>(a, w, rows, s_row)) return;
    const int lane = lane_id(), r = lane % 16, g = lane / 16, wave = threadIdx.x / WAVE;
    O *out = static_cast<O *>(a.out);
    auto store = [&](int row, int64_t col, float v) { out[(int64_t)(w.m0 + row) * a.ldo + col] = (O)(s_row[row] < 0 ? 0.0f : v); };
    auto tile = [&](auto tm) {
        constexpr int TM = decltype(tm)::value, UNROLL = TM == 1 ? 4 : 2, N = TM + TN;
        const uint8_t *codes[N], *scales[N];   // of x's lines, then the matrix's
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t row = max(s_row[min(i * 16 + r, rows - 1)], (int64_t)0);
            codes[i] = x.codes + row * x.ld_codes + g * 16;
            scales[i] = x.scales + row * x.ld_scales + g;
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = min(w.n0 + j * 16 + r, (int)a.n - 1);
            codes[TM + j] = m.codes + w.group * m.stride_codes + n * m.ld_codes + g * 16;
            scales[TM + j] = m.scales + w.group * m.stride_scales + n * m.ld_scales + g;
        }
        f32x4 acc[TM][TN] = {};
        const int whole = (int)(a.c / 128), steps = (int)((a.c + 127) / 128);
        int t = wave;
        for (; t + (UNROLL - 1) * WAVES < whole; t += UNROLL * WAVES) {
            u32x4 v[UNROLL][N];
            uint32_t s[UNROLL][N];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    v[u][k] = *reinterpret_cast<const u32x4 *>(codes[k] + (t + u * WAVES) * 64);
                    s[u][k] = scales[k][(t + u * WAVES) * 4];
                }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) mma_mx4(acc[i][j], v[u][TM + j], s[u][TM + j], v[u][i], s[u][i]);
        }
        for (; t < steps; t += WAVES) {
            u32x4 v[N];
            uint32_t s[N];
            const int valid = (int)a.c - (t * 128 + g * MX4_BLOCK);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                v[k] = valid > 0 ? *reinterpret_cast<const u32x4 *>(codes[k] + t * 64) : u32x4{};
                s[k] = valid > 0 ? scales[k][t * 4] : 127u;
                if (k < TM) v[k] = first_codes(v[k], valid);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) mma_mx4(acc[i][j], v[TM + j], s[TM + j], v[i], s[i]);
        }
        const float first[(TM * TN * 256 + WAVES * WAVE - 1) / (WAVES * WAVE)] = {};
        few_finish<O, TM, TN, WAVES>(acc, first, rows, w.n0, a.n, s_sums, store);
    };
    if (rows <= 16) tile(std::integral_constant<int, 1>{});
    else if (rows <= 32) tile(std::integral_constant<int, 2>{});
    else tile(std::integral_constant<int, 4>{});
}

template <class O, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES> hipError_t launch_tile(const GmmArgs &a, const Mx4Args &x, const Mx4Args &m, hipStream_t s)
{
    const Grid g = grid_of<GM_ROWS>(a, BM, BN);
    constexpr int threads = WAVES_M * WAVES_N * WAVE;
    if (g.blocks * threads >= (1ll << 32)) return TOO_MANY_TILES;
    hipLaunchKernelGGL((k_gmm_mx4_mx4<O, BM, BN, WAVES_M, WAVES_N, STAGES>), dim3((uint32_t)g.blocks), dim3(threads), 0, s, a, x, m, (int)g.nt);
    return hipGetLastError();
}

template <class O> hipError_t pick(const GmmArgs &a, const Mx4Args &x, const Mx4Args &m, hipStream_t s)
{
    const int64_t groups = std::min(a.groups, a.rows);
    auto m_tiles = [&](int64_t bm) { return std::max(groups, a.rows / bm + groups / 2); };
    auto tiles = [&](int64_t bm, int64_t bn) { return (double)m_tiles(bm) * (double)((a.n + bn - 1) / bn); };
    if (groups > 0 && groups * ((a.n + 63) / 64) < 256 && a.rows <= groups * 24) {
        hipLaunchKernelGGL((k_few_mx4_mx4<O, 1, 8>), few_grid(a, 16), dim3(8 * WAVE), 0, s, a, x, m);
        return hipGetLastError();
    }
    if constexpr (sizeof(O) == 2)   // (results of 32 bits do not fit the operands' place in LDS)
        if (tiles(128, 128) >= 512 && launches<GM_ROWS>(a, 256, 256, 512)) return launch_tile<O, 256, 256, 2, 4, 2>(a, x, m, s);
    if (tiles(64, 64) >= 512 || !launches<GM_ROWS>(a, 64, 64, 256)) return launch_tile<O, 128, 128, 2, 2, 2>(a, x, m, s);
    return launch_tile<O, 64, 64, 4, 1, 4>(a, x, m, s);
}

}  // namespace

hipError_t launch_grouped_mx4_mx4(const ocean_groups &g, const ocean_mx4 &x, const ocean_mx4 &w, int dtype, void *y, int64_t ldy, hipStream_t s)
{
    if (g.rows == 0 || w.rows == 0) return hipSuccess;
    GmmArgs a{};
    a.out = y, a.ldo = ldy;
    a.ptr = g.group_ptr, a.groups = g.experts, a.rows = g.rows;
    a.n = w.rows, a.c = w.inner;
    a.index = g.row_index, a.index_rows = g.row_index ? g.x_rows : g.rows;
    Mx4Args mx = mx4_args(x), mw = mx4_args(w);
    if (g.x_rows == 0 || w.inner == 0) a.c = 0, a.index_rows = 0, a.index = nullptr, mx.blocks = mw.blocks = 0;
    return with_type(dtype, [&](auto t) { return pick<decltype(t)>(a, mx, mw, s); });
}

}  // namespace ocean
