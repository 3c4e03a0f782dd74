// Products of ragged groups of rows with their group's matrix, both in four bits, on the scaled matrix instructions: 16 x 16 results from 128 numbers
// of c, each lane with one block of a line and its scale.
#include "mx4_tiles.hpp"

namespace ocean {

// (codes as bytes: 64 bytes of a line are 128 numbers of c, a fragment of 16 bytes one block)
template <> struct FragOf<uint8_t> { using type = u32x4; };

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int MMA_BLOCKS = 4, STEP_BLOCKS = LINE / 16;   // blocks of a line in a matrix instruction, in a step

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

// A tile, STAGES steps of 128 bytes of c (256 numbers) of both operands in LDS, and the scales of the periods of two steps that they belong to: 16
// bytes of a line at a time (4 bytes a step, each a line of memory looked up, cost more than the codes: 32668 rows of 4096 by eight 8192 x 4096 746 us).
// There now 650 to 690 us, 3.2 to 3.4 PFLOP/s; matrix cores are busy 43 %, LDS 34 %.  A step is a chain: without its loads it would be a sixth shorter, with a quarter of its
// products a quarter, and a tile's 16 steps have a beginning and an end that nothing overlaps, as one workgroup fills a compute unit's LDS.
// FAR: lines of x by 64-bit addresses, for those that 32-bit offsets do not reach (32000 rows gathered from 4.4 GB, eight 4096 x 4224, 500 us; 16 rows at a time 1855).  There is no range check on that way: pieces behind a line's end are its last one, which
// end_lines clears as it does the others.
template <class O, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES, bool FAR>
__global__ void __launch_bounds__(WAVES_M * WAVES_N * WAVE, 2) k_gmm_mx4_mx4(GmmArgs a, Mx4Args x, Mx4Args m, int nt)
{
    constexpr int THREADS = WAVES_M * WAVES_N * WAVE, WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 16, TN = WN / 16;
    using TL = Tile<uint8_t, false, false, BM, THREADS, LINE>;
    using TR = Tile<uint8_t, false, true, BN, THREADS, LINE>;
    constexpr int LINES = BM + BN, CODES = TL::BYTES + TR::BYTES, PERIODS = STAGES / 2 + 1, PERIOD_BLOCKS = 2 * STEP_BLOCKS;
    static_assert(STAGES % 2 == 0 && (LINES % THREADS == 0 || THREADS % LINES == 0), "as many scales a period for all waves");
    constexpr int SCALE_LOADS = LINES > THREADS ? LINES / THREADS : 1;
    __shared__ __align__(16) char lds[STAGES * CODES];
    __shared__ __align__(16) uint32_t s_scales[PERIODS][LINES][4];   // lines of x, then of the matrix
    RowsTile w;
    if (!rows_tile<O>(a, BM, BN, nt, w)) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), lane = lane_id(), r = lane % 16, g = lane / 16;
    const int wm = (wave / WAVES_N) * WM, wn = (wave % WAVES_N) * WN;
    const int depth = m.blocks * 16, steps = (m.blocks + STEP_BLOCKS - 1) / STEP_BLOCKS;   // bytes of a line
    const uint8_t *w_codes = m.codes + w.group * m.stride_codes, *w_scales = m.scales + w.group * m.stride_scales;

    const int64_t first = a.index ? 0 : w.m0;
    const Memory l_codes = memory_at(x.codes + first * x.ld_codes), r_codes = memory_at(w_codes + (int64_t)w.n0 * m.ld_codes);
    using Off = std::conditional_t<FAR, int64_t, uint32_t>;
    Off off_l[TL::LOADS], off_s[SCALE_LOADS];   // (FAR: without the piece, which the end of the line decides)
    uint32_t off_r[TR::LOADS];
#pragma unroll
    for (int i = 0; i < TL::LOADS; ++i) off_l[i] = (Off)(tile_row(a, w, TL::line_of(tid, i)) - first) * (Off)x.ld_codes + (FAR ? 0 : TL::piece_of(tid, i) * 16);
#pragma unroll
    for (int i = 0; i < TR::LOADS; ++i) off_r[i] = (uint32_t)min(TR::line_of(tid, i), (int)a.n - 1 - w.n0) * (uint32_t)m.ld_codes + TR::piece_of(tid, i) * 16;
    // (a wave's lines are all of one operand; where there are more threads than lines, some load the same.  The matrix's lie as a wave takes them, 16 side by side: as
    // 1 line in 4, 16 bytes each, they met on the same banks, a third of the cycles that LDS was used)
    const uint8_t *l_scales = x.scales + first * x.ld_scales, *r_scales = w_scales + (int64_t)w.n0 * m.ld_scales;
#pragma unroll
    for (int i = 0; i < SCALE_LOADS; ++i) {
        const int line = (i * THREADS + tid) % LINES;
        off_s[i] = line < BM ? (Off)(tile_row(a, w, line) - first) * (Off)x.ld_scales : (Off)min(tile_line<true>((line - BM) / 16, line % 16), (int)a.n - 1 - w.n0) * (Off)m.ld_scales;
    }
    // (the order of the steps is that of k_gmm_mx4, by periods)
    const int whole = (int)(a.c / (STEP_BLOCKS * MX4_BLOCK)), periods = whole / 2, turn = periods == 0 ? 0 : (w.n0 / BN + w.group * 5) % periods;
    auto period = [&](int p) { return p >= periods ? p : p + turn >= periods ? p + turn - periods : p + turn; };
    // (in `parts` parts, the part-th now)
    auto fetch = [&](int t_, int buffer, auto part_, auto parts_) {
        constexpr int PART = decltype(part_)::value, PARTS = decltype(parts_)::value;
        const int p = period(t_ / 2), t = p * 2 + t_ % 2, left = depth - t * LINE;
        char *to = lds + buffer * CODES + wave * (WAVE * 16);
        if (PART == 0 && t_ % 2 == 0) {
#pragma unroll
            for (int i = 0; i < SCALE_LOADS; ++i) {
                const int line = (i * THREADS + wave * WAVE) % LINES;
                char *const scales = reinterpret_cast<char *>(s_scales[t_ / 2 % PERIODS][line]);
                if constexpr (FAR) load_to_lds((line < BM ? l_scales : r_scales) + off_s[i] + p * PERIOD_BLOCKS, scales);
                else memory_to_lds<16>(memory_at(line < BM ? l_scales : r_scales), off_s[i], p * PERIOD_BLOCKS, scales);
            }
        }
#pragma unroll
        for (int i = TL::LOADS * PART / PARTS; i < TL::LOADS * (PART + 1) / PARTS; ++i) {
            if constexpr (FAR) load_to_lds(x.codes + first * x.ld_codes + off_l[i] + min(t * LINE + TL::piece_of(tid, i) * 16, depth - 16), to + i * THREADS * 16);
            else memory_to_lds<16>(l_codes, TL::piece_of(tid, i) * 16 < left ? off_l[i] : NOWHERE, t * LINE, to + i * THREADS * 16);
        }
#pragma unroll
        for (int i = TR::LOADS * PART / PARTS; i < TR::LOADS * (PART + 1) / PARTS; ++i)
            memory_to_lds<16>(r_codes, TR::piece_of(tid, i) * 16 < left ? off_r[i] : NOWHERE, t * LINE, to + TL::BYTES + i * THREADS * 16);
    };

    // The end of the lines: of this thread's pieces, codes of x behind it become 0 and scales of blocks behind it 1 (an empty block's could be NaN).
    auto end_lines = [&](int t, char *buffer) {
#pragma unroll
        for (int i = 0; i < TL::LOADS; ++i) {
            const int valid = (int)a.c - (t * STEP_BLOCKS + TL::piece_of(tid, i)) * MX4_BLOCK;
            u32x4 *piece = reinterpret_cast<u32x4 *>(buffer + (i * THREADS + tid) * 16);
            if (valid < MX4_BLOCK) *piece = first_codes(*piece, valid);
        }
#pragma unroll
        for (int i = 0; i < SCALE_LOADS; ++i) {
            uint32_t *scales = s_scales[t / 2 % PERIODS][(i * THREADS + tid) % LINES];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int there = m.blocks - (t / 2 * PERIOD_BLOCKS + k * MMA_BLOCKS);
                if (there < MMA_BLOCKS) scales[k] = there <= 0 ? 0x7f7f7f7fu : (scales[k] & ((1u << 8 * there) - 1u)) | 0x7f7f7f7fu << 8 * there;
            }
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    };

    const uint32_t at_l = TL::place(wm), at_r = TR::place(wn);
    f32x4 acc[TM][TN] = {};
    // A step in portions: 128 numbers of c of all the wave's columns and AT_ONCE of its 16s of rows, the next portion's reads under way meanwhile (all at once
    // don't fit the registers beside the sums).
    constexpr int AT_ONCE = TM < 4 ? TM : 4, PER_HALF = TM / AT_ONCE, PORTIONS = 2 * PER_HALF, LOAD_PARTS = 1;
    auto multiply = [&](int t, int buffer, auto load) {
        const char *from = lds + buffer * CODES;
        const uint32_t *scales = s_scales[t / 2 % PERIODS][0] + t % 2 * 2;
        u32x4 fr[2][TN], fl[2][AT_ONCE];
        uint32_t sr[2][TN], sl[2][AT_ONCE];
        auto read = [&](auto portion) {
            constexpr int p = decltype(portion)::value, h = p / PER_HALF, i0 = p % PER_HALF * AT_ONCE;
            if constexpr (i0 == 0) {
                TR::template read<h>(from + TL::BYTES, at_r, fr[h]);
#pragma unroll
                for (int j = 0; j < TN; ++j) sr[h][j] = scales[(BM + wn + j * 16 + r) * 4 + h] >> (8 * g);
            }
            TL::template read<h>(from + tile_line<false>(i0, 0) * LINE, at_l, fl[p & 1]);
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) sl[p & 1][i] = scales[(wm + tile_line<false>(i0 + i, r)) * 4 + h] >> (8 * g);
        };
        auto portion = [&](auto portion) {
            constexpr int p = decltype(portion)::value, h = p / PER_HALF, i0 = p % PER_HALF * AT_ONCE;
            if constexpr (p < PORTIONS) {
                if constexpr (p + 1 < PORTIONS) read(std::integral_constant<int, p + 1>{});
                if constexpr (p < LOAD_PARTS) load(std::integral_constant<int, p>{});
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) mma_mx4(acc[i0 + i][j], fr[h][j], sr[h][j], fl[p & 1][i], sl[p & 1][i]);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        read(std::integral_constant<int, 0>{});
        portion(std::integral_constant<int, 0>{});
        portion(std::integral_constant<int, 1>{});
        portion(std::integral_constant<int, 2>{});
        portion(std::integral_constant<int, 3>{});
    };
#pragma unroll
    for (int t = 0; t < STAGES - 1; ++t)
        if (t < steps) fetch(t, t, std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
    int buffer = 0;
    for (int t = 0; t < steps; ++t) {
        // This wave's part of the step is in LDS (loads come back in order: all but those of later steps), and what it read of the step before has
        // come; then everyone's is, and nobody reads the buffer of the step before any more.
        constexpr int LATER = (STAGES - 2) * (TL::LOADS + TR::LOADS) + (STAGES - 2) / 2 * SCALE_LOADS;
        static_assert(LATER < 64, "what the counter holds");
        asm volatile("" ::: "memory");
        if (t + STAGES - 2 < steps) __builtin_amdgcn_s_waitcnt(0x0070 | (LATER & 15) | (LATER >> 4) << 14);
        else __builtin_amdgcn_s_waitcnt(0x0070);
        asm volatile("" ::: "memory");
        if (t == whole) end_lines(t, lds + buffer * CODES);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        multiply(t, buffer, [&](auto part) {   // (in place of the step before)
            if (t + STAGES - 1 < steps) fetch(t + STAGES - 1, buffer == 0 ? STAGES - 1 : buffer - 1, part, std::integral_constant<int, LOAD_PARTS>{});
        });
        buffer = buffer + 1 == STAGES ? 0 : buffer + 1;
    }
    store_tile<O, BM, BN, WAVES_M, WAVES_N, true, sizeof(lds)>(a, w, acc, lds);
}

// Few rows: the matrix is read once, straight into registers, a block and its scale a lane.
template <class O, int TN, int WAVES>
__global__ void __launch_bounds__(WAVES * WAVE, 2) k_few_mx4_mx4(GmmArgs a, Mx4Args x, Mx4Args m)
{
    constexpr int ROWS = 16, U = TN == 2 ? 4 : 2;
    __shared__ __align__(16) float s_sums[few_lds(TN, WAVES)];
    __shared__ __align__(16) uint8_t s_scales[2][TN * 16 * FewScales<TN, WAVES>::PITCH];
    RowsTile w;
    if (!few_rows_tile<O, ROWS, TN * 16>(a, w)) return;
    const int lane = lane_id(), r = lane % 16, g = lane / 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int whole = (int)(a.c / 128), steps = (int)((a.c + 127) / 128), rows = min(ROWS, w.hi - w.m0);
    const uint8_t *codes[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) codes[j] = m.codes + w.group * m.stride_codes + min(w.n0 + j * 16 + r, (int)a.n - 1) * m.ld_codes;
    // (on their way while the row is found)
    FewScales<TN, WAVES> scales(m.scales + w.group * m.stride_scales, m.ld_scales, w.n0, a.n, m.blocks);
    Mx4Batch<TN, U> b;
    if (steps > 0) b.load(codes, min(wave * 4, steps - 1), g, m.blocks);
    const int slot = w.m0 + min(r, rows - 1);
    const int64_t number = a.index ? a.index[slot] : slot, row = (uint64_t)number < (uint64_t)a.index_rows ? number : 0;   // (0: its result is replaced by 0)
    const uint8_t *x_codes[1] = {x.codes + row * x.ld_codes}, *x_scales = x.scales + row * x.ld_scales;
    f32x4 acc[1][TN] = {};
    // U steps from t0 on; END: some of them may reach behind the lines' end.
    auto multiply = [&](int t0, auto end) {
        Mx4Batch<1, U> xs;
        xs.load(x_codes, t0, g, m.blocks);
        const uint8_t *words[1] = {x_scales + (int64_t)t0 * 4};
        xs.load_scales(words);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (decltype(end)::value) {
                const int valid = t0 + u < steps ? (int)max(min(a.c - ((int64_t)(t0 + u) * 128 + g * MX4_BLOCK), (int64_t)MX4_BLOCK), (int64_t)0) : 0;
                b.end(u, valid);
                xs.end(u, valid);
            }
#pragma unroll
            for (int j = 0; j < TN; ++j)
                mma_mx4(acc[0][j], __builtin_bit_cast(u32x4, b.v[u][j]), b.s[j][u] >> 8 * g, __builtin_bit_cast(u32x4, xs.v[u][0]), xs.s[0][u] >> 8 * g);
        }
    };
    for (int pass = 0; pass * WAVES * 4 < steps; ++pass) {
        scales.store(s_scales[pass & 1]);
        __syncthreads();
        scales.next();
        const int first = (pass * WAVES + wave) * 4;
#pragma unroll
        for (int i = 0; i < 4; i += U) {
            const int t = first + i, t_next = i + U < 4 ? t + U : first + WAVES * 4;
            if (t >= steps) break;
            const uint8_t *words[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) words[j] = s_scales[pass & 1] + (j * 16 + r) * FewScales<TN, WAVES>::PITCH + (wave * 4 + i) * 4;
            b.load_scales(words);
            if (t + U <= whole) multiply(t, std::false_type{});
            else multiply(t, std::true_type{});
            if (t_next < steps) b.load(codes, t_next, g, m.blocks);
        }
    }
    O *out = static_cast<O *>(a.out);
    few_meet<1, TN, WAVES>(acc, rows, w.n0, a.n, s_sums, [&](int i, int64_t col, float v) {
        const int64_t of = a.index ? a.index[w.m0 + i] : w.m0 + i;
        out[(int64_t)(w.m0 + i) * a.ldo + col] = (O)((uint64_t)of < (uint64_t)a.index_rows ? v : 0.0f);
    });
}

template <class O, int BM, int BN, int WAVES_M, int WAVES_N, int STAGES, bool FAR = false> hipError_t launch_tile(const GmmArgs &a, const Mx4Args &x, const Mx4Args &m, hipStream_t s)
{
    const Grid g = grid_of<GM_ROWS>(a, BM, BN);
    constexpr int threads = WAVES_M * WAVES_N * WAVE;
    if (g.blocks * threads >= (1ll << 32)) return TOO_MANY_TILES;
    hipLaunchKernelGGL((k_gmm_mx4_mx4<O, BM, BN, WAVES_M, WAVES_N, STAGES, FAR>), dim3((uint32_t)g.blocks), dim3(threads), 0, s, a, x, m, (int)g.nt);
    return hipGetLastError();
}

template <class O> hipError_t pick(const GmmArgs &a, const Mx4Args &x, const Mx4Args &m, hipStream_t s)
{
    // Up to 12 rows a group by themselves (us here and in tiles: 16 groups of 6 rows, 4096 x 4096, 25 and 28, eight of 8 15 and 16, of 16 19 and 16).
    const int64_t groups = std::min(a.groups, a.rows);
    if (groups > 0 && a.rows <= groups * 12 && a.n <= (1 << 20) && a.rows / 16 + groups < 65535)
        return with_columns_and_waves(a, [&](auto tn, auto waves) {
            constexpr int TN = decltype(tn)::value, WAVES = decltype(waves)::value;
            hipLaunchKernelGGL((k_few_mx4_mx4<O, TN, WAVES>), few_grid(a, 16, TN * 16), dim3(WAVES * WAVE), 0, s, a, x, m);
            return hipGetLastError();
        });
    constexpr TileTimes TIMES = {12.5, 3.5, 0.0248, 26, 19.5, 41, 32};
    // (32-bit offsets reach 4 GB: 256 lines side by side, or all of x where its rows are gathered)
    const bool far = !offsets_fit(a.index ? std::max<int64_t>(a.index_rows, 256) : 256, std::max(x.ld_codes, x.ld_scales), 1);
    const int lines = pick_lines(a, TIMES, sizeof(O) == 2 && !far);   // (results of 32 bits do not fit the operands' place in LDS)
    if (far) return lines == 64 ? launch_tile<O, 64, 64, 4, 1, 4, true>(a, x, m, s) : launch_tile<O, 128, 128, 2, 2, 2, true>(a, x, m, s);
    if (lines == 64) return launch_tile<O, 64, 64, 4, 1, 4>(a, x, m, s);
    if constexpr (sizeof(O) == 2)
        if (lines == 256) return launch_tile<O, 256, 256, 2, 4, 2>(a, x, m, s);
    return launch_tile<O, 128, 128, 2, 2, 2>(a, x, m, s);
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
