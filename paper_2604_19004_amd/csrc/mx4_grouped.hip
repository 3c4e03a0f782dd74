// Products of ragged groups of rows with their group's matrix in four bits, rows in their own type.
//
// Every number of four bits is a bfloat16 number, every float16 number the sum of two and every single precision number of three: so all products can be
// made by the bfloat16 matrix instructions, x in 1, 2 or 3 parts (exactly: single precision at a third of their rate is three times that of its own).  float16 goes
// through its own as long as it holds the matrix's numbers (mx4_far), and through two parts where it does not.
//
// A matrix number that is infinite makes NaN of a part that is 0, which the second and third may be where x is not: results that are NaN are looked at once more (Settle).  All
// parts of a number have its sign, so a sum that is infinite is right.
#include "mx4_tiles.hpp"

namespace ocean {

namespace {

template <class T> constexpr int PARTS_OF = std::is_same<T, bf16_t>::value ? 1 : std::is_same<T, f16_t>::value ? 2 : 3;

// 8 numbers as sums of bfloat16 numbers: each part takes the 8 leading bits of what is left, the last one the rest.  An infinite number or NaN is its first part.
template <class T> __device__ __forceinline__ void split(const T (&x)[8], bf16x8 (&out)[PARTS_OF<T>])
{
    constexpr int PARTS = PARTS_OF<T>;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if constexpr (PARTS == 1) {
            out[0][k] = x[k];
        } else {
            float left = (float)x[k];
            const bool finite = (__float_as_uint(left) & 0x7f800000u) != 0x7f800000u;
            const uint32_t quiet = left != left ? 0x00400000u : 0u;
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                const uint32_t bits = (__float_as_uint(left) | (p == 0 ? quiet : 0u)) & 0xffff0000u;
                out[p][k] = __builtin_bit_cast(bf16_t, (uint16_t)(bits >> 16));
                left = finite ? left - __uint_as_float(bits) : 0.0f;
            }
        }
    }
}
// The same in 4 operations a number and one a pair and part, where this is the time: numbers that are not finite, whose rest is NaN, are looked for with one more,
// and then it goes the other way (in tiles, 2048 rows by eight 4096 x 4096: 380 us and 340; beside few rows the branch costs more than it saves).
__device__ __forceinline__ void split_finite(const float (&x)[8], bf16x8 (&out)[3])
{
    uint32_t words[3][4];
    float other = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        float left[2] = {x[k], x[k + 1]};
        other = fmaf(left[1], 0.0f, fmaf(left[0], 0.0f, other));
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            words[p][k / 2] = __builtin_amdgcn_perm(__float_as_uint(left[1]), __float_as_uint(left[0]), 0x07060302);
#pragma unroll
            for (int i = 0; i < 2; ++i) left[i] -= __uint_as_float(__float_as_uint(left[i]) & 0xffff0000u);
        }
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) out[p] = __builtin_bit_cast(bf16x8, words[p]);
    if (other != other) split<float>(x, out);
}

// Results that came out as NaN, of columns for which the matrix has scales of infinite numbers: the sum from the definition in 64 bits where that is infinite.  As slow as it is
// simple (512 rows of ones by two 1024 x 1024 of nothing else, 1.0 ms); matrices that mx4_quantize has made have no such scale, and looking for one is what a NaN costs there (8000 rows of
// NaN, single precision, across 8192 x 4096: 3.7 ms, with what the other way of split takes).
//
// The arguments are read anew where they are wanted: kept until here, their registers cost every tile 1 to 2 % (eight groups of 256 rows, 4096 x 4096, float, 300 us and 293).
struct ProductArgs {
    GmmArgs a;
    Mx4Args m;
};
static_assert(alignof(GmmArgs) == alignof(Mx4Args) && sizeof(ProductArgs) == sizeof(GmmArgs) + sizeof(Mx4Args), "as a kernel's arguments lie");
__device__ __forceinline__ const ProductArgs &product_args_again()
{
    auto p = (const __attribute__((address_space(4))) ProductArgs *)__builtin_amdgcn_kernarg_segment_ptr();   // (a kernel's first two arguments)
    asm volatile("" : "+s"(p));
    return *(const ProductArgs *)p;
}
template <class T, bool RCOL> struct Settle {
    int group;

    __device__ __forceinline__ const uint8_t *scale_at(const Mx4Args &m, int64_t line, int64_t number) const { return m.scales + group * m.stride_scales + line * m.ld_scales + number / MX4_BLOCK; }
    // (RCOL: bit i, whether the i-th block of the WN columns from `first` on has such a scale in any line, 64 lines at a time; all lanes of the wave)
    template <int WN> __device__ __forceinline__ uint32_t of_wave(int first) const
    {
        uint32_t mine = 0, all = 0;
        if constexpr (RCOL) {
            const ProductArgs &args = product_args_again();
            const Mx4Args m = args.m;
            const int64_t depth = args.a.c;
#pragma unroll 2
            for (int64_t c = lane_id(); c < depth; c += WAVE)
#pragma unroll
                for (int i = 0; i < WN / MX4_BLOCK; ++i) mine |= (uint32_t)mx4_infinite(*scale_at(m, c, min(first / MX4_BLOCK + i, m.blocks - 1) * (int64_t)MX4_BLOCK)) << i;
#pragma unroll
            for (int i = 0; i < WN / MX4_BLOCK; ++i) all |= (uint32_t)(__any(mine >> i & 1u) != 0) << i;
        }
        return all;
    }
    __device__ __forceinline__ bool of_column(int64_t n, int first = 0, uint32_t blocks = 0) const
    {
        if constexpr (RCOL) return blocks >> (n - first) / MX4_BLOCK & 1u;
        const ProductArgs &args = product_args_again();
        const Mx4Args m = args.m;
        const int64_t depth = args.a.c;
        bool infinite = false;
#pragma unroll 8
        for (int64_t c = 0; c < depth; c += MX4_BLOCK) infinite |= mx4_infinite(*scale_at(m, n, c));
        return infinite;
    }
    __device__ __forceinline__ float result(int slot, int64_t n) const
    {
        const ProductArgs &args = product_args_again();
        const GmmArgs a = args.a;
        const Mx4Args m = args.m;
        const int64_t row = a.index ? a.index[slot] : slot;
        if ((uint64_t)row >= (uint64_t)a.index_rows) return 0.0f;
        const T *x = static_cast<const T *>(a.l) + row * a.ldl;
        constexpr int AT_ONCE = RCOL ? 2 : 4;   // (more spill in tiles of 256 x 256 across)
        double sum = 0.0;
#pragma unroll AT_ONCE
        for (int64_t c = 0; c < a.c; ++c) {
            const int64_t line = RCOL ? c : n, at = RCOL ? n : c;
            const uint32_t codes = m.codes[group * m.stride_codes + line * m.ld_codes + at / 2];
            bf16_t e[8];
            mx4_widen<bf16_t>(codes >> at % 2 * 4, mx4_scale(*scale_at(m, line, at)), e);
            sum += (double)(float)x[c] * (double)(float)e[0];   // (finite products are below 2^256)
        }
        return fabs(sum) == INFINITY ? (float)sum : NAN;
    }
};

// Whether a tile has a scale that float16 does not take; every thread calls it.
template <bool RCOL, int BN, int THREADS> __device__ __forceinline__ bool any_far(const Mx4Args &m, const uint8_t *scales, int n0, int64_t n, int depth)
{
    bool far = false;
    if constexpr (RCOL) {   // (BN / 32 blocks of every line)
        constexpr int BLOCKS = BN / MX4_BLOCK;
        const int block = min(n0 / MX4_BLOCK + (int)threadIdx.x % BLOCKS, m.blocks - 1);
#pragma unroll 4
        for (int c = threadIdx.x / BLOCKS; c < depth; c += THREADS / BLOCKS) far |= mx4_far(scales[c * m.ld_scales + block]);
    } else {
        constexpr int EACH = 8;   // threads a line
        for (int i = threadIdx.x / EACH; i < min((int64_t)BN, n - n0); i += THREADS / EACH)
#pragma unroll 2
            for (int b = threadIdx.x % EACH * 16; b < m.blocks; b += EACH * 16) {
                const uint4 v = *reinterpret_cast<const uint4 *>(scales + (n0 + i) * m.ld_scales + b);
                const uint32_t words[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int k = 0; k < 16; ++k) far |= b + k < m.blocks && mx4_far(words[k / 4] >> k % 4 * 8 & 255u);
            }
    }
    return __syncthreads_or(far);
}

// A tile: x straight to LDS (16 bits, whole pieces) or through registers, where single precision is split; the matrix's codes through registers, where they are widened.
// STAGES steps are under way, in LDS or registers: the next one, or in small tiles, which wait for memory, three (512 rows of 4095 by 4095 x 4096, bfloat16, through
// registers: 58 us and 50).  Large ones are bound by the matrix cores under the card's power: 32668 rows by eight 8192 x 4096, bf16, 1811 us, 1210 TFLOP/s; small and short
// ones by the way of a step, which has loads, LDS and matrix cores one after the other.
template <class T, bool RCOL, int BM, int BN, int WAVES_M, int WAVES_N, bool ASYNC, int STAGES>
__global__ void __launch_bounds__(WAVES_M * WAVES_N * WAVE, 2) k_gmm_mx4(GmmArgs a, Mx4Args m, int nt)
{
    constexpr int THREADS = WAVES_M * WAVES_N * WAVE, WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 16, TN = WN / 16, PARTS = sizeof(T) == 4 ? 3 : 1;
    using S = std::conditional_t<sizeof(T) == 4, bf16_t, T>;   // what LDS holds (float16 with far scales: of the matrix, bfloat16)
    constexpr bool HALF = std::is_same<T, f16_t>::value;
    constexpr int STEP_C = STEP<S>;
    static_assert(!ASYNC || PARTS == 1, "parts are made in registers");
    using TL = Tile<S, false, false, BM, THREADS, LINE>;
    using TR = Tile<S, RCOL, !RCOL, BN, THREADS, LINE>;
    constexpr int X_BYTES = PARTS * TL::BYTES, X_STEPS = ASYNC ? STAGES : 2;
    static_assert(STAGES == 2 || STAGES == 4, "the loop's steps");
    // A thread's share of the matrix's step: E numbers of a line side by side, in one block.
    constexpr int E = BN * STEP_C / THREADS, WORDS = E / 8, A_LINE = (RCOL ? BN : STEP_C) / E;
    static_assert(E == 16 || E == 32, "part of a block");
    __shared__ __align__(16) char lds[X_STEPS * X_BYTES + 2 * TR::BYTES];
    char *const lds_r = lds + X_STEPS * X_BYTES;
    RowsTile w;
    if (!rows_tile<T>(a, BM, BN, nt, w)) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
    const int wm = (wave / WAVES_N) * WM, wn = (wave % WAVES_N) * WN;
    const int depth = (int)a.c, steps = (depth + STEP_C - 1) / STEP_C;

    // Offsets of the thread's pieces of x from `x_memory` (ASYNC, in bytes), or its lines' rows (elements).
    const int64_t first = a.index ? 0 : w.m0;
    const Memory x_memory = memory_at(static_cast<const T *>(a.l) + first * a.ldl);
    uint32_t off[ASYNC ? TL::LOADS : 1];
    int64_t row[ASYNC ? 1 : TL::LOADS];
#pragma unroll
    for (int i = 0; i < TL::LOADS; ++i) {
        if constexpr (ASYNC) off[i] = (uint32_t)(((tile_row(a, w, TL::line_of(tid, i)) - first) * a.ldl + TL::piece_of(tid, i) * 8) * 2);
        else row[i] = tile_row(a, w, TL::line_of(tid, i)) * a.ldl;
    }
    // The thread's line (a row of the matrix, or one c) and its part of it; what comes of columns behind the end is not stored.
    const int line = tid / A_LINE, part = tid % A_LINE;
    const uint8_t *codes = m.codes + w.group * m.stride_codes, *scales = m.scales + w.group * m.stride_scales;
    if constexpr (!RCOL) codes += w.n0 * m.ld_codes, scales += w.n0 * m.ld_scales;
    uint32_t code_off, scale_off;
    if constexpr (RCOL) {
        const int block = min((w.n0 + part * E) / MX4_BLOCK, m.blocks - 1);
        code_off = (uint32_t)(line * (int)m.ld_codes + block * 16 + part * E % MX4_BLOCK / 2);
        scale_off = (uint32_t)(line * (int)m.ld_scales + block);
    } else {
        const int n = min(line, (int)a.n - 1 - w.n0);
        code_off = (uint32_t)n * (uint32_t)m.ld_codes + part * (E / 2);
        scale_off = (uint32_t)n * (uint32_t)m.ld_scales + part * E / MX4_BLOCK;
    }

    // (float16 with far scales is a walk of its own: beside the other one, its registers would be that one's too)
    auto run = [&](auto far) {
        constexpr bool WIDE = decltype(far)::value;
        struct Raw { uint4 v[sizeof(T) / 2]; };
        Raw kept[ASYNC ? 1 : STAGES][ASYNC ? 1 : TL::LOADS];
        uint32_t kept_codes[STAGES][WORDS], kept_scale[STAGES];   // step t's in t % STAGES
        // Workgroups begin at different steps and go round, so that they don't all read lines that begin in the same memory channels; what is left
        // of the lines behind whole steps comes last.
        const int whole = depth / STEP_C, turn = whole == 0 ? 0 : (w.n0 / BN + w.group * 5) % whole;
        auto at = [&](int t) { return t == whole ? t : t + turn >= whole ? t + turn - whole : t + turn; };
        auto scale_place = [&](int c0) -> uint32_t { return RCOL ? scale_off : scale_off + c0 / MX4_BLOCK; };
        // (steps that are not there are fetched as zeros, from no memory, so that every step has as many loads)
        auto fetch = [&](int t_, auto slot_) {
            constexpr int slot = decltype(slot_)::value;
            const int t = t_ < steps ? at(t_) : 0, c0 = t * STEP_C, left = t_ < steps ? min(STEP_C, depth - c0) : 0;
            const bool there = RCOL ? line < left : t_ < steps && c0 + part * E < m.blocks * MX4_BLOCK;
            const Memory code_memory = memory_at(RCOL ? codes + (int64_t)c0 * m.ld_codes : codes), scale_memory = memory_at(RCOL ? scales + (int64_t)c0 * m.ld_scales : scales);
            // (zeros: a code of 0 is 0 at any scale but NaN.  The scale as its word: a byte would be widened, and waited for, where it is loaded)
            const uint32_t code_at = there ? code_off : NOWHERE, scale_at = there ? scale_place(c0) & ~3u : NOWHERE;
            if constexpr (WORDS == 4) {
                const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(code_memory, code_at, RCOL ? 0 : c0 / 2, 0));
#pragma unroll
                for (int j = 0; j < 4; ++j) kept_codes[slot][j] = v[j];
            } else {
                const auto v = __builtin_amdgcn_raw_buffer_load_b64(code_memory, code_at, RCOL ? 0 : c0 / 2, 0);
                kept_codes[slot][0] = v[0], kept_codes[slot][1] = v[1];
            }
            kept_scale[slot] = __builtin_amdgcn_raw_buffer_load_b32(scale_memory, scale_at, 0, 0);
            if constexpr (ASYNC) {
                char *to = lds + slot * X_BYTES + wave * (WAVE * 16);
#pragma unroll
                for (int i = 0; i < TL::LOADS; ++i)
                    memory_to_lds<16>(x_memory, TL::piece_of(tid, i) * 8 < left ? off[i] : NOWHERE, (uint32_t)c0 * 2, to + i * THREADS * 16);
            } else {
                const T *x = static_cast<const T *>(a.l) + c0;
#pragma unroll
                for (int i = 0; i < TL::LOADS; ++i) {
                    const T *p = x + row[i] + TL::piece_of(tid, i) * 8;
                    const int valid = left - TL::piece_of(tid, i) * 8;
#pragma unroll
                    for (int j = 0; j < (int)sizeof(T) / 2; ++j)
                        kept[slot][i].v[j] = left == STEP_C ? load_any(reinterpret_cast<const char *>(p + j * PIECE<T>)) : load_piece(p + j * PIECE<T>, valid - j * PIECE<T>);
                }
            }
        };
        auto stash = [&](int t_, auto slot_) {
            constexpr int slot = decltype(slot_)::value;
            if constexpr (!ASYNC) {
                char *to = lds + slot % X_STEPS * X_BYTES;
#pragma unroll
                for (int i = 0; i < TL::LOADS; ++i) {
                    if constexpr (PARTS == 1) {
                        *reinterpret_cast<uint4 *>(to + (i * THREADS + tid) * 16) = kept[slot][i].v[0];
                    } else {
                        bf16x8 p[PARTS];
                        split_finite(__builtin_bit_cast(decltype(Vec<T, 8>{}), kept[slot][i]).e, p);
#pragma unroll
                        for (int k = 0; k < PARTS; ++k) *reinterpret_cast<bf16x8 *>(to + k * TL::BYTES + (i * THREADS + tid) * 16) = p[k];
                    }
                }
            }
            uint32_t (&words)[WORDS] = kept_codes[slot];
            if (!RCOL && t_ == whole) {   // (codes behind the lines' end meet zeros of x, but may be infinite numbers)
#pragma unroll
                for (int j = 0; j < WORDS; ++j) words[j] = mx4_first(words[j], depth - (t_ * STEP_C + part * E + j * 8));
            }
            const int swizzle = RCOL ? col_xor<S, TR::PIECES>(line) : row_xor<!RCOL, TR::PIECES>(line);
            char *to_line = lds_r + slot % 2 * TR::BYTES + line * TR::PIECES * 16;
            const float scale = mx4_scale(kept_scale[slot] >> scale_place(at(t_) * STEP_C) % 4 * 8 & 255u);
            auto widen = [&](auto type) {
                using W = decltype(type);
#pragma unroll
                for (int j = 0; j < WORDS; ++j) *reinterpret_cast<Frag<W> *>(to_line + ((part * WORDS + j) ^ swizzle) * 16) = mx4_fragment<W>(words[j], scale);
            };
            widen(std::conditional_t<WIDE, bf16_t, S>{});
        };

        const uint32_t at_l = TL::place(wm), at_r = TR::place(wn);
        f32x4 acc[TM][TN] = {};
        // (single precision: the sums of 256 products are put aside, as in k_gmm)
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
        // A step in portions: half of its c, one part of x and AT_ONCE of the wave's 16s of rows, the next portion's reads under way meanwhile; load() brings the next
        // step on its way behind the first reads (before them, the waves wait for its addresses to be taken).
        constexpr int AT_ONCE = TM < 4 ? TM : 4, PER_PART = TM / AT_ONCE, PER_HALF = PARTS * PER_PART, PORTIONS = 2 * PER_HALF;
        auto multiply = [&](int slot, auto load) {
            const char *from = lds + slot % X_STEPS * X_BYTES, *from_r = lds_r + slot % 2 * TR::BYTES;
            Frag<S> fr[2][TN], fl[2][AT_ONCE];
            auto read = [&](auto portion) {
                constexpr int q = decltype(portion)::value, h = q / PER_HALF, p = PARTS - 1 - q % PER_HALF / PER_PART, i0 = q % PER_PART * AT_ONCE;
                if constexpr (q % PER_HALF == 0) TR::template read<h>(from_r, at_r, fr[h]);
                TL::template read<h>(from + p * TL::BYTES + tile_line<false>(i0, 0) * LINE, at_l, fl[q & 1]);
            };
            auto portion = [&](auto portion) {
                constexpr int q = decltype(portion)::value, h = q / PER_HALF, i0 = q % PER_PART * AT_ONCE;
                if constexpr (q < PORTIONS) {
                    if constexpr (q + 1 < PORTIONS) read(std::integral_constant<int, q + 1>{});
                    if constexpr (q == 0) load();
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i) {
                        if constexpr (WIDE) {
                            bf16x8 x[PARTS_OF<f16_t>];
                            split<f16_t>(__builtin_bit_cast(decltype(Vec<f16_t, 8>{}), fl[q & 1][i]).e, x);
#pragma unroll
                            for (int k = PARTS_OF<f16_t> - 1; k >= 0; --k)
#pragma unroll
                                for (int j = 0; j < TN; ++j) mma_part(acc[i0 + i][j], __builtin_bit_cast(bf16x8, fr[h][j]), x[k], 0);
                            __builtin_amdgcn_sched_barrier(0);   // (one after the other: registers)
                        } else {
#pragma unroll
                            for (int j = 0; j < TN; ++j) mma_part(acc[i0 + i][j], fr[h][j], fl[q & 1][i], 0);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            read(std::integral_constant<int, 0>{});
            portion(std::integral_constant<int, 0>{});
            portion(std::integral_constant<int, 1>{});
            portion(std::integral_constant<int, 2>{});
            portion(std::integral_constant<int, 3>{});
            portion(std::integral_constant<int, 4>{});
            portion(std::integral_constant<int, 5>{});
            static_assert(PORTIONS <= 6);
        };
        using std::integral_constant;
        auto each_slot = [&](auto f) {
            f(integral_constant<int, 0>{});
            f(integral_constant<int, 1>{});
            if constexpr (STAGES == 4) {
                f(integral_constant<int, 2>{});
                f(integral_constant<int, 3>{});
            }
        };
        each_slot([&](auto slot) {
            if constexpr (decltype(slot)::value < STAGES - 1) fetch(decltype(slot)::value, slot);
        });
        stash(0, integral_constant<int, 0>{});
        // This wave's part of the step is in LDS (loads come back in order: all but those of the steps behind it), and what it read of the step before
        // has come; then everyone's is, and nobody reads the places of the step before any more.
        auto meet = [&](auto later) {
            constexpr int LATER = decltype(later)::value;
            static_assert(LATER < 16, "what the counter's low bits hold");
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(ASYNC ? 0x0070 | LATER : 0xc07f);   // (registers are waited for where they are used)
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        int t0 = 0;
        for (; t0 + STAGES <= steps; t0 += STAGES)
            each_slot([&](auto slot_) {   // (the last ones fetch steps that are not there: zeros, and no branch for which registers of loads under way would be moved)
                constexpr int slot = decltype(slot_)::value, NEXT = (slot + 1) % STAGES, LAST = (slot + STAGES - 1) % STAGES;
                const int t = t0 + slot;
                meet(integral_constant<int, (STAGES - 2) * (2 + (ASYNC ? TL::LOADS : 0))>{});
                multiply(slot, [&] { fetch(t + STAGES - 1, integral_constant<int, LAST>{}); });
                if (ASIDE && t % 4 == 3) put_aside();
                stash(t + 1, integral_constant<int, NEXT>{});
            });
        each_slot([&](auto slot_) {   // (fewer than STAGES are left, and all of them are under way)
            constexpr int slot = decltype(slot_)::value;
            if constexpr (slot < STAGES - 1)
                if (t0 + slot < steps) {
                    meet(integral_constant<int, 0>{});
                    multiply(slot, [] {});
                    stash(t0 + slot + 1, integral_constant<int, slot + 1>{});
                }
        });
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): steps that are not there also write their zeros to LDS, where the results go now
        asm volatile("" ::: "memory");
        if constexpr (ASIDE) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] += sums[i][j];
        }
        if constexpr (PARTS > 1 || WIDE)
            store_tile<T, BM, BN, WAVES_M, WAVES_N, !RCOL, sizeof(lds)>(a, w, acc, lds, Settle<T, RCOL>{w.group});
        else
            store_tile<T, BM, BN, WAVES_M, WAVES_N, !RCOL, sizeof(lds)>(a, w, acc, lds);
    };
    if constexpr (HALF) {
        if (any_far<RCOL, BN, THREADS>(m, m.scales + w.group * m.stride_scales, w.n0, a.n, depth)) {
            run(std::true_type{});
            return;
        }
    }
    run(std::false_type{});
}

// Few rows: the matrix is read once, straight into registers.  A lane's 32 numbers of c are those of its block, in four matrix instructions; x is read
// to match.  Bound by the matrix's bytes: sixteen groups of 4 rows, 4096 x 4096, 31 us, 4.6 TB/s; two of one row, 8192 x 4096, 11.3 us, 3.2 TB/s, where the beginning is a third.
// Two steps under way a wave: with one 16 and 36 us, with four, or registers cut to four waves a SIMD, 12 and 31, 15 and 40.
template <class T, int ROWS, int TN, int WAVES>
__global__ void __launch_bounds__(WAVES * WAVE, 2) k_few_mx4(GmmArgs a, Mx4Args m)
{
    constexpr int PARTS = PARTS_OF<T>;
    __shared__ __align__(16) float s_sums[few_lds(TN, WAVES)];
    __shared__ __align__(16) uint8_t s_scales[2][TN * 16 * FewScales<TN, WAVES>::PITCH];
    __shared__ int64_t s_row[ROWS];
    RowsTile w;
    if (!few_rows_tile<T, ROWS, TN * 16>(a, w)) return;
    const int lane = lane_id(), r = lane % 16, g = lane / 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const uint8_t *codes[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) codes[j] = m.codes + w.group * m.stride_codes + min(w.n0 + j * 16 + r, (int)a.n - 1) * m.ld_codes;
    const int whole = (int)(a.c / 128), steps = (int)((a.c + 127) / 128), rows = min(ROWS, w.hi - w.m0);
    T *out = static_cast<T *>(a.out);
    bool nan = false;   // (a result of this thread)
    auto store = [&](int row, int64_t col, float v) {
        v = s_row[row] < 0 ? 0.0f : v;
        nan |= v != v;
        out[(int64_t)(w.m0 + row) * a.ldo + col] = (T)v;
    };
    auto tile = [&](auto tm) {
        constexpr int TM = decltype(tm)::value, U = TM == 4 || sizeof(T) * TM > 4 ? 1 : sizeof(T) * TM * TN > 4 ? 2 : 4;
        // (on their way while the rows are found)
        FewScales<TN, WAVES> scales(m.scales + w.group * m.stride_scales, m.ld_scales, w.n0, a.n, m.blocks);
        Mx4Batch<TN, U> b;
        if (steps > 0) b.load(codes, min(wave * 4, steps - 1), g, m.blocks);
        if ((int)threadIdx.x < rows) {
            const int64_t row = a.index ? a.index[w.m0 + threadIdx.x] : w.m0 + threadIdx.x;
            s_row[threadIdx.x] = (uint64_t)row < (uint64_t)a.index_rows ? row : -1;
        }
        __syncthreads();
        const T *x[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) x[i] = static_cast<const T *>(a.l) + max(s_row[min(i * 16 + r, rows - 1)], (int64_t)0) * a.ldl + g * MX4_BLOCK;
        f32x4 acc[TM][TN] = {};
        struct Eight { uint4 v[sizeof(T) / 2]; };
        // U steps from t0 on.  ANY: some of them may reach behind the lines' end, and float16 goes in parts.
        auto multiply = [&](int t0, auto any) {
            constexpr bool ANY = decltype(any)::value;
            using W = std::conditional_t<!ANY && sizeof(T) == 2, T, bf16_t>;   // (what the matrix's numbers become)
            Eight xs[U][TM][4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                int valid = MX4_BLOCK;
                if constexpr (ANY) {
                    valid = t0 + u < steps ? (int)max(min(a.c - ((int64_t)(t0 + u) * 128 + g * MX4_BLOCK), (int64_t)MX4_BLOCK), (int64_t)0) : 0;
                    b.end(u, valid);
                }
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int p = 0; p < (int)sizeof(T) / 2; ++p) {
                            const T *at = x[i] + (int64_t)(t0 + u) * 128 + q * 8 + p * PIECE<T>;
                            xs[u][i][q].v[p] = ANY ? load_piece(at, valid - q * 8 - p * PIECE<T>) : load_any(reinterpret_cast<const char *>(at));
                        }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    Frag<W> fw[TN];
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const uint4 &v = b.v[u][j];
                        fw[j] = mx4_fragment<W>(q == 0 ? v.x : q == 1 ? v.y : q == 2 ? v.z : v.w, mx4_scale(b.scale(u, j, g)));
                    }
#pragma unroll
                    for (int i = 0; i < TM; ++i) {
                        if constexpr (std::is_same<T, W>::value) {
#pragma unroll
                            for (int j = 0; j < TN; ++j) mma_part(acc[i][j], fw[j], __builtin_bit_cast(Frag<W>, xs[u][i][q].v[0]), 0);
                        } else {
                            bf16x8 p[PARTS];
                            split<T>(__builtin_bit_cast(decltype(Vec<T, 8>{}), xs[u][i][q]).e, p);
#pragma unroll
                            for (int k = PARTS - 1; k >= 0; --k)
#pragma unroll
                                for (int j = 0; j < TN; ++j) mma_part(acc[i][j], fw[j], p[k], 0);
                        }
                    }
                    if (ANY) __builtin_amdgcn_sched_barrier(0);   // (so that this takes no more registers than the other one)
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
                bool far = false;
                if constexpr (std::is_same<T, f16_t>::value) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int j = 0; j < TN; ++j) far |= mx4_far(b.scale(u, j, g));
                    far = __any(far);
                }
                if (t + U <= whole && !far) multiply(t, std::false_type{});
                else multiply(t, std::true_type{});
                if (t_next < steps) b.load(codes, t_next, g, m.blocks);
            }
        }
        few_meet<TM, TN, WAVES>(acc, rows, w.n0, a.n, s_sums, store);
    };
    if (ROWS == 16 || rows <= 16) tile(std::integral_constant<int, 1>{});
    else if constexpr (ROWS >= 32) {
        if (ROWS == 32 || rows <= 32) tile(std::integral_constant<int, 2>{});
        else if constexpr (ROWS == 64) tile(std::integral_constant<int, 4>{});
    }
    if constexpr (PARTS > 1) {
        constexpr int COLS = TN * 16, AT_ONCE = WAVES * WAVE / COLS;
        static_assert(WAVES * WAVE % COLS == 0 && 16 % AT_ONCE == 0, "a thread stores one column's results");
        const Settle<T, false> settle{w.group};
        const int64_t n = w.n0 + threadIdx.x % COLS;
        if (nan && settle.of_column(n)) {   // (each thread goes through what few_meet had it store)
#pragma unroll 1
            for (int row = threadIdx.x / COLS; row < rows; row += AT_ONCE) {
                T *to = out + (int64_t)(w.m0 + row) * a.ldo + n;
                if (*to != *to) *to = (T)settle.result(w.m0 + row, n);
            }
        }
    }
}

template <class T, bool RCOL, int BM, int BN, int WAVES_M, int WAVES_N, bool ASYNC, int STAGES = 2> hipError_t launch_tile(const GmmArgs &a, const Mx4Args &m, hipStream_t s)
{
    const Grid g = grid_of<GM_ROWS>(a, BM, BN);
    constexpr int threads = WAVES_M * WAVES_N * WAVE;
    if (g.blocks * threads >= (1ll << 32)) return TOO_MANY_TILES;
    hipLaunchKernelGGL((k_gmm_mx4<T, RCOL, BM, BN, WAVES_M, WAVES_N, ASYNC, STAGES>), dim3((uint32_t)g.blocks), dim3(threads), 0, s, a, m, (int)g.nt);
    return hipGetLastError();
}

// Rows are few where the matrix's bytes are the time: up to 20 a group, and up to 64 where there are not enough groups and columns for the chip (4096 x 4096, us in k_few_mx4
// and in tiles: eight groups of 8 rows 19 and 35, of 16 22 and 35, of 24 45 and 35; one group of 16 12 and 25, of 40 17 and 24, of 64 21 and 24).
bool few_rows(const GmmArgs &a)
{
    const int64_t groups = std::min(a.groups, a.rows);
    return groups > 0 && a.rows <= groups * (fills_chip(a) ? 20 : 64) && a.n <= (1 << 20) && a.rows / 16 + groups < 65535;
}

template <class T, bool RCOL> hipError_t pick(const GmmArgs &a, const Mx4Args &m, bool straight, hipStream_t s)
{
    if constexpr (!RCOL) {
        if (few_rows(a)) {
            auto launch = [&](auto rows, auto tn, auto waves) {
                constexpr int ROWS = decltype(rows)::value, TN = decltype(tn)::value, WAVES = decltype(waves)::value;
                hipLaunchKernelGGL((k_few_mx4<T, ROWS, TN, WAVES>), few_grid(a, ROWS, TN * 16), dim3(WAVES * WAVE), 0, s, a, m);
                return hipGetLastError();
            };
            using std::integral_constant;
            const int64_t groups = std::min(a.groups, a.rows);
            return with_columns_and_waves(a, [&](auto tn, auto waves) {
                if (a.rows <= groups * 10) return launch(integral_constant<int, 16>{}, tn, waves);
                if (a.rows <= groups * 22) return launch(integral_constant<int, 32>{}, tn, waves);
                return launch(integral_constant<int, 64>{}, integral_constant<int, 2>{}, waves);   // (more columns leave no registers; here they are 2)
            });
        }
    }
    // (single precision, 4096 columns and c = 4096: tiles of 128 x 128 were as fast for 2048 rows as those of 64 x 64, 367 us and 369, and slower for 512, 185 and 105;
    // these take 340 and 93 since)
    if constexpr (sizeof(T) == 4) return launch_tile<T, RCOL, 64, 64, 4, 1, false, 4>(a, m, s);
    else {
        constexpr TileTimes TIMES = {26, 10, 0.0555, 74, 50, 104, 92};
        const int lines = pick_lines(a, TIMES, straight);
        if (!straight) return lines == 64 ? launch_tile<T, RCOL, 64, 64, 4, 1, false, 4>(a, m, s) : launch_tile<T, RCOL, 128, 128, 2, 2, false>(a, m, s);
        if (lines == 64) return launch_tile<T, RCOL, 64, 64, 4, 1, true, 4>(a, m, s);
        return lines == 128 ? launch_tile<T, RCOL, 128, 128, 2, 2, true>(a, m, s) : launch_tile<T, RCOL, 256, 256, 2, 4, true>(a, m, s);
    }
}

}  // namespace

hipError_t launch_grouped_mx4(const ocean_groups &g, int dtype, const void *x, int64_t ldx, const ocean_mx4 &w, bool transposed, void *y, int64_t ldy, hipStream_t s)
{
    const int64_t outer = transposed ? w.inner : w.rows, inner = transposed ? w.rows : w.inner;
    if (g.rows == 0 || outer == 0) return hipSuccess;
    GmmArgs a{};
    a.l = x, a.ldl = ldx;
    a.out = y, a.ldo = ldy;
    a.ptr = g.group_ptr, a.groups = g.experts, a.rows = g.rows;
    a.n = outer, a.c = inner;
    a.index = g.row_index, a.index_rows = g.row_index ? g.x_rows : g.rows;
    if (g.x_rows == 0 || inner == 0) a.c = 0, a.index_rows = 0, a.index = nullptr;
    const Mx4Args m = mx4_args(w);
    // (the rows of a tile lie within 256 lines, gathered ones anywhere in x)
    // (whole pieces: a piece of x lies before its row's end or behind it)
    const bool straight = dtype != OCEAN_F32 && pieces_aligned(x, ldx, 0, 2) && inner % 8 == 0 && offsets_fit(g.row_index ? std::max<int64_t>(g.x_rows, 256) : 256, ldx, 2);
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return transposed ? pick<T, true>(a, m, straight, s) : pick<T, false>(a, m, straight, s);
    });
}

}  // namespace ocean
