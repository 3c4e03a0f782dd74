// The products of gmm.hpp for few rows: the right matrix is read once, straight into registers, and that is the time it takes.
//
// A workgroup has TN * 16 columns and all of c: its waves take every WAVES-th 128 bytes of c, 16 lines at a time as the matrix cores want
// them, and their sums meet in LDS.  Rows come from the cache (each workgroup reads them all).  Nothing passes through LDS
// on its way in: no two waves need the same bytes of the right matrix.
#pragma once

#include "gmm.hpp"

namespace ocean {

namespace {

template <class T, bool ALIGNED> __device__ __forceinline__ Frag<T> few_load(const T *p, int64_t valid)
{
    if constexpr (ALIGNED) return valid > 0 ? *reinterpret_cast<const Frag<T> *>(p) : Frag<T>{};
    else return __builtin_bit_cast(Frag<T>, load_piece(p, (int)max(min(valid, (int64_t)PIECE<T>), (int64_t)0)));
}

// The waves' sums meet: [wave][row][column], a line of columns padded by four so that rows lie on different banks.
template <class T, int TM, int TN, int WAVES, class Store>
__device__ __forceinline__ void few_finish(const f32x4 (&acc)[TM][TN], const float (&first)[(TM * TN * 256 + WAVES * WAVE - 1) / (WAVES * WAVE)], int rows,
                                           int64_t n0, int64_t n, float *lds, Store store)
{
    const int lane = lane_id(), r = lane % 16, g = lane / 16, wave = threadIdx.x / WAVE;
    constexpr int COLS = TN * 16, LD = COLS + 4;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) *reinterpret_cast<f32x4 *>(lds + (wave * TM * 16 + i * 16 + r) * LD + j * 16 + g * 4) = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int o = 0; o < (TM * TN * 256 + WAVES * WAVE - 1) / (WAVES * WAVE); ++o) {
        const int k = o * WAVES * WAVE + threadIdx.x, row = k / COLS, col = k % COLS;
        if (row >= rows || n0 + col >= n) continue;
        float v = 0.0f;
#pragma unroll
        for (int s = 0; s < WAVES; ++s) v += lds[(s * TM * 16 + row) * LD + col];
        store(row, n0 + col, v + first[o]);
    }
}

// What is added to the products of this thread's results, worked out before they are (its loads are under way with theirs).
template <int TM, int TN, int WAVES, class First>
__device__ __forceinline__ void few_first(float (&first)[(TM * TN * 256 + WAVES * WAVE - 1) / (WAVES * WAVE)], int rows, int64_t n0, int64_t n, First f)
{
#pragma unroll
    for (int o = 0; o < (TM * TN * 256 + WAVES * WAVE - 1) / (WAVES * WAVE); ++o) {
        const int k = o * WAVES * WAVE + threadIdx.x, row = k / (TN * 16), col = k % (TN * 16);
        first[o] = row < rows && n0 + col < n ? f(row, n0 + col) : 0.0f;
    }
}

// The workgroup's columns, n0 .. n0 + 16 TN - 1, of `rows` rows (1 .. 16 TM), numbers row_of[] of x (-1: what comes of it is not
// used).  store(row, column, sum) is called once for each of them that there is; the sum begins with first(row, column).
template <class T, int TM, int TN, int WAVES, bool ALIGNED, class First, class Store>
__device__ __forceinline__ void few_tile(const T *x, int64_t ldx, const int64_t *row_of, int rows, const T *w, int64_t ldw, int64_t n0, int64_t n,
                                         int64_t c, float *lds, First f, Store store)
{
    float first[(TM * TN * 256 + WAVES * WAVE - 1) / (WAVES * WAVE)];
    few_first<TM, TN, WAVES>(first, rows, n0, n, f);
    const int lane = lane_id(), r = lane % 16, g = lane / 16, wave = threadIdx.x / WAVE;
    constexpr int S = STEP<T>, P = PIECE<T>, UNROLL = TM + TN <= 3 ? 4 : 2;
    const T *xp[TM], *wp[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) xp[i] = x + max(row_of[min(i * 16 + r, rows - 1)], (int64_t)0) * ldx + g * P;
#pragma unroll
    for (int j = 0; j < TN; ++j) wp[j] = w + min(n0 + j * 16 + r, n - 1) * ldw + g * P;
    f32x4 acc[TM][TN] = {};
    const int64_t whole = c / S;   // steps without a tail
    int64_t t = wave;
    for (; t + (UNROLL - 1) * WAVES < whole; t += UNROLL * WAVES) {
        Frag<T> fw[UNROLL][2][TN], fx[UNROLL][2][TM];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t at = (t + u * WAVES) * S + h * 4 * P;
#pragma unroll
                for (int j = 0; j < TN; ++j) fw[u][h][j] = few_load<T, ALIGNED>(wp[j] + at, P);
#pragma unroll
                for (int i = 0; i < TM; ++i) fx[u][h][i] = few_load<T, ALIGNED>(xp[i] + at, P);
            }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) mma<T>(acc, fw[u][h], fx[u][h]);
    }
    for (; t * S < c; t += WAVES) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = t * S + h * 4 * P, valid = c - at - g * P;
            Frag<T> fw[TN], fx[TM];
#pragma unroll
            for (int j = 0; j < TN; ++j) fw[j] = few_load<T, ALIGNED>(wp[j] + at, valid);
#pragma unroll
            for (int i = 0; i < TM; ++i) fx[i] = few_load<T, ALIGNED>(xp[i] + at, valid);
            mma<T>(acc, fw, fx);
        }
    }
    few_finish<T, TM, TN, WAVES>(acc, first, rows, n0, n, lds, store);
}

// The same where a line of the right matrix is one c (its columns lie side by side).  The matrix cores want 8
// (4) c of one column in a lane, so the lines pass through LDS, which gives them back transposed: each wave has a ring of RING pieces of its own,
// 4 KB (32 or 16 lines of 64 columns) each, filled FEW_RING - 1 ahead, straight from memory or (unaligned) through registers; no wave waits for another.  `lds` holds
// the rings, then the sums.
constexpr int FEW_COLS = 64, FEW_RING = 4, FEW_STAGE = 4096;
template <class T, int TM, int WAVES, bool ALIGNED, class Store>
__device__ __forceinline__ void few_tile_col(const T *x, int64_t ldx, const int64_t *row_of, int rows, const T *w, int64_t ldw, int64_t n0, int64_t n,
                                             int64_t c, char *lds, Store store)
{
    const int lane = lane_id(), r = lane % 16, g = lane / 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    constexpr int P = PIECE<T>, LINES = STEP<T> / 2, LOADS = FEW_STAGE / 16 / WAVE, TN = FEW_COLS / 16;
    char *ring = lds + wave * FEW_RING * FEW_STAGE;
    using Stage = Tile<T, true, false, FEW_COLS, WAVE, 64>;
    const uint32_t at_w = Stage::place(0);
    const T *xp[TM], *wp[LOADS];
    int line[LOADS], room[LOADS];   // (columns of a piece that there are)
    uint4 kept[FEW_RING][ALIGNED ? 1 : LOADS];
#pragma unroll
    for (int i = 0; i < TM; ++i) xp[i] = x + max(row_of[min(i * 16 + r, rows - 1)], (int64_t)0) * ldx + g * P;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int64_t col = n0 + Stage::piece_of(lane, i) * P;
        line[i] = Stage::line_of(lane, i);
        wp[i] = w + line[i] * ldw + (ALIGNED ? min(col, n - P) : col);
        room[i] = (int)max(min(n - col, (int64_t)P), (int64_t)0);
    }
    const int64_t stages = (c + LINES - 1) / LINES;                                  // of all waves, taken in turn
    const int64_t mine = stages > wave ? (stages - wave + WAVES - 1) / WAVES : 0;     // of this wave
    auto fill = [&](int64_t k, int slot, Frag<T> (&fx)[TM], uint4 (&kept_now)[ALIGNED ? 1 : LOADS]) {
        const int64_t c0 = (wave + k * WAVES) * LINES;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            if constexpr (!ALIGNED) kept_now[i] = load_piece(wp[i] + c0 * ldw, c0 + line[i] < c ? room[i] : 0);
            else load_to_lds(c0 + line[i] < c ? static_cast<const void *>(wp[i] + c0 * ldw) : &g_zero_piece, ring + slot * FEW_STAGE + i * WAVE * 16);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) fx[i] = few_load<T, ALIGNED>(xp[i] + c0, c - c0 - g * P);
    };
    f32x4 acc[TM][TN] = {};
    Frag<T> fx[FEW_RING][TM];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < FEW_RING - 1; ++k)
        if (k < mine) fill(k, k, fx[k], kept[k]);
    for (int64_t k0 = 0; k0 < mine; k0 += FEW_RING) {
#pragma unroll
        for (int u = 0; u < FEW_RING; ++u) {
            const int64_t k = k0 + u;
            if (k >= mine) break;
            // The slot that is filled next was read in the turn before: those reads have come back.
            __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
            const bool more = k + FEW_RING - 1 < mine;
            if (more) fill(k + FEW_RING - 1, (u + FEW_RING - 1) % FEW_RING, fx[(u + FEW_RING - 1) % FEW_RING], kept[(u + FEW_RING - 1) % FEW_RING]);
            // Loads come back in order: all but those of the FEW_RING - 1 stages behind this one.
            // (Each is one instruction: some lane's c lies before the end.)
            [[maybe_unused]] constexpr int LATER = (FEW_RING - 1) * (LOADS + TM);
            if constexpr (!ALIGNED) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) *reinterpret_cast<uint4 *>(ring + u * FEW_STAGE + (i * WAVE + lane) * 16) = kept[u][i];
                __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
            } else {
                asm volatile("" ::: "memory");
                if (more) __builtin_amdgcn_s_waitcnt(0x0f70 | (LATER & 15) | (LATER >> 4) << 14);
                else __builtin_amdgcn_s_waitcnt(0x0f70);
            }
            wave_sync();
            Frag<T> fw[TN];
            Stage::template read<0>(ring + u * FEW_STAGE, at_w, fw);
            mma<T>(acc, fw, fx[u]);
            wave_sync();
        }
    }
    const float first[(TM * TN * 256 + WAVES * WAVE - 1) / (WAVES * WAVE)] = {};
    few_finish<T, TM, TN, WAVES>(acc, first, rows, n0, n, reinterpret_cast<float *>(lds), store);
}

}  // namespace

}  // namespace ocean
