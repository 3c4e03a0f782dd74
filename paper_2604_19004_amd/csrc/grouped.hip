// Products of ragged groups of rows with their group's matrix, and the gradient of the matrices.
#include <algorithm>

#include "gmm.hpp"

namespace ocean {

namespace {

struct GmmArgs {
    const void *l, *r;
    void *out;
    int64_t ldl, ldr, ldo;
    int64_t stride;            // elements from a group's matrix (R, or with ragged c the output) to the next's
    const int64_t *ptr;        // groups + 1 offsets into `rows`
    int64_t groups, rows;      // rows: slots; the ragged dimension
    int64_t m, n, c;           // sizes of the dimensions that are not ragged
    const int32_t *index;      // row of x of each slot, or null
    int64_t index_rows;
    int index_on_r;            // (ragged c) x is the right operand
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

template <class T, bool LCOL, bool RCOL, int BM, int BN, int WAVES_M, int WAVES_N, bool ASYNC, bool RAGGED_C>
__global__ void __launch_bounds__(WAVES_M * WAVES_N * WAVE, 2) k_gmm(GmmArgs a, int64_t mt, int64_t nt)
{
    constexpr int THREADS = WAVES_M * WAVES_N * WAVE, WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 16, TN = WN / 16;
    static_assert(WN % 64 == 0, "four interleaved tiles");
    using TL = Tile<T, LCOL, false, BM, THREADS>;
    using TR = Tile<T, RCOL, true, BN, THREADS>;
    constexpr int BUFFER = TL::BYTES + TR::BYTES;
    __shared__ __align__(16) char lds[2 * BUFFER];

    int64_t mi, ni, group = 0, lo = 0, hi = 0, c_lo = 0, c_hi = a.c;
    const int64_t item = by_die(blockIdx.x, gridDim.x);
    if constexpr (RAGGED_C) {
        group = item / (mt * nt);
        if (group >= a.groups) return;
        banded(item - group * mt * nt, mt, nt, 4, mi, ni);
        group_range(a, group, c_lo, c_hi);
        lo = mi * BM;
        hi = a.m;
    } else {
        if (item >= mt * nt) return;
        banded(item, mt, nt, 4, mi, ni);
        int64_t used;
        if (!find_tile(a, mi, BM, group, lo, hi, used)) {   // no rows left: clear those of no group
            const int64_t first = min(max(a.ptr[0], (int64_t)0), a.rows), last = min(max(a.ptr[a.groups], first), a.rows);
            const int64_t outside = a.rows - (last - first), width = min((int64_t)BN, a.n - ni * BN);
            for (int64_t i = (mi - used) * BM; i < outside; i += (mt - used) * BM) {
                const int64_t count = min((int64_t)BM, outside - i) * width;
                for (int64_t k = threadIdx.x; k < count; k += THREADS) {
                    const int64_t row = i + k / width;
                    static_cast<T *>(a.out)[(row < first ? row : row - first + last) * a.ldo + ni * BN + k % width] = (T)0.0f;
                }
            }
            return;
        }
    }
    const int64_t n0 = ni * BN, m0 = lo;
    const T *lbase = static_cast<const T *>(a.l), *rbase = static_cast<const T *>(a.r) + (RAGGED_C ? 0 : group * a.stride);
    T *out = static_cast<T *>(a.out) + (RAGGED_C ? group * a.stride : 0);
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
            if (!RAGGED_C && a.index) {
                row = a.index[row];
                if ((uint64_t)row >= (uint64_t)a.index_rows) row = 0;   // (its result is replaced by 0)
            }
            lp[i] = lbase + row * a.ldl + piece * PIECE<T>;
        } else {
            const int64_t col = min(m0 + piece * PIECE<T>, ASYNC ? a.m - PIECE<T> : a.m);
            lp[i] = lbase + (c_lo + line) * a.ldl + col;
        }
    }
#pragma unroll
    for (int i = 0; i < TR::LOADS; ++i) {
        const int line = TR::line_of(i), piece = TR::piece_of(i);
        if constexpr (!RCOL) {
            rp[i] = rbase + min(n0 + line, a.n - 1) * a.ldr + piece * PIECE<T>;
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
            if (RAGGED_C && a.index && !a.index_on_r && c < depth) {
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
            if (RAGGED_C && a.index && a.index_on_r && c < depth) {
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
    const bool wide = a.ldo % PIECE<T> == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t row = m0 + wm + i * 16 + r;
        if (row >= hi) continue;
        bool zero = false;
        if (!RAGGED_C && a.index) zero = (uint64_t)(int64_t)a.index[row] >= (uint64_t)a.index_rows;
#pragma unroll
        for (int b = 0; b < TN / 4; ++b) {
            const int64_t col = n0 + wn + b * 64 + g * 16;
            T v[16];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) v[j * 4 + k] = (T)(zero ? 0.0f : acc[i][b * 4 + j][k]);
            T *p = out + row * a.ldo + col;
#pragma unroll
            for (int j = 0; j < 16; j += PIECE<T>) {
                if (wide && col + j + PIECE<T> <= a.n) {
                    Vec<T, PIECE<T>> o;
#pragma unroll
                    for (int k = 0; k < PIECE<T>; ++k) o.e[k] = v[j + k];
                    *reinterpret_cast<Vec<T, PIECE<T>> *>(p + j) = o;
                } else {
#pragma unroll
                    for (int k = 0; k < PIECE<T>; ++k)
                        if (col + j + k < a.n) p[j + k] = v[j + k];
                }
            }
        }
    }
}

inline int64_t up8(int64_t n) { return (n + 7) & ~(int64_t)7; }

template <class T, bool LCOL, bool RCOL, int BM, int BN, int WAVES_M, int WAVES_N, bool ASYNC, bool RAGGED_C>
hipError_t launch_gmm(const GmmArgs &a, hipStream_t s)
{
    const int64_t nt = (a.n + BN - 1) / BN;
    const int64_t mt = RAGGED_C ? (a.m + BM - 1) / BM : a.rows / BM + std::min(a.groups, a.rows) + 1;
    const int64_t blocks = up8(mt * nt * (RAGGED_C ? a.groups : 1));
    constexpr int threads = WAVES_M * WAVES_N * WAVE;
    if (blocks * threads >= (1ll << 32)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((k_gmm<T, LCOL, RCOL, BM, BN, WAVES_M, WAVES_N, ASYNC, RAGGED_C>), dim3((uint32_t)blocks), dim3(threads), 0, s, a, mt, nt);
    return hipGetLastError();
}

bool pieces_aligned(const void *p, int64_t ld, int64_t stride, int size)
{
    const int e = 16 / size;
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % e == 0 && stride % e == 0;
}

template <class T, bool LCOL, bool RCOL, bool RAGGED_C> hipError_t pick_tile(const GmmArgs &a, bool aligned, hipStream_t s)
{
    if constexpr (sizeof(T) == 2) {
        const int64_t rows = RAGGED_C ? a.m : a.rows / std::max<int64_t>(a.groups, 1);
        if (aligned && rows >= 256 && a.n >= 256) return launch_gmm<T, LCOL, RCOL, 256, 256, 2, 4, true, RAGGED_C>(a, s);
    }
    if (aligned) return launch_gmm<T, LCOL, RCOL, 128, 128, 2, 2, true, RAGGED_C>(a, s);
    return launch_gmm<T, LCOL, RCOL, 128, 128, 2, 2, false, RAGGED_C>(a, s);
}

}  // namespace

hipError_t launch_grouped_matmul(const ocean_groups &g, int dtype, int64_t inner, int64_t outer, const void *x, int64_t ldx, const void *w,
                                 int64_t ldw, int64_t stride, bool transposed, void *y, int64_t ldy, hipStream_t s)
{
    if (g.rows == 0 || outer == 0) return hipSuccess;
    const int size = type_size(dtype), e = 16 / size;
    GmmArgs a{x, w, y, ldx, ldw, ldy, stride, g.group_ptr, g.experts, g.rows, 0, outer, inner, g.row_index, g.x_rows, 0};
    if (g.x_rows == 0 || inner == 0) a.c = 0, a.index_rows = 0, a.index = nullptr;
    const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(w, ldw, stride, size) && inner % e == 0 && (!transposed || outer % e == 0);
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return transposed ? pick_tile<T, false, true, false>(a, aligned, s) : pick_tile<T, false, false, false>(a, aligned, s);
    });
}

hipError_t launch_grouped_weight_grad(const ocean_groups &g, int dtype, int64_t inner, int64_t outer, const void *dy, int64_t lddy, const void *x,
                                      int64_t ldx, void *dw, int64_t lddw, int64_t stride, bool transposed, hipStream_t s)
{
    if (g.experts == 0 || inner == 0 || outer == 0) return hipSuccess;
    const int size = type_size(dtype), e = 16 / size;
    // the matrix is outer x inner: its rows come from dy, its columns from x; transposed, the other way round
    GmmArgs a{transposed ? x : dy, transposed ? dy : x, dw, transposed ? ldx : lddy, transposed ? lddy : ldx, lddw, stride, g.group_ptr, g.experts,
              g.rows, transposed ? inner : outer, transposed ? outer : inner, 0, g.row_index, g.x_rows, transposed ? 0 : 1};
    if (g.x_rows == 0) a.rows = 0;   // (nothing to add up)
    const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(dy, lddy, 0, size) && inner % e == 0 && outer % e == 0;
    return with_type(dtype, [&](auto t) { return pick_tile<decltype(t), true, true, true>(a, aligned, s); });
}

}  // namespace ocean
