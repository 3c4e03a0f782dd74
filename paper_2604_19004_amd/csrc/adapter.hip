// A shared projection with a low-rank adapter for each row beside it, adapters of many requests in one batch.
//
// Few rows: a wave forms four of a row's inner products with its adapter, then a workgroup that has a few columns of the shared projection
// begins each result with the adapter's part, a dot product over the rank in 32 bits.
// More: rows are put in the order of their adapters, x * A^T is a product of ragged groups (few columns: c is cut into stretches to fill
// the chip, the stretches' sums are added up in a fixed order), and the shared projection's tiles go on, after their own c, with the products with B.
#include "few.hpp"

namespace ocean {

namespace {

inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

struct AdapterSpace {
    int32_t *perm;        // [rows] row of each slot
    int32_t *slot_id;     // [rows] its adapter, -1: none
    int64_t *ptr;         // [adapters + 1] slots of each adapter; those without one follow
    float *part;          // [stretches][rows][rank_up]
    void *h;              // [rows][parts * rank_up]
    float *row_scale;     // [rows]
    int64_t stretches, c_part;
    int rank_up;
    size_t bytes;
};

AdapterSpace adapter_space(void *at, int64_t rows, int64_t inner, int64_t adapters, int64_t rank, int dtype)
{
    AdapterSpace w{};
    const int size = type_size(dtype), e = 16 / size, step = LINE / size;
    w.rank_up = (int)((rank + e - 1) / e * e);
    // enough workgroups for two on each compute unit, and four steps at least in a stretch
    const int64_t tiles = std::max<int64_t>(1, (rows + 63) / 64 * ((rank + 63) / 64)), steps = (inner + step - 1) / step;
    w.stretches = std::max<int64_t>(1, std::min((512 + tiles - 1) / tiles, steps / 4));
    w.c_part = std::max<int64_t>(1, (steps + w.stretches - 1) / w.stretches) * step;
    w.stretches = std::max<int64_t>(1, (inner + w.c_part - 1) / w.c_part);
    char *p = static_cast<char *>(at);
    auto take = [&](size_t n) { char *q = p + w.bytes; w.bytes += up256(n); return q; };
    w.perm = reinterpret_cast<int32_t *>(take((size_t)rows * 4));
    w.slot_id = reinterpret_cast<int32_t *>(take((size_t)rows * 4));
    w.ptr = reinterpret_cast<int64_t *>(take((size_t)(adapters + 1) * 8));
    w.part = reinterpret_cast<float *>(take((size_t)w.stretches * rows * w.rank_up * 4));
    w.row_scale = reinterpret_cast<float *>(take((size_t)rows * 4));
    w.h = take((size_t)rows * w.rank_up * (size == 2 ? 2 : 1) * size);
    return w;
}

// Slots of every adapter.  The order of an adapter's rows is that of arrival and may change from call to call: no result depends on
// it, since a row's sums do not depend on its place in a tile.  One workgroup (6000 rows 8 us of the 255 that all of it takes).
__global__ void __launch_bounds__(1024) k_order_rows(const int32_t *ids, int64_t rows, int adapters, AdapterSpace w)
{
    __shared__ uint32_t s_at[OCEAN_ADAPTER_MAX + 1];
    __shared__ uint32_t s_wave[1024 / WAVE];
    for (int e = threadIdx.x; e <= adapters; e += 1024) s_at[e] = 0;
    __syncthreads();
    // Rows side by side often have the same adapter: a wave takes the places of up to four of them at once, the others one by one.
    auto take = [&](bool there, uint32_t e, auto got) {
        for (int i = 0; i < 4; ++i) {
            const unsigned long long left = __ballot(there);
            if (!left) return;
            const uint32_t first = wave_read_lane_u32(e, __ffsll(left) - 1);
            const unsigned long long same = __ballot(there && e == first);
            uint32_t at = 0;
            if (lane_id() == __ffsll(same) - 1) at = atomicAdd(&s_at[first], (uint32_t)__popcll(same));
            at = wave_read_lane_u32(at, __ffsll(same) - 1);
            if (there && e == first) {
                got(at + (uint32_t)__popcll(same & ((1ull << lane_id()) - 1)));
                there = false;
            }
        }
        if (there) got(atomicAdd(&s_at[e], 1u));
    };
    for (int64_t i0 = 0; i0 < rows; i0 += 1024) {
        const int64_t i = i0 + threadIdx.x;
        take(i < rows, i < rows ? min((uint32_t)ids[i], (uint32_t)adapters) : 0u, [](uint32_t) {});
    }
    __syncthreads();
    uint32_t before = 0;
    for (int e0 = 0; e0 <= adapters; e0 += 1024) {
        const int e = e0 + threadIdx.x;
        const uint32_t n = e <= adapters ? s_at[e] : 0u, incl = wave_inclusive_scan_u32(n);
        if (lane_id() == WAVE - 1) s_wave[threadIdx.x / WAVE] = incl;
        __syncthreads();
        uint32_t mine = before + incl - n;
        for (int i = 0; i < 1024 / WAVE; ++i) {
            if (i < (int)threadIdx.x / WAVE) mine += s_wave[i];
            before += s_wave[i];
        }
        if (e <= adapters) {
            s_at[e] = mine;
            w.ptr[e] = mine;   // (of `adapters`: where those without one begin)
        }
        __syncthreads();
    }
    for (int64_t i0 = 0; i0 < rows; i0 += 1024) {
        const int64_t i = i0 + threadIdx.x;
        const uint32_t e = i < rows ? min((uint32_t)ids[i], (uint32_t)adapters) : 0u;
        take(i < rows, e, [&](uint32_t at) {
            w.perm[at] = (int32_t)i;
            w.slot_id[at] = e < (uint32_t)adapters ? (int32_t)e : -1;
        });
    }
}

// h = scale * the stretches' sums, one wave a slot.  The row is divided by the power of two of its largest finite magnitude (row_scale, given
// back when its products are added), and a 16-bit type holds it as its rounding and the rounding of what is left: 16 or 22 bits
// together; 8 or 11 alone would be off by as much as the result's own rounding.  float16 ends at 2^-24, so the row's largest is put at 2^14: of a
// number beside a much larger one 2^-39 of that may be lost, and nothing overflows.  Of an infinity nothing is left.  Columns behind the
// adapter's rank are 0.
template <class T>
__global__ void __launch_bounds__(256) k_finish_shrink(AdapterSpace w, int64_t rows, int rank, const int32_t *ranks, const float *scale)
{
    constexpr int MOST = OCEAN_ADAPTER_MAX_RANK / WAVE;
    const int lane = lane_id();
    const int64_t n = rows * w.rank_up;
    for (int64_t slot = (int64_t)blockIdx.x * (256 / WAVE) + threadIdx.x / WAVE; slot < rows; slot += (int64_t)gridDim.x * (256 / WAVE)) {
        const int id = w.slot_id[slot];
        if (id < 0) continue;
        const int used = ranks ? min(ranks[id], rank) : rank;
        const float c = scale ? scale[id] : 1.0f;
        float v[MOST] = {};
        uint32_t largest = 0;
#pragma unroll
        for (int i = 0; i < MOST; ++i) {
            const int r = i * WAVE + lane;
            if (r < used) {
                for (int64_t s = 0; s < w.stretches; ++s) v[i] += w.part[s * n + slot * w.rank_up + r];
                v[i] *= c;
            }
            const uint32_t magnitude = __float_as_uint(v[i]) & 0x7fffffffu;
            if (magnitude < 0x7f800000u) largest = max(largest, magnitude);
        }
        largest = wave_max_u32(largest);
        constexpr int TOP = std::is_same<T, f16_t>::value ? 14 : 0;   // the exponent that the largest is given
        const int exponent = max((int)(largest >> 23) - TOP, 1) - 127;
        if (lane == 0) w.row_scale[slot] = ldexpf(1.0f, exponent);
        T *h = static_cast<T *>(w.h);
#pragma unroll
        for (int i = 0; i < MOST; ++i) {
            const int r = i * WAVE + lane;
            if (r >= w.rank_up) continue;
            const float x = ldexpf(v[i], -exponent);
            if constexpr (sizeof(T) == 4) {
                h[slot * w.rank_up + r] = x;
            } else {
                const T hi = (T)x;
                h[slot * 2 * w.rank_up + r] = hi;
                h[slot * 2 * w.rank_up + w.rank_up + r] = isinf(x) ? (T)0.0f : (T)(x - (float)hi);
            }
        }
    }
}

// Few rows.  h[row][r .. r + 3] = scale * x[row] * A^T, one wave each; nothing for rows without an adapter and behind its rank.  Bound by the wave's
// own chain of loads (48 rows, rank 16, c = 4096 in bfloat16: 5 us).
constexpr int FEW_R = 4;
template <class T, bool ALIGNED>
__global__ void __launch_bounds__(256) k_shrink_few(ocean_adapters l, const int32_t *ids, const T *x, int64_t ldx, int64_t inner, int64_t rows,
                                                    float *h, int rank_up)
{
    const int parts = (int)((l.rank + FEW_R - 1) / FEW_R), lane = lane_id();
    const int64_t item = (int64_t)blockIdx.x * (256 / WAVE) + threadIdx.x / WAVE;
    if (item >= rows * parts) return;
    const int64_t row = item / parts;
    const int r0 = (int)(item - row * parts) * FEW_R;
    const int64_t id = ids[row];
    if ((uint64_t)id >= (uint64_t)l.adapters) return;
    const int used = l.ranks ? (int)min((int64_t)l.ranks[id], l.rank) : (int)l.rank;
    if (r0 >= used) return;
    const T *xr = x + row * ldx, *ar[FEW_R];
#pragma unroll
    for (int j = 0; j < FEW_R; ++j) ar[j] = static_cast<const T *>(l.a) + id * l.stride_a + min(r0 + j, used - 1) * l.ld_a;
    constexpr int P = PIECE<T>;
    float sum[FEW_R] = {};
#pragma unroll 2
    for (int64_t c = lane * P; c < inner; c += WAVE * P) {
        const Frag<T> v = few_load<T, ALIGNED>(xr + c, inner - c);
#pragma unroll
        for (int j = 0; j < FEW_R; ++j) {
            const Frag<T> a = few_load<T, ALIGNED>(ar[j] + c, inner - c);
#pragma unroll
            for (int i = 0; i < P; ++i) sum[j] += (float)v[i] * (float)a[i];
        }
    }
#pragma unroll
    for (int j = 0; j < FEW_R; ++j) {
        const float v = wave_sum(sum[j]);
        if (lane == 0 && r0 + j < used) h[row * rank_up + r0 + j] = l.scale ? v * l.scale[id] : v;
    }
}

// The shared projection of 16, 32, 48 or 64 rows (blockIdx.y-th 64) and TN * 16 columns, each result begun with the adapter's part.  Up to 16 rows it
// is bound by W's bytes (4096 x 4096 in bfloat16: 9 us), with more by the rows, which every workgroup reads from the L2 (48: 19 us, 17 without adapters).
constexpr int FEW_ROWS = 64;
// Few rows: up to 128, and more while one round holds the workgroups, two on a compute unit, and the adapters' rows, which each row reads for itself, are
// not many.  In bfloat16, rows of 24 adapters, without tiles and in them, us:
//   up to 128 rows, 4096 x 4096: 128 of rank 16 38 and 52, 64 57 and 75, 256 132 and 191 (192 rows, 64 adapters of rank 16: 61 and 61).  Who shares an adapter is
//   not known here: all rows with the same one take 36 and 44, 54 and 46, 130 and 68, each with its own 39 and 90, 72 and 199, 217 and 776;
//   2048 -> 2048, 128 rows of rank 64 29 and 58; wider results are less apart (4096 -> 8192, 128 of rank 16 60 and 53).
//   512 workgroups: 256 x 2048 -> 2048 28 and 33 (rank 16), 43 and 45 (64); 513: 192 x 2000 -> 2736 35 and 33, 57 and 49.
//   Lines of 10 KB: 256 x 5000 -> 2048 49 and 55, 65 and 66; 6144 -> 2048 68 and 64, 83 and 75, but 256 workgroups, 192 x 6144 -> 1360, 42 and 64, 54 and 80.
//   In single precision tiles are slower at any length: 256 x 8192 -> 2048 167 and 240, 192 and 253.
//   Rows * rank: 512 x 2000 -> 512 of rank 64 34 and 37, 640 columns 43 and 38 (256 x 1280 of rank 64, 16384: 38 and 43).
inline bool few_enough(int64_t rows, int64_t inner, int64_t outer, int64_t rank, int size)
{
    if (outer >= 1ll << 27) return false;   // (a launch has fewer than 2^32 threads, 512 for 16 columns)
    const int64_t workgroups = (outer + 15) / 16 * ((rows + FEW_ROWS - 1) / FEW_ROWS);
    return rows <= 128 || (rows * rank <= 20480 && workgroups <= (size == 4 || inner * size <= 10240 ? 512 : 256));
}
template <class T, int TN, int WAVES, bool ALIGNED>
__global__ void __launch_bounds__(WAVES * WAVE, 2) k_adapter_few(ocean_adapters l, const int32_t *ids, const T *x, int64_t ldx, int64_t inner, int64_t rows,
                                                                 const T *w, int64_t ldw, int64_t outer, T *y, int64_t ldy, const float *h, int rank_up)
{
    __shared__ __align__(16) float s_sum[WAVES * FEW_ROWS * (TN * 16 + 4)];
    __shared__ int64_t s_row[FEW_ROWS];
    __shared__ int32_t s_id[FEW_ROWS], s_used[FEW_ROWS];
    const int64_t m0 = (int64_t)blockIdx.y * FEW_ROWS, n0 = (int64_t)blockIdx.x * TN * 16;
    const int count = (int)min((int64_t)FEW_ROWS, rows - m0);
    if ((int)threadIdx.x < count) {
        const int64_t id = ids[m0 + threadIdx.x];
        const bool has = (uint64_t)id < (uint64_t)l.adapters;
        s_row[threadIdx.x] = m0 + threadIdx.x;
        s_id[threadIdx.x] = has ? (int32_t)id : 0;
        s_used[threadIdx.x] = !has ? 0 : l.ranks ? (int)min((int64_t)l.ranks[id], l.rank) : (int)l.rank;
    }
    __syncthreads();
    auto first = [&](int row, int64_t col) {
        const int used = s_used[row];
        float v = 0.0f;
        if (used > 0) {
            const T *b = static_cast<const T *>(l.b) + (int64_t)s_id[row] * l.stride_b + col * l.ld_b;
            const float *hr = h + (m0 + row) * rank_up;
#pragma unroll 4
            for (int r = 0; r < used; r += PIECE<T>) {
                const Frag<T> p = __builtin_bit_cast(Frag<T>, load_piece(b + r, used - r));
#pragma unroll
                for (int i = 0; i < PIECE<T>; ++i)
                    if (r + i < used) v += hr[r + i] * (float)p[i];
            }
        }
        return v;
    };
    auto store = [&](int row, int64_t col, float v) { y[(m0 + row) * ldy + col] = (T)v; };
    auto tile = [&](auto tm) {
        few_tile<T, decltype(tm)::value, TN, WAVES, ALIGNED>(x, ldx, s_row, count, w, ldw, n0, outer, inner, s_sum, first, store);
    };
    if (count <= 16) tile(std::integral_constant<int, 1>{});
    else if (count <= 32) tile(std::integral_constant<int, 2>{});
    else if (count <= 48) tile(std::integral_constant<int, 3>{});
    else tile(std::integral_constant<int, 4>{});
}

template <class T>
hipError_t launch_few_rows(const ocean_adapters &l, const int32_t *ids, int64_t rows, int64_t inner, int64_t outer, const T *x, int64_t ldx, const T *w,
                           int64_t ldw, T *y, int64_t ldy, float *h, int rank_up, bool none, hipStream_t s)
{
    const int size = sizeof(T);
    ocean_adapters used = l;
    if (none) used.adapters = 0;
    if (!none) {
        const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(l.a, l.ld_a, l.stride_a, size) && inner % PIECE<T> == 0;
        const dim3 grid((uint32_t)((rows * ((l.rank + FEW_R - 1) / FEW_R) + 3) / 4));
        if (aligned) hipLaunchKernelGGL((k_shrink_few<T, true>), grid, dim3(256), 0, s, used, ids, x, ldx, inner, rows, h, rank_up);
        else hipLaunchKernelGGL((k_shrink_few<T, false>), grid, dim3(256), 0, s, used, ids, x, ldx, inner, rows, h, rank_up);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(w, ldw, 0, size) && inner % PIECE<T> == 0;
    auto launch = [&](auto tn, auto waves, auto al) {
        constexpr int TN = decltype(tn)::value, WAVES = decltype(waves)::value;
        const dim3 grid((uint32_t)((outer + TN * 16 - 1) / (TN * 16)), (uint32_t)((rows + FEW_ROWS - 1) / FEW_ROWS));
        hipLaunchKernelGGL((k_adapter_few<T, TN, WAVES, decltype(al)::value>), grid, dim3(WAVES * WAVE), 0, s, used, ids, x, ldx, inner, rows, w, ldw,
                           outer, y, ldy, h, rank_up);
        return hipGetLastError();
    };
    const std::integral_constant<int, 1> one{};
    const std::integral_constant<int, 2> two{};
    const std::integral_constant<int, 8> eight{};
    // Columns of a workgroup: every one reads all rows, and all compute units should have one (64 adapters of rank 16, 4096 x 4096: 32 rows 23
    // us with 16 columns and 27 with 32, 96 rows 42 and 38; 4096 x 1024, 48 rows 37 and 48).
    if (rows > 64 && outer >= 4096) return aligned ? launch(two, eight, std::true_type{}) : launch(two, eight, std::false_type{});
    return aligned ? launch(one, eight, std::true_type{}) : launch(one, eight, std::false_type{});
}

}  // namespace

size_t adapter_workspace(int64_t rows, int64_t inner, int64_t outer, int64_t adapters, int64_t rank, int dtype)
{
    return adapter_space(nullptr, rows, inner, adapters, rank, dtype).bytes;
}

hipError_t launch_adapter(const ocean_adapters &l, const int32_t *ids, int dtype, int64_t rows, int64_t inner, int64_t outer, const void *x,
                          int64_t ldx, const void *w, int64_t ldw, void *y, int64_t ldy, void *workspace, hipStream_t s)
{
    if (rows == 0 || outer == 0) return hipSuccess;
    const int size = type_size(dtype), e = 16 / size, rank = (int)l.rank;
    const bool none = l.adapters == 0 || rank == 0 || inner == 0;
    const int64_t adapters = none ? 0 : l.adapters;
    const bool x_fits = offsets_fit(std::max<int64_t>(rows, 256), ldx, size);
    const AdapterSpace sp = adapter_space(workspace, rows, inner, l.adapters, l.rank, dtype);
    if (few_enough(rows, inner, outer, l.rank, size)) {
        return with_type(dtype, [&](auto t) {
            using T = decltype(t);
            return launch_few_rows(l, ids, rows, inner, outer, static_cast<const T *>(x), ldx, static_cast<const T *>(w), ldw, static_cast<T *>(y), ldy,
                                   sp.part, sp.rank_up, none, s);
        });
    }
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        GmmArgs shrink{};
        shrink.l = x, shrink.ldl = ldx, shrink.rows = rows, shrink.c = inner;
        shrink.index = sp.perm, shrink.index_rows = rows;
        GmmArgs a = shrink;
        shrink.r = l.a, shrink.ldr = l.ld_a, shrink.stride = l.stride_a;
        shrink.out = sp.part, shrink.ldo = sp.rank_up;
        shrink.ptr = sp.ptr, shrink.groups = adapters;
        shrink.n = rank, shrink.c_part = sp.c_part;
        a.r = w, a.ldr = ldw;
        a.out = y, a.ldo = ldy, a.n = outer;
        a.slot_id = sp.slot_id, a.adapters = adapters;
        a.h = sp.h, a.row_scale = sp.row_scale, a.b = l.b, a.ldb = l.ld_b, a.stride_b = l.stride_b, a.ranks = l.ranks, a.rank = rank, a.rank_up = sp.rank_up;
        const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(w, ldw, 0, size) && inner % e == 0 && x_fits && offsets_fit(256, ldw, size);
        if (!some_tile_launches<T, GM_EXPAND>(a, aligned) || (!none && !launches<GM_SHRINK>(shrink, 64, 64, 256))) return TOO_MANY_TILES;
        hipLaunchKernelGGL(k_order_rows, dim3(1), dim3(1024), 0, s, ids, rows, (int)adapters, sp);
        hipError_t r = hipGetLastError();
        if (r != hipSuccess) return r;
        if (!none) {
            const bool whole = pieces_aligned(x, ldx, 0, size) && pieces_aligned(l.a, l.ld_a, l.stride_a, size) && inner % e == 0 && x_fits &&
                               offsets_fit(256, l.ld_a, size);
            r = whole ? launch_gmm<T, false, false, 64, 64, 4, 1, true, 2, GM_SHRINK, float>(shrink, s)
                      : launch_gmm<T, false, false, 64, 64, 4, 1, false, 2, GM_SHRINK, float>(shrink, s);
            if (r != hipSuccess) return r;
            hipLaunchKernelGGL((k_finish_shrink<T>), dim3((uint32_t)std::min((rows + 3) / 4, (int64_t)1 << 20)), dim3(256), 0, s, sp, rows, rank,
                               l.ranks, l.scale);
            r = hipGetLastError();
            if (r != hipSuccess) return r;
        }
        return launch_tiles<T, false, false, GM_EXPAND>(a, [&](int64_t bm) { return (rows + bm - 1) / bm; }, aligned, s);
    });
}

}  // namespace ocean
