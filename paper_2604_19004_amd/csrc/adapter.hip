// A shared projection with a low-rank adapter for each row beside it, adapters of many requests in one batch.
//
// Rows are put in the order of their adapters, x * A^T is a product of ragged groups (few columns: c is cut into stretches to fill
// the chip, the stretches' sums are added up in a fixed order), and the shared projection's tiles go on, after their own c, with the products with B.
#include "gmm.hpp"

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
// it, since a row's sums do not depend on its place in a tile.
__global__ void __launch_bounds__(1024) k_order_rows(const int32_t *ids, int64_t rows, int adapters, AdapterSpace w)
{
    __shared__ uint32_t s_at[OCEAN_ADAPTER_MAX + 1];
    __shared__ uint32_t s_wave[1024 / WAVE];
    for (int e = threadIdx.x; e <= adapters; e += 1024) s_at[e] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < rows; i += 1024) {
        const uint32_t e = min((uint32_t)ids[i], (uint32_t)adapters);
        atomicAdd(&s_at[e], 1u);
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
    for (int64_t i = threadIdx.x; i < rows; i += 1024) {
        const uint32_t e = min((uint32_t)ids[i], (uint32_t)adapters), at = atomicAdd(&s_at[e], 1u);
        w.perm[at] = (int32_t)i;
        w.slot_id[at] = e < (uint32_t)adapters ? (int32_t)e : -1;
    }
}

// h = scale * the stretches' sums, one wave a slot.  The row is divided by the power of two of its largest magnitude (row_scale, given
// back when its products are added), and a 16-bit type holds it as its rounding and the rounding of what is left: 16 or 22 bits
// together, whatever the range of the type; 8 or 11 alone would be off by as much as the result's own rounding.  Columns behind the
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
            largest = max(largest, __float_as_uint(v[i]) & 0x7fffffffu);
        }
        largest = wave_max_u32(largest);
        const int exponent = largest >= 0x7f800000u ? 0 : max((int)(largest >> 23), 1) - 127;   // (infinite or NaN rows stay as they are)
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
                h[slot * 2 * w.rank_up + w.rank_up + r] = (T)(x - (float)hi);
            }
        }
    }
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
    hipLaunchKernelGGL(k_order_rows, dim3(1), dim3(1024), 0, s, ids, rows, (int)adapters, sp);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        GmmArgs a{};
        a.l = x, a.ldl = ldx, a.rows = rows, a.c = inner;
        a.index = sp.perm, a.index_rows = rows;
        if (!none) {
            a.r = l.a, a.ldr = l.ld_a, a.stride = l.stride_a;
            a.out = sp.part, a.ldo = sp.rank_up;
            a.ptr = sp.ptr, a.groups = adapters;
            a.n = rank, a.c_part = sp.c_part;
            const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(l.a, l.ld_a, l.stride_a, size) && inner % e == 0 && x_fits &&
                                 offsets_fit(256, l.ld_a, size);
            hipError_t r = aligned ? launch_gmm<T, false, false, 64, 64, 4, 1, true, 2, GM_SHRINK, float>(a, s)
                                   : launch_gmm<T, false, false, 64, 64, 4, 1, false, 2, GM_SHRINK, float>(a, s);
            if (r != hipSuccess) return r;
            hipLaunchKernelGGL((k_finish_shrink<T>), dim3((uint32_t)std::min((rows + 3) / 4, (int64_t)1 << 20)), dim3(256), 0, s, sp, rows, rank,
                               l.ranks, l.scale);
            r = hipGetLastError();
            if (r != hipSuccess) return r;
        }
        a.r = w, a.ldr = ldw, a.stride = 0;
        a.out = y, a.ldo = ldy, a.n = outer;
        a.slot_id = sp.slot_id, a.adapter_ptr = sp.ptr, a.adapters = adapters;
        a.h = sp.h, a.row_scale = sp.row_scale, a.b = l.b, a.ldb = l.ld_b, a.stride_b = l.stride_b, a.ranks = l.ranks, a.rank = rank, a.rank_up = sp.rank_up;
        const bool aligned = pieces_aligned(x, ldx, 0, size) && pieces_aligned(w, ldw, 0, size) && inner % e == 0 && x_fits && offsets_fit(256, ldw, size);
        return launch_tiles<T, false, false, GM_EXPAND>(a, [&](int64_t bm) { return (rows + bm - 1) / bm; }, aligned, s);
    });
}

}  // namespace ocean
