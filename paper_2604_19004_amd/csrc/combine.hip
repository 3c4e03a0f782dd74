// The routing matrix times the dense rows that the experts gave, and its gradients.
#include <algorithm>
#include <initializer_list>

#include "routed.hpp"

namespace ocean {

namespace {

// The most elements a load takes, up to 16 bytes, such that no row of any of the matrices breaks its alignment.
struct Operand { const void *p; int64_t ld; };
int vector_width(int size, int64_t width, std::initializer_list<Operand> ops)
{
    int v = 16 / size;
    for (; v > 1; v >>= 1) {
        bool ok = width % v == 0;
        for (const Operand &o : ops) ok = ok && (o.p == nullptr || (reinterpret_cast<uintptr_t>(o.p) % (v * size) == 0 && o.ld % v == 0));
        if (ok) break;
    }
    return v;
}
template <class T, class F> hipError_t with_vector(int v, F f)
{
    if (v == 8) {
        if constexpr (sizeof(T) == 2) return f(std::integral_constant<int, 8>{});
    }
    if (v == 4) return f(std::integral_constant<int, 4>{});
    if (v == 2) return f(std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, 1>{});
}

// A row's entries, within the arrays whatever the offsets say.
__device__ __forceinline__ void row_range(const ocean_routing &r, int64_t t, int64_t &lo, int64_t &hi)
{
    const int64_t cap = r.tokens * r.k;
    lo = min(max(r.row_ptr[t], (int64_t)0), cap);
    hi = min(max(r.row_ptr[t + 1], lo), cap);
}

// out[t] = sum val[p] y[slot[p]].  Each thread has V elements of a row of the result and passes over the row's entries; bound by the rows' bytes, and
// a few rows by the launch (37 of 2047 in half precision, two entries each: 3 us).
template <class T, int V>
__global__ void __launch_bounds__(256) k_combine(ocean_routing r, const T *y, int64_t width, int64_t ldy, T *out, int64_t ldo, int64_t pieces)
{
    const int64_t cap = r.tokens * r.k;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < r.tokens * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / pieces, at = (i - t * pieces) * V;
        int64_t lo, hi;
        row_range(r, t, lo, hi);
        float sum[V] = {};
        for (int64_t p = lo; p < hi; ++p) {
            const int64_t slot = r.slot[p];
            if ((uint64_t)slot >= (uint64_t)cap) continue;
            const float w = r.val ? r.val[p] : 1.0f;
            const auto v = *reinterpret_cast<const Vec<T, V> *>(y + slot * ldy + at);
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += w * (float)v.e[j];
        }
        Vec<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.e[j] = (T)sum[j];
        *reinterpret_cast<Vec<T, V> *>(out + t * ldo + at) = o;
    }
}

// `split` waves a token, each with every split-th of its entries: the row of dout goes to the entries' rows, and its products with the rows that the
// experts gave are summed up across the lanes.  Rows that no entry names are cleared.  Bound by the bytes: 16384 rows of 2048 in bfloat16, four entries
// each, 125 us or 4.8 TB/s (a large copy has 4.9).
template <class T, int V>
__global__ void __launch_bounds__(256) k_combine_backward(ocean_routing r, const T *dout, int64_t ldo, const T *y, int64_t ldy, int64_t width,
                                                          T *dy, int64_t lddy, float *dval, int split)
{
    const int lane = lane_id();
    const int64_t wave = (int64_t)blockIdx.x * (256 / WAVE) + threadIdx.x / WAVE, waves = (int64_t)gridDim.x * (256 / WAVE), cap = r.tokens * r.k;
    const int64_t n = min(max(r.row_ptr[r.tokens], (int64_t)0), cap);
    for (int64_t item = wave; item < r.tokens * split; item += waves) {
        const int64_t t = item / split;
        int64_t lo, hi;
        row_range(r, t, lo, hi);
        for (int64_t p = lo + (item - t * split); p < hi; p += split) {
            const int64_t slot = r.slot[p];
            const bool there = (uint64_t)slot < (uint64_t)cap;
            const float w = r.val ? r.val[p] : 1.0f;
            float dot = 0.0f;
            if (there) {
                for (int64_t at = lane * V; at < width; at += WAVE * V) {
                    const auto d = *reinterpret_cast<const Vec<T, V> *>(dout + t * ldo + at);
                    Vec<T, V> o;
#pragma unroll
                    for (int j = 0; j < V; ++j) o.e[j] = (T)(w * (float)d.e[j]);
                    *reinterpret_cast<Vec<T, V> *>(dy + slot * lddy + at) = o;
                    if (dval) {
                        const auto v = *reinterpret_cast<const Vec<T, V> *>(y + slot * ldy + at);
#pragma unroll
                        for (int j = 0; j < V; ++j) dot += (float)d.e[j] * (float)v.e[j];
                    }
                }
            }
            if (dval) {
                dot = wave_sum(dot);
                if (lane == 0) dval[p] = dot;
            }
        }
    }
    for (int64_t s = n + wave; s < cap; s += waves) {
        for (int64_t at = lane * V; at < width; at += WAVE * V) *reinterpret_cast<Vec<T, V> *>(dy + s * lddy + at) = Vec<T, V>{};
        if (dval && lane == 0) dval[s] = 0.0f;
    }
}

}  // namespace

hipError_t launch_combine(const ocean_routing &r, const void *y, int dtype, int64_t width, int64_t ldy, void *out, int64_t ldo, hipStream_t s)
{
    if (r.tokens == 0 || width == 0) return hipSuccess;
    return with_type(dtype, [&](auto e) {
        using T = decltype(e);
        return with_vector<T>(vector_width(sizeof(T), width, {{y, ldy}, {out, ldo}}), [&](auto v) {
            constexpr int V = decltype(v)::value;
            const int64_t pieces = width / V;
            hipLaunchKernelGGL((k_combine<T, V>), dim3((uint32_t)std::min((r.tokens * pieces + 255) / 256, (int64_t)1 << 22)), dim3(256), 0, s, r,
                               static_cast<const T *>(y), width, ldy, static_cast<T *>(out), ldo, pieces);
            return hipGetLastError();
        });
    });
}

hipError_t launch_combine_backward(const ocean_routing &r, const void *dout, int64_t ldo, const void *y, int64_t ldy, int dtype,
                                   int64_t width, void *dy, int64_t lddy, float *dval, hipStream_t s)
{
    if (r.tokens == 0) return hipSuccess;
    return with_type(dtype, [&](auto e) {
        using T = decltype(e);
        return with_vector<T>(vector_width(sizeof(T), width, {{dout, ldo}, {dval ? y : nullptr, ldy}, {dy, lddy}}), [&](auto v) {
            constexpr int V = decltype(v)::value;
            // A wave an entry (16384 rows of 2048 in bfloat16, four entries each, 125 us and with a wave a row 133; 2019 of 6464 in single precision, seven
            // each, 164 and 271), but not where many rows are only written (without dval, 32768 of 1024, eight each, 169 and 131; 16384 of 2048 75 and 89).
            const int split = dval || r.tokens * r.k <= 65536 ? r.k : 1;
            hipLaunchKernelGGL((k_combine_backward<T, V>), dim3((uint32_t)std::min((r.tokens * split + 3) / 4, (int64_t)1 << 20)), dim3(256), 0, s, r,
                               static_cast<const T *>(dout), ldo, static_cast<const T *>(y), ldy, width, static_cast<T *>(dy), lddy, dval, split);
            return hipGetLastError();
        });
    });
}

}  // namespace ocean
