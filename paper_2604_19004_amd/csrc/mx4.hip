// Matrices to microscaled four bits and back.  Both are bound by memory: a lane has 8 numbers (16 bytes of a 16-bit type, 4 of codes), four
// lanes a block, and neighbouring lanes neighbouring numbers.  8192 x 4096, bf16: 16.3 to 17.8 us there, 85 MB at 4.8 to 5.2 TB/s
// as a copy, and 14.2 to 14.6 back, where the codes are still in the caches.
#include <algorithm>

#include "mx4.hpp"

namespace ocean {

namespace {

constexpr int TPB = 256;

// Calls f(matrix, row, unit, step) for the rows and the first unit (of 8 numbers) of this thread; 2^lanes_log threads share a row.  Threads of a
// block of 32 go together.
template <class F> __device__ __forceinline__ void each_row(const ocean_mx4 &q, int lanes_log, F f)
{
    const int per = TPB >> lanes_log;
    for (int64_t row = (int64_t)blockIdx.x * per + (threadIdx.x >> lanes_log); row < q.count * q.rows; row += (int64_t)gridDim.x * per) {
        const int64_t e = (uint32_t)row / (uint32_t)q.rows;   // (below 2^31)
        f(e, row - e * q.rows, (int)(threadIdx.x & ((1 << lanes_log) - 1)) + ((int)blockIdx.y << lanes_log), (int)gridDim.y << lanes_log);
    }
}

// (units: with those of the scales' padding)
template <class T, bool ALIGNED>
__global__ void __launch_bounds__(TPB) k_mx4_quantize(const T *x, int64_t ldx, int64_t stride, ocean_mx4 q, int units, int lanes_log)
{
    each_row(q, lanes_log, [&](int64_t e, int64_t i, int first, int step) {
        const T *from = x + e * stride + i * ldx;
        uint8_t *codes = q.codes + e * q.stride_codes + i * q.ld_codes, *scales = q.scales + e * q.stride_scales + i * q.ld_scales;
        for (int u = first; u < units; u += step) {
            T v[8];
            load8<T, ALIGNED>(from + (int64_t)u * 8, (int)min(max(q.inner - (int64_t)u * 8, (int64_t)0), (int64_t)8), v);
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint((float)v[k]) & 0x7fffffffu);
            top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false));   // quad_perm [1,0,3,2]
            top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false));   // quad_perm [2,3,0,1]
            const uint32_t s = mx4_scale_of(top);
            const bool block = (int64_t)(u & ~3) * 8 < q.inner;   // (else: padding of the scales)
            if (block) *reinterpret_cast<uint32_t *>(codes + (int64_t)u * 4) = s == 255u ? 0u : mx4_narrow(v, mx4_scale(s));
            if ((u & 3) == 0) scales[u / 4] = block ? (uint8_t)s : (uint8_t)0;
        }
    });
}

template <class T, bool ALIGNED>
__global__ void __launch_bounds__(TPB) k_mx4_dequantize(ocean_mx4 q, T *out, int64_t ldo, int64_t stride, int units, int lanes_log)
{
    each_row(q, lanes_log, [&](int64_t e, int64_t i, int first, int step) {
        const uint8_t *codes = q.codes + e * q.stride_codes + i * q.ld_codes, *scales = q.scales + e * q.stride_scales + i * q.ld_scales;
        T *to = out + e * stride + i * ldo;
        for (int u = first; u < units; u += step) {
            T v[8];
            mx4_widen<T>(*reinterpret_cast<const uint32_t *>(codes + (int64_t)u * 4), mx4_scale(scales[u / 4]), v);
            store8<T, ALIGNED>(to + (int64_t)u * 8, (int)min(q.inner - (int64_t)u * 8, (int64_t)8), v);
        }
    });
}

// Threads that share a row of `units`: a power of two (at most a workgroup's, at least a block's four), so that no thread divides; and the workgroups along it.
struct Shape { int lanes_log; dim3 grid; };
Shape shape_of(int64_t rows, int64_t units)
{
    int log = 2;
    while (log < 8 && (int64_t)1 << log < units) ++log;
    const int64_t per = TPB >> log, across = std::min<int64_t>((units + (1 << log) - 1) >> log, 64);
    return Shape{log, dim3((uint32_t)std::min<int64_t>((rows + per - 1) / per, 1 << 20), (uint32_t)across)};
}

}  // namespace

hipError_t launch_mx4_quantize(const void *x, int dtype, int64_t ldx, int64_t stride, const ocean_mx4 &q, hipStream_t s)
{
    if (q.count == 0 || q.rows == 0 || q.inner == 0) return hipSuccess;
    const int units = (int)((mx4_blocks(q.inner) + 15) / 16 * 64);
    const Shape shape = shape_of(q.count * q.rows, units);
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, shape.grid, dim3(TPB), 0, s, static_cast<const T *>(x), ldx, stride, q, units, shape.lanes_log);
            return hipGetLastError();
        };
        return pieces_aligned(x, ldx, stride, sizeof(T)) ? launch(k_mx4_quantize<T, true>) : launch(k_mx4_quantize<T, false>);
    });
}

hipError_t launch_mx4_dequantize(const ocean_mx4 &q, int dtype, void *out, int64_t ldo, int64_t stride, hipStream_t s)
{
    if (q.count == 0 || q.rows == 0 || q.inner == 0) return hipSuccess;
    const int units = (int)((q.inner + 7) / 8);
    const Shape shape = shape_of(q.count * q.rows, units);
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, shape.grid, dim3(TPB), 0, s, q, static_cast<T *>(out), ldo, stride, units, shape.lanes_log);
            return hipGetLastError();
        };
        return pieces_aligned(out, ldo, stride, sizeof(T)) ? launch(k_mx4_dequantize<T, true>) : launch(k_mx4_dequantize<T, false>);
    });
}

}  // namespace ocean
