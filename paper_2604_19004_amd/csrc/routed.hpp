// Declarations shared by the translation units of the routed products (ocean_routed.h): element types, small wave reductions, launches.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "ocean_internal.hpp"
#include "ocean_routed.h"

namespace ocean {

int set_error(int code, const char *msg) noexcept;   // ocean_api.hip: the message behind ocean_last_error

using bf16_t = __bf16;
using f16_t = _Float16;

template <class T> struct TypeTraits;
template <> struct TypeTraits<float> { static constexpr int code = OCEAN_F32; static constexpr float lowest = -3.402823466e38f; };
template <> struct TypeTraits<bf16_t> { static constexpr int code = OCEAN_BF16; static constexpr float lowest = -3.3895313892515355e38f; };
template <> struct TypeTraits<f16_t> { static constexpr int code = OCEAN_F16; static constexpr float lowest = -65504.0f; };

// What a launch function returns, and nothing has been launched then, where a result has more tiles than one launch takes.
constexpr hipError_t TOO_MANY_TILES = hipErrorInvalidConfiguration;

inline int type_size(int dtype) { return dtype == OCEAN_F32 ? 4 : 2; }

#if defined(__HIPCC__)
// V consecutive elements moved by one load or store.
template <class T, int V> struct alignas(sizeof(T) * V) Vec { T e[V]; };

// Sum over the 64 lanes of a wave, as a wave-uniform number, by the moves of wave_inclusive_scan_u32.  The tree is the same
// each time, and so is the rounding.  Every lane must be active.
__device__ __forceinline__ float wave_sum(float v)
{
    auto moved = [](float x, auto ctrl, auto rows) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
    };
    using std::integral_constant;
    v += moved(v, integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});   // row_shr:1
    v += moved(v, integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});   // row_shr:2
    v += moved(v, integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});   // row_shr:4
    v += moved(v, integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});   // row_shr:8
    v += moved(v, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // row_bcast:15, rows 1 and 3
    v += moved(v, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});   // row_bcast:31, rows 2 and 3
    return __uint_as_float(wave_read_lane_u32(__float_as_uint(v), WAVE - 1));
}
#endif

// Calls f with a value of the element type behind a dtype code.
template <class F> inline hipError_t with_type(int dtype, F f)
{
    if (dtype == OCEAN_F32) return f(float{});
    if (dtype == OCEAN_BF16) return f(bf16_t{});
    return f(f16_t{});
}

// route.hip
size_t route_workspace(int64_t tokens, int64_t experts, int32_t k);
hipError_t launch_route(const void *logits, int dtype, int64_t ld, bool normalize, const ocean_routing &r, void *workspace, hipStream_t s);
hipError_t launch_route_backward(const ocean_routing &r, const float *dval, const void *logits, int dtype, int64_t ld, bool normalize,
                                 void *dlogits, int64_t ldd, hipStream_t s);

// combine.hip
hipError_t launch_combine(const ocean_routing &r, const void *y, int dtype, int64_t width, int64_t ldy, void *out, int64_t ldo, hipStream_t s);
hipError_t launch_combine_backward(const ocean_routing &r, const void *dout, int64_t ldo, const void *y, int64_t ldy, int dtype,
                                   int64_t width, void *dy, int64_t lddy, float *dval, hipStream_t s);

// grouped.hip
hipError_t launch_grouped_matmul(const ocean_groups &g, int dtype, int64_t inner, int64_t outer, const void *x, int64_t ldx, const void *w,
                                 int64_t ldw, int64_t stride, bool transposed, void *y, int64_t ldy, hipStream_t s);
hipError_t launch_grouped_weight_grad(const ocean_groups &g, int dtype, int64_t inner, int64_t outer, const void *dy, int64_t lddy, const void *x,
                                      int64_t ldx, void *dw, int64_t lddw, int64_t stride, bool transposed, hipStream_t s);

// adapter.hip
size_t adapter_workspace(int64_t rows, int64_t inner, int64_t outer, int64_t adapters, int64_t rank, int dtype);
hipError_t launch_adapter(const ocean_adapters &l, const int32_t *ids, int dtype, int64_t rows, int64_t inner, int64_t outer, const void *x,
                          int64_t ldx, const void *w, int64_t ldw, void *y, int64_t ldy, void *workspace, hipStream_t s);

}  // namespace ocean
