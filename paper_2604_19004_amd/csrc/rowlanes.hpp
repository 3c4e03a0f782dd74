// Rows of logits in the lanes of a wave: their order, reductions over the lanes that share a row, how many lanes and columns each.
#pragma once

#include <type_traits>

#include "routed.hpp"

namespace ocean {

namespace {

// Whole numbers in the order of the values; 0 stands for a masked logit, below every other.  -0 and 0 are the same.
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b >> 31) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) { return __uint_as_float((key >> 31) ? (key & 0x7fffffffu) : ~key); }

template <class T> __device__ __forceinline__ uint32_t logit_key(T v)
{
    const float x = (float)v;
    if (!(x > TypeTraits<T>::lowest)) return 0;   // (NaN as well)
    return order_key(fminf(x, -TypeTraits<T>::lowest));
}

// Moves among the G lanes that share a row, every lane receiving the result: inside 16 lanes by lane swaps (neighbours, pairs, mirrored halves
// of 8, mirrored rows of 16), over the whole wave by the prefix moves of ocean_internal.hpp.  All lanes must be active.
template <class F> __device__ __forceinline__ uint32_t row16(uint32_t v, F f)
{
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));    // quad_perm [1,0,3,2]
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));    // quad_perm [2,3,0,1]
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));   // row_half_mirror
    return f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, false));   // row_mirror
}
template <int G> __device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    if constexpr (G == 16) return row16(v, [](uint32_t x, uint32_t y) { return max(x, y); });
    else return wave_max_u32(v);
}
template <int G> __device__ __forceinline__ float lanes_sum(float v)
{
    if constexpr (G == 16)
        return __uint_as_float(row16(__float_as_uint(v), [](uint32_t x, uint32_t y) { return __float_as_uint(__uint_as_float(x) + __uint_as_float(y)); }));
    else return wave_sum(v);
}

// Calls f with the lanes that share a row and the columns of a lane as constants.
template <class F> hipError_t with_columns(int64_t experts, F f)
{
    using std::integral_constant;
    if (experts <= 16) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (experts <= 32) return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
    if (experts <= 64) return f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    if (experts <= 128) return f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    if (experts <= 256) return f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    if (experts <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    return f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

}  // namespace

}  // namespace ocean
