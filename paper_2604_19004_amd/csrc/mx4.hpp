// Microscaled four bits in registers: 8 codes of a word to 8 numbers of a type and back, by the conversions of gfx950 (exact, and to the nearest
// with ties to the even code, over all scales, subnormal results and operands among them).
#pragma once

#include "experts.hpp"
#include "gmm.hpp"

namespace ocean {

namespace {

typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 mx_f16x2 __attribute__((ext_vector_type(2)));

// 2^(s - 127) as the conversions want it: they take the exponent's bits (0: 2^-127, 255: NaN).
__device__ __forceinline__ float mx4_scale(uint32_t s) { return __uint_as_float(s << 23); }

// The 8 numbers of a word.
template <class T> __device__ __forceinline__ void mx4_widen(uint32_t codes, float scale, T (&out)[8])
{
    auto pair = [&](auto sel) {
        constexpr int B = decltype(sel)::value;
        if constexpr (std::is_same<T, bf16_t>::value) {
            const mx_bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B);
            out[2 * B] = v[0], out[2 * B + 1] = v[1];
        } else {
            const mx_f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, B);
            out[2 * B] = (T)v[0], out[2 * B + 1] = (T)v[1];   // (float16: rounded here)
        }
    };
    pair(std::integral_constant<int, 0>{});
    pair(std::integral_constant<int, 1>{});
    pair(std::integral_constant<int, 2>{});
    pair(std::integral_constant<int, 3>{});
}

// The same as a fragment of the matrix instructions; float16 has all numbers whose scale is not far (below).
template <class T> __device__ __forceinline__ Frag<T> mx4_fragment(uint32_t codes, float scale)
{
    if constexpr (std::is_same<T, f16_t>::value) {
        const mx_f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1),
                       c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3);
        return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
        bf16_t e[8];
        mx4_widen<bf16_t>(codes, scale, e);
        return bf16x8{e[0], e[1], e[2], e[3], e[4], e[5], e[6], e[7]};
    }
}
// Whether float16 does not hold numbers of this scale: 6 * 2^(s - 127) is beyond it from 141 on, 2^(s - 128) is below its 2^-24 up to 103.  Numbers of scales up to
// 51 count as 0 there: 2^31 products of them with float16 numbers come to less than half its least number.  (255 stays NaN.)
__device__ __forceinline__ bool mx4_far(uint32_t s) { return (s > 140u && s != 255u) || (s > 51u && s < 104u); }

// Whether bfloat16 has no number for some of this scale's, which are infinite there (4 * 2^126 and on, 2 * 2^127 and on).
__device__ __forceinline__ bool mx4_infinite(uint32_t s) { return s - 253u < 2u; }

// And back.
template <class T> __device__ __forceinline__ uint32_t mx4_narrow(const T (&x)[8], float scale)
{
    uint32_t w = 0;
    auto pair = [&](auto sel) {
        constexpr int B = decltype(sel)::value;
        if constexpr (std::is_same<T, bf16_t>::value) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, mx_bf16x2{x[2 * B], x[2 * B + 1]}, scale, B);
        else if constexpr (std::is_same<T, f16_t>::value) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, mx_f16x2{x[2 * B], x[2 * B + 1]}, scale, B);
        else w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2 * B], x[2 * B + 1], scale, B);
    };
    pair(std::integral_constant<int, 0>{});
    pair(std::integral_constant<int, 1>{});
    pair(std::integral_constant<int, 2>{});
    pair(std::integral_constant<int, 3>{});
    return w;
}

// The scale's byte of a block whose largest magnitude has these bits: the exponent two lower (the largest number becomes 4 to 8 units), not below 2^-127.
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t top)
{
    const uint32_t exponent = top >> 23;
    return top == 0 ? 127u : exponent == 255u ? 255u : max(exponent, 2u) - 2u;
}

// 8 numbers at p, of which `valid` are there (0 for the others).
template <class T, bool ALIGNED> __device__ __forceinline__ void load8(const T *p, int valid, T (&out)[8])
{
    constexpr int E = PIECE<T>;
#pragma unroll
    for (int j = 0; j < 8 / E; ++j) {
        const uint4 v = ALIGNED && valid >= 8 ? reinterpret_cast<const uint4 *>(p)[j] : load_piece(p + j * E, valid - j * E);
        const Vec<T, E> e = __builtin_bit_cast(Vec<T, E>, v);
#pragma unroll
        for (int k = 0; k < E; ++k) out[j * E + k] = e.e[k];
    }
}
template <class T, bool ALIGNED> __device__ __forceinline__ void store8(T *p, int valid, const T (&x)[8])
{
    constexpr int E = PIECE<T>;
#pragma unroll
    for (int j = 0; j < 8 / E; ++j) {
        Vec<T, E> e;
#pragma unroll
        for (int k = 0; k < E; ++k) e.e[k] = x[j * E + k];
        if (valid >= (j + 1) * E) {
            if constexpr (ALIGNED) *reinterpret_cast<uint4 *>(p + j * E) = __builtin_bit_cast(uint4, e);
            else store_any<false>(p + j * E, e);
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (j * E + k < valid) p[j * E + k] = e.e[k];
        }
    }
}

// Codes of a word without those from the valid-th on.
__device__ __forceinline__ uint32_t mx4_first(uint32_t codes, int valid)
{
    return valid >= 8 ? codes : valid <= 0 ? 0u : codes & ((1u << (4 * valid)) - 1u);
}

}  // namespace

}  // namespace ocean
