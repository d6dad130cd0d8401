// MXFP4 elements on the device, shared by the quantisation and the products.
#pragma once

#include "gs_lowbit.h"

namespace gs {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Scale byte of a block whose largest magnitude has the bit pattern m.
__device__ __forceinline__ int mx4_exponent(uint32_t m)
{
    const int k = (int)(m >> 23);
    return k == 255 ? 255 : k > 2 ? k - 2 : 0;
}

typedef u16 u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Two bf16 numbers a word: the larger magnitudes, which order as their bits do.
__device__ __forceinline__ u16x2 larger_magnitudes(u16x2 top, uint32_t w)
{
    return __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w & 0x7fff7fffu));
}

// Elements 2 PAIR and 2 PAIR + 1 (two floats, or two bf16 in a word) under scale s =
// mx_scale() of their block, as e2m1 in byte PAIR of w: one rounding, to nearest even,
// and clamped, all by the conversion.
template <int PAIR> __device__ __forceinline__ uint32_t mx4_pair(uint32_t w, float a, float b, float s)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, s, PAIR);
}
template <int PAIR> __device__ __forceinline__ uint32_t mx4_pair(uint32_t w, uint32_t ab, float s)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, ab), s, PAIR);
}

// A lane's E elements of a block (4 or 8, of bf16 8).
template <class T, int E> struct Mx4Lane;
template <int E> struct Mx4Lane<float, E> {
    typename Elems<float, E>::type x;
    // Bit pattern (of fp32) of the largest magnitude.
    __device__ __forceinline__ uint32_t magnitude() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < E; e++) m = larger(m, __float_as_uint(x[e]) & 0x7fffffffu);
        return m;
    }
    // As e2m1, the first in the low bits; zeros for E8 = 255.
    __device__ __forceinline__ uint32_t codes(int E8) const
    {
        const float s = mx_scale(E8);
        uint32_t w = mx4_pair<1>(mx4_pair<0>(0, x[0], x[1], s), x[2], x[3], s);
        if constexpr (E == 8) w = mx4_pair<3>(mx4_pair<2>(w, x[4], x[5], s), x[6], x[7], s);
        return E8 == 255 ? 0 : w;
    }
};
template <> struct Mx4Lane<u16, 8> {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    words x;
    __device__ __forceinline__ Mx4Lane(const typename Elems<u16, 8>::type &v) : x(__builtin_bit_cast(words, v)) {}
    __device__ __forceinline__ uint32_t magnitude() const
    {
        u16x2 top = {};
#pragma unroll
        for (int p = 0; p < 4; p++) top = larger_magnitudes(top, x[p]);
        const uint32_t t = __builtin_bit_cast(uint32_t, top);
        return larger(t << 16, t & 0xffff0000u);
    }
    __device__ __forceinline__ uint32_t codes(int E8) const
    {
        const float s = mx_scale(E8);
        const uint32_t w = mx4_pair<3>(mx4_pair<2>(mx4_pair<1>(mx4_pair<0>(0, x[0], s), x[1], s), x[2], s), x[3], s);
        return E8 == 255 ? 0 : w;
    }
};

// X (rows x cols of dtype) along its rows into codes and scales in the layout
// of gs_mxfp4, enqueued on s.
void mx4_quantize_rows(const void *X, int64_t ldx, int dtype, int64_t rows, int64_t cols, uint8_t *codes,
                       uint8_t *scales, hipStream_t s);

}  // namespace gs
