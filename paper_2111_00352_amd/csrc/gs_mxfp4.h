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

// Eight elements under scale byte E as e2m1, the first in the low bits (round to
// nearest even and clamped by the conversion); zeros for E = 255.  The scaling is
// exact but for numbers far below the smallest e2m1 step.
__device__ __forceinline__ uint32_t mx4_pack8(const float *x, int E)
{
    const float inv = mx_inverse(E);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0] * inv, x[1] * inv, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2] * inv, x[3] * inv, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4] * inv, x[5] * inv, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6] * inv, x[7] * inv, 1.0f, 3);
    return E == 255 ? 0 : w;
}

// Four elements likewise.
__device__ __forceinline__ uint16_t mx4_pack4(const float *x, int E)
{
    const float inv = mx_inverse(E);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0] * inv, x[1] * inv, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2] * inv, x[3] * inv, 1.0f, 1);
    return E == 255 ? 0 : (uint16_t)w;
}

// X (rows x cols of dtype) along its rows into codes and scales in the layout
// of gs_mxfp4, enqueued on s.
void mx4_quantize_rows(const void *X, int64_t ldx, int dtype, int64_t rows, int64_t cols, uint8_t *codes,
                       uint8_t *scales, hipStream_t s);

}  // namespace gs
