// Shared pieces of the microscaled formats (8-bit saved activations, MXFP4):
// scale bytes, dense elements of either type, and the walk of row-wise kernels
// over blocks of 32 columns.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>
#include <utility>

#include "gs_internal.h"

namespace gs {

constexpr int kMxBlock = 32;             // columns of a block
constexpr int64_t kMxMaxCols = 1 << 24;  // widest matrix of either format

// ------------------------------------------------------------------ layouts

inline int64_t saved_code_pitch(int64_t cols) { return ceil_div(cols, kMxBlock) * kMxBlock; }
inline int64_t saved_scale_pitch(int64_t cols) { return ceil_div(cols, kMxBlock); }
// MXFP4 columns with their padding: a product takes 64 or 128 of them a step.
inline int64_t mx4_cols(int64_t cols) { return cols <= 64 ? ceil_div(cols, 64) * 64 : ceil_div(cols, 128) * 128; }

// Throws unless n rows of `cols` elements with leading dimension ld (elements
// of `size` bytes) at p are a valid operand.
void check_operand(const char *name, const void *p, int64_t rows, int64_t cols, int64_t ld, int size);
void check_saved(const gs_saved *A, bool relu_only);
void check_mxfp4(const gs_mxfp4 *A);
int dtype_size(int dtype);  // bytes of a gs_dtype, throws for others
// Whether a call that moves `bytes` goes past the caches; operands with their leading dimensions.
bool streams(double bytes, int64_t cols, int size, std::initializer_list<std::pair<const void *, int64_t>> operands);

// --------------------------------------------------------------- scale bytes

// 2^(E-127), NaN for E = 255.
__device__ __forceinline__ float mx_scale(int E)
{
    return __int_as_float(E == 255 ? 0x7fc00000 : E == 0 ? 0x00400000 : E << 23);
}
// 2^(127-E) for E <= 253, 0 for 255.
__device__ __forceinline__ float mx_inverse(int E) { return __int_as_float((E == 255 ? 0 : 254 - E) << 23); }

// Maximum over aligned groups of 4 or 8 lanes (of magnitudes' bit patterns,
// which order as the magnitudes do, NaN above infinity).
template <int L> __device__ __forceinline__ uint32_t group_max(uint32_t v)
{
    static_assert(L == 4 || L == 8);
    auto step = [&](uint32_t w) { v = w > v ? w : v; };
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));  // lanes 1 0 3 2
    step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));  // lanes 2 3 0 1
    if constexpr (L == 8) step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));  // 7 .. 0
    return v;
}

// ----------------------------------------------------------- dense elements

typedef unsigned short u16;
template <class T, int E> struct Elems;
template <int E> struct Elems<float, E> {
    typedef float type __attribute__((ext_vector_type(E), aligned(4)));
};
template <int E> struct Elems<u16, E> {  // bf16
    typedef u16 type __attribute__((ext_vector_type(E), aligned(2)));
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(u16 x) { return __int_as_float((int)x << 16); }

// Rounds to the nearest bf16, ties to even; a NaN stays one.
__device__ __forceinline__ u16 to_bf16(float x)
{
    return __builtin_bit_cast(u16, (__bf16)x);
}
template <class T> __device__ __forceinline__ T from_f32(float x)
{
    if constexpr (sizeof(T) == 4)
        return x;
    else
        return to_bf16(x);
}

// E elements from p, of which the first `valid` are in the row; zeros after them.
// NT: past the caches' replacement (as data that no one reads again soon).
// The end of a row is stored in up to three PIECES of 4, 2 and 1 elements (100,000 x 257
// bf16 values of saved codes 15.3 us, element by element 16.1), but loaded by elements
// (pieces, put together afterwards: quantising these rows 20.8 us instead of 18.5).
template <class T, int E, bool NT = false>
__device__ __forceinline__ typename Elems<T, E>::type load_elems(const T *p, int64_t valid)
{
    typename Elems<T, E>::type v;
    if (valid >= E) {
        if constexpr (NT)
            v = __builtin_nontemporal_load(reinterpret_cast<const typename Elems<T, E>::type *>(p));
        else
            v = *reinterpret_cast<const typename Elems<T, E>::type *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < E; i++) v[i] = i < valid ? p[i] : T(0);
    }
    return v;
}
template <class T, int E, bool NT = false, bool PIECES = true>
__device__ __forceinline__ void store_elems(T *p, typename Elems<T, E>::type v, int64_t valid)
{
    if (valid >= E) {
        if constexpr (NT)
            __builtin_nontemporal_store(v, reinterpret_cast<typename Elems<T, E>::type *>(p));
        else
            *reinterpret_cast<typename Elems<T, E>::type *>(p) = v;
    } else if constexpr (!PIECES) {
#pragma unroll
        for (int i = 0; i < E; i++)
            if (i < valid) p[i] = v[i];
    } else {
        static_assert(E == 4 || E == 8);
        const int n = valid > 0 ? (int)valid : 0;
        typename Elems<T, 4>::type q4;
        typename Elems<T, 2>::type q2;
#pragma unroll
        for (int i = 0; i < 4; i++) q4[i] = v[i];
#pragma unroll
        for (int i = 0; i < 2; i++) q2[i] = E == 8 && n & 4 ? v[E / 2 + i] : v[i];
        const T low = n & 2 ? v[2] : v[0], high = n & 2 ? v[E - 2] : v[E / 2];
        if (E == 8 && n & 4) *reinterpret_cast<typename Elems<T, 4>::type *>(p) = q4;
        if (n & 2) *reinterpret_cast<typename Elems<T, 2>::type *>(p + (n & 4)) = q2;
        if (n & 1) p[n & 6] = E == 8 && n & 4 ? high : low;
    }
}

// ------------------------------------------------------------------ 8-bit codes

// Codes of E neighbouring elements.
template <int E> struct Codes;
template <> struct Codes<4> {
    typedef uint32_t type;
};
template <> struct Codes<8> {
    typedef uint2 type;
};
template <int E> __device__ __forceinline__ uint32_t code_word(const typename Codes<E>::type &c, int w)
{
    if constexpr (E == 4)
        return c;
    else
        return w ? c.y : c.x;
}
template <int E> __device__ __forceinline__ typename Codes<E>::type code_words(const uint32_t *w)
{
    if constexpr (E == 4)
        return w[0];
    else
        return make_uint2(w[0], w[1]);
}

// 1.5 * 2^23: the sum with a number below 2^22 is rounded to a whole one, whose low bits
// are those of the sum.
constexpr float kWhole = 12582912.0f;

// Signed codes of E elements of a block of 32, whose other elements the neighbouring lanes
// (an aligned group of 32 / E) hold, and the block's scale byte.
template <int E> struct Saved8 {
    typename Codes<E>::type codes;
    uint8_t scale;
};
template <int E> __device__ __forceinline__ Saved8<E> save8_signed(const float (&y)[E])
{
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < E; e++) {
        const uint32_t b = __float_as_uint(y[e]) & 0x7fffffffu;
        m = b > m ? b : m;
    }
    const int k = (int)(group_max<kMxBlock / E>(m) >> 23);
    const int E8 = k == 255 ? 255 : k > 7 ? k - 6 : 1;
    const float inv = mx_inverse(E8);
    uint32_t w[E / 4];
#pragma unroll
    for (int q = 0; q < E / 4; q++) {
        uint32_t c[4];
#pragma unroll
        for (int e = 0; e < 4; e++)
            c[e] = __float_as_uint(__builtin_amdgcn_fmed3f(__builtin_fmaf(y[4 * q + e], inv, kWhole), kWhole - 127, kWhole + 127));
        w[q] = __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400) | __builtin_amdgcn_perm(c[3], c[2], 0x04000c0c);
        if (E8 == 255) w[q] = 0;
    }
    return {code_words<E>(w), (uint8_t)E8};
}

// ------------------------------------------------------------- block walk

// Row-wise kernels see a matrix as rows * d blocks of 32 columns in row-major
// order, each block as 32 / E units of E elements, a unit a lane.  A workgroup
// takes kUnits units at a time and splits their block numbers into row and
// block by multiplication: the first one's (64-bit) exactly for numbers below
// 2^44 (m64 = ceil(2^64 / d), d < 2^20), the others as 32-bit offsets below
// d + 2^10 from that row's first block (m32 = ceil(2^32 / d) up to d = 2^15;
// past that they cross one row end at most).
constexpr int kUnitThreads = 256;
constexpr int kUnitRounds = 4;  // units of a thread in flight
constexpr int kUnits = kUnitThreads * kUnitRounds;

struct BlockDiv {
    uint32_t d;
    uint32_t m32;
    uint64_t m64;
};
inline BlockDiv block_div(int64_t d)
{
    BlockDiv b{(uint32_t)d, 0, 0};
    if (d > 1) {
        b.m64 = UINT64_MAX / (uint64_t)d + 1;
        b.m32 = (uint32_t)(UINT32_MAX / (uint32_t)d + 1);
    }
    return b;
}

struct BlockAt {
    int64_t row;
    int32_t blk;
};
__device__ __forceinline__ BlockAt block_first(const BlockDiv &b, int64_t g)
{
    const int64_t row = b.d == 1 ? g : (int64_t)__umul64hi((uint64_t)g, b.m64);
    return BlockAt{row, (int32_t)(g - row * b.d)};
}
__device__ __forceinline__ BlockAt block_step(const BlockDiv &b, const BlockAt &first, uint32_t off)
{
    const uint32_t x = (uint32_t)first.blk + off;
    const uint32_t q = b.d == 1 ? x : b.d > 32768 ? (x >= b.d ? 1u : 0u) : __umulhi(x, b.m32);
    return BlockAt{first.row + q, (int32_t)(x - q * b.d)};
}

// Workgroups for `units` units; a launch holds fewer than 2^32 threads, so the
// kernels loop.
inline unsigned unit_grid(int64_t units) { return (unsigned)std::min<int64_t>(ceil_div(units, kUnits), 1 << 20); }

}  // namespace gs
