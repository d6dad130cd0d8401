// Rows of a dense matrix held by groups of lanes: how many lanes and 16-byte pieces a row
// takes, sums and maxima over a group, and tensors whose type a call names.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "gs_device.h"
#include "gs_lowbit.h"

namespace gs {

// A matrix that a call reads or writes, its sizes in bytes; NULL: not there.
struct Extent {
    const void *p;
    int64_t rows, width, pitch;
};
// Refuses an output that shares bytes with an operand.  Of matrices of one pitch, parts of the
// same rows may lie beside each other, and with `same` the operand may be the output itself.
inline void check_apart(const char *output, const Extent &out, const char *name, const Extent &in, bool same = false)
{
    if (!out.p || !in.p || out.rows == 0 || in.rows == 0) return;
    const int64_t a = (int64_t)(uintptr_t)out.p, b = (int64_t)(uintptr_t)in.p;
    if (a + (out.rows - 1) * out.pitch + out.width <= b || b + (in.rows - 1) * in.pitch + in.width <= a) return;
    if (out.pitch == in.pitch) {
        if (same && a == b) return;
        const int64_t d = ((b - a) % out.pitch + out.pitch) % out.pitch;
        if (d >= out.width && d + in.width <= out.pitch) return;
    }
    fail(GS_ERR_INVALID_ARG, "%s overlaps %s", output, name);
}

// Elements of 16 bytes.
template <class T> constexpr int kPiece = sizeof(T) == 4 ? 4 : 8;

// ------------------------------------------------------- sums over lanes

template <int CTRL> __device__ __forceinline__ uint32_t dpp32(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL> __device__ __forceinline__ float dpp(float v) { return __uint_as_float(dpp32<CTRL>(__float_as_uint(v))); }
template <int CTRL> __device__ __forceinline__ double dpp(double v)
{
    const uint64_t b = __double_as_longlong(v);
    return __longlong_as_double((long long)((uint64_t)dpp32<CTRL>((uint32_t)(b >> 32)) << 32 | dpp32<CTRL>((uint32_t)b)));
}

// v of the two halves of the wave (of neighbouring rows of 16 lanes), both in every lane.
template <class V> struct Both {
    V low, high;
};
__device__ __forceinline__ Both<float> halves(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ Both<float> rows16(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
template <class F> __device__ __forceinline__ Both<double> both64(double v, F &&swap)
{
    const uint64_t b = __double_as_longlong(v);
    const Both<float> lo = swap(__uint_as_float((uint32_t)b)), hi = swap(__uint_as_float((uint32_t)(b >> 32)));
    auto join = [](float h, float l) {
        return __longlong_as_double((long long)((uint64_t)__float_as_uint(h) << 32 | __float_as_uint(l)));
    };
    return {join(hi.low, lo.low), join(hi.high, lo.high)};
}
__device__ __forceinline__ Both<double> halves(double v) { return both64(v, [](float x) { return halves(x); }); }
__device__ __forceinline__ Both<double> rows16(double v) { return both64(v, [](float x) { return rows16(x); }); }

// op over aligned groups of L lanes (a power of two up to 64), the same bits in each of
// them: every step combines two lanes' values, and op is commutative.
template <int L, class V, class Op> __device__ __forceinline__ V group_fold(V v, Op &&op)
{
    if constexpr (L > 1) v = op(v, dpp<0xB1>(v));    // lanes 1 0 3 2
    if constexpr (L > 2) v = op(v, dpp<0x4E>(v));    // lanes 2 3 0 1
    if constexpr (L > 4) v = op(v, dpp<0x141>(v));   // lanes 7 .. 0
    if constexpr (L > 8) v = op(v, dpp<0x140>(v));   // lanes 15 .. 0
    if constexpr (L > 16) {
        const Both<V> b = rows16(v);
        v = op(b.low, b.high);
    }
    if constexpr (L > 32) {
        const Both<V> b = halves(v);
        v = op(b.low, b.high);
    }
    return v;
}
// The same for whole numbers.
template <int L, class Op> __device__ __forceinline__ uint32_t group_fold_u(uint32_t v, Op &&op)
{
    return __float_as_uint(group_fold<L>(__uint_as_float(v), [&](float a, float b) {
        return __uint_as_float(op(__float_as_uint(a), __float_as_uint(b)));
    }));
}
template <int L, class V> __device__ __forceinline__ V group_sum(V v)
{
    return group_fold<L>(v, [](V a, V b) { return a + b; });
}

// The same over a row that L lanes hold, or all waves of a workgroup of L > 64 threads: tmp is
// L / 64 values in LDS; ends with a barrier then.
template <int L, class V, class Op> __device__ __forceinline__ V row_fold(V v, V *tmp, Op &&op)
{
    if constexpr (L <= kWave) {
        return group_fold<L>(v, op);
    } else {
        v = group_fold<kWave>(v, op);
        if (threadIdx.x % kWave == 0) tmp[threadIdx.x / kWave] = v;
        __syncthreads();
        V t = tmp[0];
#pragma unroll
        for (int w = 1; w < L / kWave; w++) t = op(t, tmp[w]);
        __syncthreads();
        return t;
    }
}
template <int L, class V> __device__ __forceinline__ V row_sum(V v, V *tmp)
{
    return row_fold<L>(v, tmp, [](V a, V b) { return a + b; });
}

// N sums at once, with one pair of barriers (tmp: N * L / 64 values).
template <int L, int N> __device__ __forceinline__ void row_sums(float (&v)[N], float *tmp)
{
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = group_sum<(L < kWave ? L : kWave)>(v[i]);
    if constexpr (L > kWave) {
        if (threadIdx.x % kWave == 0)
#pragma unroll
            for (int i = 0; i < N; i++) tmp[threadIdx.x / kWave * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = tmp[i];
#pragma unroll
        for (int w = 1; w < L / kWave; w++)
#pragma unroll
            for (int i = 0; i < N; i++) v[i] += tmp[w * N + i];
        __syncthreads();
    }
}

// -------------------------------------------------------------- row ends
//
// 16 bytes of a row from column `col` on, whatever is left of the row: the last ones are loaded
// as the row's last 16 bytes and moved into place afterwards, so that no load waits for a
// branch.  (Element by element, the gradient of a norm of 99,991 x 257 bf16 took 98 us.)

template <class T> struct RowPiece {
    static constexpr int E = kPiece<T>;
    typedef typename Elems<T, E>::type V;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    V v;
    int shift;  // elements to move it down by; E and more: nothing of it is in the row

    // col below any number, cols >= 1; in: the row exists (else nothing is read of it)
    template <bool NT = false> __device__ __forceinline__ void load(const T *row, int col, int cols, bool in = true)
    {
        if (cols >= E) {
            const int at = col < cols - E ? col : cols - E;
            shift = in ? col - at : E;
            if (in) v = load_elems<T, E, NT>(row + at, E);
        } else {
            shift = 0;
            v = load_elems<T, E>(row + col, in ? cols - col : 0);
        }
    }
    __device__ __forceinline__ static T from_bits(uint32_t b)
    {
        if constexpr (sizeof(T) == 4)
            return __uint_as_float(b);
        else
            return (T)b;
    }
    // The elements, `fill` (twice its bits in bf16) in the place of those behind the row.
    __device__ __forceinline__ V get(int col, int cols, uint32_t fill = 0) const
    {
        u32x4 w = __builtin_bit_cast(u32x4, v);
        if (cols < E) {
            if (fill) {
                V o = v;
#pragma unroll
                for (int e = 0; e < E; e++)
                    if (col + e >= cols) o[e] = from_bits(fill);
                return o;
            }
            return v;
        }
        if (__any(shift != 0)) {
            auto move = [&](int words) {
                u32x4 o;
#pragma unroll
                for (int i = 0; i < 4; i++) o[i] = i + words < 4 ? w[i + words < 4 ? i + words : 0] : fill;
                return o;
            };
            constexpr int ONE = sizeof(T) == 4 ? 1 : 2;  // elements of a word
            if constexpr (sizeof(T) == 2) {
                const u32x4 o = {w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16 | fill << 16};
                w = shift & 1 ? o : w;
            }
            w = shift & ONE ? move(1) : w;
            w = shift & 2 * ONE ? move(2) : w;
            const u32x4 none = {fill, fill, fill, fill};
            w = shift >= E ? none : w;
        }
        return __builtin_bit_cast(V, w);
    }
};

// -------------------------------------------------------------- held rows

constexpr int kRowThreads = 256;

// A row is held by L lanes (a wave's, or all of a workgroup's), R pieces of 16 bytes in each.
// Neighbouring lanes hold neighbouring pieces.
template <class T, int L, int R> struct RowAt {
    static constexpr int E = kPiece<T>;
    static constexpr int kRows = L <= kRowThreads ? kRowThreads / L : 1;  // of a workgroup
    static constexpr int kThreads = L <= kRowThreads ? kRowThreads : L;
    __device__ __forceinline__ static int lane() { return threadIdx.x % L; }
    __device__ __forceinline__ static int64_t first_row() { return (int64_t)blockIdx.x * kRows + threadIdx.x / L; }
    __device__ __forceinline__ static int64_t row_step() { return (int64_t)gridDim.x * kRows; }
    __device__ __forceinline__ static int col(int i) { return (i * L + lane()) * E; }
};

// (L, R) that hold a row of `pieces` 16-byte pieces, R at most RMOST and L from LLEAST to LMOST;
// go(L, R) as integral constants.  False: the row is wider.  Few pieces a lane: their registers
// leave room for the waves that hide the loads.
template <int LLEAST, int LMOST, int RMOST, class Go> bool with_row(int64_t pieces, Go &&go)
{
    auto one = [&](auto l, auto below, auto r) {  // (what `below` lanes hold is theirs)
        constexpr int L = decltype(l)::value, R = decltype(r)::value;
        if constexpr (L < LLEAST || L > LMOST || R > RMOST || (L > LLEAST && L * R <= decltype(below)::value * RMOST)) {
            return false;
        } else {
            if (pieces > (int64_t)L * R) return false;
            go(l, r);
            return true;
        }
    };
    using std::integral_constant;
    auto all = [&](auto l, auto below) {
        return one(l, below, integral_constant<int, 1>{}) || one(l, below, integral_constant<int, 2>{}) ||
               one(l, below, integral_constant<int, 3>{}) || one(l, below, integral_constant<int, 4>{});
    };
    const integral_constant<int, 4> l4;
    const integral_constant<int, 8> l8;
    const integral_constant<int, 16> l16;
    const integral_constant<int, 32> l32;
    const integral_constant<int, 64> l64;
    const integral_constant<int, 256> l256;
    const integral_constant<int, 512> l512;
    return all(l4, l4) || all(l8, l4) || all(l16, l8) || all(l32, l16) || all(l64, l32) || all(l256, l64) || all(l512, l256);
}

// Keeps the elements as they lie in registers: bf16 numbers are widened again where they are
// used again, which takes half the registers of keeping both.
template <class V> __device__ __forceinline__ void as_they_lie(V &v)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    u32x4 w = __builtin_bit_cast(u32x4, v);
    asm("" : "+v"(w));
    v = __builtin_bit_cast(V, w);
}

// Element i of an fp32 or bf16 array (wide: fp32).
__device__ __forceinline__ float load_either(const void *p, bool wide, int64_t i)
{
    return wide ? ((const float *)p)[i] : to_f32(((const u16 *)p)[i]);
}
// E of them (a weight for each column) from column c on, ones without an array, zeros past the last.
template <int E> __device__ __forceinline__ void load_weights(const void *p, bool wide, int c, int cols, float (&w)[E])
{
    if (!p) {
#pragma unroll
        for (int e = 0; e < E; e++) w[e] = 1.0f;
    } else if (c + E <= cols) {
        if (wide) {
#pragma unroll
            for (int q = 0; q < E / 4; q++) {
                const auto v = load_elems<float, 4>((const float *)p + c + 4 * q, 4);
#pragma unroll
                for (int e = 0; e < 4; e++) w[4 * q + e] = v[e];
            }
        } else {
            const auto v = load_elems<u16, E>((const u16 *)p + c, E);
#pragma unroll
            for (int e = 0; e < E; e++) w[e] = to_f32(v[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; e++) w[e] = c + e < cols ? load_either(p, wide, c + e) : 0.0f;
    }
}

}  // namespace gs
