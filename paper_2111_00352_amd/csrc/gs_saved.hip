// Activations kept in 8 bits for the backward pass: a layer's input is read
// twice by its gradient (the weight gradient H^T G and the mask of the ReLU
// below it), once per step, and is otherwise the largest thing a full-batch
// step keeps.  Blocks of 32 columns share a power-of-two step, so a value is a
// code of at most 8 significant bits times a power of two: saving and reading
// back are exact fp32 operations, and the matrix cores take it as bf16 without
// rounding.
//
// Everything here but the weight gradient is a stream: one pass, bound by
// memory.  A lane holds 16 bytes of a block, so that a wave's loads and stores are
// contiguous, and a block's lanes find its largest magnitude among themselves; four
// such pieces of a lane are in flight.  Measured, with what the matrices themselves
// hold: saving 2,000,000 x 128 fp32 by a ReLU 331 us (6.9 TB/s), 99,991 x 257 bf16 as
// it is 18 us; their values 182 us (7.1 TB/s) and 15 us; the masked gradient of
// 204,800 x 256 bf16 44 us (5.9 TB/s).  At 100 MB and less launch and drain show (2 to
// 3 us a call), and the instructions an element: 17.3 us for the ragged matrix, 18.8
// with a rounding, two bounds, a conversion and a shift for each code.
#include <algorithm>
#include <initializer_list>
#include <utility>

#include "gs_device.h"
#include "gs_lowbit.h"

namespace gs {

int dtype_size(int dtype)
{
    if (dtype != GS_F32 && dtype != GS_BF16) fail(GS_ERR_INVALID_ARG, "unknown element type %d", dtype);
    return dtype == GS_F32 ? 4 : 2;
}

void check_operand(const char *name, const void *p, int64_t rows, int64_t cols, int64_t ld, int size)
{
    if (rows > 0 && cols > 0 && !p) fail(GS_ERR_INVALID_ARG, "%s is null", name);
    if (ld < cols) fail(GS_ERR_INVALID_ARG, "%s: leading dimension below the width", name);
    if ((uintptr_t)p % size) fail(GS_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    if (rows > 1 && ld > (((int64_t)1 << 62) / size - cols) / (rows - 1))
        fail(GS_ERR_INVALID_ARG, "%s: span is not addressable", name);
}

static void check_shape(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0 || rows > INT32_MAX) fail(GS_ERR_INVALID_ARG, "bad matrix size");
    if (cols > kMxMaxCols) fail(GS_ERR_UNSUPPORTED, "at most 2^24 columns");
}

void check_saved(const gs_saved *A, bool relu_only)
{
    if (!A) fail(GS_ERR_INVALID_ARG, "null saved activations");
    check_shape(A->rows, A->cols);
    if (A->act != GS_ACT_NONE && A->act != GS_ACT_RELU) fail(GS_ERR_INVALID_ARG, "unknown activation %d", A->act);
    if (relu_only && A->act != GS_ACT_RELU) fail(GS_ERR_INVALID_ARG, "activations were not saved by a ReLU");
    if (A->rows > 0 && A->cols > 0 && (!A->codes || !A->scales)) fail(GS_ERR_INVALID_ARG, "null saved array");
    if ((uintptr_t)A->codes % 16) fail(GS_ERR_INVALID_ARG, "saved codes are not 16-byte aligned");
}

void check_mxfp4(const gs_mxfp4 *A)
{
    if (!A) fail(GS_ERR_INVALID_ARG, "null MXFP4 matrix");
    check_shape(A->rows, A->cols);
    if (A->rows > 0 && A->cols > 0 && (!A->codes || !A->scales)) fail(GS_ERR_INVALID_ARG, "null MXFP4 array");
    if ((uintptr_t)A->codes % 16 || (uintptr_t)A->scales % 4)
        fail(GS_ERR_INVALID_ARG, "MXFP4 codes are not 16-byte or scales not 4-byte aligned");
}

namespace {

// Lanes of a block: 16 bytes of the dense operand each.
template <class T> constexpr int kUnitElems = sizeof(T) == 4 ? 4 : 8;

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

// For each of this thread's units load(i, unit, row, first column, columns left in
// the row from there), i the round, then use(...) likewise.
template <int E, class Load, class Use>
__device__ __forceinline__ void walk_units(int64_t units, const BlockDiv &div, int64_t cols, Load &&load, Use &&use)
{
    constexpr int L = kMxBlock / E;
    for (int64_t u0 = (int64_t)blockIdx.x * kUnits; u0 < units; u0 += (int64_t)gridDim.x * kUnits) {
        const BlockAt first = block_first(div, u0 / L);
        int64_t row[kUnitRounds];
        int32_t col[kUnitRounds];
#pragma unroll
        for (int i = 0; i < kUnitRounds; i++) {
            const uint32_t t = i * kUnitThreads + threadIdx.x;
            const BlockAt at = block_step(div, first, t / L);
            row[i] = at.row;
            col[i] = at.blk * kMxBlock + (t % L) * E;
            if (u0 + t < units) load(i, u0 + t, row[i], col[i], cols - col[i]);
        }
#pragma unroll
        for (int i = 0; i < kUnitRounds; i++) {
            const int64_t u = u0 + i * kUnitThreads + threadIdx.x;
            // (units are whole blocks: the lanes of a block are all inside or all outside)
            if (u < units) use(i, u, row[i], col[i], cols - col[i]);
        }
    }
}

// 1.5 * 2^23: the sum with a number below 2^22 is rounded to a whole one, whose low bits
// are those of the sum.
constexpr float kWhole = 12582912.0f;

template <class T, bool RELU, bool NT>
__global__ __launch_bounds__(kUnitThreads) void k_save(const T *__restrict__ P, int64_t ldp, int64_t cols,
                                                       int64_t units, BlockDiv div, uint8_t *__restrict__ codes,
                                                       uint8_t *__restrict__ scales, T *__restrict__ H, int64_t ldh)
{
    constexpr int E = kUnitElems<T>, L = kMxBlock / E;
    typename Elems<T, E>::type v[kUnitRounds];
    walk_units<E>(
        units, div, cols,
        [&](int i, int64_t, int64_t row, int32_t col, int64_t left) { v[i] = load_elems<T, E, NT>(P + row * ldp + col, left); },
        [&](int i, int64_t u, int64_t row, int32_t col, int64_t left) {
            float h[E];
            bool on[E];
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float x = to_f32(v[i][e]);
                on[e] = !(x <= 0.0f);
                h[e] = RELU && !on[e] ? 0.0f : x;
                const uint32_t b = __float_as_uint(h[e]) & 0x7fffffffu;
                m = b > m ? b : m;
            }
            const int k = (int)(group_max<L>(m) >> 23);
            const int s = k - (RELU ? 7 : 6);
            const int E8 = k == 255 ? 255 : s > 1 ? s : 1;
            const float inv = mx_inverse(E8);
            uint32_t w[E / 4];
#pragma unroll
            for (int q = 0; q < E / 4; q++) {
                uint32_t c[4];
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    // (nearest whole number, ties to even, in the low byte; a NaN gives the lower bound)
                    const float r = __builtin_amdgcn_fmed3f(__builtin_fmaf(h[4 * q + e], inv, kWhole), kWhole + (RELU ? 1 : -127),
                                                            kWhole + (RELU ? 255 : 127));
                    c[e] = __float_as_uint(r);
                    if (RELU) c[e] = on[4 * q + e] ? c[e] : 0;
                }
                w[q] = __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400) | __builtin_amdgcn_perm(c[3], c[2], 0x04000c0c);
                if (!RELU && E8 == 255) w[q] = 0;
            }
            *reinterpret_cast<typename Codes<E>::type *>(codes + u * E) = code_words<E>(w);
            if (u % L == 0) scales[u / L] = (uint8_t)E8;
            if constexpr (RELU) {
                if (H && left > 0) {
                    typename Elems<T, E>::type o;
#pragma unroll
                    for (int e = 0; e < E; e++) o[e] = on[e] ? v[i][e] : T(0);
                    store_elems<T, E, NT>(H + row * ldh + col, o, left);
                }
            } else {
                if (H && left > 0) store_elems<T, E, NT>(H + row * ldh + col, v[i], left);
            }
        });
}

template <class T, bool NT>
__global__ __launch_bounds__(kUnitThreads) void k_relu_grad(const uint8_t *__restrict__ codes, int64_t cols,
                                                            int64_t units, BlockDiv div, const T *dH, int64_t ldh,
                                                            T *dP, int64_t ldp)
{
    constexpr int E = kUnitElems<T>;
    typename Elems<T, E>::type v[kUnitRounds];
    typename Codes<E>::type c[kUnitRounds];
    walk_units<E>(
        units, div, cols,
        [&](int i, int64_t u, int64_t row, int32_t col, int64_t left) {
            c[i] = *reinterpret_cast<const typename Codes<E>::type *>(codes + u * E);
            v[i] = load_elems<T, E, NT>(dH + row * ldh + col, left);
        },
        [&](int i, int64_t, int64_t row, int32_t col, int64_t left) {
            typename Elems<T, E>::type o;
#pragma unroll
            for (int e = 0; e < E; e++) o[e] = code_word<E>(c[i], e / 4) >> (8 * (e % 4)) & 255 ? v[i][e] : T(0);
            if (left > 0) store_elems<T, E, NT>(dP + row * ldp + col, o, left);
        });
}

template <class T, bool NT>
__global__ __launch_bounds__(kUnitThreads) void k_saved_values(const uint8_t *__restrict__ codes,
                                                               const uint8_t *__restrict__ scales, int is_signed,
                                                               int64_t cols, int64_t units, BlockDiv div,
                                                               T *__restrict__ out, int64_t ld)
{
    constexpr int E = kUnitElems<T>, L = kMxBlock / E;
    typename Codes<E>::type c[kUnitRounds];
    int E8[kUnitRounds];
    const uint32_t flip = is_signed ? 0x80808080u : 0;
    const float zero = is_signed ? 128.0f : 0.0f;
    walk_units<E>(
        units, div, cols,
        [&](int i, int64_t u, int64_t, int32_t, int64_t) {
            c[i] = *reinterpret_cast<const typename Codes<E>::type *>(codes + u * E);
            E8[i] = scales[u / L];
        },
        [&](int i, int64_t, int64_t row, int32_t col, int64_t left) {
            typename Elems<T, E>::type o;
            const float s = mx_scale(E8[i]);
#pragma unroll
            for (int e = 0; e < E; e++) {
                // (signed codes as unsigned ones 128 above)
                const uint32_t b = (code_word<E>(c[i], e / 4) ^ flip) >> (8 * (e % 4)) & 255;
                o[e] = from_f32<T>(((float)b - zero) * s);  // (exact in bf16 too)
            }
            if (left > 0) store_elems<T, E, NT>(out + row * ld + col, o, left);
        });
}

// Whether a call streams past the caches: when what it moves is more than the
// memory-side cache holds for its next reader, and rows are whole 16-byte pieces
// (others share lines between accesses).  Saving and reading back n x 128 fp32:
// 100,000 rows 30.5 us in the caches, 32.0 us past them; 200,000 68.4 and 61.8;
// 2,000,000 631 and 530.
constexpr double kStreamBytes = 200e6;
bool streams(double bytes, int64_t cols, int size, std::initializer_list<std::pair<const void *, int64_t>> operands)
{
    if (bytes < kStreamBytes || cols * size % 16) return false;
    for (const auto &[p, ld] : operands)
        if ((uintptr_t)p % 16 || ld * size % 16) return false;
    return true;
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" {

int gs_saved_layout(int64_t cols, int64_t *code_pitch, int64_t *scale_pitch)
{
    return guarded([&] {
        if (!code_pitch || !scale_pitch) fail(GS_ERR_INVALID_ARG, "null output");
        check_shape(0, cols);
        *code_pitch = saved_code_pitch(cols);
        *scale_pitch = saved_scale_pitch(cols);
    });
}

int gs_save_activation(const void *P, int64_t ldp, int dtype, const gs_saved *out, void *H, int64_t ldh,
                       gs_stream stream)
{
    return guarded([&] {
        check_saved(out, false);
        const int size = dtype_size(dtype);
        check_operand("P", P, out->rows, out->cols, ldp, size);
        if (H) check_operand("H", H, out->rows, out->cols, ldh, size);
        if (out->rows == 0 || out->cols == 0) return;
        const int64_t nb = saved_scale_pitch(out->cols);
        auto go = [&](auto kernel, auto type) {
            using T = decltype(type);
            const int64_t units = out->rows * nb * (kMxBlock / kUnitElems<T>);
            kernel<<<unit_grid(units), kUnitThreads, 0, (hipStream_t)stream>>>(
                (const T *)P, ldp, out->cols, units, block_div(nb), out->codes, out->scales, (T *)H, ldh);
        };
        const double bytes = (double)out->rows * out->cols * (size * (H ? 2 : 1) + 1);
        const bool nt = streams(bytes, out->cols, size, {{P, ldp}, {H, H ? ldh : ldp}});
        const bool relu = out->act == GS_ACT_RELU;
        if (dtype == GS_F32) {
            if (nt)
                relu ? go(k_save<float, true, true>, 0.0f) : go(k_save<float, false, true>, 0.0f);
            else
                relu ? go(k_save<float, true, false>, 0.0f) : go(k_save<float, false, false>, 0.0f);
        } else {
            if (nt)
                relu ? go(k_save<u16, true, true>, u16(0)) : go(k_save<u16, false, true>, u16(0));
            else
                relu ? go(k_save<u16, true, false>, u16(0)) : go(k_save<u16, false, false>, u16(0));
        }
        GS_HIP(hipGetLastError());
    });
}

int gs_saved_dequantize(const gs_saved *A, void *out, int64_t ld, int dtype, gs_stream stream)
{
    return guarded([&] {
        check_saved(A, false);
        check_operand("out", out, A->rows, A->cols, ld, dtype_size(dtype));
        if (A->rows == 0 || A->cols == 0) return;
        const int64_t nb = saved_scale_pitch(A->cols);
        auto go = [&](auto type) {
            using T = decltype(type);
            const int64_t units = A->rows * nb * (kMxBlock / kUnitElems<T>);
            const double bytes = (double)A->rows * A->cols * (sizeof(T) + 1);
            const auto kernel = streams(bytes, A->cols, sizeof(T), {{out, ld}}) ? k_saved_values<T, true> : k_saved_values<T, false>;
            kernel<<<unit_grid(units), kUnitThreads, 0, (hipStream_t)stream>>>(
                A->codes, A->scales, A->act == GS_ACT_NONE, A->cols, units, block_div(nb), (T *)out, ld);
        };
        dtype == GS_F32 ? go(0.0f) : go(u16(0));
        GS_HIP(hipGetLastError());
    });
}

int gs_relu_grad(const gs_saved *A, const void *dH, int64_t ldh, int dtype, void *dP, int64_t ldp, gs_stream stream)
{
    return guarded([&] {
        check_saved(A, true);
        const int size = dtype_size(dtype);
        check_operand("dH", dH, A->rows, A->cols, ldh, size);
        check_operand("dP", dP, A->rows, A->cols, ldp, size);
        if (A->rows == 0 || A->cols == 0) return;
        const int64_t nb = saved_scale_pitch(A->cols);
        auto go = [&](auto type) {
            using T = decltype(type);
            const int64_t units = A->rows * nb * (kMxBlock / kUnitElems<T>);
            const double bytes = (double)A->rows * A->cols * (2 * sizeof(T) + 1);
            const auto kernel = streams(bytes, A->cols, sizeof(T), {{dH, ldh}, {dP, ldp}}) ? k_relu_grad<T, true> : k_relu_grad<T, false>;
            kernel<<<unit_grid(units), kUnitThreads, 0, (hipStream_t)stream>>>(
                A->codes, A->cols, units, block_div(nb), (const T *)dH, ldh, (T *)dP, ldp);
        };
        dtype == GS_F32 ? go(0.0f) : go(u16(0));
        GS_HIP(hipGetLastError());
    });
}

}  // extern "C"
