// MXFP4 (OCP Microscaling, e2m1 elements, blocks of 32 with a power-of-two
// scale): quantisation along the rows or the columns of a dense matrix, and the
// values back.  Each is one pass, bound by memory: 100,000 x 128 fp32 in 12.7 us (4.6
// TB/s), their values in 12 us; 2 to 3 us of each are the launch's start and drain.  The
// element conversions of gfx950 take the block's scale, so an element costs little more
// than its share of the largest magnitude.
#include <algorithm>

#include "gs_device.h"
#include "gs_lowbit.h"
#include "gs_mxfp4.h"

namespace gs {
namespace {

// A lane takes 16 bytes of the dense operand: four or eight columns, so that a load
// or store of a wave is contiguous.
template <class T> constexpr int kLaneCols = 16 / sizeof(T);
template <int E> struct Nibbles;
template <> struct Nibbles<4> {
    typedef u16 type;
};
template <> struct Nibbles<8> {
    typedef uint32_t type;
};

template <class T>
__global__ __launch_bounds__(kUnitThreads) void k_mx4_rows(const T *__restrict__ X, int64_t ldx, int64_t cols,
                                                           int64_t units, BlockDiv div, uint8_t *__restrict__ codes,
                                                           uint8_t *__restrict__ scales)
{
    constexpr int E = kLaneCols<T>, L = kMxBlock / E;
    typename Elems<T, E>::type v[kUnitRounds];
    for (int64_t u0 = (int64_t)blockIdx.x * kUnits; u0 < units; u0 += (int64_t)gridDim.x * kUnits) {
        const BlockAt first = block_first(div, u0 / L);
#pragma unroll
        for (int i = 0; i < kUnitRounds; i++) {
            const uint32_t t = i * kUnitThreads + threadIdx.x;
            const BlockAt at = block_step(div, first, t / L);
            const int32_t col = at.blk * kMxBlock + (t % L) * E;
            if (u0 + t < units) v[i] = load_elems<T, E>(X + at.row * ldx + col, cols - col);
        }
#pragma unroll
        for (int i = 0; i < kUnitRounds; i++) {
            const int64_t u = u0 + i * kUnitThreads + threadIdx.x;
            if (u >= units) continue;  // (whole blocks)
            const Mx4Lane<T, E> x{v[i]};
            const int E8 = mx4_exponent(group_max<L>(x.magnitude()));
            reinterpret_cast<typename Nibbles<E>::type *>(codes)[u] = (typename Nibbles<E>::type)x.codes(E8);
            if (u % L == 0) scales[u / L] = (uint8_t)E8;
        }
    }
}

// Along the columns: out row c holds column c of X.  A workgroup takes 256 rows x 64
// columns of X, a wave a block of 32 rows at a time: lane (g, j) = (lane / 8, lane % 8)
// loads eight neighbouring columns (8 j on) of rows 4 g .. 4 g + 3, so that a load
// reads whole lines, finds the columns' largest magnitudes across the eight g and
// packs its four rows of each column into two bytes.  The codes go out through LDS,
// where they meet those of the other blocks, as 128 contiguous bytes of an out row.
// Neighbouring workgroups take neighbouring columns, the rest of the same rows of X:
// 4096 x 4096 bf16 11.0 us, 13.6 us with neighbours along the rows; 8192 x 8192 38.5 and
// 49 us.  Finding maxima by lane swaps, which fold two columns at once, instead of through
// LDS made that 9.5 us (4.5 TB/s; 128 x 128 fp32 5.2 -> 3.6 us).
constexpr int kColTile = 64;
constexpr int kRowTile = 256;
constexpr int kColBlocks = kRowTile / kMxBlock;

// Swaps a's lanes 32 .. 63 with b's lanes 0 .. 31, and a's lanes 16 .. 31 and 48 .. 63
// with b's 0 .. 15 and 32 .. 47.
__device__ __forceinline__ void swap_halves(uint32_t &a, uint32_t &b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
__device__ __forceinline__ void swap_rows(uint32_t &a, uint32_t &b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
// The largest m[c] over the eight lanes with this lane's j, for two of the eight columns c:
// 2 (lane / 16) and the next one.  Each swap folds two columns at once.
__device__ __forceinline__ void max_over_rows(uint32_t (&m)[8], uint32_t (&top)[2])
{
#pragma unroll
    for (int c = 0; c < 4; c++) {
        swap_halves(m[c], m[c + 4]);
        m[c] = larger(m[c], m[c + 4]);
    }
#pragma unroll
    for (int c = 0; c < 2; c++) {
        swap_rows(m[c], m[c + 2]);
        const uint32_t v = larger(m[c], m[c + 2]);
        top[c] = larger(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true));  // row_ror:8
    }
}

// All eight columns' values in every lane, from that distribution.
__device__ __forceinline__ void to_all_rows(const uint32_t (&v)[2], uint32_t (&all)[8])
{
#pragma unroll
    for (int c = 0; c < 2; c++) {
        all[c] = all[c + 2] = v[c];
        swap_rows(all[c], all[c + 2]);
    }
#pragma unroll
    for (int c = 0; c < 4; c++) {
        all[c + 4] = all[c];
        swap_halves(all[c], all[c + 4]);
    }
}

// Four rows of eight columns in a lane.
template <class T> struct ColLane;
template <> struct ColLane<float> {
    float x[8][4];
    __device__ __forceinline__ void set(int i, typename Elems<float, 8>::type v)
    {
#pragma unroll
        for (int c = 0; c < 8; c++) x[c][i] = v[c];
    }
    __device__ __forceinline__ void magnitudes(uint32_t (&m)[8]) const
    {
#pragma unroll
        for (int c = 0; c < 8; c++) {
            m[c] = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) m[c] = larger(m[c], __float_as_uint(x[c][i]) & 0x7fffffffu);
        }
    }
    __device__ __forceinline__ u16 pack(int c, float s) const
    {
        return (u16)mx4_pair<1>(mx4_pair<0>(0, x[c][0], x[c][1], s), x[c][2], x[c][3], s);
    }
};
template <> struct ColLane<u16> {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    u32x4 x[4];  // two columns a word
    __device__ __forceinline__ void set(int i, typename Elems<u16, 8>::type v) { x[i] = __builtin_bit_cast(u32x4, v); }
    __device__ __forceinline__ void magnitudes(uint32_t (&m)[8]) const
    {
#pragma unroll
        for (int p = 0; p < 4; p++) {
            u16x2 top = {};
#pragma unroll
            for (int i = 0; i < 4; i++)
                top = larger_magnitudes(top, x[i][p]);
            const uint32_t t = __builtin_bit_cast(uint32_t, top);
            m[2 * p] = t << 16;
            m[2 * p + 1] = t & 0xffff0000u;
        }
    }
    __device__ __forceinline__ u16 pack(int c, float s) const
    {
        const uint32_t pick = c % 2 ? 0x07060302 : 0x05040100;
        auto rows = [&](int i) { return __builtin_amdgcn_perm(x[i + 1][c / 2], x[i][c / 2], pick); };
        return (u16)mx4_pair<1>(mx4_pair<0>(0, rows(0), s), rows(2), s);
    }
};

template <class T>
__global__ __launch_bounds__(256) void k_mx4_cols(const T *__restrict__ X, int64_t ldx, int64_t rows, int64_t cols,
                                                  int64_t col_tiles, int64_t tiles, int64_t code_pitch,
                                                  int64_t scale_pitch, uint8_t *__restrict__ codes,
                                                  uint8_t *__restrict__ scales)
{
    constexpr int kPitch = kColBlocks * 16 + 16;  // (the shift spreads columns over banks)
    __shared__ __align__(16) uint8_t tile[kColTile * kPitch];
    __shared__ uint8_t exps[kColTile][kColBlocks];
    const int wave = threadIdx.x / kWave, g = threadIdx.x % kWave / 8, j = threadIdx.x % 8;
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int64_t r0 = (t / col_tiles) * kRowTile, c0 = (t % col_tiles) * kColTile, left = cols - c0 - 8 * j;
#pragma unroll
        for (int h = 0; h < kColBlocks / 4; h++) {
            const int blk = 4 * h + wave;
            ColLane<T> x;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int64_t row = r0 + 32 * blk + 4 * g + i;
                typename Elems<T, 8>::type v = {};
                if (row < rows) v = load_elems<T, 8>(X + row * ldx + c0 + 8 * j, left);
                x.set(i, v);
            }
            uint32_t m[8], top[2], s[2], scale[8];
            x.magnitudes(m);
            max_over_rows(m, top);
#pragma unroll
            for (int c = 0; c < 2; c++) {
                const int E8 = mx4_exponent(top[c]);
                if (g % 2 == 0) exps[8 * j + g + c][blk] = (uint8_t)E8;
                s[c] = __float_as_uint(mx_scale(E8));
            }
            to_all_rows(s, scale);
#pragma unroll
            for (int c = 0; c < 8; c++)  // (a block with a NaN or an infinity has zeros)
                *reinterpret_cast<u16 *>(tile + (8 * j + c) * kPitch + 16 * blk + 2 * g) =
                    scale[c] < 0x7f800000u ? x.pack(c, __uint_as_float(scale[c])) : 0;
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kColTile * kColBlocks / 256; q++) {
            const int e = q * 256 + threadIdx.x, c = e / kColBlocks, blk = e % kColBlocks;
            const int64_t at = r0 / kMxBlock + blk;  // block of the out row
            if (c0 + c < cols && at < scale_pitch) {
                *reinterpret_cast<uint4 *>(codes + (c0 + c) * code_pitch + at * 16) =
                    *reinterpret_cast<const uint4 *>(tile + c * kPitch + 16 * blk);
                scales[(c0 + c) * scale_pitch + at] = exps[c][blk];
            }
        }
        __syncthreads();
    }
}

// Codes 2 PAIR and 2 PAIR + 1 of w under scale s as two bf16 (exactly).
template <int PAIR> __device__ __forceinline__ uint32_t mx4_values2(uint32_t w, float s)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, PAIR));
}

template <class T>
__global__ __launch_bounds__(kUnitThreads) void k_mx4_values(const uint8_t *__restrict__ codes,
                                                             const uint8_t *__restrict__ scales, int64_t code_pitch,
                                                             int64_t scale_pitch, int64_t cols, int64_t units,
                                                             BlockDiv div, T *__restrict__ out, int64_t ld)
{
    constexpr int E = kLaneCols<T>, L = kMxBlock / E;
    typename Nibbles<E>::type w[kUnitRounds];
    int E8[kUnitRounds];
    int64_t row[kUnitRounds];
    int32_t col[kUnitRounds];
    for (int64_t u0 = (int64_t)blockIdx.x * kUnits; u0 < units; u0 += (int64_t)gridDim.x * kUnits) {
        const BlockAt first = block_first(div, u0 / L);
#pragma unroll
        for (int i = 0; i < kUnitRounds; i++) {
            const uint32_t t = i * kUnitThreads + threadIdx.x;
            const BlockAt at = block_step(div, first, t / L);
            row[i] = at.row;
            col[i] = at.blk * kMxBlock + (t % L) * E;
            if (u0 + t < units) {
                w[i] = *reinterpret_cast<const typename Nibbles<E>::type *>(codes + row[i] * code_pitch + col[i] / 2);
                E8[i] = scales[row[i] * scale_pitch + at.blk];
            }
        }
#pragma unroll
        for (int i = 0; i < kUnitRounds; i++) {
            const int64_t u = u0 + i * kUnitThreads + threadIdx.x;
            if (u >= units || col[i] >= cols) continue;
            const float s = mx_scale(E8[i]);
            typename Elems<T, E>::type o;
            if constexpr (E == 8) {
                uint4 p = make_uint4(mx4_values2<0>(w[i], s), mx4_values2<1>(w[i], s), mx4_values2<2>(w[i], s), mx4_values2<3>(w[i], s));
                if (E8[i] == 255) p = make_uint4(0x7fc07fc0, 0x7fc07fc0, 0x7fc07fc0, 0x7fc07fc0);
                o = __builtin_bit_cast(typename Elems<T, E>::type, p);
            } else {
                const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.0f, 0);
                const f32x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.0f, 1);
                o = typename Elems<T, E>::type{p0[0] * s, p0[1] * s, p1[0] * s, p1[1] * s};
            }
            store_elems<T, E>(out + row[i] * ld + col[i], o, cols - col[i]);
        }
    }
}

}  // namespace

void mx4_quantize_rows(const void *X, int64_t ldx, int dtype, int64_t rows, int64_t cols, uint8_t *codes,
                       uint8_t *scales, hipStream_t s)
{
    const int64_t nb = mx4_cols(cols) / kMxBlock;
    if (rows * nb == 0) return;
    auto go = [&](auto type) {
        using T = decltype(type);
        const int64_t units = rows * nb * (kMxBlock / kLaneCols<T>);
        k_mx4_rows<T><<<unit_grid(units), kUnitThreads, 0, s>>>((const T *)X, ldx, cols, units, block_div(nb), codes, scales);
    };
    dtype == GS_F32 ? go(0.0f) : go(u16(0));
    GS_HIP(hipGetLastError());
}

}  // namespace gs

using namespace gs;

extern "C" {

int gs_mxfp4_layout(int64_t cols, int64_t *code_pitch, int64_t *scale_pitch)
{
    return guarded([&] {
        if (!code_pitch || !scale_pitch) fail(GS_ERR_INVALID_ARG, "null output");
        if (cols < 0) fail(GS_ERR_INVALID_ARG, "bad matrix size");
        if (cols > kMxMaxCols) fail(GS_ERR_UNSUPPORTED, "at most 2^24 columns");
        *code_pitch = mx4_cols(cols) / 2;
        *scale_pitch = mx4_cols(cols) / kMxBlock;
    });
}

int gs_mxfp4_quantize(const void *X, int64_t ldx, int dtype, int64_t rows, int64_t cols, int axis,
                      const gs_mxfp4 *out, gs_stream stream)
{
    return guarded([&] {
        check_mxfp4(out);
        if (axis != 0 && axis != 1) fail(GS_ERR_INVALID_ARG, "axis is 0 or 1");
        if (out->rows != (axis ? rows : cols) || out->cols != (axis ? cols : rows))
            fail(GS_ERR_INVALID_ARG, "the MXFP4 matrix has another shape");
        check_operand("X", X, rows, cols, ldx, dtype_size(dtype));
        if (rows == 0 || cols == 0) return;
        const hipStream_t s = (hipStream_t)stream;
        if (axis == 1) {
            mx4_quantize_rows(X, ldx, dtype, rows, cols, out->codes, out->scales, s);
            return;
        }
        const int64_t padded = mx4_cols(rows), col_tiles = ceil_div(cols, kColTile);
        const int64_t tiles = ceil_div(padded, kRowTile) * col_tiles;
        const unsigned grid = (unsigned)std::min<int64_t>(tiles, 1 << 20);
        auto go = [&](auto type) {
            using T = decltype(type);
            k_mx4_cols<T><<<grid, 256, 0, s>>>((const T *)X, ldx, rows, cols, col_tiles, tiles, padded / 2,
                                              padded / kMxBlock, out->codes, out->scales);
        };
        dtype == GS_F32 ? go(0.0f) : go(u16(0));
        GS_HIP(hipGetLastError());
    });
}

int gs_mxfp4_dequantize(const gs_mxfp4 *A, void *out, int64_t ld, int dtype, gs_stream stream)
{
    return guarded([&] {
        check_mxfp4(A);
        check_operand("out", out, A->rows, A->cols, ld, dtype_size(dtype));
        if (A->rows == 0 || A->cols == 0) return;
        // (blocks of the matrix, without the padding of its rows)
        const int64_t nb = ceil_div(A->cols, kMxBlock), padded = mx4_cols(A->cols);
        auto go = [&](auto type) {
            using T = decltype(type);
            const int64_t units = A->rows * nb * (kMxBlock / kLaneCols<T>);
            k_mx4_values<T><<<unit_grid(units), kUnitThreads, 0, (hipStream_t)stream>>>(
                A->codes, A->scales, padded / 2, padded / kMxBlock, A->cols, units, block_div(nb), (T *)out, ld);
        };
        dtype == GS_F32 ? go(0.0f) : go(u16(0));
        GS_HIP(hipGetLastError());
    });
}

}  // extern "C"
