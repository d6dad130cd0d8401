// C = A . B^T for MXFP4 operands on the scaled matrix instructions
// (V_MFMA_SCALE_F32_32X32X64_F8F6F4): a lane holds one block of 32 elements of
// its row as 16 bytes and the block's scale byte, which is the layout of the
// format itself.
#include <algorithm>

#include "gs_device.h"
#include "gs_mxfp4.h"

namespace gs {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x16 mfma_fp4(const uint4 &a, int sa, const uint4 &b, int sb, f32x16 c)
{
    const i32x8 x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    const i32x8 y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, 0, sa, 0, sb);
}

// Where C goes: element (row, col) as T, 0 where the mask's code is 0.
template <class T> struct Out {
    T *c;
    int64_t ld;
    const uint8_t *mask;
    int64_t mask_pitch;
    __device__ __forceinline__ void store(int64_t row, int64_t col, float v) const
    {
        if (mask && mask[row * mask_pitch + col] == 0) v = 0.0f;
        c[row * ld + col] = from_f32<T>(v);
    }
};

// Four waves, 128 x 128 of C, a wave 64 x 64; operands straight from memory.
template <class T>
__global__ __launch_bounds__(256) void k_matmul(const uint8_t *__restrict__ ac, const uint8_t *__restrict__ as,
                                                const uint8_t *__restrict__ bc, const uint8_t *__restrict__ bs,
                                                int64_t m, int64_t n, int kpad, int64_t tiles_n, int64_t tiles, Out<T> out)
{
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t cp = kpad / 2, sp = kpad / kMxBlock;
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int64_t m0 = (t / tiles_n) * 128 + (wave / 2) * 64, n0 = (t % tiles_n) * 128 + (wave % 2) * 64;
        f32x16 acc[2][2] = {};
        int64_t ra[2], rb[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            ra[i] = std::min<int64_t>(m0 + 32 * i + lane % 32, m - 1);
            rb[i] = std::min<int64_t>(n0 + 32 * i + lane % 32, n - 1);
        }
        for (int k = 0; k < kpad; k += 64) {
            uint4 a[2], b[2];
            int sa[2], sb[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const int blk = k / 32 + lane / 32;
                a[i] = *reinterpret_cast<const uint4 *>(ac + ra[i] * cp + blk * 16);
                b[i] = *reinterpret_cast<const uint4 *>(bc + rb[i] * cp + blk * 16);
                sa[i] = as[ra[i] * sp + blk];
                sb[i] = bs[rb[i] * sp + blk];
            }
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int j = 0; j < 2; j++) acc[i][j] = mfma_fp4(a[i], sa[i], b[j], sb[j], acc[i][j]);
        }
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int j = 0; j < 2; j++)
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const int64_t row = m0 + 32 * i + 8 * (e / 4) + 4 * (lane / 32) + e % 4;
                    const int64_t col = n0 + 32 * j + lane % 32;
                    if (row < m && col < n) out.store(row, col, acc[i][j][e]);
                }
    }
}

uint64_t round256(uint64_t x) { return (x + 255) / 256 * 256; }

void check_sizes(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || n < 0 || k < 0 || m > INT32_MAX || n > INT32_MAX) fail(GS_ERR_INVALID_ARG, "bad product size");
    if (k > kMxMaxCols) fail(GS_ERR_UNSUPPORTED, "at most 2^24 columns");
}

// Workspace: A's codes and scales when A is dense.
uint64_t workspace(int64_t m, int64_t k, int a_dtype)
{
    if (a_dtype < 0) return 0;
    return round256((uint64_t)m * mx4_cols(k) / 2) + round256((uint64_t)m * mx4_cols(k) / kMxBlock);
}

void check_out(int64_t m, int64_t n, const gs_saved *mask, void *C, int64_t ldc, int dtype)
{
    check_operand("C", C, m, n, ldc, dtype_size(dtype));
    if (mask) {
        check_saved(mask, true);
        if (mask->rows != m || mask->cols != n) fail(GS_ERR_INVALID_ARG, "the mask has another shape than the product");
    }
}

void check_work(const void *work, uint64_t have, uint64_t need)
{
    if (need && (!work || have < need))
        fail(GS_ERR_INVALID_ARG, "workspace of %llu bytes is below the %llu needed",
             (unsigned long long)(work ? have : 0), (unsigned long long)need);
    if ((uintptr_t)work % 16) fail(GS_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
}

void multiply(const gs_mxfp4 &A, const gs_mxfp4 &B, const gs_saved *mask, void *C, int64_t ldc, int dtype,
              hipStream_t s)
{
    const int64_t m = A.rows, n = B.rows;
    if (m == 0 || n == 0) return;
    const int kpad = (int)mx4_cols(A.cols);
    const int64_t tiles_n = ceil_div(n, 128), tiles = ceil_div(m, 128) * tiles_n;
    const unsigned grid = (unsigned)std::min<int64_t>(tiles, 1 << 20);
    auto go = [&](auto type) {
        using T = decltype(type);
        const Out<T> out{(T *)C, ldc, mask ? mask->codes : nullptr, mask ? saved_code_pitch(n) : 0};
        k_matmul<T><<<grid, 256, 0, s>>>(A.codes, A.scales, B.codes, B.scales, m, n, kpad, tiles_n, tiles, out);
    };
    dtype == GS_F32 ? go(0.0f) : go(u16(0));
    GS_HIP(hipGetLastError());
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" {

int gs_mxfp4_matmul_workspace(int64_t m, int64_t n, int64_t k, int a_dtype, uint64_t *bytes)
{
    return guarded([&] {
        if (!bytes) fail(GS_ERR_INVALID_ARG, "null output");
        check_sizes(m, n, k);
        if (a_dtype != -1) dtype_size(a_dtype);
        *bytes = workspace(m, k, a_dtype);
    });
}

int gs_mxfp4_matmul(const gs_mxfp4 *A, const gs_mxfp4 *B, const gs_saved *mask, void *C, int64_t ldc, int dtype,
                    void *work, uint64_t work_bytes, gs_stream stream)
{
    return guarded([&] {
        check_mxfp4(A);
        check_mxfp4(B);
        if (A->cols != B->cols) fail(GS_ERR_INVALID_ARG, "A and B have different widths");
        check_out(A->rows, B->rows, mask, C, ldc, dtype);
        check_work(work, work_bytes, workspace(A->rows, A->cols, -1));
        multiply(*A, *B, mask, C, ldc, dtype, (hipStream_t)stream);
    });
}

int gs_mxfp4_matmul_dense(const void *A, int64_t lda, int a_dtype, int64_t m, const gs_mxfp4 *B,
                          const gs_saved *mask, void *C, int64_t ldc, int dtype, void *work, uint64_t work_bytes,
                          gs_stream stream)
{
    return guarded([&] {
        check_mxfp4(B);
        check_sizes(m, B->rows, B->cols);
        check_operand("A", A, m, B->cols, lda, dtype_size(a_dtype));
        check_out(m, B->rows, mask, C, ldc, dtype);
        check_work(work, work_bytes, workspace(m, B->cols, a_dtype));
        uint8_t *codes = (uint8_t *)work;
        const gs_mxfp4 q{m, B->cols, codes, codes + round256((uint64_t)m * mx4_cols(B->cols) / 2)};
        mx4_quantize_rows(A, lda, a_dtype, m, B->cols, q.codes, q.scales, (hipStream_t)stream);
        multiply(q, *B, mask, C, ldc, dtype, (hipStream_t)stream);
    });
}

}  // extern "C"
