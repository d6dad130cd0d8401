// C = A . B^T for MXFP4 operands on the scaled matrix instructions
// (V_MFMA_SCALE_F32_32X32X64_F8F6F4): a lane holds one block of 32 elements of
// its row as 16 bytes and the block's scale byte, which is the layout of the
// format itself.
#include <algorithm>
#include <type_traits>

#include "gs_device.h"
#include "gs_mxfp4.h"

namespace gs {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(4)));

// c + a . b for 32 x 64 of A and B: 16 bytes a lane (row lane % 32, elements 32 *
// (lane / 32) onwards), scale bytes in byte OP of sa and sb.
template <int OP> __device__ __forceinline__ f32x16 mfma_fp4(u32x4 a, int sa, u32x4 b, int sb, f32x16 c)
{
    const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i32x8 y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, OP, sa, OP, sb);
}

// Where C goes: element (row, col) as T, 0 where the mask's code is 0.
template <class T, bool MASK> struct Out {
    T *c;
    int64_t ld;
    const uint8_t *mask;
    int64_t mask_pitch;
    __device__ __forceinline__ void store(int64_t row, int64_t col, float v) const
    {
        if (MASK && mask[row * mask_pitch + col] == 0) v = 0.0f;
        c[row * ld + col] = from_f32<T>(v);
    }
};

// Four waves, 128 x 128 of C, a wave 64 x 64; operands straight from memory.
template <class T, bool MASK>
__global__ __launch_bounds__(256) void k_matmul(const uint8_t *__restrict__ ac, const uint8_t *__restrict__ as,
                                                const uint8_t *__restrict__ bc, const uint8_t *__restrict__ bs,
                                                int64_t m, int64_t n, int kpad, int64_t tiles_n, int64_t tiles,
                                                Out<T, MASK> out)
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
            u32x4 a[2], b[2];
            int sa[2], sb[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const int blk = k / 32 + lane / 32;
                a[i] = *reinterpret_cast<const u32x4 *>(ac + ra[i] * cp + blk * 16);
                b[i] = *reinterpret_cast<const u32x4 *>(bc + rb[i] * cp + blk * 16);
                sa[i] = as[ra[i] * sp + blk];
                sb[i] = bs[rb[i] * sp + blk];
            }
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int j = 0; j < 2; j++) acc[i][j] = mfma_fp4<0>(a[i], sa[i], b[j], sb[j], acc[i][j]);
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

// ------------------------------------------------------------ large products
//
// A workgroup of four waves makes a tile of 64 WT x 64 WT, a wave a quarter of it
// (WT x WT instructions of 32 x 32 for every 64 of k), 256 of k a step.  Codes go
// from memory to LDS without passing registers; two buffers hold the step that is
// multiplied and the next one.  A row of a step is 128 bytes, whose eight 16-byte
// pieces lie in LDS in an order that depends on the row (piece ^ row % 8), so that
// the 32 rows an instruction reads spread over all banks; the loads put them there
// by choosing which piece of the row each lane fetches.
//
// The fragments of a step are read as four quarters of 64.  The last quarter is
// multiplied only after the next step's barrier, while that step's first quarters
// are read: the matrix cores have work across the barrier.  The next step's loads
// are issued after a step's last LDS read, so they have three quarters of a step
// until the barrier waits for them.
//
// Scale words (one for 128 of k) are read four at a time (512 of k) by one thread a
// row, a run ahead, and lie in LDS by word, so a wave reads 32 neighbouring words.
constexpr int kStepK = 256;

template <int WT> struct TileLds {
    static constexpr int kRows = 64 * WT;
    static constexpr int kStage = 2 * kRows * (kStepK / 2);
    __align__(1024) uint8_t codes[2][kStage];  // A's rows, then B's
    uint32_t scales[2][4][2 * kRows];
};

__device__ __forceinline__ void load_to_lds(const uint8_t *g, uint8_t *l)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)g,
                                     (__attribute__((address_space(3))) void *)l, 16, 0, 0);
}

// kpad >= 512, a multiple of 128.
template <class T, bool MASK, int WT>
__global__ __launch_bounds__(256, WT == 4 ? 1 : 2) void k_tile(const uint8_t *__restrict__ ac,
                                                               const uint8_t *__restrict__ as,
                                                               const uint8_t *__restrict__ bc,
                                                               const uint8_t *__restrict__ bs, int64_t m, int64_t n,
                                                               int kpad, int64_t tiles_m, int64_t tiles_n,
                                                               Out<T, MASK> out)
{
    constexpr int BM = 64 * WT, LD = 2 * WT, SL = 2 * BM / 256;
    __shared__ TileLds<WT> lds;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int64_t cp = kpad / 2;
    const int sp = kpad / kMxBlock;
    // an XCD takes a contiguous run of tiles, in panels of 8 rows of them
    const int64_t t = xcd_tile(blockIdx.x, tiles_m * tiles_n);
    const int64_t panel = t / (8 * tiles_n), in = t % (8 * tiles_n), ph = std::min<int64_t>(8, tiles_m - 8 * panel);
    const int64_t m0 = (8 * panel + in % ph) * BM, n0 = (in / ph) * BM;
    const int wm = wave / 2, wn = wave % 2, r = lane % 32, half = lane / 32;

    // Loads to LDS: a wave's load q fills rows 8 (wave LD + q) .. + 7 of a buffer.
    // Rows past the last one repeat it (their results are not stored).
    const int piece = (lane % 8) ^ (lane / 8);
    uint32_t offa[LD], offb[LD];
    const uint8_t *ga = ac + m0 * cp, *gb = bc + n0 * cp;
#pragma unroll
    for (int q = 0; q < LD; q++) {
        const int row = 8 * (wave * LD + q) + lane / 8;
        offa[q] = (uint32_t)(std::min<int64_t>(row, m - 1 - m0) * cp) + piece * 16;
        offb[q] = (uint32_t)(std::min<int64_t>(row, n - 1 - n0) * cp) + piece * 16;
    }
    auto issue = [&](int k, int buf) {
        const uint8_t *a = ga + k / 2, *b = gb + k / 2;
        uint8_t *to = lds.codes[buf] + 1024 * LD * wave;
        // (half a step is left at the end of the row: its upper half is not read)
        const uint32_t back = k + kStepK > kpad && piece >= 4 ? 64u : 0u;
#pragma unroll
        for (int q = 0; q < LD; q++) {
            load_to_lds(a + (offa[q] - back), to + 1024 * q);
            load_to_lds(b + (offb[q] - back), to + BM * 128 + 1024 * q);
        }
    };
    // Scales: four words from 512 run on, moved back to the row's last four at its
    // end; the words keep their places in a run of four.
    const uint8_t *gs[SL];
#pragma unroll
    for (int i = 0; i < SL; i++) {
        const int row = threadIdx.x + 256 * i;
        gs[i] = row < BM ? as + (m0 + std::min<int64_t>(row, m - 1 - m0)) * sp
                         : bs + (n0 + std::min<int64_t>(row - BM, n - 1 - n0)) * sp;
    }
    u32x4 sw[SL];
    auto load_scales = [&](int run) {
#pragma unroll
        for (int i = 0; i < SL; i++)
            sw[i] = *reinterpret_cast<const u32x4u *>(gs[i] + std::min(16 * run, sp - 16));
    };
    auto write_scales = [&](int run) {
        const int shift = (16 * run - std::min(16 * run, sp - 16)) / 4;
#pragma unroll
        for (int i = 0; i < SL; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) lds.scales[run & 1][(j - shift) & 3][threadIdx.x + 256 * i] = sw[i][j];
    };
    u32x4 fa[4][WT], fb[4][WT];
    uint32_t sa[2][WT], sb[2][WT];
    const int ra = wm * WT * 4096 + r * 128, rb = BM * 128 + wn * WT * 4096 + r * 128;
    auto read = [&](int buf, int q) {
        const uint8_t *p = lds.codes[buf] + ((2 * q + half) ^ (r & 7)) * 16;
#pragma unroll
        for (int i = 0; i < WT; i++) {
            fa[q][i] = *reinterpret_cast<const u32x4 *>(p + ra + i * 4096);
            fb[q][i] = *reinterpret_cast<const u32x4 *>(p + rb + i * 4096);
        }
    };
    auto read_scales = [&](int step, int h) {  // of the step's half h
        const uint32_t *p = lds.scales[step >> 1 & 1][2 * (step & 1) + h];
#pragma unroll
        for (int i = 0; i < WT; i++) {
            sa[h][i] = p[wm * WT * 32 + r + 32 * i];
            sb[h][i] = p[BM + wn * WT * 32 + r + 32 * i];
        }
    };
    f32x16 acc[WT][WT] = {};
    auto mul = [&](auto q) {
        constexpr int Q = decltype(q)::value;
#pragma unroll
        for (int i = 0; i < WT; i++)
#pragma unroll
            for (int j = 0; j < WT; j++)
                acc[i][j] = mfma_fp4<2 * (Q & 1)>(fa[Q][i], (int)(sa[Q / 2][i] >> 8 * half), fb[Q][j],
                                                  (int)(sb[Q / 2][j] >> 8 * half), acc[i][j]);
    };
    using Q0 = std::integral_constant<int, 0>;
    using Q1 = std::integral_constant<int, 1>;
    using Q2 = std::integral_constant<int, 2>;
    using Q3 = std::integral_constant<int, 3>;

    auto loads_done = [] {  // every wave's loads to LDS have arrived, and its reads are over
        __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
        __syncthreads();
    };
    const int steps = (kpad + kStepK - 1) / kStepK;  // the last one may be half a step
    issue(0, 0);
    load_scales(0);
    write_scales(0);
    load_scales(1);
    loads_done();
    read(0, 0), read(0, 1), read(0, 2), read(0, 3);
    read_scales(0, 0), read_scales(0, 1);
    issue(kStepK, 1);
    mul(Q0{}), mul(Q1{}), mul(Q2{});
    // Within a step the order of the instructions is laid down: an LDS read or a load
    // for every multiplication, which takes longer.
    auto interleave = [](auto kind, int count) {
#pragma unroll
        for (int i = 0; i < count; i++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(decltype(kind)::value, 1, 0);
        }
    };
    using LdsRead = std::integral_constant<int, 0x100>;
    using Load = std::integral_constant<int, 0x010>;
    auto full_step = [&](int s) {
        read(s & 1, 0), read(s & 1, 1);
        read_scales(s, 0);
        mul(Q3{});
        interleave(LdsRead{}, 4 * WT + WT);
        __builtin_amdgcn_sched_barrier(0);
        read(s & 1, 2), read(s & 1, 3);
        read_scales(s, 1);
        issue((s + 1) * kStepK, (s & 1) ^ 1);
        mul(Q0{}), mul(Q1{}), mul(Q2{});
        interleave(LdsRead{}, 4 * WT + WT);
        interleave(Load{}, 2 * LD);
        __builtin_amdgcn_sched_barrier(0);
    };
    int s = 1;
    for (; s < steps - 2; s += 2) {
        loads_done();
        write_scales((s + 1) / 2);
        load_scales((s + 3) / 2);
        full_step(s);
        loads_done();
        full_step(s + 1);
    }
    if (s < steps - 1) {
        loads_done();
        write_scales((s + 1) / 2);
        full_step(s++);
    }
    loads_done();
    read(s & 1, 0), read(s & 1, 1);
    read_scales(s, 0);
    mul(Q3{});
    mul(Q0{}), mul(Q1{});
    if (kpad % kStepK == 0) {
        read(s & 1, 2), read(s & 1, 3);
        read_scales(s, 1);
        mul(Q2{}), mul(Q3{});
    }

    const int64_t row0 = m0 + 32 * wm * WT + 4 * half, col0 = n0 + 32 * wn * WT + r;
#pragma unroll
    for (int i = 0; i < WT; i++)
#pragma unroll
        for (int e = 0; e < 16; e++) {
            const int64_t row = row0 + 32 * i + 8 * (e / 4) + e % 4;
            if (row < m) {
#pragma unroll
                for (int j = 0; j < WT; j++)
                    if (col0 + 32 * j < n) out.store(row, col0 + 32 * j, acc[i][j][e]);
            }
            __builtin_amdgcn_sched_barrier(0);  // (addresses of a row at a time)
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
    auto typed = [&](auto type, auto masked) {
        using T = decltype(type);
        constexpr bool MASK = decltype(masked)::value;
        const Out<T, MASK> out{(T *)C, ldc, mask ? mask->codes : nullptr, mask ? saved_code_pitch(n) : 0};
        auto tiled = [&](auto wt) {
            constexpr int WT = decltype(wt)::value;
            const int64_t tm = ceil_div(m, 64 * WT), tn = ceil_div(n, 64 * WT);
            k_tile<T, MASK, WT><<<(unsigned)(tm * tn), 256, 0, s>>>(A.codes, A.scales, B.codes, B.scales, m, n, kpad, tm, tn, out);
        };
        if (kpad >= 512 && ceil_div(m, 256) * ceil_div(n, 256) < (1 << 22)) {
            ceil_div(m, 256) * ceil_div(n, 256) >= 128 ? tiled(std::integral_constant<int, 4>{}) : tiled(std::integral_constant<int, 2>{});
            return;
        }
        const int64_t tiles_n = ceil_div(n, 128), tiles = ceil_div(m, 128) * tiles_n;
        const unsigned grid = (unsigned)std::min<int64_t>(tiles, 1 << 20);
        k_matmul<T, MASK><<<grid, 256, 0, s>>>(A.codes, A.scales, B.codes, B.scales, m, n, kpad, tiles_n, tiles, out);
    };
    auto go = [&](auto type) { mask ? typed(type, std::true_type{}) : typed(type, std::false_type{}); };
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
