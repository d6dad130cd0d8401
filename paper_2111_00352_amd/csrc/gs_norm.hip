// Root-mean-square norm of the rows of H = X + R (R: the residual stream, may be absent),
//
//   r = (mean H^2 + eps)^(-1/2),   Y = H r w,
//
// with Y dense or in the 8 bits of saved activations, and its gradient: with x = H r and
// u = dY w
//
//   dX = dH + r (u - x mean(u x)),   dw = sum over rows of dY x.
//
// H is rounded to its type before anything is made of it, so that the backward pass, which
// reads it from memory, sees the numbers that were normalised.  Squares are exact in 64
// bits and summed there: no row is too large for its r, or too small while r is below 2^128 (past
// that, with eps 0, it is infinite), and a row's sum costs a few instructions beside the loads
// that bound these kernels.
//
// Both directions are one pass over memory, which bounds them: a row stays in registers between
// its sum and its results.  2,000,000 x 128 fp32 with a residual into 8 bits takes 512 us (6.5
// TB/s), the norm alone 335 (6.1), its gradient 611 (5.0); 20,000 x 8192 bf16 109 (6.0) and 238 (4.1).
// Rows at odd offsets, whose 16-byte pieces straddle their loads' lines, cost up to a fifth more.
// The gradient of bf16 rows that fill part of a workgroup's lanes is bound by its instructions and two
// barriers a row: 186,011 x 1344 510 us (2.9 TB/s), where 200,000 x 1024 take 212 (5.8).
#include <algorithm>
#include <type_traits>

#include "gs_rows.h"

namespace gs {
namespace {

// t^(-1/2): the instruction's value, a step of Newton's method on, which has over 32 bits right.
__device__ __forceinline__ float inverse_root(double t)
{
    const double y = __builtin_amdgcn_rsq(t);
    return (float)(t > 0.0 && t < __builtin_inf() ? y * __builtin_fma(-0.5 * t * y, y, 1.5) : y);
}

template <class T, int L, int R, bool SAVE, bool NT>
__global__ __launch_bounds__((RowAt<T, L, R>::kThreads)) void k_norm(const T *__restrict__ X, int64_t ldx, const T *__restrict__ Res,
                                                                 int64_t ldr, const void *__restrict__ w, bool w32, double eps,
                                                                 int64_t n, int cols, T *__restrict__ H, int64_t ldh,
                                                                 T *__restrict__ Y, int64_t ldy, uint8_t *__restrict__ codes,
                                                                 uint8_t *__restrict__ scales, int blocks,
                                                                 float *__restrict__ rstd)
{
    using At = RowAt<T, L, R>;
    constexpr int E = At::E;
    using V = typename Elems<T, E>::type;
    __shared__ double tmp[L > kWave ? L / kWave : 1];
    float wt[R][E];
#pragma unroll
    for (int i = 0; i < R; i++) load_weights<E>(w, w32, At::col(i), cols, wt[i]);
    const double inv = 1.0 / cols;
    // (rows of a wave that are past the last one go along: every lane takes part in the sums)
    for (int64_t row = At::first_row(), at = (int64_t)blockIdx.x * At::kRows; at < n; row += At::row_step(), at += At::row_step()) {
        const bool in = row < n;
        V v[R];
        RowPiece<T> x[R], q[R];
#pragma unroll
        for (int i = 0; i < R; i++) x[i].template load<NT>(X + row * ldx, At::col(i), cols, in);
        if (Res)
#pragma unroll
            for (int i = 0; i < R; i++) q[i].template load<NT>(Res + row * ldr, At::col(i), cols, in);
#pragma unroll
        for (int i = 0; i < R; i++) v[i] = x[i].get(At::col(i), cols);
        if (Res) {
#pragma unroll
            for (int i = 0; i < R; i++) {
                const V t = q[i].get(At::col(i), cols);
#pragma unroll
                for (int e = 0; e < E; e++) v[i][e] = from_f32<T>(to_f32(v[i][e]) + to_f32(t[e]));
                store_elems<T, E, NT>(H + row * ldh + At::col(i), v[i], in ? cols - At::col(i) : 0);
            }
        }
        double ss = 0.0;
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int e = 0; e < E; e++) {
                const double h = (double)to_f32(v[i][e]);
                ss = __builtin_fma(h, h, ss);
            }
        ss = row_sum<L>(ss, tmp);
        const float r = inverse_root(ss * inv + eps);
#pragma unroll
        for (int i = 0; i < R; i++) as_they_lie(v[i]);
        if (in && At::lane() == 0) rstd[row] = r;
#pragma unroll
        for (int i = 0; i < R; i++) {
            float y[E];
#pragma unroll
            for (int e = 0; e < E; e++) y[e] = to_f32(v[i][e]) * r * wt[i][e];
            if constexpr (!SAVE) {
                V o;
#pragma unroll
                for (int e = 0; e < E; e++) o[e] = from_f32<T>(y[e]);
                store_elems<T, E, NT>(Y + row * ldy + At::col(i), o, in ? cols - At::col(i) : 0);
            } else {
                const Saved8<E> c = save8_signed<E>(y);
                if (in && At::col(i) < blocks * kMxBlock) {
                    const int64_t u = row * blocks * kMxBlock + At::col(i);
                    *reinterpret_cast<typename Codes<E>::type *>(codes + u) = c.codes;
                    if (At::col(i) % kMxBlock == 0) scales[u / kMxBlock] = c.scale;
                }
            }
        }
    }
}

// Gradient.  part: a row of `cols` partial sums of dw for each workgroup, or NULL.
template <class T, int L, int R, bool NT>
__global__ __launch_bounds__((RowAt<T, L, R>::kThreads)) void k_norm_grad(const T *__restrict__ H, int64_t ldh, const float *__restrict__ rstd,
                                                                      const T *__restrict__ dY, int64_t ldy, const void *__restrict__ w,
                                                                      bool w32, const T *dH, int64_t ldd, int64_t n, int cols, T *dX,
                                                                      int64_t ldx, float *__restrict__ part)
{
    using At = RowAt<T, L, R>;
    constexpr int E = At::E;
    using V = typename Elems<T, E>::type;
    constexpr int kSums = L <= kWave ? kRowThreads / kWave : 1;
    __shared__ float tmp[L > kWave ? L / kWave : 1];
    __shared__ float sums[L <= kWave ? kSums : 1][L <= kWave ? L * R * E : 1];
    float wt[R][E], dw[R][E];
#pragma unroll
    for (int i = 0; i < R; i++) {
        load_weights<E>(w, w32, At::col(i), cols, wt[i]);
#pragma unroll
        for (int e = 0; e < E; e++) dw[i][e] = 0.0f;
    }
    const float inv = 1.0f / (float)cols;
    // the next row is loaded while this one is worked on
    RowPiece<T> hp[R], gp[R], dp[R];
    float r_next;
    auto load = [&](int64_t row) {
        const bool in = row < n;
        r_next = in ? rstd[row] : 0.0f;
#pragma unroll
        for (int i = 0; i < R; i++) {
            hp[i].template load<NT>(H + row * ldh, At::col(i), cols, in);
            gp[i].template load<NT>(dY + row * ldy, At::col(i), cols, in);
            if (dH) dp[i].template load<NT>(dH + row * ldd, At::col(i), cols, in);
        }
    };
    load(At::first_row());
    for (int64_t row = At::first_row(), at = (int64_t)blockIdx.x * At::kRows; at < n; row += At::row_step(), at += At::row_step()) {
        const bool in = row < n;
        V h[R], g[R], d[R];
        const float r = r_next;
#pragma unroll
        for (int i = 0; i < R; i++) {
            h[i] = hp[i].get(At::col(i), cols);
            g[i] = gp[i].get(At::col(i), cols);
            if (dH) d[i] = dp[i].get(At::col(i), cols);
        }
        load(row + At::row_step());
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float x = to_f32(h[i][e]) * r, y = to_f32(g[i][e]);
                dot = __builtin_fmaf(y * wt[i][e], x, dot);
                dw[i][e] = __builtin_fmaf(y, x, dw[i][e]);
            }
        dot = row_sum<L>(dot, tmp) * inv;
#pragma unroll
        for (int i = 0; i < R; i++) {
            as_they_lie(h[i]);
            as_they_lie(g[i]);
            V o;
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float x = to_f32(h[i][e]) * r, u = to_f32(g[i][e]) * wt[i][e];
                const float t = r * __builtin_fmaf(-x, dot, u);
                o[e] = from_f32<T>(dH ? t + to_f32(d[i][e]) : t);
            }
            store_elems<T, E, NT>(dX + row * ldx + At::col(i), o, in ? cols - At::col(i) : 0);
        }
    }
    if (!part) return;
    float *to = part + (int64_t)blockIdx.x * cols;
    if constexpr (L > kWave) {
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int e = 0; e < E; e++)
                if (At::col(i) + e < cols) to[At::col(i) + e] = dw[i][e];
    } else {
        // over the rows of a wave by lane swaps, over the waves through LDS
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int e = 0; e < E; e++) {
                float s = dw[i][e];
                if constexpr (L == 8) s += dpp<0x128>(s);  // row_ror:8
                if constexpr (L <= 16) {
                    const Both<float> b = rows16(s);
                    s = b.low + b.high;
                }
                if constexpr (L <= 32) {
                    const Both<float> b = halves(s);
                    s = b.low + b.high;
                }
                if (threadIdx.x % kWave < L) sums[threadIdx.x / kWave][At::col(i) + e] = s;
            }
        __syncthreads();
        for (int c = threadIdx.x; c < cols; c += kRowThreads) {
            float s = 0.0f;
#pragma unroll
            for (int v = 0; v < kSums; v++) s += sums[v][c];
            to[c] = s;
        }
    }
}

// Rows wider than a workgroup holds: two passes over each.
constexpr int kWideThreads = 1024;

template <class T, bool SAVE>
__global__ __launch_bounds__(kWideThreads) void k_norm_wide(const T *__restrict__ X, int64_t ldx, const T *__restrict__ Res,
                                                           int64_t ldr, const void *__restrict__ w, bool w32, double eps, int64_t n,
                                                           int cols, T *H, int64_t ldh, T *__restrict__ Y, int64_t ldy,
                                                           uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, int blocks,
                                                           float *__restrict__ rstd)
{
    constexpr int E = kPiece<T>;
    using V = typename Elems<T, E>::type;
    __shared__ double tmp[kWideThreads / kWave];
    const double inv = 1.0 / cols;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        double ss = 0.0;
        for (int c = threadIdx.x * E; c < cols; c += kWideThreads * E) {
            V v = load_elems<T, E>(X + row * ldx + c, cols - c);
            if (Res) {
                const V q = load_elems<T, E>(Res + row * ldr + c, cols - c);
#pragma unroll
                for (int e = 0; e < E; e++) v[e] = from_f32<T>(to_f32(v[e]) + to_f32(q[e]));
                store_elems<T, E>(H + row * ldh + c, v, cols - c);  // (read again by this thread)
            }
#pragma unroll
            for (int e = 0; e < E; e++) {
                const double h = (double)to_f32(v[e]);
                ss = __builtin_fma(h, h, ss);
            }
        }
        ss = row_sum<kWideThreads>(ss, tmp);
        const float r = inverse_root(ss * inv + eps);
        if (threadIdx.x == 0) rstd[row] = r;
        const T *from = Res ? H + row * ldh : X + row * ldx;
        const int end = SAVE ? blocks * kMxBlock : cols;
        for (int c0 = 0; c0 < end; c0 += kWideThreads * E) {  // (all lanes of a wave: blocks are found across lanes)
            const int c = c0 + threadIdx.x * E;
            const V v = load_elems<T, E>(from + c, cols - c);
            float y[E], wt[E];
            load_weights<E>(w, w32, c, cols, wt);
#pragma unroll
            for (int e = 0; e < E; e++) y[e] = c + e < cols ? to_f32(v[e]) * r * wt[e] : 0.0f;
            if constexpr (!SAVE) {
                V o;
#pragma unroll
                for (int e = 0; e < E; e++) o[e] = from_f32<T>(y[e]);
                store_elems<T, E>(Y + row * ldy + c, o, cols - c);
            } else {
                const Saved8<E> s = save8_signed<E>(y);
                if (c < end) {
                    const int64_t u = row * blocks * kMxBlock + c;
                    *reinterpret_cast<typename Codes<E>::type *>(codes + u) = s.codes;
                    if (c % kMxBlock == 0) scales[u / kMxBlock] = s.scale;
                }
            }
        }
    }
}

// mean(u x) of a row.
template <class T>
__global__ __launch_bounds__(kWideThreads) void k_norm_dot(const T *__restrict__ H, int64_t ldh, const float *__restrict__ rstd,
                                                          const T *__restrict__ dY, int64_t ldy, const void *__restrict__ w, bool w32,
                                                          int64_t n, int cols, float *__restrict__ dots)
{
    constexpr int E = kPiece<T>;
    __shared__ float tmp[kWideThreads / kWave];
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const float r = rstd[row];
        float dot = 0.0f, run = 0.0f;
        int k = 0;
        for (int c = threadIdx.x * E; c < cols; c += kWideThreads * E) {
            const auto h = load_elems<T, E>(H + row * ldh + c, cols - c);
            const auto g = load_elems<T, E>(dY + row * ldy + c, cols - c);
            float wt[E];
            load_weights<E>(w, w32, c, cols, wt);
#pragma unroll
            for (int e = 0; e < E; e++)
                if (c + e < cols) run = __builtin_fmaf(to_f32(g[e]) * wt[e], to_f32(h[e]) * r, run);
            if (++k % 16 == 0) {
                dot += run;
                run = 0.0f;
            }
        }
        dot = row_sum<kWideThreads>(dot + run, tmp);
        if (threadIdx.x == 0) dots[row] = dot / (float)cols;
    }
}
// dX and, of each workgroup row's share of the rows, sums of dw: a thread a column.
template <class T>
__global__ __launch_bounds__(kRowThreads) void k_norm_grad_wide(const T *__restrict__ H, int64_t ldh, const float *__restrict__ rstd,
                                                                const T *__restrict__ dY, int64_t ldy, const void *__restrict__ w,
                                                                bool w32, const T *dH, int64_t ldd, int64_t n, int cols, T *dX,
                                                                int64_t ldx, const float *__restrict__ dots, float *__restrict__ part)
{
    const int c = blockIdx.x * kRowThreads + threadIdx.x;
    if (c >= cols) return;
    const float wt = w ? load_either(w, w32, c) : 1.0f;
    float sum = 0.0f, run = 0.0f;
    int k = 0;
    for (int64_t row = blockIdx.y; row < n; row += gridDim.y) {
        const float r = rstd[row], x = to_f32(H[row * ldh + c]) * r, y = to_f32(dY[row * ldy + c]);
        const float t = r * __builtin_fmaf(-x, dots[row], y * wt);
        dX[row * ldx + c] = from_f32<T>(dH ? t + to_f32(dH[row * ldd + c]) : t);
        run = __builtin_fmaf(y, x, run);
        if (++k % kChainFold == 0) {
            sum += run;
            run = 0.0f;
        }
    }
    if (part) part[(int64_t)blockIdx.y * cols + c] = sum + run;
}

// ------------------------------------------------------------------- launch

// Partial rows of dw: a workgroup's share of the rows is summed in its registers, so a few
// workgroups a compute unit, and no more than 32 MB of partials.
template <class T> constexpr int kGradPieces = sizeof(T) == 4 ? 4 : 2;  // of a lane (bf16 takes 50 registers for each)
struct NormGradPlan {
    int64_t blocks;
    bool wide;
};
template <class T> NormGradPlan norm_grad_plan(int64_t n, int64_t cols)
{
    NormGradPlan p{0, false};
    const int64_t most = std::max<int64_t>(1, (32 << 20) / 4 / std::max<int64_t>(1, cols));
    const bool held = with_row<8, 512, kGradPieces<T>>(ceil_div(cols, kPiece<T>), [&](auto l, auto r) {
        using At = RowAt<T, decltype(l)::value, decltype(r)::value>;
        const int64_t steps = std::max<int64_t>(1, ceil_div(n, (int64_t)At::kRows));  // of kRows rows
        p.blocks = ceil_div(steps, ceil_div(steps, std::min<int64_t>(768, most)));   // (equal shares)
    });
    if (!held) {
        p.wide = true;
        p.blocks = std::max<int64_t>(1, std::min<int64_t>(n, most));
    }
    return p;
}
uint64_t norm_grad_need(int64_t n, int64_t cols, int dtype)
{
    const NormGradPlan p = dtype == GS_F32 ? norm_grad_plan<float>(n, cols) : norm_grad_plan<u16>(n, cols);
    return (uint64_t)(p.blocks * cols + (p.wide ? n : 0)) * 4;
}

void check_norm(int64_t n, int64_t cols, int w_dtype)
{
    if (n < 0 || n > INT32_MAX || cols < 1) fail(GS_ERR_INVALID_ARG, "bad matrix size");
    if (cols > kMxMaxCols) fail(GS_ERR_UNSUPPORTED, "at most 2^24 columns");
    dtype_size(w_dtype);
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" {

int gs_rms_norm(const void *X, int64_t ldx, const void *R, int64_t ldr, int dtype, int64_t rows, int64_t cols, const void *w,
                int w_dtype, double eps, void *H, int64_t ldh, void *Y, int64_t ldy, const gs_saved *saved, float *rstd,
                gs_stream stream)
{
    return guarded([&] {
        const int size = dtype_size(dtype);
        check_norm(rows, cols, w_dtype);
        if (!(eps >= 0.0) || eps > 1e300) fail(GS_ERR_INVALID_ARG, "eps must be at least 0 and finite");
        check_operand("X", X, rows, cols, ldx, size);
        if (R) {
            check_operand("R", R, rows, cols, ldr, size);
            check_operand("H", H, rows, cols, ldh, size);
        }
        if (Y && saved) fail(GS_ERR_INVALID_ARG, "one of Y and saved is given");
        if (saved) {
            check_saved(saved, false);
            if (saved->act != GS_ACT_NONE) fail(GS_ERR_INVALID_ARG, "a norm is saved with GS_ACT_NONE");
            if (saved->rows != rows || saved->cols != cols) fail(GS_ERR_INVALID_ARG, "saved has another shape");
        } else {
            check_operand("Y", Y, rows, cols, ldy, size);
        }
        if (rows > 0 && !rstd) fail(GS_ERR_INVALID_ARG, "rstd is null");
        if (w && (uintptr_t)w % dtype_size(w_dtype)) fail(GS_ERR_INVALID_ARG, "w is not aligned to its elements");
        if (rows == 0) return;
        const auto extent = [&](const void *p, int64_t ld) { return Extent{p, rows, cols * size, ld * size}; };
        const Extent x = extent(X, ldx), r = extent(R, ldr), h = extent(R ? H : nullptr, ldh), y = extent(Y, ldy);
        check_apart("H", h, "X", x, true), check_apart("H", h, "R", r, true);
        check_apart("Y", y, "X", x), check_apart("Y", y, "R", r), check_apart("Y", y, "H", h);
        if (saved) {
            const Extent codes = {saved->codes, rows, saved_code_pitch(cols), saved_code_pitch(cols)};
            const Extent scales = {saved->scales, rows, saved_scale_pitch(cols), saved_scale_pitch(cols)};
            for (const Extent &part : {codes, scales})
                check_apart("saved", part, "X", x), check_apart("saved", part, "R", r), check_apart("saved", part, "H", h);
        }
        const hipStream_t s = (hipStream_t)stream;
        const int blocks = (int)saved_scale_pitch(cols);
        const double bytes = (double)rows * cols * (size * (R ? 3 : 1) + (saved ? 1 : size));
        const bool nt = streams(bytes, cols, size, {{X, ldx}, {R, R ? ldr : ldx}, {H, R ? ldh : ldx}, {Y, Y ? ldy : ldx}});
        auto go = [&](auto type, auto save) {
            using T = decltype(type);
            constexpr bool SAVE = decltype(save)::value;
            uint8_t *codes = saved ? saved->codes : nullptr, *scales = saved ? saved->scales : nullptr;
            // Workgroups that go on to further rows load the weights once for them: 87,335 x 2048 bf16 into
            // 8 bits 117 us by 8,192 workgroups, 125 by one for each set of rows, 1,000,000 x 17 fp32 30 and
            // 39; fp32 rows of three pieces a lane and more keep the chip busier without (2,000,000 x 128 with
            // a residual 536 and 513).
            auto run = [&](auto kernel, int64_t grid, int threads, bool once) {
                kernel<<<(unsigned)std::min<int64_t>(grid, once ? 1 << 20 : 8192), threads, 0, s>>>(
                    (const T *)X, ldx, (const T *)R, ldr, w, w_dtype == GS_F32, eps, rows, (int)cols, (T *)H, ldh, (T *)Y, ldy, codes,
                    scales, blocks, rstd);
            };
            const int64_t pieces = SAVE ? (int64_t)blocks * (kMxBlock / kPiece<T>) : ceil_div(cols, kPiece<T>);
            const bool held = with_row<8, 512, 4>(pieces, [&](auto l, auto r) {
                constexpr int L = decltype(l)::value, N = decltype(r)::value;
                using At = RowAt<T, L, N>;
                constexpr bool ONCE = sizeof(T) == 4 && N >= 3;
                nt ? run(k_norm<T, L, N, SAVE, true>, ceil_div(rows, (int64_t)At::kRows), At::kThreads, ONCE)
                   : run(k_norm<T, L, N, SAVE, false>, ceil_div(rows, (int64_t)At::kRows), At::kThreads, ONCE);
            });
            if (!held) run(k_norm_wide<T, SAVE>, rows, kWideThreads, false);
        };
        if (dtype == GS_F32)
            saved ? go(0.0f, std::true_type{}) : go(0.0f, std::false_type{});
        else
            saved ? go(u16(0), std::true_type{}) : go(u16(0), std::false_type{});
        GS_HIP(hipGetLastError());
    });
}

int gs_rms_norm_grad_workspace(int64_t rows, int64_t cols, int dtype, uint64_t *bytes)
{
    return guarded([&] {
        if (!bytes) fail(GS_ERR_INVALID_ARG, "null output");
        dtype_size(dtype);
        check_norm(rows, cols, GS_F32);
        *bytes = norm_grad_need(rows, cols, dtype);
    });
}

int gs_rms_norm_grad(const void *H, int64_t ldh, const float *rstd, const void *dY, int64_t ldy, int dtype, int64_t rows,
                     int64_t cols, const void *w, int w_dtype, const void *dH, int64_t ldd, void *dX, int64_t ldx, float *dw,
                     void *work, uint64_t work_bytes, gs_stream stream)
{
    return guarded([&] {
        const int size = dtype_size(dtype);
        check_norm(rows, cols, w_dtype);
        check_operand("H", H, rows, cols, ldh, size);
        check_operand("dY", dY, rows, cols, ldy, size);
        if (dH) check_operand("dH", dH, rows, cols, ldd, size);
        check_operand("dX", dX, rows, cols, ldx, size);
        if (rows > 0 && !rstd) fail(GS_ERR_INVALID_ARG, "rstd is null");
        if (w && (uintptr_t)w % dtype_size(w_dtype)) fail(GS_ERR_INVALID_ARG, "w is not aligned to its elements");
        const uint64_t need = norm_grad_need(rows, cols, dtype);
        if (work_bytes < need || !work)
            fail(GS_ERR_INVALID_ARG, "workspace of %llu bytes is below the %llu needed",
                 (unsigned long long)(work ? work_bytes : 0), (unsigned long long)need);
        const auto extent = [&](const void *p, int64_t ld) { return Extent{p, rows, cols * size, ld * size}; };
        const Extent dx = extent(dX, ldx);
        check_apart("dX", dx, "H", extent(H, ldh)), check_apart("dX", dx, "dY", extent(dY, ldy));
        check_apart("dX", dx, "dH", extent(dH, ldd), true);
        const Extent partial = {work, 1, (int64_t)need, (int64_t)need};
        check_apart("work", partial, "H", extent(H, ldh)), check_apart("work", partial, "dY", extent(dY, ldy));
        check_apart("work", partial, "dH", extent(dH, ldd)), check_apart("work", partial, "dX", dx);
        const hipStream_t s = (hipStream_t)stream;
        float *part = (float *)work;
        const double bytes = (double)rows * cols * size * (dH ? 4 : 3);
        const bool nt = streams(bytes, cols, size, {{H, ldh}, {dY, ldy}, {dH, dH ? ldd : ldh}, {dX, ldx}});
        auto go = [&](auto type) {
            using T = decltype(type);
            const NormGradPlan p = norm_grad_plan<T>(rows, cols);
            if (p.wide) {
                float *dots = part + p.blocks * cols;
                if (rows > 0)
                    k_norm_dot<T><<<(unsigned)std::min<int64_t>(rows, 1 << 20), kWideThreads, 0, s>>>(
                        (const T *)H, ldh, rstd, (const T *)dY, ldy, w, w_dtype == GS_F32, rows, (int)cols, dots);
                k_norm_grad_wide<T><<<dim3((unsigned)ceil_div(cols, kRowThreads), (unsigned)p.blocks), kRowThreads, 0, s>>>(
                    (const T *)H, ldh, rstd, (const T *)dY, ldy, w, w_dtype == GS_F32, (const T *)dH, ldd, rows, (int)cols, (T *)dX,
                    ldx, dots, dw ? part : nullptr);
            } else {
                with_row<8, 512, kGradPieces<T>>(ceil_div(cols, kPiece<T>), [&](auto l, auto r) {
                    constexpr int L = decltype(l)::value, N = decltype(r)::value;
                    auto run = [&](auto kernel) {
                        kernel<<<(unsigned)p.blocks, RowAt<T, L, N>::kThreads, 0, s>>>(
                            (const T *)H, ldh, rstd, (const T *)dY, ldy, w, w_dtype == GS_F32, (const T *)dH, ldd, rows, (int)cols,
                            (T *)dX, ldx, dw ? part : nullptr);
                    };
                    nt ? run(k_norm_grad<T, L, N, true>) : run(k_norm_grad<T, L, N, false>);
                });
            }
            GS_HIP(hipGetLastError());
            if (dw) reduce_partials(part, (int)p.blocks, cols, dw, s);
        };
        dtype == GS_F32 ? go(0.0f) : go(u16(0));
    });
}

}  // extern "C"
