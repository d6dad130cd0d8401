// Scores of rows of logits s (n x v), with c = 1 / temperature:
//
//   m = max s,  S = sum exp(c (s - m)),  log p_j = c (s_j - m) - log S
//
// and from them the log probability of a given class, the entropy
// log S - sum exp(x) x / S (x = c (s - m)), the k best classes, the loss of a student
// against a teacher's k best classes, and the gradients of these.  Logits of -inf (masked
// classes) have probability 0 and add nothing; a row of nothing else, or one with a NaN or
// +inf, has no distribution and gives NaN.
//
// Everything is one pass over the logits.  Rows that a wave (or eight of its lanes) holds
// stay in registers between the maximum and the sums; wider ones are read by a workgroup
// with a running maximum and sums in every thread, which are rescaled when the maximum
// moves and joined at the end.
#include <algorithm>

#include "gs_rows.h"

namespace gs {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_inff();

// exp(x), x <= 0 or NaN; 0 below 2^-126.
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// Whole numbers in the order of the values: -0 as +0, every NaN above +inf, 0 below everything.
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return x != x ? 0xffffffffu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

struct ClassIds {
    const void *p;
    bool wide;  // 64-bit
    __device__ __forceinline__ int64_t at(int64_t i) const { return wide ? ((const int64_t *)p)[i] : ((const int32_t *)p)[i]; }
};

struct ScoreOut {
    float *lp, *entropy;
    float2 *stats;
    int top;
    int32_t *top_ids;
    float *top_lp;
};

// What a row's results are made of.
struct RowStats {
    float m, S, X;  // maximum, sum of exp(x), sum of exp(x) x
};

__device__ __forceinline__ void write_scores(const RowStats &t, float logS, int64_t row, const ScoreOut &out, const ClassIds &ids,
                                             float given, int64_t id, int v)
{
    if (out.stats) out.stats[row] = make_float2(t.m, t.S);
    if (out.entropy) out.entropy[row] = logS - t.X / t.S;
    if (out.lp) out.lp[row] = id < 0 ? 0.0f : id < v ? given - t.m - logS : __builtin_nanf("");
}

// The loss of a row against its teacher, over L lanes (a wave's, or a workgroup of L).
struct Teacher {
    ClassIds ids;
    const void *t;
    bool t32;
    int k;
    float c;     // 1 / temperature
    float scale;  // temperature^2
};
template <class T, int L>
__device__ __forceinline__ void write_loss(const RowStats &st, float logS, const T *s, int64_t row, bool in, int v, const Teacher &te,
                                           int lane, float *tmp, float *loss)
{
    auto each = [&](auto &&f) {
        for (int i = lane; i < te.k; i += L) {
            const int64_t at = row * te.k + i;
            const int64_t id = in ? te.ids.at(at) : -1;
            const float t = in ? load_either(te.t, te.t32, at) : 0.0f;
            if (id >= 0 && !(t == -kInf)) f(id, t);
        }
    };
    float tm = -kInf;
    each([&](int64_t, float t) { tm = fmaxf(tm, t); });
    tm = row_fold<L>(tm, tmp, [](float a, float b) { return fmaxf(a, b); });
    float W = 0.0f, D = 0.0f, any = 0.0f;
    each([&](int64_t id, float t) {
        const float d = (t - tm) * te.c, w = exp_neg(d);
        const float x = id < v ? (to_f32(s[id]) - st.m) * te.c : __builtin_nanf("");
        W += w;
        if (!(w == 0.0f)) D = __builtin_fmaf(w, d - x, D);
        if (id >= v) D = x;
        any = 1.0f;
    });
    W = row_sum<L>(W, tmp);
    D = row_sum<L>(D, tmp);
    any = row_sum<L>(any, tmp);
    if (in && lane == 0) loss[row] = any > 0.0f ? te.scale * (D / W + (logS - logf(W))) : 0.0f;
}

// ------------------------------------------------------------ rows in registers

template <class T, int L, int R, bool TEACHER, bool NT>
__global__ __launch_bounds__(kRowThreads) void k_scores_held(const T *__restrict__ s, int64_t ld, int64_t n, int v, ClassIds ids,
                                                            Teacher te, ScoreOut out)
{
    using At = RowAt<T, L, R>;
    constexpr int E = At::E;
    using V = typename Elems<T, E>::type;
    for (int64_t row = At::first_row(), at = (int64_t)blockIdx.x * At::kRows; at < n; row += At::row_step(), at += At::row_step()) {
        const bool in = row < n;
        const T *p = s + row * ld;
        float x[R][E];
        {
            V q[R];
#pragma unroll
            for (int i = 0; i < R; i++) q[i] = load_elems<T, E, NT>(p + At::col(i), in ? v - At::col(i) : 0);
#pragma unroll
            for (int i = 0; i < R; i++)
#pragma unroll
                for (int e = 0; e < E; e++) x[i][e] = At::col(i) + e < v ? to_f32(q[i][e]) : -kInf;
        }
        int64_t id = -1;
        float given = 0.0f;
        if constexpr (!TEACHER) {
            if (in && out.lp && At::lane() == 0) {
                id = ids.at(row);
                if (id >= 0 && id < v) given = to_f32(p[id]);
            }
        }
        RowStats t{-kInf, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int e = 0; e < E; e++) t.m = fmaxf(t.m, x[i][e]);
        t.m = group_fold<L>(t.m, [](float a, float b) { return fmaxf(a, b); });
        const float c = TEACHER ? te.c : 1.0f;
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float d = (x[i][e] - t.m) * c, w = exp_neg(d);
                t.S += w;
                if constexpr (!TEACHER) t.X += w == 0.0f ? 0.0f : w * d;
            }
        t.S = group_sum<L>(t.S);
        if constexpr (!TEACHER) t.X = group_sum<L>(t.X);
        const float logS = logf(t.S);
        if constexpr (TEACHER) {
            write_loss<T, L>(t, logS, p, row, in, v, te, At::lane(), (float *)nullptr, out.lp);
            if (in && At::lane() == 0) out.stats[row] = make_float2(t.m, t.S);
        } else {
            if (in && At::lane() == 0) write_scores(t, logS, row, out, ids, given, id, v);
            // the best, one after another: the largest left, of the lowest index
            if (out.top) {
                uint32_t key[R][E];
#pragma unroll
                for (int i = 0; i < R; i++)
#pragma unroll
                    for (int e = 0; e < E; e++) key[i][e] = At::col(i) + e < v ? order_key(x[i][e]) : 0;
                for (int j = 0; j < out.top; j++) {
                    uint32_t best = 0;
                    int col = 0x7fffffff;
#pragma unroll
                    for (int i = 0; i < R; i++)
#pragma unroll
                        for (int e = 0; e < E; e++)
                            if (key[i][e] > best) {
                                best = key[i][e];
                                col = At::col(i) + e;
                            }
                    const uint32_t top = group_fold_u<L>(best, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
                    col = best == top ? col : 0x7fffffff;
                    col = (int)group_fold_u<L>((uint32_t)col, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
                    if (in && At::lane() == 0) {
                        out.top_ids[row * out.top + j] = col;
                        out.top_lp[row * out.top + j] = key_value(top) - t.m - logS;
                    }
#pragma unroll
                    for (int i = 0; i < R; i++)
#pragma unroll
                        for (int e = 0; e < E; e++)
                            if (At::col(i) + e == col) key[i][e] = 0;
                }
            }
        }
    }
}

// --------------------------------------------------------------- wide rows
//
// A workgroup a row.  The k best are found in the same pass: k of the 256 largest values of
// groups of threads over the first part of the row bound the k-th best from below, and what
// is not below that bound is collected in LDS, a few times k of it; its order decides.  Where
// that is more than LDS holds (long runs of equal logits, rows that ascend) or the row has a
// NaN, the k-th best is found digit by digit in passes of its own.
constexpr int kWideUnits = 4;      // pieces of a thread in flight
constexpr int kTopGroups = 256;
constexpr int kTopKeep = 3072;     // collected at most
constexpr int kTopMax = 128;

typedef unsigned long long u64;
// Orders by value, then by the lower index.
__device__ __forceinline__ u64 order64(uint32_t key, int64_t col) { return (u64)key << 32 | (uint32_t)~(uint32_t)col; }

template <int NT> struct WideLds {
    uint32_t group[kTopGroups];
    u64 keep[kTopKeep];
    int kept;
    uint32_t hist[256];
    u64 prefix;
    int left;
};

// The k-th largest of the workgroup's 256 groups' keys (0 where fewer groups have one), found
// by one wave bit by bit; every thread passes its own.
template <int NT> __device__ __forceinline__ uint32_t bound_of_groups(uint32_t key, int k, WideLds<NT> &lds)
{
    constexpr int G = NT / kTopGroups;
    static_assert(G == 1 || G == 4);
    if constexpr (G == 4) key = group_fold_u<4>(key, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
    if (threadIdx.x % G == 0) lds.group[threadIdx.x / G] = key;
    __syncthreads();
    if (threadIdx.x < kWave) {
        uint32_t g[kTopGroups / kWave], t = 0;
#pragma unroll
        for (int i = 0; i < kTopGroups / kWave; i++) g[i] = lds.group[i * kWave + threadIdx.x];
        for (int b = 31; b >= 0; b--) {
            int c = 0;
#pragma unroll
            for (int i = 0; i < kTopGroups / kWave; i++) c += __popcll(__ballot(g[i] >= (t | 1u << b)));
            if (c >= k) t |= 1u << b;
        }
        if (threadIdx.x == 0) lds.group[0] = t;
    }
    __syncthreads();
    return lds.group[0];
}

// The k best of a row, digit by digit: 4 of the key, 3 of the index.
template <class T, int NT>
__device__ __forceinline__ void top_by_digits(const T *p, int v, int k, WideLds<NT> &lds)
{
    if (threadIdx.x == 0) {
        lds.prefix = 0;
        lds.left = k;
    }
    for (int shift = 56; shift >= 0; shift -= 8) {
        if (shift == 24) continue;  // (indexes have 24 bits: their complements' upper eight are ones)
        for (int i = threadIdx.x; i < 256; i += NT) lds.hist[i] = 0;
        __syncthreads();
        const u64 prefix = lds.prefix;
        const u64 mask = shift == 56 ? 0 : ~0ull << (shift + 8);
        for (int c0 = 0; c0 < v; c0 += NT) {
            const int c = c0 + threadIdx.x;
            const u64 o = c < v ? order64(order_key(to_f32(p[c])), c) : 0;
            const bool on = c < v && (o & mask) == (prefix & mask);
            const uint32_t digit = (uint32_t)(o >> shift) & 255;
            const u64 who = __ballot(on);
            if (who) {
                const uint32_t first = __shfl(digit, __ffsll(who) - 1, kWave);
                if (__ballot(on && digit == first) == who) {  // (runs of equal digits as one)
                    if ((int)(threadIdx.x % kWave) == __ffsll(who) - 1) atomicAdd(&lds.hist[first], (uint32_t)__popcll(who));
                } else if (on) {
                    atomicAdd(&lds.hist[digit], 1u);
                }
            }
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int left = lds.left, d = 255;
            for (; d > 0 && (int)lds.hist[d] < left; d--) left -= lds.hist[d];
            lds.left = left;
            lds.prefix = prefix | (u64)d << shift | (shift == 32 ? 0xff000000ull : 0);
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) lds.kept = 0;
    __syncthreads();
    const u64 least = lds.prefix;
    for (int c = threadIdx.x; c < v; c += NT) {
        const u64 o = order64(order_key(to_f32(p[c])), c);
        if (o >= least) {
            const int at = atomicAdd(&lds.kept, 1);
            if (at < kTopKeep) lds.keep[at] = o;
        }
    }
    __syncthreads();
}

template <class T, int NTH, bool TEACHER, bool TOP>
__global__ __launch_bounds__(NTH) void k_scores_wide(const T *__restrict__ s, int64_t ld, int64_t n, int v, ClassIds ids, Teacher te,
                                                    ScoreOut out)
{
    constexpr int E = kPiece<T>, U = kWideUnits;
    using V = typename Elems<T, E>::type;
    __shared__ std::conditional_t<TOP, WideLds<NTH>, uint8_t> lds;
    __shared__ float fold[NTH / kWave];
    const float c = TEACHER ? te.c : 1.0f;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T *p = s + row * ld;
        if constexpr (TOP) {
            if (threadIdx.x == 0) lds.kept = 0;  // (bound_of_groups' barriers come before its first use)
        }
        RowStats t{-kInf, 0.0f, 0.0f};
        float least = kInf;  // collected from here on
        for (int c0 = 0; c0 < v; c0 += NTH * U * E) {
            V q[U];
#pragma unroll
            for (int i = 0; i < U; i++) {
                const int col = c0 + (i * NTH + threadIdx.x) * E;
                q[i] = load_elems<T, E>(p + col, v - col);
            }
            float m = t.m;
            float x[U][E];
#pragma unroll
            for (int i = 0; i < U; i++)
#pragma unroll
                for (int e = 0; e < E; e++) {
                    x[i][e] = c0 + (i * NTH + (int)threadIdx.x) * E + e < v ? to_f32(q[i][e]) : -kInf;
                    m = fmaxf(m, x[i][e]);
                }
            const float base = m == -kInf ? 0.0f : m;
            const float d0 = t.m == -kInf ? 0.0f : (t.m - base) * c, f = exp_neg(d0);
            if constexpr (!TEACHER) t.X = f * __builtin_fmaf(t.S, d0, t.X);
            t.S *= f;
            t.m = m;
#pragma unroll
            for (int i = 0; i < U; i++)
#pragma unroll
                for (int e = 0; e < E; e++) {
                    const float d = (x[i][e] - base) * c, w = exp_neg(d);
                    t.S += w;
                    if constexpr (!TEACHER) t.X += w == 0.0f ? 0.0f : w * d;
                }
            if constexpr (TOP) {
                if (c0 == 0) {
                    const bool some = (int)threadIdx.x * E < v;
                    least = key_value(std::max(bound_of_groups<NTH>(some ? order_key(m) : 0, out.top, lds), 0x007fffffu));
                }
                float here = -kInf;
#pragma unroll
                for (int i = 0; i < U; i++)
#pragma unroll
                    for (int e = 0; e < E; e++) here = fmaxf(here, x[i][e]);
                if (here >= least) {
#pragma unroll
                    for (int i = 0; i < U; i++)
#pragma unroll
                        for (int e = 0; e < E; e++) {
                            const int col = c0 + (i * NTH + (int)threadIdx.x) * E + e;
                            if (x[i][e] >= least && col < v) {
                                const int at = atomicAdd(&lds.kept, 1);
                                if (at < kTopKeep) lds.keep[at] = order64(order_key(x[i][e]), col);
                            }
                        }
                }
            }
        }
        // the threads' sums joined
        {
            const float m = row_fold<NTH>(t.m, fold, [](float a, float b) { return fmaxf(a, b); });
            const float base = m == -kInf ? 0.0f : m;
            const float d0 = t.m == -kInf ? 0.0f : (t.m - base) * c, f = exp_neg(d0);
            if constexpr (!TEACHER) t.X = row_sum<NTH>(f * __builtin_fmaf(t.S, d0, t.X), fold);
            t.S = row_sum<NTH>(t.S * f, fold);
            t.m = m;
            if (m == -kInf) t.S = __builtin_nanf("");
        }
        const float logS = logf(t.S);
        if constexpr (TEACHER) {
            write_loss<T, NTH>(t, logS, p, row, true, v, te, threadIdx.x, fold, out.lp);
            if (threadIdx.x == 0) out.stats[row] = make_float2(t.m, t.S);
        } else if (threadIdx.x == 0) {
            const int64_t id = out.lp ? ids.at(row) : -1;
            write_scores(t, logS, row, out, ids, id >= 0 && id < v ? to_f32(p[id]) : 0.0f, id, v);
        }
        if constexpr (TOP) {
            // (a barrier lies between the last collected and here)
            if (lds.kept > kTopKeep || t.S != t.S) top_by_digits<T, NTH>(p, v, out.top, lds);
            const int kept = lds.kept < kTopKeep ? lds.kept : kTopKeep;
            for (int i = threadIdx.x; i < kept; i += NTH) {
                const u64 mine = lds.keep[i];
                int rank = 0;
                for (int j = 0; j < kept; j++) rank += lds.keep[j] > mine;
                if (rank < out.top) {
                    out.top_ids[row * out.top + rank] = (int32_t)~(uint32_t)mine;
                    out.top_lp[row * out.top + rank] = key_value((uint32_t)(mine >> 32)) - t.m - logS;
                }
            }
            __syncthreads();  // (before the next row's)
        }
    }
}

// ---------------------------------------------------------------- gradients

// Rows (L lanes each), or pieces of rows of a workgroup (L = kRowThreads: blockIdx.y the
// piece, of `span` columns).
struct GradIn {
    const float2 *stats;
    const float *g, *e, *entropy;  // NULL: none
};

template <class T, int L, bool NT>
__global__ __launch_bounds__(kRowThreads) void k_scores_grad(const T *s, int64_t ld, int64_t n, int v, int span, ClassIds ids, GradIn a,
                                                            T *out, int64_t ldo)
{
    constexpr int E = kPiece<T>, U = 4;
    using V = typename Elems<T, E>::type;
    constexpr int kRows = kRowThreads / L;
    const int lane = threadIdx.x % L, c1 = blockIdx.y * span, c2 = c1 + span < v ? c1 + span : v;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / L; row < n; row += (int64_t)gridDim.x * kRows) {
        const float2 st = a.stats[row];
        const int64_t id = a.g ? ids.at(row) : -1;
        float g = a.g && id >= 0 ? a.g[row] : 0.0f;
        if (id >= v) g = __builtin_nanf("");
        const float e0 = a.e ? a.e[row] : 0.0f, H = a.e ? a.entropy[row] : 0.0f;
        const float inv = 1.0f / st.y, shift = H - logf(st.y);
        for (int c0 = c1 + lane * E; c0 < c2; c0 += L * E * U) {
            V q[U];
#pragma unroll
            for (int i = 0; i < U; i++) q[i] = load_elems<T, E, NT>(s + row * ld + c0 + i * L * E, c2 - c0 - i * L * E);
#pragma unroll
            for (int i = 0; i < U; i++) {
                const int col = c0 + i * L * E;
                V o;
#pragma unroll
                for (int e = 0; e < E; e++) {
                    const float x = to_f32(q[i][e]) - st.x, p = exp_neg(x) * inv;
                    float d = -g * p;
                    if (a.e) d = __builtin_fmaf(-e0, p == 0.0f ? 0.0f : p * (x + shift), d);
                    if (col + e == id) d += g;
                    o[e] = from_f32<T>(d);
                }
                store_elems<T, E, NT>(out + row * ldo + col, o, c2 - col);
            }
        }
    }
}

// Waits for this thread's stores, then for the other threads of the workgroup.
__device__ __forceinline__ void stores_meet()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// The distillation loss's gradient.  The elements at the teacher's classes, which may be the
// same class twice, are made by a lane for each of them and stored over what the row's pass
// left there.  LDS: per row `kp` ids, weights and values.
template <class T, int L, bool NT>
__global__ __launch_bounds__(kRowThreads) void k_distill_grad(const T *s, int64_t ld, int64_t n, int v, int span, Teacher te, GradIn a,
                                                             int kp, T *out, int64_t ldo)
{
    constexpr int E = kPiece<T>, U = 4;
    using V = typename Elems<T, E>::type;
    constexpr int kRows = kRowThreads / L;
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ float fold[kRowThreads / kWave];
    const int lane = threadIdx.x % L, c1 = blockIdx.y * span, c2 = c1 + span < v ? c1 + span : v;
    int *id = (int *)lds + 3 * kp * (threadIdx.x / L);
    float *w = (float *)id + kp, *val = w + kp;
    for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < n; r0 += (int64_t)gridDim.x * kRows) {
        const int64_t row = r0 + threadIdx.x / L;
        const bool in = row < n;
        const float2 st = in ? a.stats[row] : make_float2(0.0f, 1.0f);
        const float inv = 1.0f / st.y;
        float tm = -kInf, bad = 0.0f;
        for (int i = lane; i < kp; i += L) {
            const int64_t at = row * te.k + i;
            int64_t j = in && i < te.k ? te.ids.at(at) : -1;
            const float t = j >= 0 ? load_either(te.t, te.t32, at) : 0.0f;
            if (t == -kInf) j = -1;
            if (j >= v) bad = 1.0f;
            id[i] = j < v ? (int)j : -1;
            w[i] = t;
            if (j >= 0) tm = fmaxf(tm, t);
        }
        tm = row_fold<L>(tm, fold, [](float x, float y) { return fmaxf(x, y); });
        float W = 0.0f;
        for (int i = lane; i < kp; i += L) {
            w[i] = id[i] >= 0 ? exp_neg((w[i] - tm) * te.c) : 0.0f;
            W += w[i];
        }
        W = row_sum<L>(W, fold);
        bad = row_sum<L>(bad, fold);
        float any = 0.0f;
        for (int i = lane; i < te.k; i += L) any += id[i] >= 0 ? 1.0f : 0.0f;
        any = row_sum<L>(any, fold);
        // (NaN where the teacher's weights are, 0 where the row has none of them)
        const float gT = bad > 0.0f ? __builtin_nanf("") : any > 0.0f && in ? a.g[row] / te.c * (W / W) : 0.0f;
        __syncthreads();
        for (int i = lane; i < te.k; i += L) {
            const int j = id[i];
            if (j < c1 || j >= c2) continue;
            float q = 0.0f;
            for (int o = 0; o < kp; o += 4) {
                const int4 jj = *reinterpret_cast<const int4 *>(id + o);
                const float4 ww = *reinterpret_cast<const float4 *>(w + o);
                q += jj.x == j ? ww.x : 0.0f;
                q += jj.y == j ? ww.y : 0.0f;
                q += jj.z == j ? ww.z : 0.0f;
                q += jj.w == j ? ww.w : 0.0f;
            }
            const float x = (to_f32(s[row * ld + j]) - st.x) * te.c;
            val[i] = gT * (exp_neg(x) * inv - q / W);
        }
        __syncthreads();  // (out may be s: its elements have been read)
        const bool none = gT == 0.0f;
        for (int c0 = c1 + lane * E; c0 < c2 && in; c0 += L * E * U) {
            V q[U];
#pragma unroll
            for (int i = 0; i < U; i++) q[i] = load_elems<T, E, NT>(s + row * ld + c0 + i * L * E, c2 - c0 - i * L * E);
#pragma unroll
            for (int i = 0; i < U; i++) {
                const int col = c0 + i * L * E;
                V o;
#pragma unroll
                for (int e = 0; e < E; e++)
                    o[e] = none ? T(0) : from_f32<T>(gT * (exp_neg((to_f32(q[i][e]) - st.x) * te.c) * inv));
                store_elems<T, E, NT>(out + row * ldo + col, o, c2 - col);
            }
        }
        stores_meet();
        for (int i = lane; i < te.k; i += L)
            if (id[i] >= c1 && id[i] < c2) out[row * ldo + id[i]] = from_f32<T>(val[i]);
        __syncthreads();  // (before the next rows')
    }
}

// ------------------------------------------------------------------- launch

void check_logits(const void *s, int64_t ld, int dtype, int64_t n, int64_t v)
{
    const int size = dtype_size(dtype);
    if (n < 0 || n > INT32_MAX || v < 1) fail(GS_ERR_INVALID_ARG, "bad matrix size");
    if (v > kMxMaxCols) fail(GS_ERR_UNSUPPORTED, "at most 2^24 classes");
    check_operand("logits", s, n, v, ld, size);
}
ClassIds check_ids(const char *name, const void *p, int id_bytes, int64_t n)
{
    if (id_bytes != 4 && id_bytes != 8) fail(GS_ERR_INVALID_ARG, "%s have 4 or 8 bytes", name);
    if (n > 0 && !p) fail(GS_ERR_INVALID_ARG, "%s are null", name);
    if ((uintptr_t)p % id_bytes) fail(GS_ERR_INVALID_ARG, "%s are not aligned", name);
    return {p, id_bytes == 8};
}
Teacher check_teacher(const void *ids, int id_bytes, const void *t, int t_dtype, int64_t n, int64_t k, double temperature)
{
    if (k < 1) fail(GS_ERR_INVALID_ARG, "a teacher has at least one class");
    if (k > kTopMax) fail(GS_ERR_UNSUPPORTED, "a teacher has at most %d classes", kTopMax);
    if (!(temperature >= 1e-3) || !(temperature <= 1e3)) fail(GS_ERR_INVALID_ARG, "temperature must be 0.001 to 1000");
    const int size = dtype_size(t_dtype);
    if (n > 0 && !t) fail(GS_ERR_INVALID_ARG, "the teacher's logits are null");
    if ((uintptr_t)t % size) fail(GS_ERR_INVALID_ARG, "the teacher's logits are not aligned");
    return {check_ids("the teacher's classes", ids, id_bytes, n), t, t_dtype == GS_F32, (int)k, (float)(1.0 / temperature),
            (float)(temperature * temperature)};
}

// Rows up to 64 pieces of 16 bytes are held by eight lanes, up to 512 by a wave.
template <class T, bool TEACHER>
void launch_scores(const T *s, int64_t ld, int64_t n, int64_t v, const ClassIds &ids, const Teacher &te, const ScoreOut &out,
                   hipStream_t st)
{
    const int64_t pieces = ceil_div(v, kPiece<T>);
    const bool nt = streams((double)n * v * sizeof(T), v, sizeof(T), {{s, ld}});
    bool done = false;
    if (pieces <= 512)
        done = with_row(pieces, [&](auto l, auto r) {
            constexpr int L = decltype(l)::value, R = decltype(r)::value;
            if constexpr (L <= kWave) {
                const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(n, (int64_t)(kRowThreads / L)), 1 << 20);
                nt ? k_scores_held<T, L, R, TEACHER, true><<<grid, kRowThreads, 0, st>>>(s, ld, n, (int)v, ids, te, out)
                   : k_scores_held<T, L, R, TEACHER, false><<<grid, kRowThreads, 0, st>>>(s, ld, n, (int)v, ids, te, out);
            }
        });
    if (done) return;
    const unsigned grid = (unsigned)std::min<int64_t>(n, 1 << 20);
    auto go = [&](auto kernel, int threads) { kernel<<<grid, threads, 0, st>>>(s, ld, n, (int)v, ids, te, out); };
    const bool large = pieces > 4096;
    if constexpr (TEACHER)
        large ? go(k_scores_wide<T, 1024, true, false>, 1024) : go(k_scores_wide<T, 256, true, false>, 256);
    else if (out.top)
        large ? go(k_scores_wide<T, 1024, false, true>, 1024) : go(k_scores_wide<T, 256, false, true>, 256);
    else
        large ? go(k_scores_wide<T, 1024, false, false>, 1024) : go(k_scores_wide<T, 256, false, false>, 256);
}

// go(L, span, grid): eight lanes a row up to 64 pieces, a wave up to 1024, else a workgroup
// for 16 pieces a thread.
template <class T, class Go> void grad_shape(int64_t n, int64_t v, Go &&go)
{
    const int64_t pieces = ceil_div(v, kPiece<T>);
    auto grid = [&](int64_t rows) { return (unsigned)std::min<int64_t>(ceil_div(n, rows), 1 << 20); };
    if (pieces <= 64)
        go(std::integral_constant<int, 8>{}, (int)v, dim3(grid(kRowThreads / 8)));
    else if (pieces <= 1024)
        go(std::integral_constant<int, 64>{}, (int)v, dim3(grid(kRowThreads / 64)));
    else {
        const int span = kRowThreads * 16 * kPiece<T>;
        const unsigned parts = (unsigned)ceil_div(v, span);
        go(std::integral_constant<int, kRowThreads>{}, span, dim3((unsigned)std::min<int64_t>(n, (1 << 22) / parts), parts));
    }
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" {

int gs_log_probs(const void *s, int64_t ld, int dtype, int64_t n, int64_t v, const void *ids, int id_bytes, float *logp,
                 float *entropy, float *stats, int64_t top, int32_t *top_ids, float *top_logp, gs_stream stream)
{
    return guarded([&] {
        check_logits(s, ld, dtype, n, v);
        if (top < 0 || top > v) fail(GS_ERR_INVALID_ARG, "top must be 0 to the number of classes");
        if (top > kTopMax) fail(GS_ERR_UNSUPPORTED, "top is at most %d", kTopMax);
        const ClassIds id = logp ? check_ids("ids", ids, id_bytes, n) : ClassIds{nullptr, false};
        if (n > 0 && top > 0 && (!top_ids || !top_logp)) fail(GS_ERR_INVALID_ARG, "null output");
        if (n == 0) return;
        const ScoreOut out{logp, entropy, (float2 *)stats, (int)top, top_ids, top_logp};
        const Teacher none{};
        if (dtype == GS_F32)
            launch_scores<float, false>((const float *)s, ld, n, v, id, none, out, (hipStream_t)stream);
        else
            launch_scores<u16, false>((const u16 *)s, ld, n, v, id, none, out, (hipStream_t)stream);
        GS_HIP(hipGetLastError());
    });
}

int gs_log_probs_grad(const void *s, int64_t ld, int dtype, int64_t n, int64_t v, const void *ids, int id_bytes, const float *stats,
                      const float *dlogp, const float *dentropy, const float *entropy, void *out, int64_t ldo, gs_stream stream)
{
    return guarded([&] {
        check_logits(s, ld, dtype, n, v);
        check_operand("out", out, n, v, ldo, dtype_size(dtype));
        const ClassIds id = dlogp ? check_ids("ids", ids, id_bytes, n) : ClassIds{nullptr, false};
        if (n > 0 && (!stats || (dentropy && !entropy))) fail(GS_ERR_INVALID_ARG, "null statistics");
        if ((uintptr_t)stats % 8) fail(GS_ERR_INVALID_ARG, "stats are not 8-byte aligned");
        if (n == 0) return;
        const GradIn a{(const float2 *)stats, dlogp, dentropy, entropy};
        auto go = [&](auto type) {
            using T = decltype(type);
            const bool nt = streams(2.0 * n * v * sizeof(T), v, sizeof(T), {{s, ld}, {out, ldo}});
            grad_shape<T>(n, v, [&](auto l, int span, dim3 grid) {
                constexpr int L = decltype(l)::value;
                auto run = [&](auto kernel) {
                    kernel<<<grid, kRowThreads, 0, (hipStream_t)stream>>>((const T *)s, ld, n, (int)v, span, id, a, (T *)out, ldo);
                };
                nt ? run(k_scores_grad<T, L, true>) : run(k_scores_grad<T, L, false>);
            });
        };
        dtype == GS_F32 ? go(0.0f) : go(u16(0));
        GS_HIP(hipGetLastError());
    });
}

int gs_distill_loss(const void *s, int64_t ld, int dtype, int64_t n, int64_t v, const void *top_ids, int id_bytes,
                    const void *top_logits, int t_dtype, int64_t k, double temperature, float *loss, float *stats, gs_stream stream)
{
    return guarded([&] {
        check_logits(s, ld, dtype, n, v);
        const Teacher te = check_teacher(top_ids, id_bytes, top_logits, t_dtype, n, k, temperature);
        if (n > 0 && (!loss || !stats)) fail(GS_ERR_INVALID_ARG, "null output");
        if ((uintptr_t)stats % 8) fail(GS_ERR_INVALID_ARG, "stats are not 8-byte aligned");
        if (n == 0) return;
        const ScoreOut out{loss, nullptr, (float2 *)stats, 0, nullptr, nullptr};
        const ClassIds none{nullptr, false};
        if (dtype == GS_F32)
            launch_scores<float, true>((const float *)s, ld, n, v, none, te, out, (hipStream_t)stream);
        else
            launch_scores<u16, true>((const u16 *)s, ld, n, v, none, te, out, (hipStream_t)stream);
        GS_HIP(hipGetLastError());
    });
}

int gs_distill_grad(const void *s, int64_t ld, int dtype, int64_t n, int64_t v, const void *top_ids, int id_bytes,
                    const void *top_logits, int t_dtype, int64_t k, double temperature, const float *stats, const float *dloss,
                    void *out, int64_t ldo, gs_stream stream)
{
    return guarded([&] {
        check_logits(s, ld, dtype, n, v);
        check_operand("out", out, n, v, ldo, dtype_size(dtype));
        const Teacher te = check_teacher(top_ids, id_bytes, top_logits, t_dtype, n, k, temperature);
        if (n > 0 && (!stats || !dloss)) fail(GS_ERR_INVALID_ARG, "null statistics or gradient");
        if ((uintptr_t)stats % 8) fail(GS_ERR_INVALID_ARG, "stats are not 8-byte aligned");
        if (n == 0) return;
        const GradIn a{(const float2 *)stats, dloss, nullptr, nullptr};
        const int kp = (int)ceil_div(k, 4) * 4;
        auto go = [&](auto type) {
            using T = decltype(type);
            grad_shape<T>(n, v, [&](auto l, int span, dim3 grid) {
                constexpr int L = decltype(l)::value;
                k_distill_grad<T, L, false><<<grid, kRowThreads, (kRowThreads / L) * 3 * kp * 4, (hipStream_t)stream>>>(
                    (const T *)s, ld, n, (int)v, span, te, a, kp, (T *)out, ldo);
            });
        };
        dtype == GS_F32 ? go(0.0f) : go(u16(0));
        GS_HIP(hipGetLastError());
    });
}

}  // extern "C"
