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
//
// fp32 rows are bound by memory (2,000,000 x 47: 83 us, 4.8 TB/s), wide bf16 rows by the
// instructions of two bytes' exponential and sums (2048 x 128,000 with the 20 best 154 us, 3.4 TB/s;
// 4096 x 50,257 against 64 alternatives 116 us, 3.5).
#include <algorithm>

#include "gs_rows.h"

namespace gs {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_inff();
template <class T> constexpr uint32_t kNegInf = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;

// exp(x), x <= 0 or NaN; 0 below 2^-126.
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// In the place of lower powers, down to -inf, whose weights are 0 long since: its product with what is
// summed, or with a gradient, is finite.
constexpr float kLeast = -0x1p10f;

// The weights of a row's logits are 2^((x - m) k), with k = c log2(e).  (As 2^(x k - m k), with
// one operation less, they would not be right where m k leaves the type's range: rows of its
// lowest number.)
struct Scale {
    float k, m;
    __device__ __forceinline__ Scale(float k_, float m_) : k(k_), m(m_ == -kInf ? 0.0f : m_) {}
    __device__ __forceinline__ float power(float x) const { return (x - m) * k; }
    // Of what was summed with m, where the maximum is `next` from now on (m may have been the type's lowest
    // number, of classes masked with it, or -1e38).
    __device__ __forceinline__ float power_at(const Scale &next) const { return fmaxf((m - next.m) * k, kLeast); }
};
constexpr float kLn2 = 0.6931471805599453f;

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
    // From the sums of the weights, and of weight times power.
    __device__ __forceinline__ void set(float sum, float powers)
    {
        S = m == -kInf ? __builtin_nanf("") : sum;
        X = powers * kLn2;
    }
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
    float c;      // 1 / temperature
    float k2;     // log2(e) / temperature
    float scale;  // temperature^2
    float tiny;   // c / kLossUnit
};
// What the sum of weight times (log q' - log p') is divided by: a hundred of them stay finite for classes that
// the student masked with its type's lowest number, at any temperature.
constexpr float kLossUnit = 0x1p24f;
// Alternative i of a row: its class (negative: none) and what teacher and student give it.
template <class T> struct Alternative {
    int64_t id;
    float t, s;
    __device__ __forceinline__ void load(const Teacher &te, int64_t row, int i, bool in)
    {
        const int64_t at = row * te.k + i;
        id = in && i < te.k ? te.ids.at(at) : -1;
        t = id >= 0 ? load_either(te.t, te.t32, at) : 0.0f;
    }
    __device__ __forceinline__ void look_up(const T *p, int v)  // (in memory or in LDS)
    {
        if (t == -kInf) id = -1;
        s = id < 0 ? 0.0f : id < v ? to_f32(p[id]) : __builtin_nanf("");
    }
};
// The loss, and the statistics that its gradient takes: m, S, the teacher's largest logit and
// 1 / the sum of its weights; 0 instead of that for a row without alternatives, NaN where a
// class is not there.  first: the lane's first alternative, looked up.
template <class T, int L>
__device__ __forceinline__ void write_loss(const RowStats &st, float logS, const T *p, int64_t row, bool in, int v, const Teacher &te,
                                           int lane, const Alternative<T> &first, float *tmp, float *loss, float4 *stats)
{
    auto each = [&](auto &&f) {
        if (first.id >= 0) f(first);
        for (int i = lane + L; i < te.k; i += L) {
            Alternative<T> a;
            a.load(te, row, i, in);
            a.look_up(p, v);
            if (a.id >= 0) f(a);
        }
    };
    float tm = -kInf;
    each([&](const Alternative<T> &a) { tm = fmaxf(tm, a.t); });
    tm = row_fold<L>(tm, tmp, [](float a, float b) { return fmaxf(a, b); });
    // of the weights, of weight (log q' - log p') / kLossUnit, of the alternatives (infinity for one that is not there)
    float sums[3] = {0.0f, 0.0f, 0.0f};
    each([&](const Alternative<T> &a) {
        const float d = a.t - tm, w = exp_neg(d * te.c), x = (a.s - st.m) * te.tiny;
        sums[0] += w;
        if (!(w == 0.0f) || x != x) sums[1] = __builtin_fmaf(w, d * te.tiny - x, sums[1]);
        sums[2] += a.id < v ? 1.0f : kInf;
    });
    row_sums<L, 3>(sums, tmp);
    if (in && lane == 0) {
        loss[row] = sums[2] > 0.0f ? __builtin_fmaf(te.scale * kLossUnit, sums[1] / sums[0], te.scale * (logS - logf(sums[0]))) : 0.0f;
        stats[row] = make_float4(st.m, st.S, tm, sums[2] == kInf ? __builtin_nanf("") : sums[2] > 0.0f ? 1.0f / sums[0] : 0.0f);
    }
}

// ------------------------------------------------------------ rows in registers

// (where there are more sets of rows than workgroups in a launch, 2^20, the next ones are loaded while these
// are worked on; L > 64: a workgroup's row, no alternatives.  Each of the best classes is a scan of the row in
// registers: 200,000 x 1000 fp32 153 us, 369 with 8 of them, 2,093 with 64.)
template <class T, int L, int R, bool TEACHER, bool NT>
__global__ __launch_bounds__(kRowThreads) void k_scores_held(const T *__restrict__ s, int64_t ld, int64_t n, int v, ClassIds ids,
                                                            Teacher te, ScoreOut out)
{
    using At = RowAt<T, L, R>;
    constexpr int E = At::E;
    using V = typename Elems<T, E>::type;
    __shared__ float tmp[3 * kRowThreads / kWave];
    RowPiece<T> q[R];
    Alternative<T> ahead;
    int64_t id_ahead = -1;
    auto load = [&](int64_t row) {
        const bool in = row < n;
#pragma unroll
        for (int i = 0; i < R; i++) q[i].template load<NT>(s + row * ld, At::col(i), v, in);
        if constexpr (TEACHER)
            ahead.load(te, row, At::lane(), in);
        else
            id_ahead = in && out.lp && At::lane() == 0 ? ids.at(row) : -1;
    };
    load(At::first_row());
    for (int64_t row = At::first_row(), at = (int64_t)blockIdx.x * At::kRows; at < n; row += At::row_step(), at += At::row_step()) {
        const bool in = row < n;
        const T *p = s + row * ld;
        float x[R][E];
#pragma unroll
        for (int i = 0; i < R; i++) {
            const V t = q[i].get(At::col(i), v, kNegInf<T>);
#pragma unroll
            for (int e = 0; e < E; e++) x[i][e] = to_f32(t[e]);
        }
        Alternative<T> first = ahead;
        const int64_t id = id_ahead;
        float given = 0.0f;
        if constexpr (TEACHER)
            first.look_up(p, v);
        else if (id >= 0 && id < v)
            given = to_f32(p[id]);
        load(row + At::row_step());
        RowStats t{-kInf, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int e = 0; e < E; e++) t.m = fmaxf(t.m, x[i][e]);
        t.m = row_fold<L>(t.m, tmp, [](float a, float b) { return fmaxf(a, b); });
        const Scale by(TEACHER ? te.k2 : kLog2e, t.m);
        float sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < R; i++)
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float d = by.power(x[i][e]), w = __builtin_amdgcn_exp2f(d);
                sums[0] += w;
                if constexpr (!TEACHER) sums[1] = __builtin_fmaf(w, fmaxf(d, kLeast), sums[1]);
            }
        if constexpr (TEACHER)
            sums[0] = row_sum<L>(sums[0], tmp);
        else
            row_sums<L, 2>(sums, tmp);
        t.set(sums[0], sums[1]);
        const float logS = logf(t.S);
        if constexpr (TEACHER) {
            write_loss<T, L>(t, logS, p, row, in, v, te, At::lane(), first, tmp, out.lp, (float4 *)out.stats);
        } else {
            if (in && At::lane() == 0) write_scores(t, logS, row, out, ids, given, id, v);
            // the best, one after another: the largest left, of the lowest index
            if (L <= kWave && out.top) {
                constexpr int G = L <= kWave ? L : kWave;
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
                    const uint32_t top = group_fold_u<G>(best, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
                    col = best == top ? col : 0x7fffffff;
                    col = (int)group_fold_u<G>((uint32_t)col, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
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

// ------------------------------------------------- short rows, one behind the other
//
// Up to 128 logits a row, rows that follow each other without a gap: a workgroup copies its rows'
// bytes to LDS as whole aligned lines and takes rows from there, L lanes a row, every L-th
// element a lane's; gradients go back the same way.  (In pieces of 16 bytes of each row: gradient of
// 2,000,000 x 47 fp32 223 us for 149, of 1,500,000 x 64 190 for 147, distillation 145 and 283 for 127 and
// 221, 125 and 231 for 113 and 201.  Scores alone are not quicker so: 88 and 91, 80 and 90.)
constexpr int kFlatMost = 128;

// Rows in LDS: behind each other, with a piece between them where whole pieces make a row and
// an even number of them would put many rows on the same banks.
struct FlatRows {
    int v, pitch;
    uint32_t m;  // ceil(2^24 / v): i / v = i m / 2^24 for i below 2^16 (v <= 128)
    template <class T> static FlatRows of(int v)
    {
        constexpr int E = kPiece<T>;
        return {v, v % E == 0 && v / E % 2 == 0 ? v + E : v, (uint32_t)(((1u << 24) + v - 1) / v)};
    }
    __device__ __forceinline__ int place(int i) const  // of element i of the rows
    {
        return pitch == v ? i : i + (int)((uint64_t)(uint32_t)i * m >> 24) * (pitch - v);
    }
    template <class T, int L> __host__ __device__ int elems() const  // of LDS, for whole pieces
    {
        constexpr int E = kPiece<T>;
        return (kRowThreads / L * pitch + E - 1) / E * E;
    }
};
// Copies `count` elements between memory and LDS (16-byte aligned both).
template <class T> __device__ __forceinline__ void flat_load(const T *from, T *to, int count, const FlatRows &f)
{
    constexpr int E = kPiece<T>;
    for (int i = threadIdx.x * E; i < count; i += kRowThreads * E)
        *reinterpret_cast<typename Elems<T, E>::type *>(to + f.place(i)) = load_elems<T, E, true>(from + i, count - i);
}
template <class T> __device__ __forceinline__ void flat_store(T *to, const T *from, int count, const FlatRows &f)
{
    constexpr int E = kPiece<T>;
    for (int i = threadIdx.x * E; i < count; i += kRowThreads * E)
        store_elems<T, E, true>(to + i, *reinterpret_cast<const typename Elems<T, E>::type *>(from + f.place(i)), count - i);
}

// The loss against a teacher.
template <class T, int L, int C>
__global__ __launch_bounds__(kRowThreads) void k_flat_loss(const T *__restrict__ s, int64_t n, FlatRows f, Teacher te, ScoreOut out)
{
    constexpr int ROWS = kRowThreads / L;
    extern __shared__ __align__(16) uint8_t lds[];
    T *all = (T *)lds;
    const int v = f.v, lane = threadIdx.x % L, mine = threadIdx.x / L;
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < n; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = r0 + mine;
        const bool in = row < n;
        const T *p = all + mine * f.pitch;
        Alternative<T> first;
        first.load(te, row, lane, in);
        flat_load(s + r0 * v, all, (int)std::min<int64_t>(ROWS, n - r0) * v, f);
        __syncthreads();
        float x[C], sum = 0.0f;
        RowStats t{-kInf, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < C; i++) {
            const int c = lane + L * i;
            x[i] = in && c < v ? to_f32(p[c]) : -kInf;
            t.m = fmaxf(t.m, x[i]);
        }
        t.m = group_fold<L>(t.m, [](float a, float b) { return fmaxf(a, b); });
        const Scale by(te.k2, t.m);
#pragma unroll
        for (int i = 0; i < C; i++) sum += __builtin_amdgcn_exp2f(by.power(x[i]));
        t.set(group_sum<L>(sum), 0.0f);
        first.look_up(p, v);
        write_loss<T, L>(t, logf(t.S), p, row, in, v, te, lane, first, (float *)nullptr, out.lp, (float4 *)out.stats);
        __syncthreads();  // (before the next rows')
    }
}

// --------------------------------------------------------------- wide rows
//
// A workgroup a row.  The k best are found in the same pass: k of the 256 largest values of
// groups of threads over the first part of the row bound the k-th best from below, and what
// is not below that bound is collected in LDS, a few times k of it; its order decides.  Where
// that is more than LDS holds (long runs of equal logits, rows that ascend) or the row has a
// NaN, the k-th best is found digit by digit in passes of its own.
template <class T> constexpr int kWideUnits = sizeof(T) == 4 ? 4 : 2;  // pieces of a thread at a time, 16 elements
constexpr int kTopGroups = 256;
constexpr int kTopKeep = 2880;     // collected at most
constexpr int kTopMax = 128;

typedef unsigned long long u64;
// Orders by value, then by the lower index.
__device__ __forceinline__ u64 order64(uint32_t key, int64_t col) { return (u64)key << 32 | (uint32_t)~(uint32_t)col; }

template <int NT> struct WideLds {
    uint32_t group[kTopGroups];
    uint32_t bound;  // (not among the groups: waves still read it when the next bound's keys are written)
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
        if (threadIdx.x == 0) lds.bound = t;
    }
    __syncthreads();
    return lds.bound;
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
    constexpr int E = kPiece<T>, U = kWideUnits<T>;
    using V = typename Elems<T, E>::type;
    __shared__ std::conditional_t<TOP, WideLds<NTH>, uint8_t> lds;
    __shared__ float fold[3 * NTH / kWave];
    const float k = TEACHER ? te.k2 : kLog2e;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T *p = s + row * ld;
        if constexpr (TOP) {
            if (threadIdx.x == 0) lds.kept = 0;  // (bound_of_groups' barriers come before its first use)
        }
        Alternative<T> first;
        if constexpr (TEACHER) first.load(te, row, threadIdx.x, true);
        float top = -kInf, sums[2] = {0.0f, 0.0f};
        Scale by(k, top);
        float least = kInf;  // collected from here on
        int parts = 0;
        RowPiece<T> q[U];
#pragma unroll
        for (int i = 0; i < U; i++) q[i].load(p, (i * NTH + (int)threadIdx.x) * E, v);
        for (int c0 = 0; c0 < v; c0 += NTH * U * E) {
            float x[U][E], high[U], here = -kInf;
#pragma unroll
            for (int i = 0; i < U; i++) {
                const V w = q[i].get(c0 + (i * NTH + (int)threadIdx.x) * E, v, kNegInf<T>);
                high[i] = -kInf;
#pragma unroll
                for (int e = 0; e < E; e++) {
                    x[i][e] = to_f32(w[e]);
                    high[i] = fmaxf(high[i], x[i][e]);
                }
                here = fmaxf(here, high[i]);
            }
            if (c0 + NTH * U * E < v)  // (the next ones while these are worked on)
#pragma unroll
                for (int i = 0; i < U; i++) q[i].load(p, c0 + ((U + i) * NTH + (int)threadIdx.x) * E, v);
            if (here > top) {
                const Scale next(k, here);
                const float up = top == -kInf ? 0.0f : by.power_at(next), f = __builtin_amdgcn_exp2f(up);
                if constexpr (!TEACHER) sums[1] = f * __builtin_fmaf(sums[0], up, sums[1]);
                sums[0] *= f;
                top = here;
                by = next;
            }
#pragma unroll
            for (int i = 0; i < U; i++)
#pragma unroll
                for (int e = 0; e < E; e++) {
                    const float d = by.power(x[i][e]), w = __builtin_amdgcn_exp2f(d);
                    sums[0] += w;
                    if constexpr (!TEACHER) sums[1] = __builtin_fmaf(w, fmaxf(d, kLeast), sums[1]);
                }
            if constexpr (TOP) {
                // (after 1, 2, 4 .. parts, of all that has been seen)
                if ((parts & (parts + 1)) == 0) {
                    const bool some = (int)threadIdx.x * E < v;
                    least = key_value(std::max(bound_of_groups<NTH>(some ? order_key(top) : 0, out.top, lds), 0x007fffffu));
                }
                parts++;
#pragma unroll
                for (int i = 0; i < U; i++)
                    if (high[i] >= least) {
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
        if constexpr (TEACHER) first.look_up(p, v);
        // the threads' sums joined
        RowStats t;
        {
            t.m = row_fold<NTH>(top, fold, [](float a, float b) { return fmaxf(a, b); });
            const Scale all(k, t.m);
            const float up = top == -kInf ? 0.0f : by.power_at(all), f = __builtin_amdgcn_exp2f(up);
            float both[2] = {sums[0] * f, f * __builtin_fmaf(sums[0], up, sums[1])};
            row_sums<NTH, 2>(both, fold);
            t.set(both[0], both[1]);
        }
        const float logS = logf(t.S);
        if constexpr (TEACHER) {
            write_loss<T, NTH>(t, logS, p, row, true, v, te, threadIdx.x, first, fold, out.lp, (float4 *)out.stats);
        } else if (threadIdx.x == 0) {
            const int64_t id = out.lp ? ids.at(row) : -1;
            write_scores(t, logS, row, out, ids, id >= 0 && id < v ? to_f32(p[id]) : 0.0f, id, v);
        }
        if constexpr (TOP) {
            // (a barrier lies between the last collected and here)
            if (lds.kept > kTopKeep || t.S != t.S) top_by_digits<T, NTH>(p, v, out.top, lds);
            // Much was collected with bounds from the row's first parts: only what the whole row's leaves is
            // ordered, as that takes the square of its number (2048 x 128,000 bf16, the 128 best:
            // 206 us, and 603 without).
            if (lds.kept > kTopGroups && lds.kept <= kTopKeep) {
                const int all = lds.kept;
                const bool some = (int)threadIdx.x * E < v;
                const uint32_t bound = std::max(bound_of_groups<NTH>(some ? order_key(top) : 0, out.top, lds), 0x007fffffu);
                if (threadIdx.x == 0) lds.kept = 0;
                __syncthreads();
                for (int i = 0; i < all; i += NTH) {
                    const u64 held = i + (int)threadIdx.x < all ? lds.keep[i + threadIdx.x] : 0;
                    __syncthreads();  // (what is written now goes where these or earlier ones were)
                    if ((uint32_t)(held >> 32) >= bound) lds.keep[atomicAdd(&lds.kept, 1)] = held;
                }
                __syncthreads();
            }
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

// Rows of L lanes, or spans of rows of a workgroup (blockIdx.y: the span), R pieces of a lane at
// a time; the next ones, of this row or of the next, are loaded while these are worked on.  Bound by
// memory: 4096 x 50,257 bf16 at odd offsets 173 us, 4.8 TB/s.

// What a lane goes through: steps of its row's span, then of the row after it.
template <class T, int L, int R, bool NT> struct GradWalk {
    static constexpr int E = kPiece<T>, STEP = L * R * E, kRows = kRowThreads / L;
    using V = typename Elems<T, E>::type;
    const T *s;
    int64_t ld, n, row, at;  // at: the workgroup's first row
    int v, c1, c2, c0;
    RowPiece<T> q[R];
    __device__ __forceinline__ static int lane() { return threadIdx.x % L; }
    __device__ __forceinline__ int col(int i) const { return c0 + (i * L + lane()) * E; }
    __device__ __forceinline__ GradWalk(const T *s_, int64_t ld_, int64_t n_, int v_, int span)
        : s(s_), ld(ld_), n(n_), row((int64_t)blockIdx.x * kRows + threadIdx.x / L), at((int64_t)blockIdx.x * kRows), v(v_),
          c1(blockIdx.y * span), c2(c1 + span < v_ ? c1 + span : v_), c0(c1)
    {
        load();
    }
    __device__ __forceinline__ void load()
    {
#pragma unroll
        for (int i = 0; i < R; i++) q[i].template load<NT>(s + row * ld, col(i), v, row < n);
    }
    __device__ __forceinline__ void take(V (&x)[R]) const
    {
#pragma unroll
        for (int i = 0; i < R; i++) x[i] = q[i].get(col(i), v);
    }
    // On to the next step; true: of the same row.
    __device__ __forceinline__ bool next()
    {
        c0 += STEP;
        const bool same = c0 < c2;
        if (!same) {
            c0 = c1;
            row += (int64_t)gridDim.x * kRows;
            at += (int64_t)gridDim.x * kRows;
        }
        load();
        return same;
    }
};
struct GradIn {
    const float *stats;
    const float *g, *e, *entropy;  // NULL: none
};

template <class T, int L, int R, bool NT>
__global__ __launch_bounds__(kRowThreads) void k_scores_grad(const T *s, int64_t ld, int64_t n, int v, int span, ClassIds ids, GradIn a,
                                                            T *out, int64_t ldo)
{
    using Walk = GradWalk<T, L, R, NT>;
    using V = typename Walk::V;
    constexpr int E = Walk::E;
    Walk walk(s, ld, n, v, span);
    struct Given {
        float2 st;
        int64_t id;
        float g, e, H;
    } ahead;
    auto look = [&](int64_t row) {
        const bool in = row < n;
        ahead.st = in ? ((const float2 *)a.stats)[row] : make_float2(0.0f, 1.0f);
        ahead.id = in && a.g ? ids.at(row) : -1;
        ahead.g = in && a.g ? a.g[row] : 0.0f;
        ahead.e = in && a.e ? a.e[row] : 0.0f;
        ahead.H = in && a.e ? a.entropy[row] : 0.0f;
    };
    look(walk.row);
    while (walk.at < n) {
        const int64_t row = walk.row;
        const Given gv = ahead;
        const float g = gv.id < 0 ? 0.0f : gv.id < v ? gv.g : __builtin_nanf("");
        const int mine = gv.id >= 0 && gv.id < v ? (int)gv.id : -1;
        // -g p - e p (log p + H) = weight (fa power + fb)
        const Scale by(kLog2e, gv.st.x);
        const float f = 1.0f / gv.st.y, fa = -gv.e * kLn2 * f, fb = (-g - gv.e * (gv.H - logf(gv.st.y))) * f;
        bool more = true;
        while (more) {
            V x[R];
            walk.take(x);
            const int c0 = walk.c0;
            more = walk.next();
            if (!more) look(walk.row);
#pragma unroll
            for (int i = 0; i < R; i++) {
                const int col = c0 + (i * L + walk.lane()) * E;
                V o;
#pragma unroll
                for (int e = 0; e < E; e++) {
                    const float d = by.power(to_f32(x[i][e])), weight = __builtin_amdgcn_exp2f(d);
                    float y = weight * (a.e ? __builtin_fmaf(fa, fmaxf(d, kLeast), fb) : fb);
                    if (col + e == mine) y += g;
                    o[e] = from_f32<T>(y);
                }
                store_elems<T, E, NT>(out + row * ldo + col, o, row < n ? walk.c2 - col : 0);
            }
        }
    }
}

// Short rows: see k_flat_loss.  TEACHER: the distillation loss's gradient, else the scores'.
constexpr int kFlatAlternatives = 32;
template <class T, int L, int C, bool TEACHER>
__global__ __launch_bounds__(kRowThreads) void k_flat_grad(const T *s, int64_t n, FlatRows f, ClassIds ids, Teacher te, GradIn a, int kp, T *out)
{
    const int v = f.v;
    constexpr int ROWS = kRowThreads / L;
    extern __shared__ __align__(16) uint8_t lds[];
    T *all = (T *)lds;
    const int lane = threadIdx.x % L, mine = threadIdx.x / L;
    T *p = all + mine * f.pitch;
    int *alt = (int *)(all + f.template elems<T, L>()) + 2 * kp * mine;  // classes and weights of the row's alternatives
    float *w = (float *)alt + kp;
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < n; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = r0 + mine;
        const bool in = row < n;
        const int count = (int)std::min<int64_t>(ROWS, n - r0) * v;
        flat_load(s + r0 * v, all, count, f);
        float m, fa = 0.0f, fb, g = 0.0f;
        int given = -1;
        if constexpr (TEACHER) {
            const float4 st = in ? ((const float4 *)a.stats)[row] : make_float4(0.0f, 1.0f, 0.0f, 0.0f);
            m = st.x;
            g = in && st.w != 0.0f ? a.g[row] / te.c + (st.w - st.w) : 0.0f;
            fb = g / st.y;
            for (int i = lane; i < kp; i += L) {
                Alternative<T> one;
                one.load(te, row, i, in);
                const bool there = one.id >= 0 && one.id < v && one.t != -kInf;
                alt[i] = there ? (int)one.id : -1;
                w[i] = there ? exp_neg((one.t - st.z) * te.c) * st.w : 0.0f;
            }
        } else {
            const float2 st = in ? ((const float2 *)a.stats)[row] : make_float2(0.0f, 1.0f);
            const int64_t id = in && a.g ? ids.at(row) : -1;
            const float e = in && a.e ? a.e[row] : 0.0f, H = in && a.e ? a.entropy[row] : 0.0f;
            g = id < 0 ? 0.0f : id < v ? a.g[row] : __builtin_nanf("");
            given = id >= 0 && id < v ? (int)id : -1;
            m = st.x;
            const float inv = 1.0f / st.y;
            fa = -e * kLn2 * inv;
            fb = (-g - e * (H - logf(st.y))) * inv;
        }
        __syncthreads();
        const Scale by(TEACHER ? te.k2 : kLog2e, m);
        float y[C];
#pragma unroll
        for (int i = 0; i < C; i++) {
            const int c = lane + L * i;
            const float d = by.power(in && c < v ? to_f32(p[c]) : 0.0f), weight = __builtin_amdgcn_exp2f(d);
            if constexpr (TEACHER) {
                y[i] = g == 0.0f ? 0.0f : weight * fb;
            } else {
                y[i] = weight * (a.e ? __builtin_fmaf(fa, fmaxf(d, kLeast), fb) : fb);
                if (c == given) y[i] += g;
            }
        }
        // (a lane's own elements: what an alternative adds to one is found before it is rounded)
        if constexpr (TEACHER) {
            for (int o = 0; o < kp; o++) {
                const int at = alt[o] - lane;
                const float add = g * w[o];
#pragma unroll
                for (int i = 0; i < C; i++)
                    if (at == L * i && g != 0.0f) y[i] -= add;
            }
        }
#pragma unroll
        for (int i = 0; i < C; i++)
            if (in && lane + L * i < v) p[lane + L * i] = from_f32<T>(y[i]);
        __syncthreads();
        flat_store(out + r0 * v, all, count, f);
        __syncthreads();  // (before the next rows')
    }
}

// What the L lanes of a row have written to LDS and stored is seen by all of them.
template <int L> __device__ __forceinline__ void lanes_meet()
{
    if constexpr (L <= kWave) {  // (a wave's LDS operations and its stores keep their order)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        asm volatile("" ::: "memory");
    } else {
        __syncthreads();  // (stores of a workgroup's waves reach memory in the order of its barriers)
    }
}

// The distillation loss's gradient.  The elements at the teacher's classes, which may be the
// same class twice, are made by a lane for each of them and stored over what the row's pass
// left there.  LDS: per row `kp` ids, weights and values.
template <class T, int L, int R, bool NT>
__global__ __launch_bounds__(kRowThreads) void k_distill_grad(const T *s, int64_t ld, int64_t n, int v, int span, Teacher te, GradIn a,
                                                             int kp, T *out, int64_t ldo)
{
    using Walk = GradWalk<T, L, R, NT>;
    using V = typename Walk::V;
    constexpr int E = Walk::E;
    extern __shared__ __align__(16) uint8_t lds[];
    int *id = (int *)lds + 3 * kp * (threadIdx.x / L);
    float *w = (float *)id + kp, *val = w + kp;
    Walk walk(s, ld, n, v, span);
    const int c1 = walk.c1, c2 = walk.c2, lane = walk.lane();
    float4 st_ahead;
    float g_ahead;
    Alternative<T> one_ahead;
    auto look = [&](int64_t row) {
        const bool in = row < n;
        st_ahead = in ? ((const float4 *)a.stats)[row] : make_float4(0.0f, 1.0f, 0.0f, 0.0f);
        g_ahead = in ? a.g[row] : 0.0f;
        one_ahead.load(te, row, lane, in);
    };
    look(walk.row);
    while (walk.at < n) {
        const int64_t row = walk.row;
        const bool in = row < n;
        const T *p = s + row * ld;
        const float4 st = st_ahead;
        const Scale by(te.k2, st.x);
        const float inv = 1.0f / st.y;
        // (NaN where the teacher's weights are or a class is not there, 0 for a row without alternatives)
        const float gT = st.w == 0.0f ? 0.0f : g_ahead / te.c + (st.w - st.w);
        // the student's probability and the teacher's at each alternative in the span
        for (int i = lane; i < kp; i += L) {
            Alternative<T> one = one_ahead;
            if (i >= L) one.load(te, row, i, in);
            const bool there = one.id >= 0 && one.id < v && one.t != -kInf;
            id[i] = there ? (int)one.id : -1;
            w[i] = there ? exp_neg((one.t - st.z) * te.c) * st.w : 0.0f;
            if (there && one.id >= c1 && one.id < c2) val[i] = __builtin_amdgcn_exp2f(by.power(to_f32(p[one.id]))) * inv;
        }
        lanes_meet<L>();  // (out may be s: its elements have been read)
        for (int i = lane; i < te.k; i += L) {
            const int j = id[i];
            if (j < c1 || j >= c2) continue;
            float sum = 0.0f;
            for (int o = 0; o < kp; o += 4) {
                const int4 jj = *reinterpret_cast<const int4 *>(id + o);
                const float4 ww = *reinterpret_cast<const float4 *>(w + o);
                sum += jj.x == j ? ww.x : 0.0f;
                sum += jj.y == j ? ww.y : 0.0f;
                sum += jj.z == j ? ww.z : 0.0f;
                sum += jj.w == j ? ww.w : 0.0f;
            }
            val[i] = gT == 0.0f ? 0.0f : gT * (val[i] - sum);
        }
        const float f = gT * inv;
        bool more = true;
        while (more) {
            V x[R];
            walk.take(x);
            const int c0 = walk.c0;
            more = walk.next();
            if (!more) look(walk.row);
#pragma unroll
            for (int i = 0; i < R; i++) {
                const int col = c0 + (i * L + lane) * E;
                V o;
#pragma unroll
                for (int e = 0; e < E; e++) o[e] = gT == 0.0f ? T(0) : from_f32<T>(f * __builtin_amdgcn_exp2f(by.power(to_f32(x[i][e]))));
                store_elems<T, E, NT>(out + row * ldo + col, o, in ? c2 - col : 0);
            }
        }
        lanes_meet<L>();
        for (int i = lane; i < te.k; i += L)
            if (id[i] >= c1 && id[i] < c2) out[row * ldo + id[i]] = from_f32<T>(val[i]);
        lanes_meet<L>();  // (before the next rows')
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
            (float)(1.4426950408889634 / temperature), (float)(temperature * temperature), (float)(1.0 / temperature) / kLossUnit};
}

// Whether rows are short and without gaps; go(L, C): lanes and elements.
template <class T> bool flat_rows(int64_t v, std::initializer_list<std::pair<const void *, int64_t>> operands)
{
    if (v > kFlatMost || v < 8) return false;
    for (const auto &[p, ld] : operands)
        if ((uintptr_t)p % 16 || ld != v) return false;
    return true;
}
template <class Go> void with_flat(int64_t v, Go &&go)
{
    using std::integral_constant;
    const integral_constant<int, 4> l4;
    const integral_constant<int, 8> l8;
    if (v <= 16)
        go(l4, integral_constant<int, 4>{});
    else if (v <= 32)
        go(l4, integral_constant<int, 8>{});
    else if (v <= 48)
        go(l4, integral_constant<int, 12>{});
    else if (v <= 64)
        go(l4, integral_constant<int, 16>{});
    else if (v <= 96)
        go(l8, integral_constant<int, 12>{});
    else
        go(l8, integral_constant<int, 16>{});
}

// Rows that a workgroup (with alternatives to find: a wave) holds stay in registers; wider
// ones take a workgroup a row, the larger the fewer they are (the chip holds 2,048 of 256 threads).
// A workgroup takes one set of rows: 2,048 that go on to further ones are slower (2,000,000 x 47:
// scores 113 and 88 us, gradient 256 and 223).
constexpr int64_t kRowBlocks = 1 << 20;
template <class T, bool TEACHER>
void launch_scores(const T *s, int64_t ld, int64_t n, int64_t v, const ClassIds &ids, const Teacher &te, const ScoreOut &out,
                   hipStream_t st)
{
    const int64_t pieces = ceil_div(v, kPiece<T>);
    // (past the caches only where a load takes whole lines: 2,000,000 x 48 86 us, past them 158)
    const bool nt = pieces > 32 && streams((double)n * v * sizeof(T), v, sizeof(T), {{s, ld}});
    if constexpr (TEACHER) {
        if (flat_rows<T>(v, {{s, ld}})) {
            with_flat(v, [&](auto l, auto c) {
                constexpr int L = decltype(l)::value, C = decltype(c)::value;
                const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(n, (int64_t)(kRowThreads / L)), kRowBlocks);
                const FlatRows f = FlatRows::of<T>((int)v);
                k_flat_loss<T, L, C><<<grid, kRowThreads, f.template elems<T, L>() * sizeof(T), st>>>(s, n, f, te, out);
            });
            return;
        }
    }
    const bool held = pieces <= (out.top ? 4 * kWave : 4 * kRowThreads) && with_row<4, kRowThreads, 4>(pieces, [&](auto l, auto r) {
        constexpr int L = decltype(l)::value, R = decltype(r)::value;
        const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(n, (int64_t)(kRowThreads / L)), kRowBlocks);
        nt ? k_scores_held<T, L, R, TEACHER, true><<<grid, kRowThreads, 0, st>>>(s, ld, n, (int)v, ids, te, out)
           : k_scores_held<T, L, R, TEACHER, false><<<grid, kRowThreads, 0, st>>>(s, ld, n, (int)v, ids, te, out);
    });
    if (held) return;
    const unsigned grid = (unsigned)std::min<int64_t>(n, 1 << 20);
    auto go = [&](auto kernel, int threads) { kernel<<<grid, threads, 0, st>>>(s, ld, n, (int)v, ids, te, out); };
    const bool large = pieces > 2048 && n < 2048;
    if constexpr (TEACHER)
        large ? go(k_scores_wide<T, 1024, true, false>, 1024) : go(k_scores_wide<T, 256, true, false>, 256);
    else if (out.top)
        large ? go(k_scores_wide<T, 1024, false, true>, 1024) : go(k_scores_wide<T, 256, false, true>, 256);
    else
        large ? go(k_scores_wide<T, 1024, false, false>, 1024) : go(k_scores_wide<T, 256, false, false>, 256);
}

// go(L, R, span, grid): rows that a workgroup holds, else spans of four steps of wider ones
// (4096 x 50,257 bf16: 192 us; whole rows 222).
template <class T, class Go> void grad_shape(int64_t n, int64_t v, Go &&go)
{
    const int64_t pieces = ceil_div(v, kPiece<T>);
    if (with_row<4, kRowThreads, 4>(pieces, [&](auto l, auto r) {
            go(l, r, (int)v, dim3((unsigned)std::min<int64_t>(ceil_div(n, (int64_t)kRowThreads / decltype(l)::value), kRowBlocks)));
        }))
        return;
    constexpr int R = 4, STEP = kRowThreads * R * kPiece<T>;
    constexpr int span = 4 * STEP;
    go(std::integral_constant<int, kRowThreads>{}, std::integral_constant<int, R>{}, span,
       dim3((unsigned)std::min<int64_t>(n, kRowBlocks), (unsigned)ceil_div(v, span)));
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
        if ((uintptr_t)stats % 8) fail(GS_ERR_INVALID_ARG, "stats are not 8-byte aligned");
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
        check_apart("out", {out, n, v * dtype_size(dtype), ldo * dtype_size(dtype)}, "logits",
                    {s, n, v * dtype_size(dtype), ld * dtype_size(dtype)}, true);
        if (n == 0) return;
        const GradIn a{stats, dlogp, dentropy, entropy};
        auto go = [&](auto type) {
            using T = decltype(type);
            if (flat_rows<T>(v, {{s, ld}, {out, ldo}})) {
                with_flat(v, [&](auto l, auto c) {
                    constexpr int L = decltype(l)::value, C = decltype(c)::value;
                    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(n, (int64_t)(kRowThreads / L)), kRowBlocks);
                    const FlatRows f = FlatRows::of<T>((int)v);
                    k_flat_grad<T, L, C, false><<<grid, kRowThreads, f.template elems<T, L>() * sizeof(T), (hipStream_t)stream>>>(
                        (const T *)s, n, f, id, Teacher{}, a, 0, (T *)out);
                });
                return;
            }
            const bool nt = streams(2.0 * n * v * sizeof(T), v, sizeof(T), {{s, ld}, {out, ldo}});
            grad_shape<T>(n, v, [&](auto l, auto r, int span, dim3 grid) {
                constexpr int L = decltype(l)::value, R = decltype(r)::value;
                auto run = [&](auto kernel) {
                    kernel<<<grid, kRowThreads, 0, (hipStream_t)stream>>>((const T *)s, ld, n, (int)v, span, id, a, (T *)out, ldo);
                };
                nt ? run(k_scores_grad<T, L, R, true>) : run(k_scores_grad<T, L, R, false>);
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
        if ((uintptr_t)stats % 16) fail(GS_ERR_INVALID_ARG, "stats are not 16-byte aligned");
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
        if ((uintptr_t)stats % 16) fail(GS_ERR_INVALID_ARG, "stats are not 16-byte aligned");
        check_apart("out", {out, n, v * dtype_size(dtype), ldo * dtype_size(dtype)}, "logits",
                    {s, n, v * dtype_size(dtype), ld * dtype_size(dtype)}, true);
        if (n == 0) return;
        const GradIn a{stats, dloss, nullptr, nullptr};
        const int kp = (int)ceil_div(k, 4) * 4;
        auto go = [&](auto type) {
            using T = decltype(type);
            if (k <= kFlatAlternatives && flat_rows<T>(v, {{s, ld}, {out, ldo}})) {
                with_flat(v, [&](auto l, auto c) {
                    constexpr int L = decltype(l)::value, C = decltype(c)::value, ROWS = kRowThreads / L;
                    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(n, (int64_t)ROWS), kRowBlocks);
                    const FlatRows f = FlatRows::of<T>((int)v);
                    const size_t lds = f.template elems<T, L>() * sizeof(T) + (size_t)ROWS * 2 * kp * 4;
                    k_flat_grad<T, L, C, true><<<grid, kRowThreads, lds, (hipStream_t)stream>>>(
                        (const T *)s, n, f, ClassIds{nullptr, false}, te, a, kp, (T *)out);
                });
                return;
            }
            grad_shape<T>(n, v, [&](auto l, auto r, int span, dim3 grid) {
                constexpr int L = decltype(l)::value, R = decltype(r)::value;
                k_distill_grad<T, L, R, false><<<grid, kRowThreads, (kRowThreads / L) * 3 * kp * 4, (hipStream_t)stream>>>(
                    (const T *)s, ld, n, (int)v, span, te, a, kp, (T *)out, ldo);
            });
        };
        dtype == GS_F32 ? go(0.0f) : go(u16(0));
        GS_HIP(hipGetLastError());
    });
}

}  // extern "C"
