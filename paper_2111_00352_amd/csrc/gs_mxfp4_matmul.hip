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
template <class T> struct Out {
    using type = T;
    T *c;
    int64_t ld;
    const uint8_t *mask;
    int64_t mask_pitch;
    bool stream = false;  // stores past the caches' replacement
    // Columns col .. col + E - 1 (col a multiple of E, E 4 or 8) as far as they are below n.
    template <int E> __device__ __forceinline__ void store_row(int64_t row, int64_t col, int64_t n, typename Elems<T, E>::type v) const
    {
        if (mask) {
            const uint32_t *p = reinterpret_cast<const uint32_t *>(mask + row * mask_pitch + col);
#pragma unroll
            for (int e = 0; e < E; e++)
                if ((p[e / 4] >> 8 * (e % 4) & 255) == 0) v[e] = T(0);
        }
        // (row ends by elements: k_narrow would spill for the pieces)
        if (stream)
            store_elems<T, E, true, false>(c + row * ld + col, v, n - col);
        else
            store_elems<T, E, false, false>(c + row * ld + col, v, n - col);
    }
};

// A wave's 32 rows x COLS columns of C on their way through LDS: accumulators hold
// four neighbouring columns of 32 rows, stores want whole lines.
template <class T, int COLS> struct Staged {
    static constexpr int E = 16 / sizeof(T);
    static constexpr int kTiles = COLS / 32;
    static constexpr int kPitch = COLS * sizeof(T) + 16;  // (the shift spreads rows over banks)
    static constexpr int kBytes = 32 * kPitch;
    static constexpr int kLanes = COLS / E, kRows = 64 / kLanes;  // lanes of a row, rows of a store
    uint8_t *lds;
    int lane;
    // acc: lane l, registers 4 g .. 4 g + 3 hold columns 8 g + 4 (l / 32) .. + 3 of row l % 32
    __device__ __forceinline__ void put(int tile, const f32x16 &acc) const
    {
#pragma unroll
        for (int g = 0; g < 4; g++) {
            typedef T quad __attribute__((ext_vector_type(4)));
            const quad v = {from_f32<T>(acc[4 * g]), from_f32<T>(acc[4 * g + 1]), from_f32<T>(acc[4 * g + 2]),
                            from_f32<T>(acc[4 * g + 3])};
            *reinterpret_cast<quad *>(lds + lane % 32 * kPitch + (32 * tile + 8 * g + 4 * (lane / 32)) * sizeof(T)) = v;
        }
    }
    // Rows m0 .. m0 + 31 below m, columns from col0 on below n.  WHOLE: all of them are,
    // there is no mask, and the stores are to go past the caches.
    template <bool WHOLE = false>
    __device__ __forceinline__ void store(const Out<T> &out, int64_t m0, int64_t m, int64_t col0, int64_t n) const
    {
        typedef T whole __attribute__((ext_vector_type(E)));
        __builtin_amdgcn_wave_barrier();  // (a wave's LDS operations keep their order)
        const int64_t col = col0 + lane % kLanes * E;
        whole v[32 / kRows];
#pragma unroll
        for (int i = 0; i < 32 / kRows; i++)
            v[i] = *reinterpret_cast<const whole *>(lds + (kRows * i + lane / kLanes) * kPitch + lane % kLanes * 16);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 32 / kRows; i++) {
            const int64_t row = m0 + kRows * i + lane / kLanes;
            if constexpr (WHOLE)
                store_elems<T, E, true>(out.c + row * out.ld + col, v[i], E);
            else if (row < m && col < n)
                out.template store_row<E>(row, col, n, v[i]);
        }
    }
};

// ------------------------------------------- many rows, up to 512 of k (layers)
//
// Bound by memory: A is read and C written once, B (a layer's weights) is small.
// A workgroup keeps a panel of B in LDS, as the fragments the instructions take;
// each wave takes 32 rows of A at a time, holds their fragments in registers and
// passes over the panel.  B is the instruction's first operand, so a lane ends up
// with four neighbouring columns of one row of C.
//
// A dense A is quantised on the way: the wave loads its rows as they lie in memory
// (8 or 4 lanes a block), finds each block's scale across those lanes and lets LDS
// turn the codes into fragments (a lane a block).
//
// 2,000,000 x 128 x 128 fp32 390 us (5.3 TB/s; reading and writing in equal parts, a
// copy of 8 GB reaches 4.8), 100,000 x 128 x 64 with fp32 operands and a mask 16.5 us (5.3
// TB/s); bf16 100,000 x 128 x 128 8.6 us, of which 2 to 3 are the launch.
constexpr int kNarrowWaves = 4;
constexpr int kNarrowMaxK = 512;
constexpr int kNarrowTmp = 64 * (16 + 1);  // bytes of LDS for a wave's quantisation
constexpr int kNarrowLine = 128;           // bytes of a row of C it stores at a time, and of LDS for that
constexpr int kNarrowOut = 32 * (kNarrowLine + 16);

// A as it is given: MXFP4 codes and scales, or dense.
struct MxRows {
    const uint8_t *codes, *scales;
    int64_t code_pitch;
    int scale_pitch;
    static constexpr double kSize = 0.5;
    int width() const { return scale_pitch * kMxBlock; }
};
template <class T> struct DenseRows {
    const T *p;
    int64_t ld;
    int cols;
    static constexpr double kSize = sizeof(T);
    int width() const { return cols; }
};

// Row source of a wave: fragments of rows m0 + lane % 32, KS times 64 of k: f[ks],
// and their scale bytes, four ks a word.  start() once with the first m0, then
// rows(m0, the one after it) for each.  Loads are issued early, into the next rows at
// the end of these, before this wave's stores to C (a load waits for the stores
// issued before it).
// FIT: kPadded rows, kFull ones (64 KS wide), or full ones that are loaded past the
// caches' replacement.
enum Fit { kPadded, kFull, kFullStream };
template <class Rows, int KS, Fit FIT> struct RowSource;

template <int KS, Fit FIT> struct RowSource<MxRows, KS, FIT> {
    const MxRows &A;
    int lane;
    u32x4 nf[KS];
    uint32_t ns[(KS + 3) / 4];
    __device__ __forceinline__ RowSource(const MxRows &A_, int lane_, uint8_t *) : A(A_), lane(lane_) {}
    __device__ __forceinline__ void start(int64_t m0)
    {
        const int64_t row = m0 + lane % 32;
        const uint8_t *c = A.codes + row * A.code_pitch, *s = A.scales + row * A.scale_pitch;
#pragma unroll
        for (int q = 0; q < (KS + 3) / 4; q++) ns[q] = 0;
#pragma unroll
        for (int ks = 0; ks < KS; ks++) {
            const int blk = 2 * ks + lane / 32;
            nf[ks] = u32x4{};
            if (FIT != kPadded || blk < A.scale_pitch) {
                nf[ks] = *reinterpret_cast<const u32x4 *>(c + 16 * blk);
                ns[ks / 4] |= (uint32_t)s[blk] << 8 * (ks % 4);
            }
        }
    }
    __device__ __forceinline__ void rows(int64_t, int64_t next, int64_t m, u32x4 *f, uint32_t *sc)
    {
#pragma unroll
        for (int ks = 0; ks < KS; ks++) f[ks] = nf[ks];
#pragma unroll
        for (int q = 0; q < (KS + 3) / 4; q++) sc[q] = ns[q];
        if (next < m) start(std::min(next, m - 32));
    }
};

// Dense rows.  tmp: this wave's kNarrowTmp bytes of LDS.
template <class T, int KS, Fit FIT> struct RowSource<DenseRows<T>, KS, FIT> {
    static constexpr int E = 16 / sizeof(T), L = kMxBlock / E;  // elements a lane, lanes a block
    static constexpr int RB = 64 / (2 * L);                     // rows of a load instruction (two blocks of each)
    static constexpr int N = 32 / RB;                           // load instructions of a slice (64 of k)
    static constexpr int kAhead = KS < 2 ? 1 : 2;               // slices
    const DenseRows<T> &A;
    int lane;
    uint8_t *tmp;
    int64_t off;  // of this lane's elements from the first row's of a load
    typename Elems<T, E>::type v[kAhead][N];
    __device__ __forceinline__ RowSource(const DenseRows<T> &A_, int lane_, uint8_t *tmp_) : A(A_), lane(lane_), tmp(tmp_)
    {
        off = lane / (2 * L) * A.ld + lane % (2 * L) * E;
    }
    __device__ __forceinline__ void load(int64_t m0, int ks)
    {
        const T *p = A.p + m0 * A.ld + 64 * ks;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const T *q = p + i * RB * A.ld + off;
            v[ks % kAhead][i] = load_elems<T, E, FIT == kFullStream>(q, FIT == kPadded ? A.cols - 64 * ks - lane % (2 * L) * E : E);
        }
    }
    __device__ __forceinline__ void start(int64_t m0)
    {
#pragma unroll
        for (int ks = 0; ks < kAhead; ks++) load(m0, ks);
    }
    __device__ __forceinline__ void rows(int64_t m0, int64_t next, int64_t m, u32x4 *f, uint32_t *sc)
    {
#pragma unroll
        for (int q = 0; q < (KS + 3) / 4; q++) sc[q] = 0;
#pragma unroll
        for (int ks = 0; ks < KS; ks++) {
#pragma unroll
            for (int i = 0; i < N; i++) {
                const Mx4Lane<T, E> x{v[ks % kAhead][i]};
                const int E8 = mx4_exponent(group_max<L>(x.magnitude()));
                // block (row, h) as lane 32 h + row of the fragment
                const int to = lane / L % 2 * 32 + i * RB + lane / (2 * L);
                if constexpr (E == 8)
                    *reinterpret_cast<uint32_t *>(tmp + 16 * to + lane % L * 4) = x.codes(E8);
                else
                    *reinterpret_cast<u16 *>(tmp + 16 * to + lane % L * 2) = (u16)x.codes(E8);
                if (lane % L == 0) tmp[1024 + to] = (uint8_t)E8;
            }
            if (ks + kAhead < KS)
                load(m0, ks + kAhead);
            else if (next < m)
                load(std::min(next, m - 32), ks + kAhead - KS);
            __builtin_amdgcn_wave_barrier();  // (a wave's LDS operations keep their order)
            f[ks] = *reinterpret_cast<const u32x4 *>(tmp + 16 * lane);
            sc[ks / 4] |= (uint32_t)tmp[1024 + lane] << 8 * (ks % 4);
            __builtin_amdgcn_wave_barrier();
        }
    }
};

template <int J, int KS>
__device__ __forceinline__ f32x16 narrow_chain(const u32x4 *b, const uint32_t *bsc, const u32x4 *f, const uint32_t *sc, f32x16 acc)
{
    if constexpr (J < KS) {
        acc = mfma_fp4<J % 4>(b[64 * J], (int)bsc[64 * (J / 4)], f[J], (int)sc[J / 4], acc);
        return narrow_chain<J + 1, KS>(b, bsc, f, sc, acc);
    } else {
        return acc;
    }
}

// Workgroup b: columns [y * panel, (y + 1) * panel) of C, y = b / gx (panel a
// multiple of 32), of the runs of 32 rows a wave the (b % gx)-th and every gx-th after it.
// Waves of a SIMD, for the registers of the rows in flight.
template <class Rows> constexpr int narrow_waves(int KS)
{
    return KS == 8 ? 2 : KS == 4 || (KS == 2 && std::is_same_v<Rows, DenseRows<float>>) ? 3 : 4;
}

// m >= 32: the last rows are taken as a full 32, some of them twice (with the same
// results).
template <class Rows, class T, int KS, Fit FIT>
__global__ __launch_bounds__(kNarrowWaves * kWave, narrow_waves<Rows>(KS)) void k_narrow(Rows A, const uint8_t *__restrict__ bc,
                                                                 const uint8_t *__restrict__ bs, int64_t m, int64_t n,
                                                                 int kpad, int panel, int gx,
                                                                 Out<T> out)
{
    constexpr int KQ = (KS + 3) / 4;
    extern __shared__ __align__(16) uint8_t lds[];
    const int tiles = panel / 32;
    u32x4 *bf = reinterpret_cast<u32x4 *>(lds);                               // [tile][ks][lane]
    uint32_t *bq = reinterpret_cast<uint32_t *>(lds + tiles * KS * 1024);     // [tile][ks / 4][lane]
    uint8_t *tmp = lds + tiles * (KS * 1024 + KQ * 256);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int64_t n0 = (int64_t)(blockIdx.x / gx) * panel;
    const int64_t cp = kpad / 2;
    const int sp = kpad / kMxBlock;
    for (int i = threadIdx.x; i < tiles * KS * 64; i += kNarrowWaves * kWave) {
        const int l = i % 64, blk = 2 * (i / 64 % KS) + l / 32;
        const int64_t row = std::min<int64_t>(n0 + i / (64 * KS) * 32 + l % 32, n - 1);
        bf[i] = blk < sp ? *reinterpret_cast<const u32x4 *>(bc + row * cp + 16 * blk) : u32x4{};
    }
    for (int i = threadIdx.x; i < tiles * KQ * 64; i += kNarrowWaves * kWave) {
        const int l = i % 64, q = i / 64 % KQ;
        const int64_t row = std::min<int64_t>(n0 + i / (64 * KQ) * 32 + l % 32, n - 1);
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int blk = 2 * (4 * q + j) + l / 32;
            if (4 * q + j < KS && blk < sp) w |= (uint32_t)bs[row * sp + blk] << 8 * j;
        }
        bq[i] = w;
    }
    __syncthreads();
    const int64_t step = (int64_t)gx * kNarrowWaves * 32;
    int64_t m0 = ((int64_t)(blockIdx.x % gx) * kNarrowWaves + wave) * 32;
    if (m0 >= m) return;
    uint8_t *own = tmp + wave * (kNarrowTmp + kNarrowOut);
    RowSource<Rows, KS, FIT> src(A, lane, own);
    const Staged<T, kNarrowLine / sizeof(T)> st{own + kNarrowTmp, lane};
    src.start(std::min(m0, m - 32));
    for (; m0 < m; m0 += step) {
        const int64_t at = std::min(m0, m - 32);
        u32x4 f[KS];
        uint32_t sc[KQ];
        src.rows(at, m0 + step, m, f, sc);
        for (int j = 0; j < tiles && n0 + 32 * j < n; j += st.kTiles) {
#pragma unroll
            for (int i = 0; i < st.kTiles; i++)  // (a second tile past the panel is not stored)
                if (i == 0 || j + i < tiles)
                    st.put(i, narrow_chain<0, KS>(bf + (j + i) * KS * 64 + lane, bq + (j + i) * KQ * 64 + lane, f, sc, f32x16{}));
            st.store(out, at, m, n0 + 32 * j, std::min<int64_t>(n, n0 + panel));
        }
    }
}

// --------------------------------------------------------- few rows, any k
//
// One row or a few against wide weights: bound by reading B once, and by latency.
// A workgroup takes 16 rows of B (so that 4,096 of them fill the chip), its eight
// waves 512 of k at a time each, all of a wave's loads in flight together, and the
// waves' sums are added in LDS.  V_MFMA_SCALE_F32_16X16X128: a lane holds block
// lane / 16 of row lane % 16, of B as it lies in memory.  A dense A
// of at most kFewInside elements is quantised into LDS by every workgroup, after its
// first loads of B are on their way.
//
// 1 x 4096 x 4096 4.4 us (9 MB, 2.0 TB/s): about 1.3 us of reading at the rate of a copy,
// the rest the launch, one round trip to memory and the join.
constexpr int kFewWaves = 8;
constexpr int kFewSteps = 4;  // of 128
constexpr int kFewRows = 64;         // of A at most, 32 where k_narrow could take them
constexpr int64_t kFewInside = 1 << 16;
constexpr int64_t kFewColumns = 1 << 26;  // of C in a launch, which holds fewer than 2^32 threads

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma_fp4_16(u32x4 a, int sa, u32x4 b, int sb, f32x4 c)
{
    const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i32x8 y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, sa, 0, sb);
}

// Blocks 4 (step + i) + lane / 16, i < kFewSteps, of a row of `blocks` blocks whose
// codes and scales start at c and s, zeros past them; scale bytes in byte 0 of sc[i].
__device__ __forceinline__ void load_chunk(const uint8_t *c, const uint8_t *s, int step, int blocks, int lane, u32x4 *f,
                                           uint32_t *sc)
{
    const int q = lane / 16;
    if (4 * (step + kFewSteps) <= blocks) {
        const u32x4 w = *reinterpret_cast<const u32x4u *>(s + 4 * step);
#pragma unroll
        for (int i = 0; i < kFewSteps; i++) {
            f[i] = *reinterpret_cast<const u32x4 *>(c + 64 * (step + i) + 16 * q);
            sc[i] = w[i] >> 8 * q;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kFewSteps; i++) {
            f[i] = u32x4{};
            sc[i] = 0;
            if (4 * (step + i) + q < blocks) {
                f[i] = *reinterpret_cast<const u32x4 *>(c + 64 * (step + i) + 16 * q);
                sc[i] = s[4 * (step + i) + q];
            }
        }
    }
}

// Quantises dense rows of A into LDS: rows of kpad / 2 + 16 bytes, then their scales.
template <class T>
__device__ __forceinline__ void few_quantise(const DenseRows<T> &A, int64_t m, int kpad, uint8_t *codes, uint8_t *scales)
{
    constexpr int E = 8, L = kMxBlock / E;
    const int per = kpad / E, units = (int)m * per;
    for (int u = threadIdx.x; u < units; u += kFewWaves * kWave) {  // (whole blocks: a multiple of 4)
        const int row = u / per, col = u % per * E;
        const Mx4Lane<T, E> x{load_elems<T, E>(A.p + row * A.ld + col, A.cols - col)};
        const int E8 = mx4_exponent(group_max<L>(x.magnitude()));
        *reinterpret_cast<uint32_t *>(codes + row * (kpad / 2 + 16) + col / 2) = x.codes(E8);
        if (u % L == 0) scales[row * (kpad / kMxBlock) + col / kMxBlock] = (uint8_t)E8;
    }
}

// MT: tiles of 16 rows of A.
template <class Rows, class T, int MT>
__global__ __launch_bounds__(kFewWaves * kWave) void k_few(Rows A, const uint8_t *__restrict__ bc,
                                                          const uint8_t *__restrict__ bs, int64_t m, int64_t n, int kpad,
                                                          Out<T> out)
{
    constexpr bool DENSE = !std::is_same_v<Rows, MxRows>;
    __shared__ f32x4 sums[kFewWaves][MT][kWave];
    extern __shared__ __align__(16) uint8_t lds[];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int blocks = kpad / kMxBlock, steps = (blocks + 3) / 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int64_t row = std::min<int64_t>(n0 + lane % 16, n - 1);
    const uint8_t *c = bc + row * (kpad / 2), *s = bs + row * (kpad / kMxBlock);
    const uint8_t *ac, *as;
    int64_t ap, sp;
    u32x4 fb[kFewSteps], fa[kFewSteps];
    uint32_t qb[kFewSteps], qa[kFewSteps];
    int step = kFewSteps * wave;
    if (step < steps) load_chunk(c, s, step, blocks, lane, fb, qb);
    if constexpr (DENSE) {
        ac = lds;
        as = lds + m * (kpad / 2 + 16);
        ap = kpad / 2 + 16;
        sp = kpad / kMxBlock;
        few_quantise(A, m, kpad, lds, lds + m * (kpad / 2 + 16));
        __syncthreads();
    } else {
        ac = A.codes;
        as = A.scales;
        ap = A.code_pitch;
        sp = A.scale_pitch;
    }
    f32x4 acc[MT] = {};
    for (; step < steps; step += kFewSteps * kFewWaves) {
        if (step != kFewSteps * wave) load_chunk(c, s, step, blocks, lane, fb, qb);
#pragma unroll
        for (int t = 0; t < MT; t++) {
            const int64_t i = std::min<int64_t>(16 * t + lane % 16, m - 1);
            load_chunk(ac + i * ap, as + i * sp, step, blocks, lane, fa, qa);
#pragma unroll
            for (int k = 0; k < kFewSteps; k++) acc[t] = mfma_fp4_16(fb[k], (int)qb[k], fa[k], (int)qa[k], acc[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < MT; t++) sums[wave][t][lane] = acc[t];
    __syncthreads();
    if (wave < MT) {
        f32x4 v = sums[0][wave][lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; w++) v += sums[w][wave][lane];
        // accumulator: lane l holds columns 4 (l / 16) .. + 3 of row l % 16 of C
        const int64_t i = 16 * wave + lane % 16, j = n0 + 4 * (lane / 16);
        if (i < m && j < n)
            out.template store_row<4>(i, j, n, typename Elems<T, 4>::type{from_f32<T>(v[0]), from_f32<T>(v[1]), from_f32<T>(v[2]), from_f32<T>(v[3])});
    }
}

// ------------------------------------------------------------ large products
//
// A workgroup of four waves makes a tile of 64 WT x 64 WT, a wave a quarter of it
// (WT x WT instructions of 32 x 32 for every 64 of k).  k is taken in chunks of 256,
// so that a row of a chunk is a whole line of 128 bytes (chunks of 128, half a line a
// row, left the kernel bound by the rate of requests to L2).  Codes go
// from memory to LDS without passing registers, a chunk ahead of the one that is
// multiplied.  A row's eight 16-byte pieces lie in LDS in an order that depends on the
// row (piece ^ row / 2 % 8), so that the rows LDS serves together (16 of 32: those whose
// row / 4 is 0, 3, 5, 6 and the others) spread over all banks; the loads put them there
// by choosing which piece each lane fetches.
//
// A chunk is multiplied as four quarters, the fragments of each read while the one
// before it is multiplied.  The last quarter of a chunk is multiplied after the
// workgroup has met to start the next one, so the matrix cores have work on both
// sides of that barrier.
//
// Scales lie in LDS as 16 bytes of a row, a run of two chunks, loaded a run ahead.
//
// 8192^3 to bf16 255 to 264 us, 4.2 to 4.3 PFLOP/s: 113 us for every 4,096 of k (4.9
// PFLOP/s) and 25 us around them, 16 of which are the stores.  The instructions alone,
// on random operands in registers, reach 6.5 to 7.0 PFLOP/s, at clocks that have fallen
// under that load; with operands that are not loaded anew the loop takes 210 us, with ones
// that are not read from LDS 250.
// Tiles of 256 x 256 leave a compute unit one workgroup, whose stores nothing covers; a
// workgroup that goes on to its next tile meanwhile was slower (261 us: what it keeps
// across the stores spills).
constexpr int kChunkK = 256;

template <int WT> struct TileLds {
    static constexpr int kRows = 64 * WT;                   // of either operand
    static constexpr int kStage = 2 * kRows * kChunkK / 2;  // A's rows, then B's
    __align__(1024) uint8_t codes[2 * kStage];
    __align__(16) uint8_t scales[2][2 * kRows * 16];
    uint8_t after[16];  // (half a chunk at the end of a row reads a word past its scales)
};

// 16 bytes a lane from p + lane_off + off to `to` and the 64 x 16 bytes after it.  The
// callers mark `to` as not overlapping with what they read from LDS meanwhile: the
// compiler then leaves the waiting to them.
__device__ __forceinline__ void load_to_lds(const uint8_t *p, uint32_t lane_off, uint32_t off, uint8_t *to)
{
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, -1, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)to, 16, lane_off, off, 0, 0);
}

// A wave's share of the loads: 2 WT of either operand a chunk and one of the scales.
// Load q fills rows 8 (wave 2 WT + q) .. + 7 of a stage; of the scale rows of both
// operands, in order, a wave takes 32 WT, 64 with each chunk.  Rows past the last one
// repeat it (their results are not stored).
template <int WT> struct TileLoads {
    uint32_t a[2 * WT], b[2 * WT];  // offsets from the tile's first row of A and B
    uint32_t s[WT / 2];             // and of the scale rows (A's or B's)
    int kpad;
    bool upper;                     // this lane's piece for even q (the other half for odd) is
                                    // in the upper half of a row of a chunk
};
template <int WT>
__device__ __forceinline__ void tile_load(uint8_t *__restrict__ to, uint8_t *__restrict__ scales_to,
                                          const uint8_t *__restrict__ ga, const uint8_t *__restrict__ gb,
                                          const uint8_t *__restrict__ gs, const TileLoads<WT> &ld, int chunk, int run,
                                          int group)
{
    // (a row that ends with half a chunk: the upper half, which is not read, repeats the lower)
    const uint32_t over = (chunk + 1) * kChunkK > ld.kpad ? 64u : 0u;
    const uint32_t back[2] = {ld.upper ? over : 0, ld.upper ? 0 : over};
#pragma unroll
    for (int q = 0; q < 2 * WT; q++) {
        load_to_lds(ga, ld.a[q] - back[q % 2], chunk * (kChunkK / 2), to + 1024 * q);
        load_to_lds(gb, ld.b[q] - back[q % 2], chunk * (kChunkK / 2), to + WT * 8192 + 1024 * q);
    }
    uint32_t so = ld.s[0];
    if constexpr (WT == 4) so = group ? ld.s[1] : so;
    load_to_lds(gs, so, std::min(16 * run, ld.kpad / kMxBlock - 16), scales_to + (WT == 4 ? group * 1024 : 0));
}

template <int WT> struct Frags {
    u32x4 a[WT], b[WT];
};
template <int WT> struct ScaleWords {  // of a chunk: 128 of k each
    uint32_t a[2][WT], b[2][WT];
};
template <int WT> struct TileReads {
    int a, b;    // this lane's row of A and B in a stage
    int sa, sb;  // and its scales in a run
    int half, swz;
    __device__ __forceinline__ void frags(const uint8_t *from, int q, Frags<WT> &f) const
    {
        const uint8_t *p = from + ((2 * q + half) ^ swz) * 16;
#pragma unroll
        for (int i = 0; i < WT; i++) {
            f.a[i] = *reinterpret_cast<const u32x4 *>(p + a + i * 4096);
            f.b[i] = *reinterpret_cast<const u32x4 *>(p + b + i * 4096);
        }
    }
    __device__ __forceinline__ void scales(const uint8_t *from, ScaleWords<WT> &s) const
    {
#pragma unroll
        for (int i = 0; i < WT; i++) {
            typedef uint32_t pair __attribute__((ext_vector_type(2), aligned(4)));
            const pair x = *reinterpret_cast<const pair *>(from + sa + i * 512);
            const pair y = *reinterpret_cast<const pair *>(from + sb + i * 512);
            s.a[0][i] = x[0], s.a[1][i] = x[1];
            s.b[0][i] = y[0], s.b[1][i] = y[1];
        }
    }
};
// Quarter Q.  B is the first operand: a lane's sums are four neighbouring columns of a row of C.
template <int Q, int WT>
__device__ __forceinline__ void tile_mul(f32x16 (&acc)[WT][WT], const Frags<WT> &f, const ScaleWords<WT> &s, int half)
{
#pragma unroll
    for (int i = 0; i < WT; i++)
#pragma unroll
        for (int j = 0; j < WT; j++)
            acc[i][j] = mfma_fp4<2 * (Q & 1)>(f.b[j], (int)(s.b[Q / 2][j] >> 8 * half), f.a[i], (int)(s.a[Q / 2][i] >> 8 * half),
                                              acc[i][j]);
}

// Of the instructions up to the next sched_barrier: COUNT groups of one
// multiplication, R LDS reads and V loads.
template <int COUNT, int R, int V> __device__ __forceinline__ void interleave()
{
#pragma unroll
    for (int i = 0; i < COUNT; i++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if constexpr (R) __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
        if constexpr (V) __builtin_amdgcn_sched_group_barrier(0x010, V, 0);
    }
}

// Fragments of A and the scales of a chunk's upper half, if keep is ~0.
template <int WT> __device__ __forceinline__ void keep_rows(Frags<WT> &f, ScaleWords<WT> &s, uint32_t keep)
{
#pragma unroll
    for (int i = 0; i < WT; i++) {
        f.a[i] &= keep;
        s.a[1][i] &= keep;
        s.b[1][i] &= keep;
    }
}

// One chunk, which lies in `from`.  held, s: the last quarter of the chunk before it
// and its scales, on return this one's.  FIRST: there is none before it.  LAST: nothing
// is loaded, and if keep is 0 instead of ~0 the chunk is half a one, whose other half
// is taken as zeros.
template <int WT, bool FIRST, bool LAST>
__device__ __forceinline__ void tile_chunk(uint8_t *__restrict__ to, uint8_t *__restrict__ scales_to,
                                           const uint8_t *__restrict__ from, const uint8_t *__restrict__ scales,
                                           const uint8_t *__restrict__ ga, const uint8_t *__restrict__ gb,
                                           const uint8_t *__restrict__ gs, const TileLoads<WT> &ld,
                                           const TileReads<WT> &rd, int chunk, uint32_t keep,
                                           f32x16 (&acc)[WT][WT], Frags<WT> &held, ScaleWords<WT> &s)
{
    Frags<WT> f;
    ScaleWords<WT> sn;
    rd.scales(scales, sn);
    rd.frags(from, 0, f);
    if constexpr (!LAST) tile_load<WT>(to, scales_to, ga, gb, gs, ld, chunk + 1, (chunk >> 1) + 1, chunk & 1);
    if constexpr (!FIRST) {
        tile_mul<3, WT>(acc, held, s, rd.half);
        interleave<2 * WT, 2, LAST ? 0 : 1>();
        interleave<WT == 4 ? 8 : 0, 0, LAST ? 0 : 1>();
    }
    __builtin_amdgcn_sched_barrier(0);
    s = sn;
    rd.frags(from, 1, held);
    tile_mul<0, WT>(acc, f, s, rd.half);
    interleave<2 * WT, 1, 0>();
    __builtin_amdgcn_sched_barrier(0);
    rd.frags(from, 2, f);
    tile_mul<1, WT>(acc, held, s, rd.half);
    interleave<2 * WT, 1, 0>();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (LAST) keep_rows(f, s, keep);
    rd.frags(from, 3, held);
    tile_mul<2, WT>(acc, f, s, rd.half);
    interleave<2 * WT, 1, 0>();
    if constexpr (LAST) keep_rows(held, s, keep);
    __builtin_amdgcn_sched_barrier(0);
}

// This wave's loads have arrived and its LDS reads are done, and so are all others'.
__device__ __forceinline__ void tile_meet()
{
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
}

// Chunks [slice * per, (slice + 1) * per) of k (the last slice: to the end), slice =
// blockIdx.y, per even, at least two of them; slice i's product goes to out i * m * n
// elements on.  kpad >= 512, a multiple of 128.
template <class T, int WT>
__global__ __launch_bounds__(256, WT == 4 ? 1 : 2) void k_tile(const uint8_t *__restrict__ ac,
                                                               const uint8_t *__restrict__ as,
                                                               const uint8_t *__restrict__ bc,
                                                               const uint8_t *__restrict__ bs, int64_t m, int64_t n,
                                                               int kpad, int per, int tiles_m, int tiles_n,
                                                               Out<T> out)
{
    constexpr int BM = 64 * WT;
    using Lds = TileLds<WT>;
    __shared__ Lds lds;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int cp = kpad / 2, sp = kpad / kMxBlock, all = (kpad + kChunkK - 1) / kChunkK;
    const int first = (int)blockIdx.y * per, chunks = blockIdx.y + 1 == gridDim.y ? all : first + per;  // the end
    // an XCD takes a contiguous run of tiles, in panels of 8 rows of them
    const int t = (int)xcd_tile(blockIdx.x, (int64_t)tiles_m * tiles_n);
    const int panel = t / (8 * tiles_n), in = t % (8 * tiles_n), ph = std::min(8, tiles_m - 8 * panel);
    // (divided in vector registers: told to be the same for all lanes)
    const int64_t m0 = (int64_t)__builtin_amdgcn_readfirstlane(8 * panel + in % ph) * BM;
    const int64_t n0 = (int64_t)__builtin_amdgcn_readfirstlane(in / ph) * BM;
    const int wm = wave / 2, wn = wave % 2, r = lane % 32;
    const int last_a = (int)std::min<int64_t>(BM, m - m0) - 1, last_b = (int)std::min<int64_t>(BM, n - n0) - 1;

    const uint8_t *ga = ac + m0 * cp, *gb = bc + n0 * cp;
    const bool of_b = wave >= 2;
    const uint8_t *gs = of_b ? bs + n0 * sp : as + m0 * sp;
    TileLoads<WT> ld;
#pragma unroll
    for (int q = 0; q < 2 * WT; q++) {
        const int row = 8 * (wave * 2 * WT + q) + lane / 8, piece = (lane % 8) ^ (row / 2 % 8);
        ld.a[q] = (uint32_t)std::min(row, last_a) * cp + piece * 16;
        ld.b[q] = (uint32_t)std::min(row, last_b) * cp + piece * 16;
    }
#pragma unroll
    for (int g = 0; g < WT / 2; g++)
        ld.s[g] = (uint32_t)std::min(wave % 2 * 32 * WT + 64 * g + lane, of_b ? last_b : last_a) * sp;
    ld.kpad = kpad;
    ld.upper = lane % 8 >= 4;
    TileReads<WT> rd;
    rd.a = (wm * WT * 32 + r) * 128, rd.b = (BM + wn * WT * 32 + r) * 128;
    rd.sa = (wm * WT * 32 + r) * 16, rd.sb = (BM + wn * WT * 32 + r) * 16;
    rd.half = lane / 32, rd.swz = r / 2 % 8;
    // Wave's places, and those of chunk c's scales (run c / 2 starts at byte
    // min(16 (c / 2), sp - 16) of a scale row).
    auto put = [&](int c) { return lds.codes + (c & 1) * Lds::kStage + 2048 * WT * wave; };
    auto put_scales = [&](int run) { return lds.scales[run & 1] + 32 * WT * 16 * wave; };
    auto codes_of = [&](int c) { return lds.codes + (c & 1) * Lds::kStage; };
    auto scales_of = [&](int c) { return lds.scales[c >> 1 & 1] + 8 * c - std::min(16 * (c >> 1), sp - 16); };

    tile_load<WT>(put(0), put_scales(first / 2), ga, gb, gs, ld, first, first / 2, 0);
    if constexpr (WT == 4) load_to_lds(gs, ld.s[1], std::min(8 * first, sp - 16), put_scales(first / 2) + 1024);
    f32x16 acc[WT][WT] = {};
    Frags<WT> held;
    ScaleWords<WT> s;
    tile_meet();
    tile_chunk<WT, true, false>(put(1), put_scales(first / 2 + 1), codes_of(0), scales_of(first), ga, gb, gs, ld, rd, first,
                                0, acc, held, s);
    int c = first + 1;
#pragma unroll 1
    for (; c < chunks - 1; c++) {
        tile_meet();
        tile_chunk<WT, false, false>(put(c + 1), put_scales((c >> 1) + 1), codes_of(c), scales_of(c), ga, gb, gs, ld, rd, c,
                                     0, acc, held, s);
    }
    tile_meet();
    tile_chunk<WT, false, true>(put(0), put_scales(0), codes_of(c), scales_of(c), ga, gb, gs, ld, rd, c,
                                chunks == all && kpad % kChunkK ? 0u : ~0u, acc, held, s);
    tile_mul<3, WT>(acc, held, s, rd.half);

    using St = Staged<T, 32 * WT>;
    static_assert(4 * St::kBytes <= 2 * Lds::kStage);
    __syncthreads();  // every wave has read the last step
    const St st{lds.codes + wave * St::kBytes, lane};
    out.c += (int64_t)blockIdx.y * m * n;
    auto store = [&](auto whole) {
#pragma unroll
        for (int i = 0; i < WT; i++) {
#pragma unroll
            for (int j = 0; j < WT; j++) st.put(j, acc[i][j]);
            st.template store<decltype(whole)::value>(out, m0 + 32 * (wm * WT + i), m, n0 + 32 * wn * WT, n);
        }
    };
    // (4096 x 8192 and more of C without a branch a piece: 8192 x 8192 x 512 in 32 bits
    // 84.9 us with them, 79.5 without, x 8192 in 16 bits 257 and 254)
    if (out.stream && !out.mask && m0 + BM <= m && n0 + BM <= n)
        store(std::true_type{});
    else
        store(std::false_type{});
}

// C from `split` partial products of m x n, added in order.
template <class T>
__global__ __launch_bounds__(256) void k_join(const float *__restrict__ part, int split, int64_t m, int64_t n, Out<T> out)
{
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, row = blockIdx.y;
    if (col >= n) return;
    Elems<float, 4>::type s = {};
    constexpr int U = 4;  // partials in flight
    for (int p = 0; p < split; p += U) {
        Elems<float, 4>::type v[U] = {};
#pragma unroll
        for (int u = 0; u < U; u++)
            if (p + u < split) v[u] = load_elems<float, 4>(part + ((int64_t)(p + u) * m + row) * n + col, n - col);
#pragma unroll
        for (int u = 0; u < U; u++) s += v[u];
    }
    out.template store_row<4>(row, col, n, typename Elems<T, 4>::type{from_f32<T>(s[0]), from_f32<T>(s[1]), from_f32<T>(s[2]), from_f32<T>(s[3])});
}

uint64_t round256(uint64_t x) { return (x + 255) / 256 * 256; }

void check_sizes(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || n < 0 || k < 0 || m > INT32_MAX || n > INT32_MAX) fail(GS_ERR_INVALID_ARG, "bad product size");
    if (k > kMxMaxCols) fail(GS_ERR_UNSUPPORTED, "at most 2^24 columns");
}

// How a product of k > 0 is formed.  Measured on both sides of each limit (us in a graph, A in
// MXFP4, C in fp32; n x k of B):
// - Under 32 rows only k_few can (k_narrow takes 32 at a time).  32 rows, k_few and k_narrow: 4096 x
//   64 3.2 and 3.0, 4096 x 256 3.4 and 3.5, 128 x 512 2.9 and 3.8; 64 rows 3.8 and 3.1, 4.2 and 3.7,
//   3.5 and 4.2.  A dense A of 32 rows is quicker by k_few: 4096 x 256 from bf16 4.0 and 6.6.
// - At a padded k of 512 both k_narrow (512 at most) and k_tile (512 at least) can: 1,000 rows, n = 500 5.2
//   and 6.0; 8,192 rows, n = 512 9.3 and 6.1; 100,000 rows, n = 128 20.8 and 26.5, n = 512 58.5 and
//   50.7.  The limit in n is right at both ends only: from 8,192 rows on tiles are quicker at n = 256
//   (6.5 and 4.9; 100,000 rows 38.5 and 27.6), at 1,000 rows k_narrow still is at n = 1024 (5.3 and 5.8).
// - Up to 64 rows and a longer k, k_few and k_tile: 64 rows, 512 x 1024 3.8 and 6.3, 4096 x 4096 8.1 and
//   11.0; with much of B the tiles are quicker already (8192 x 8192 25.7 and 16.5, 300 x 8192 12.9 and 9.5).
enum class Way { kFew, kNarrow, kTile };
Way way(int64_t m, int64_t n, int kpad)
{
    if (m < 32) return Way::kFew;
    if (kpad <= kNarrowMaxK && (kpad < 512 || n < 512)) return Way::kNarrow;
    return m <= kFewRows ? Way::kFew : Way::kTile;
}

// Columns of B that a workgroup of k_narrow keeps: 32 KB of it (KS times 64 of k).  With 32 KB
// and with 16 (us in a graph, MXFP4 to fp32): 100,000 x 1024 x 64 107 and 121, 100,000 x 300 x 384 88 and 93,
// 500,000 x 512 x 128 207 and 207, 100,000 x 512 x 256 49 and 45.  Two workgroups
// of 32 KB fit a compute unit's LDS, one of 64 KB would.
int narrow_slices(int kpad) { return kpad <= 64 ? 1 : kpad <= 128 ? 2 : kpad <= 256 ? 4 : 8; }
int64_t narrow_columns(int kpad) { return 32 * (32 / narrow_slices(kpad)); }

// Whether a dense A is quantised by the kernel that multiplies it: by k_few up to kFewInside elements,
// by k_narrow while one panel holds all of B.  Inside and in a launch before it (us in a graph, where a
// launch costs 2 us instead of the host's 3): k_few, bf16, 1 x 4096 x 4096 4.0 and 6.0, 31 x 1000 x 1024
// 5.8 and 6.8, at its limit 16 x 4096 x 4096 10.3 and 7.9; k_narrow, 100,000 x 256 x 256 from bf16 32 and 41,
// from fp32 41 and 49, past its limit 100,000 x 512 x 256 from fp32 73 and 71, x 300 x 384 127 and 117.
bool quantised_inside(int64_t m, int64_t n, int kpad)
{
    switch (way(m, n, kpad)) {
    case Way::kFew: return m <= 32 && m * kpad <= kFewInside;
    case Way::kNarrow: return n <= narrow_columns(kpad);
    default: return false;
    }
}

// Tiles of a large product, and how many slices of k they are made in.
struct TilePlan {
    int wt, split, per;
    int64_t tiles_m, tiles_n;
};
TilePlan tile_plan(int64_t m, int64_t n, int kpad)
{
    TilePlan p;
    // Tiles of 128 x 128 and of 256 x 256 (us in a graph, MXFP4 to bf16): 120 large ones, 2048 x 3840 x 1024,
    // 8.1 and 11.4; 128, 2048 x 4096 x 4096, 25 and 29; 143, 2816 x 3328 x 1152, 13.8 and 13.8; 144, 3000^3, 30 and
    // 26.5; 256, 4096^3, 51 and 38.  Small ones stay quicker where k is short: 8192 x 8192 x 1024 60 and 66.
    p.wt = ceil_div(m, 256) * ceil_div(n, 256) >= 128 ? 4 : 2;
    p.tiles_m = ceil_div(m, 64 * p.wt);
    p.tiles_n = ceil_div(n, 64 * p.wt);
    // Slices of k are for products with fewer tiles than compute units.  A chunk takes a
    // workgroup about 0.55 us; the second launch costs 4 us, and partial products are
    // written and read at about 5 TB/s: 224 x 310 x 8192 20.1 us in one, 10.1 us in eight;
    // 256 x 4096 x 4096 12.0 us in one, 19.7 us in four.
    const int chunks = (kpad + kChunkK - 1) / kChunkK;
    const int64_t idle = compute_units() / (p.tiles_m * p.tiles_n);
    p.per = chunks;
    p.split = 1;
    double best = 0;
    for (int per = 2; per < chunks; per += 2) {
        const int split = chunks / per, longest = chunks - (split - 1) * per;
        if (split < 2 || split > idle) continue;
        const double gain = 0.55 * (chunks - longest) - 4.0 - (double)split * m * n * 8 / 5e6;
        if (gain > best) {
            best = gain;
            p.per = per;
            p.split = split;
        }
    }
    return p;
}

uint64_t dense_bytes(int64_t m, int kpad) { return round256((uint64_t)m * kpad / 2) + round256((uint64_t)m * kpad / kMxBlock); }

// Workspace: A's codes and scales when A is dense and quantised first, and the
// partial products of slices of k.
uint64_t workspace(int64_t m, int64_t n, int64_t k, int a_dtype)
{
    const int kpad = (int)mx4_cols(k);
    uint64_t bytes = a_dtype < 0 || quantised_inside(m, n, kpad) ? 0 : dense_bytes(m, kpad);
    if (way(m, n, kpad) == Way::kTile)
        if (const TilePlan p = tile_plan(m, n, kpad); p.split > 1) bytes += (uint64_t)p.split * m * n * 4;
    return bytes;
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

struct Product {
    int64_t m, n;
    int kpad;
    const gs_mxfp4 *B;
    const gs_saved *mask;
    void *C;
    int64_t ldc;
    int dtype;
    hipStream_t s;
    float *part;  // for slices of k
};

// f(Out<T>) for the product's type and mask.
template <class F> void with_out(const Product &p, F &&f)
{
    auto typed = [&](auto type) {
        using T = decltype(type);
        f(Out<T>{(T *)p.C, p.ldc, p.mask ? p.mask->codes : nullptr, p.mask ? saved_code_pitch(p.n) : 0});
    };
    p.dtype == GS_F32 ? typed(0.0f) : typed(u16(0));
    GS_HIP(hipGetLastError());
}

template <class Rows> void multiply_narrow(const Product &p, const Rows &A)
{
    // Panels of 32 KB of B (two workgroups to a compute unit), fewer columns while
    // there are fewer workgroups than compute units: 512 x 512 x 256 from fp32 7.2 us, 12.4 with
    // whole panels, 8192 x 512 x 128 7.6 and 15.3 (20,000 x 128 x 128 7.7 and 7.2).
    const int KS = narrow_slices(p.kpad);
    const int64_t groups = ceil_div(p.m, 32 * kNarrowWaves);
    int64_t panel = std::min<int64_t>(ceil_div(p.n, 32) * 32, narrow_columns(p.kpad));
    while (panel > 32 && groups * ceil_div(p.n, panel) < compute_units()) panel = ceil_div(panel / 2, 32) * 32;
    const int64_t panels = ceil_div(p.n, panel);
    const int64_t gx = std::min<int64_t>(groups, std::max<int64_t>(1, 8 * compute_units() / panels));
    if (gx * panels >= 1 << 24) fail(GS_ERR_UNSUPPORTED, "the product has too many tiles");
    with_out(p, [&](auto out) {
        using T = typename decltype(out)::type;
        // C past the caches: 500,000 x 128 x 128 fp32 105 -> 81 us; and A where both are
        // far larger than these: 1,000,000 x 64 x 128 175 -> 152 us (the former: 96 us).
        out.stream = true;
        const double bytes = (double)p.m * (A.width() * Rows::kSize + p.n * sizeof(T));
        auto go = [&](auto ks, auto fit) {
            constexpr int K = decltype(ks)::value;
            const size_t lds = panel / 32 * (K * 1024 + (K + 3) / 4 * 256) + kNarrowWaves * (kNarrowTmp + kNarrowOut);
            k_narrow<Rows, T, K, decltype(fit)::value><<<(unsigned)(gx * panels), kNarrowWaves * kWave, lds, p.s>>>(
                A, p.B->codes, p.B->scales, p.m, p.n, p.kpad, (int)panel, (int)gx, out);
        };
        auto sized = [&](auto ks) {
            if (A.width() != 64 * KS) return go(ks, std::integral_constant<Fit, kPadded>{});
            if constexpr (!std::is_same_v<Rows, MxRows>)
                if (bytes > 700e6) return go(ks, std::integral_constant<Fit, kFullStream>{});
            go(ks, std::integral_constant<Fit, kFull>{});
        };
        if (KS == 1)
            sized(std::integral_constant<int, 1>{});
        else if (KS == 2)
            sized(std::integral_constant<int, 2>{});
        else if (KS == 4)
            sized(std::integral_constant<int, 4>{});
        else
            sized(std::integral_constant<int, 8>{});
    });
}

template <class Rows> void multiply_few(const Product &p, const Rows &A)
{
    with_out(p, [&](auto out) {
        using T = typename decltype(out)::type;
        auto go = [&](auto mt) {
            const size_t lds = std::is_same_v<Rows, MxRows> ? 0 : p.m * (p.kpad / 2 + 16 + p.kpad / kMxBlock);
            for (int64_t n0 = 0; n0 < p.n; n0 += kFewColumns) {
                const int64_t n = std::min(p.n - n0, kFewColumns);
                auto at = out;  // (a mask has 2^24 columns at most: it is read in the first launch only)
                at.c += n0;
                k_few<Rows, T, decltype(mt)::value><<<(unsigned)ceil_div(n, 16), kFewWaves * kWave, lds, p.s>>>(
                    A, p.B->codes + n0 * (p.kpad / 2), p.B->scales + n0 * (p.kpad / kMxBlock), p.m, n, p.kpad, at);
            }
        };
        if constexpr (std::is_same_v<Rows, MxRows>)
            if (p.m > 32) return go(std::integral_constant<int, 4>{});
        if (p.m > 16) return go(std::integral_constant<int, 2>{});
        go(std::integral_constant<int, 1>{});
    });
}

void multiply(const Product &p, const gs_mxfp4 &A)
{
    if (p.m == 0 || p.n == 0) return;
    const MxRows rows{A.codes, A.scales, p.kpad / 2, p.kpad / kMxBlock};
    const Way w = way(p.m, p.n, p.kpad);
    if (w == Way::kNarrow) return multiply_narrow(p, rows);
    if (w == Way::kFew) return multiply_few(p, rows);
    const TilePlan t = tile_plan(p.m, p.n, p.kpad);
    if (t.tiles_m * t.tiles_n >= 1 << 24) fail(GS_ERR_UNSUPPORTED, "the product has too many tiles");
    auto tiled = [&](auto wt, auto out) {
        using T = typename decltype(out)::type;
        const dim3 grid((unsigned)(t.tiles_m * t.tiles_n), (unsigned)t.split);
        k_tile<T, decltype(wt)::value><<<grid, 256, 0, p.s>>>(A.codes, A.scales, p.B->codes, p.B->scales, p.m, p.n, p.kpad, t.per,
                                                              (int)t.tiles_m, (int)t.tiles_n, out);
    };
    auto sized = [&](auto out) {
        t.wt == 4 ? tiled(std::integral_constant<int, 4>{}, out) : tiled(std::integral_constant<int, 2>{}, out);
    };
    if (t.split == 1)
        return with_out(p, [&](auto out) {
            out.stream = true;  // (4096^3 to bf16: 38.3 us, 40.4 us without; 2048^3 to fp32 10.5 and 11.4)
            sized(out);
        });
    sized(Out<float>{p.part, p.n, nullptr, 0});
    GS_HIP(hipGetLastError());
    with_out(p, [&](auto out) {
        k_join<<<dim3((unsigned)ceil_div(p.n, 1024), (unsigned)p.m), 256, 0, p.s>>>(p.part, t.split, p.m, p.n, out);
    });
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
        *bytes = workspace(m, n, k, a_dtype);
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
        check_work(work, work_bytes, workspace(A->rows, B->rows, A->cols, -1));
        multiply({A->rows, B->rows, (int)mx4_cols(B->cols), B, mask, C, ldc, dtype, (hipStream_t)stream, (float *)work}, *A);
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
        check_work(work, work_bytes, workspace(m, B->rows, B->cols, a_dtype));
        Product p{m, B->rows, (int)mx4_cols(B->cols), B, mask, C, ldc, dtype, (hipStream_t)stream, nullptr};
        if (m == 0 || p.n == 0) return;
        const int k = (int)B->cols;
        if (quantised_inside(m, p.n, p.kpad)) {
            auto rows = [&](const auto &r) { way(m, p.n, p.kpad) == Way::kNarrow ? multiply_narrow(p, r) : multiply_few(p, r); };
            a_dtype == GS_F32 ? rows(DenseRows<float>{(const float *)A, lda, k}) : rows(DenseRows<u16>{(const u16 *)A, lda, k});
            return;
        }
        uint8_t *codes = (uint8_t *)work;
        p.part = (float *)(codes + dense_bytes(m, p.kpad));
        const gs_mxfp4 q{m, B->cols, codes, codes + round256((uint64_t)m * p.kpad / 2)};
        mx4_quantize_rows(A, lda, a_dtype, m, B->cols, q.codes, q.scales, p.s);
        multiply(p, q);
    });
}

}  // extern "C"
