// Products of rows sorted by group (a node's type, a relation, an expert), each group with a
// matrix of its own: rows offsets[g] .. offsets[g + 1] - 1 belong to group g.
//
//   C = A W_g        gs_grouped_matmul
//   C = A W_g^T      the same, transposed: the gradient of A
//   dW_g = A_g^T G_g gs_grouped_weight_grad
//
// The offsets stay on the device: a launch has as many workgroups as there can be tiles, and
// each finds its group and rows itself, from a prefix sum over the groups' tiles that a wave
// makes with its lanes.
//
// Products go by tiles of 64 x 64 or 128 x 128, and where they fit by kernels for few rows (bound by the
// matrices), for large products in bf16 (by the matrix cores) and for layers of many rows (by A and C);
// weight gradients have one of their own.  A tile's operands lie in LDS by rows of 128 bytes
// along the summed index, 64 elements in bf16, 32 in fp32, so that a lane's fragment of a matrix
// instruction is 16 bytes there.  Operands whose summed index is not the one that is
// contiguous in memory are turned on their way through registers.  Activations in the 8 bits
// of a norm or a saved activation are exact in bf16 and become the product's type there too.
// fp32 operands are multiplied in fp32 (V_MFMA_F32_32X32X2_F32), but for layers.
#include <algorithm>
#include <type_traits>

#include "gs_rows.h"

namespace gs {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4v __attribute__((ext_vector_type(4)));

constexpr int kLine = 128;                                  // bytes of a row of a tile in LDS
template <class T> constexpr int kChunk = kLine / sizeof(T);  // elements along the summed index

// ------------------------------------------------------------- where a tile is

struct Offsets {
    const void *p;
    bool wide;
    int groups;
    int64_t rows;
    __device__ __forceinline__ int64_t at(int g) const
    {
        const int64_t o = wide ? ((const int64_t *)p)[g] : ((const int32_t *)p)[g];
        return o < 0 ? 0 : o < rows ? o : rows;  // (whatever they hold, rows are those there are)
    }
};

// Of the segments "rows before the first group" (0), the groups (1 ..) and "rows behind the
// last" (groups + 1), the one in which the id-th of `per` x ceil(rows / step) items lies.
struct Segment {
    int index;        // -1: there are fewer items
    int64_t r0, r1;   // its rows
    int64_t local;    // the item's number in it
    int64_t first;    // number of its first item
};
__device__ __forceinline__ int64_t lane_value(int64_t v, int lane)
{
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, lane), hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
    return (int64_t)((uint64_t)hi << 32 | lo);
}
// The same for every lane, and told to be (divisions are made in vector registers).
__device__ __forceinline__ int64_t uniform(int64_t v)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
// ends: whether the segments without a group count.  EMPTY: a group without rows has `per` items too.
// The item of workgroup `id`, SPREAD: so that each accelerator die has an equal contiguous
// run of the items there are (a launch has more workgroups than that).
template <bool EMPTY>
__device__ __forceinline__ int64_t count_items(const Offsets &o, int64_t step, int64_t per, bool ends)
{
    int64_t all = 0;
    for (int j = lane_id(); j < o.groups + 2; j += kWave) {
        if (j == 0 || j > o.groups) {
            const int64_t n = j == 0 ? o.at(0) : o.rows - o.at(o.groups);
            if (ends) all += (n + step - 1) / step * per;
        } else {
            const int64_t n = o.at(j) - o.at(j - 1), items = n > 0 ? (n + step - 1) / step : 0;
            all += (EMPTY && items == 0 ? 1 : items) * per;
        }
    }
    return (int64_t)wave_sum_u64((unsigned long long)all);
}
template <bool EMPTY, bool SPREAD>
__device__ __forceinline__ Segment find_segment(const Offsets &o, int64_t step, int64_t per, bool ends, int64_t id)
{
    // segments j0 + lane: rows, items
    auto look = [&](int j0, int64_t &r0, int64_t &r1) {
        const int j = j0 + lane_id();
        r0 = r1 = 0;
        if (j <= o.groups + 1) {
            r0 = j == 0 ? 0 : o.at(j - 1);
            r1 = j == o.groups + 1 ? o.rows : o.at(j);
            if (r1 < r0) r1 = r0;
        }
        const bool group = j >= 1 && j <= o.groups;
        int64_t items = (r1 - r0 + step - 1) / step;
        if (EMPTY && items == 0) items = 1;
        return group || (ends && j <= o.groups + 1) ? items * per : 0;
    };
    int64_t r0, r1, items = look(0, r0, r1);
    if constexpr (SPREAD) {
        const int64_t all = count_items<EMPTY>(o, step, per, ends);
        if (id >= all) return {-1, 0, 0, 0, 0};
        id = xcd_tile(id, all);
    }
    int64_t base = 0;
    for (int j0 = 0;;) {
        int64_t inc = items;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int64_t up = __shfl_up(inc, d, kWave);
            if (lane_id() >= d) inc += up;
        }
        inc += base;
        const unsigned long long past = __ballot(inc > id);
        if (past) {
            const int l = __ffsll(past) - 1;
            const int64_t first = lane_value(inc - items, l);
            return {j0 + l, lane_value(r0, l), lane_value(r1, l), id - first, first};
        }
        base = lane_value(inc, kWave - 1);
        if ((j0 += kWave) >= o.groups + 2) return {-1, 0, 0, 0, 0};
        items = look(j0, r0, r1);
    }
}

// ------------------------------------------------------------------ operands
//
// An operand of a tile: ROWS rows of the tile, chunk by chunk along the summed index k.  256
// threads load a chunk into registers (load) and put it into LDS (store), where piece p of
// row r lies at r * 128 + (p ^ r / 2 % 8) * 16: the rows that LDS serves together then spread
// over its banks.

__device__ __forceinline__ uint8_t *piece_at(uint8_t *lds, int row, int piece)
{
    return lds + row * kLine + ((piece ^ (row >> 1 & 7)) << 4);
}

// k contiguous: element (r, k) at p[r * ld + k].
template <class T> struct AlongRows {
    typedef T type;
    const T *p;
    int64_t ld;
    template <int ROWS> struct Held {
        typename Elems<T, kPiece<T>>::type v[ROWS / 32];
    };
    // Rows r0 .. below r1, k from k0 below k1.
    template <int ROWS> __device__ __forceinline__ void load(Held<ROWS> &h, int64_t r0, int64_t r1, int64_t k0, int64_t k1) const
    {
        constexpr int E = kPiece<T>;
        const int64_t k = k0 + threadIdx.x % 8 * E;
#pragma unroll
        for (int i = 0; i < ROWS / 32; i++) {
            const int64_t r = r0 + threadIdx.x / 8 + 32 * i;
            h.v[i] = load_elems<T, E>(p + r * ld + k, r < r1 ? k1 - k : 0);
        }
    }
    template <int ROWS> __device__ __forceinline__ void store(const Held<ROWS> &h, uint8_t *lds) const
    {
#pragma unroll
        for (int i = 0; i < ROWS / 32; i++)
            *reinterpret_cast<u32x4 *>(piece_at(lds, threadIdx.x / 8 + 32 * i, threadIdx.x % 8)) = __builtin_bit_cast(u32x4, h.v[i]);
    }
};

// The number of a signed code, and of codes of activations saved by a ReLU.
struct CodeValue {
    bool relu;
    __device__ __forceinline__ float operator()(uint32_t word, int byte) const
    {
        const int c = (int)(word >> (8 * byte) & 255);
        return (float)(relu ? c : (int)(int8_t)c);
    }
};

// A row of 8-bit activations, as T.
template <class T> struct SavedAlongRows {
    typedef T type;
    const uint8_t *codes, *scales;
    int64_t code_pitch, scale_pitch;
    CodeValue value;
    template <int ROWS> struct Held {
        typename Codes<kPiece<T>>::type c[ROWS / 32];
        uint8_t s[ROWS / 32];
    };
    template <int ROWS> __device__ __forceinline__ void load(Held<ROWS> &h, int64_t r0, int64_t r1, int64_t k0, int64_t k1) const
    {
        constexpr int E = kPiece<T>;
        const int64_t k = k0 + threadIdx.x % 8 * E;
#pragma unroll
        for (int i = 0; i < ROWS / 32; i++) {
            const int64_t r = r0 + threadIdx.x / 8 + 32 * i;
            h.c[i] = {};
            h.s[i] = 0;
            if (r < r1 && k < k1) {  // (codes behind the last column are 0)
                h.c[i] = *reinterpret_cast<const typename Codes<E>::type *>(codes + r * code_pitch + k);
                h.s[i] = scales[r * scale_pitch + k / kMxBlock];
            }
        }
    }
    template <int ROWS> __device__ __forceinline__ void store(const Held<ROWS> &h, uint8_t *lds) const
    {
        constexpr int E = kPiece<T>;
#pragma unroll
        for (int i = 0; i < ROWS / 32; i++) {
            typename Elems<T, E>::type v;
            const float s = mx_scale(h.s[i]);
#pragma unroll
            for (int e = 0; e < E; e++) v[e] = from_f32<T>(value(code_word<E>(h.c[i], e / 4), e % 4) * s);
            *reinterpret_cast<u32x4 *>(piece_at(lds, threadIdx.x / 8 + 32 * i, threadIdx.x % 8)) = __builtin_bit_cast(u32x4, v);
        }
    }
};

// 16 bytes of column c of E rows of `N` columns.
template <class T, int N> __device__ __forceinline__ u32x4 turned(const typename Elems<T, N>::type (&v)[kPiece<T>], int c)
{
    u32x4 o;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] = __float_as_uint(v[e][c]);
    } else if constexpr (N == 1) {
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] = v[2 * e][0] | (uint32_t)v[2 * e + 1][0] << 16;
    } else {  // halves of two words each
        typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
#pragma unroll
        for (int e = 0; e < 4; e++)
            o[e] = __builtin_amdgcn_perm(__builtin_bit_cast(words, v[2 * e + 1])[c / 2], __builtin_bit_cast(words, v[2 * e])[c / 2],
                                         c % 2 ? 0x07060302 : 0x05040100);
    }
    return o;
}

// k is the matrix's row: element (r, k) at p[k * ld + r].  A thread takes E neighbouring k of
// ROWS / 32 neighbouring r.
template <class T> struct AcrossRows {
    typedef T type;
    const T *p;
    int64_t ld;
    template <int ROWS> struct Held {
        typename Elems<T, ROWS / 32>::type v[kPiece<T>];
    };
    template <int ROWS> __device__ __forceinline__ void load(Held<ROWS> &h, int64_t r0, int64_t r1, int64_t k0, int64_t k1) const
    {
        constexpr int E = kPiece<T>, N = ROWS / 32;
        const int64_t k = k0 + threadIdx.x % 8 * E, r = r0 + threadIdx.x / 8 * N;
#pragma unroll
        for (int e = 0; e < E; e++) h.v[e] = load_elems<T, N>(p + (k + e) * ld + r, k + e < k1 ? r1 - r : 0);
    }
    template <int ROWS> __device__ __forceinline__ void store(const Held<ROWS> &h, uint8_t *lds) const
    {
        constexpr int N = ROWS / 32;
#pragma unroll
        for (int i = 0; i < N; i++)
            *reinterpret_cast<u32x4 *>(piece_at(lds, threadIdx.x / 8 * N + i, threadIdx.x % 8)) = turned<T, N>(h.v, i);
    }
};

// --------------------------------------------------------------------- tile

// c + b a^T over 32 bytes of k of 32 rows of either: a lane holds 16 bytes of row lane % 32.
// Its sums are columns 8 g + 4 (lane / 32) .. + 3 (register 4 g ..) of A's row lane % 32.
template <class T> __device__ __forceinline__ f32x16 multiply(u32x4 b, u32x4 a, f32x16 c)
{
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
    } else {
        const f32x4v x = __builtin_bit_cast(f32x4v, b), y = __builtin_bit_cast(f32x4v, a);
#pragma unroll
        for (int i = 0; i < 4; i++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
}

// The sums of a tile of 64 WT x 64 WT, over k from k0 below k1: waves 2 x 2, each WT x WT
// times 32 x 32.  Two chunks in LDS, the next one in registers.
template <class LA, class LB, int WT>
__device__ __forceinline__ void tile_sums(const LA &A, const LB &B, int64_t a0, int64_t a1, int64_t b0, int64_t b1, int64_t k0,
                                          int64_t k1, uint8_t *lds, f32x16 (&acc)[WT][WT])
{
    using T = typename LA::type;
    constexpr int ROWS = 64 * WT, STAGE = 2 * ROWS * kLine;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int ra = wave / 2 * 32 * WT + lane % 32, rb = wave % 2 * 32 * WT + lane % 32, half = lane / 32;
    typename LA::template Held<ROWS> ha;
    typename LB::template Held<ROWS> hb;
    A.template load<ROWS>(ha, a0, a1, k0, k1);
    B.template load<ROWS>(hb, b0, b1, k0, k1);
    A.template store<ROWS>(ha, lds);
    B.template store<ROWS>(hb, lds + STAGE / 2);
    __syncthreads();
    int at = 0;
    for (int64_t k = k0; k < k1; k += kChunk<T>, at ^= 1) {
        const bool more = k + kChunk<T> < k1;
        if (more) {
            A.template load<ROWS>(ha, a0, a1, k + kChunk<T>, k1);
            B.template load<ROWS>(hb, b0, b1, k + kChunk<T>, k1);
        }
        uint8_t *from = lds + at * STAGE;
#pragma unroll
        for (int q = 0; q < 4; q++) {
            u32x4 fa[WT], fb[WT];
#pragma unroll
            for (int i = 0; i < WT; i++) {
                fa[i] = *reinterpret_cast<const u32x4 *>(piece_at(from, ra + 32 * i, 2 * q + half));
                fb[i] = *reinterpret_cast<const u32x4 *>(piece_at(from + STAGE / 2, rb + 32 * i, 2 * q + half));
            }
#pragma unroll
            for (int i = 0; i < WT; i++)
#pragma unroll
                for (int j = 0; j < WT; j++) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j]);
        }
        if (more) {
            A.template store<ROWS>(ha, lds + (at ^ 1) * STAGE);
            B.template store<ROWS>(hb, lds + (at ^ 1) * STAGE + STAGE / 2);
        }
        __syncthreads();
    }
}

// Stores a wave's WT x WT sums at (r0, c0), as far as rows are below r1 and columns below c1,
// through LDS: a lane has four neighbouring columns, a store wants whole lines.
template <class T, int WT>
__device__ __forceinline__ void tile_store(const f32x16 (&acc)[WT][WT], uint8_t *lds, T *out, int64_t ld, int64_t r0, int64_t r1,
                                           int64_t c0, int64_t c1)
{
    constexpr int E = kPiece<T>, PITCH = 32 * WT * sizeof(T) + 16, LANES = 32 * WT / E, ROWS = kWave / LANES;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    uint8_t *mine = lds + wave * 32 * PITCH;
    r0 += wave / 2 * 32 * WT;
    c0 += wave % 2 * 32 * WT;
#pragma unroll
    for (int i = 0; i < WT; i++) {
#pragma unroll
        for (int j = 0; j < WT; j++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                typedef T quad __attribute__((ext_vector_type(4)));
                const quad v = {from_f32<T>(acc[i][j][4 * g]), from_f32<T>(acc[i][j][4 * g + 1]), from_f32<T>(acc[i][j][4 * g + 2]),
                                from_f32<T>(acc[i][j][4 * g + 3])};
                *reinterpret_cast<quad *>(mine + lane % 32 * PITCH + (32 * j + 8 * g + 4 * (lane / 32)) * sizeof(T)) = v;
            }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 32 / ROWS; q++) {
            const int r = ROWS * q + lane / LANES, c = lane % LANES * E;
            const auto v = *reinterpret_cast<const typename Elems<T, E>::type *>(mine + r * PITCH + c * sizeof(T));
            const int64_t row = r0 + 32 * i + r;
            if (row < r1 && c0 + c < c1) store_elems<T, E>(out + row * ld + c0 + c, v, c1 - c0 - c);
        }
        __syncthreads();
    }
}

template <int WT> constexpr int kTileLds = 2 * 2 * 64 * WT * kLine;

// Where a segment's tile starts.  Tiles of a group go in blocks of eight along its rows, all of
// the columns for each, so that operands are met again in a cache.
__device__ __forceinline__ void place_tile(const Segment &s, int side, int tiles_n, int64_t &r0, int64_t &c0)
{
    const int64_t tiles = (s.r1 - s.r0 + side - 1) / side, block = s.local / (8 * tiles_n), rest = s.local - block * 8 * tiles_n;
    const int64_t high = std::min<int64_t>(8, tiles - block * 8);
    r0 = uniform(s.r0 + (block * 8 + rest % high) * side);
    c0 = uniform(rest / high * side);
}

// Zeros in a tile of rows without a group.
template <int SIDE, class T> __device__ void zero_tile(T *C, int64_t ldc, int64_t r0, int64_t r1, int64_t c0, int64_t c1)
{
    constexpr int E = kPiece<T>, LANES = SIDE / E;
    for (int64_t r = r0 + threadIdx.x / LANES; r < std::min(r0 + SIDE, r1); r += 256 / LANES) {
        const int64_t c = c0 + threadIdx.x % LANES * E;
        if (c < c1) store_elems<T, E>(C + r * ldc + c, typename Elems<T, E>::type{}, c1 - c);
    }
}

// C's tiles, of any form.  Bound by latency where it is taken: a tile has few chunks, each a trip
// through registers (one ahead) and LDS.  30,011 rows x 255 to 47 columns, 40 groups, bf16: 10.5 us.
// Large products in fp32, bound by the matrix cores, reach 121 TFLOP/s (8192 x 4096 x 4096).
template <class LA, class LB, class TO, int WT>
__global__ __launch_bounds__(256, WT == 1 ? 4 : 2) void k_grouped(LA A, LB W, int64_t w_step, Offsets off, int64_t k, int64_t n, bool fill,
                                                                  int tiles_n, TO *__restrict__ C, int64_t ldc)
{
    __shared__ __align__(1024) uint8_t lds[kTileLds<WT>];
    constexpr int SIDE = 64 * WT;
    const Segment s = find_segment<false, true>(off, SIDE, tiles_n, fill, blockIdx.x);
    if (s.index < 0) return;
    int64_t r0, c0;
    place_tile(s, SIDE, tiles_n, r0, c0);
    f32x16 acc[WT][WT];
#pragma unroll
    for (int i = 0; i < WT; i++)
#pragma unroll
        for (int j = 0; j < WT; j++) acc[i][j] = f32x16{};
    if (s.index >= 1 && s.index <= off.groups) {
        LB B = W;
        B.p += (s.index - 1) * w_step;
        tile_sums<LA, LB, WT>(A, B, r0, s.r1, c0, n, 0, k, lds, acc);
    }
    tile_store<TO, WT>(acc, lds, C, ldc, r0, s.r1, c0, n);
}

// ------------------------------------------------------------------ few rows
//
// Up to 32 rows of a group a workgroup: bound by reading the groups' matrices.  Four waves share
// 32 N columns and split k, a step of two pieces (16 in bf16, 8 in fp32) each at a time; a lane
// loads the fragments of its N columns straight from memory, turned in registers where k is the
// matrix's row, two steps ahead.  The waves' sums meet in LDS.  16 rows of as many groups, 4096 x 4096
// bf16, take 81 us: 537 MB at 6.7 TB/s.

constexpr int kFewWaves = 4;

// 16 bytes along k of a row of A, from k on, `valid` elements of them.
template <class T> __device__ __forceinline__ u32x4 row_piece(const AlongRows<T> &A, int64_t r, int64_t k, int64_t valid)
{
    return __builtin_bit_cast(u32x4, load_elems<T, kPiece<T>>(A.p + r * A.ld + k, valid));
}
template <class T> __device__ __forceinline__ u32x4 row_piece(const SavedAlongRows<T> &A, int64_t r, int64_t k, int64_t valid)
{
    constexpr int E = kPiece<T>;
    typename Elems<T, E>::type v{};
    if (valid > 0) {  // (codes behind the last column are 0)
        const auto c = *reinterpret_cast<const typename Codes<E>::type *>(A.codes + r * A.code_pitch + k);
        const float s = mx_scale(A.scales[r * A.scale_pitch + k / kMxBlock]);
#pragma unroll
        for (int e = 0; e < E; e++) v[e] = from_f32<T>(A.value(code_word<E>(c, e / 4), e % 4) * s);
    }
    return __builtin_bit_cast(u32x4, v);
}

template <class LA, class T, bool TURN, int N, class TO>
__global__ __launch_bounds__(kFewWaves * kWave, N == 4 ? 2 : 3) void k_grouped_few(LA A, const T *__restrict__ W, int64_t ldw, int64_t w_step, Offsets off,
                                                                    int64_t k, int64_t n, bool fill, int tiles_n, TO *__restrict__ C,
                                                                    int64_t ldc)
{
    constexpr int E = kPiece<T>, STEP = 2 * E, SIDE = 32 * N;
    __shared__ float red[kFewWaves][16][kWave];
    const Segment s = find_segment<false, true>(off, 32, tiles_n, fill, blockIdx.x);
    if (s.index < 0) return;
    const int64_t r0 = uniform(s.r0 + s.local / tiles_n * 32), c0 = uniform(s.local % tiles_n * SIDE);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, half = lane / 32;
    const int64_t rows = std::min<int64_t>(32, s.r1 - r0);
    if (s.index < 1 || s.index > off.groups) {
        for (int i = threadIdx.x; i < 32 * SIDE; i += kFewWaves * kWave)
            if (i / SIDE < rows && c0 + i % SIDE < n) C[(r0 + i / SIDE) * ldc + c0 + i % SIDE] = TO(0);
        return;
    }
    const T *B = W + (s.index - 1) * w_step;
    const int64_t row = r0 + std::min<int64_t>(lane % 32, rows - 1);
    // A lane's columns (n >= N).  TURN: N neighbouring ones, moved back from the end (several
    // lanes then have the same); else N of them 32 apart, the last one for those past it.
    auto column = [&](int l, int i) -> int64_t {
        if constexpr (TURN)
            return std::min(c0 + l * N, n - N) + i;
        else
            return std::min(c0 + l + 32 * i, n - 1);
    };
    struct Step {
        u32x4 a;
        typename Elems<T, N>::type v[TURN ? E : 1];
        u32x4 w[TURN ? 1 : N];
    };
    const T *base[TURN ? 1 : N];
#pragma unroll
    for (int i = 0; i < (TURN ? 1 : N); i++) base[i] = B + (TURN ? column(lane % 32, 0) + half * E * ldw : column(lane % 32, i) * ldw + half * E);
    auto load = [&](Step &t, int64_t at) {  // whole steps
        t.a = row_piece(A, row, at + half * E, E);
        if constexpr (TURN) {
            const T *p = base[0] + at * ldw;
#pragma unroll
            for (int e = 0; e < E; e++) t.v[e] = load_elems<T, N, true>(p + e * ldw, N);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) t.w[i] = __builtin_bit_cast(u32x4, load_elems<T, E, true>(base[i] + at, E));
        }
    };
    auto load_end = [&](Step &t, int64_t at) {  // zeros from k on
        const int64_t ka = at + half * E;
        t.a = row_piece(A, row, ka, k - ka);
        if constexpr (TURN) {
#pragma unroll
            for (int e = 0; e < E; e++) t.v[e] = load_elems<T, N>(base[0] + (at + e) * ldw, ka + e < k ? N : 0);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) t.w[i] = __builtin_bit_cast(u32x4, load_elems<T, E>(base[i] + at, k - ka));
        }
    };
    f32x16 acc[N];
#pragma unroll
    for (int i = 0; i < N; i++) acc[i] = f32x16{};
    auto work = [&](const Step &t) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            if constexpr (TURN)
                acc[i] = multiply<T>(turned<T, N>(t.v, i), t.a, acc[i]);
            else
                acc[i] = multiply<T>(t.w[i], t.a, acc[i]);
        }
    };
    constexpr int64_t NEXT = kFewWaves * STEP;
    const int64_t whole = k - STEP;  // the last place a whole step can start at
    Step t0, t1, t2;
    int64_t at = wave * STEP;
    if (at <= whole) load(t0, at);
    if (at + NEXT <= whole) load(t1, at + NEXT);
    for (; at + 2 * NEXT <= whole; at += 3 * NEXT) {
        load(t2, at + 2 * NEXT);
        work(t0);
        if (at + 3 * NEXT <= whole) load(t0, at + 3 * NEXT);
        work(t1);
        if (at + 4 * NEXT <= whole) load(t1, at + 4 * NEXT);
        work(t2);
    }
    if (at <= whole) {
        work(t0);
        at += NEXT;
        if (at <= whole) {
            work(t1);
            at += NEXT;
        }
    }
    if (at < k) {
        load_end(t0, at);
        work(t0);
    }
    // Sums of the matrix's columns 8 (e / 4) + 4 half + e % 4 (of 32) by A's row lane % 32.
#pragma unroll
    for (int i = 0; i < N; i++) {
        if (i) __syncthreads();
#pragma unroll
        for (int e = 0; e < 16; e++) red[wave][e][lane] = acc[i][e];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 16 / kFewWaves; q++) {
            const int e = wave * (16 / kFewWaves) + q;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kFewWaves; w++) v += red[w][e][lane];
            const int l = 8 * (e / 4) + 4 * half + e % 4;
            const int64_t c = column(l, i);
            if (lane % 32 < rows && c < n) C[(r0 + lane % 32) * ldc + c] = from_f32<TO>(v);
        }
    }
}

// -------------------------------------------------------------- large tiles
//
// bf16 tiles of 256 x 256, a wave 128 x 128 of it: of what LDS serves in a cycle the
// fragments take half then (all of it at 128 x 128).  Rows of whole aligned 16-byte pieces,
// k in whole chunks.  A goes from memory to LDS without passing registers, two chunks ahead; W
// comes through registers, where it is turned if its k is not contiguous, and is loaded a
// chunk before it is stored.  The last quarter of a chunk is multiplied after the workgroup has
// met, while the next one's first fragments are read.  16,384 x 4096 x 4096 in 16 equal groups takes
// 543 us, 1.01 PFLOP/s: with one workgroup a compute unit nothing covers a chunk's end, nor a
// tile's first loads and its stores.

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, -1, 0x00020000);
}

// A: eight rows of a chunk a load, eight loads of a wave: rows 64 wave + 8 q .. + 7.  Offsets of
// this lane's row and piece (in the order in which LDS wants them) from the tile's first row;
// rows past the last one repeat it.
struct TileLoad {
    uint32_t at[8];
    __device__ __forceinline__ void set(int64_t rows, int64_t ld)
    {
        const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
#pragma unroll
        for (int q = 0; q < 8; q++) {
            const int row = 64 * wave + 8 * q + lane / 8, piece = lane % 8 ^ (row >> 1 & 7);
            at[q] = (uint32_t)(std::min<int64_t>(row, rows - 1) * ld * 2) + piece * 16;
        }
    }
    __device__ __forceinline__ void go(const __amdgpu_buffer_rsrc_t &from, uint32_t k_bytes, uint8_t *__restrict__ to) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
        for (int q = 0; q < 8; q++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)(to + (64 * wave + 8 * q) * kLine), 16,
                                                     at[q], k_bytes, 0, 0);
    }
};
// W: eight neighbouring k of eight neighbouring columns in a thread (TURN: W is k x n), or of
// eight columns 32 apart (n x k).
template <bool TURN> struct TileWeights {
    uint32_t at[TURN ? 1 : 8], step;
    u32x4 v[8];
    __device__ __forceinline__ void set(int64_t cols, int64_t ld)
    {
        const int64_t piece = threadIdx.x % 8, c = threadIdx.x / 8;
        if constexpr (TURN) {
            step = (uint32_t)ld * 2;
            at[0] = (uint32_t)(piece * 8 * ld * 2 + std::min<int64_t>(c * 8, cols - 8) * 2);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) at[i] = (uint32_t)(std::min<int64_t>(c + 32 * i, cols - 1) * ld * 2 + piece * 16);
        }
    }
    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t &from, uint32_t k_bytes)
    {
#pragma unroll
        for (int e = 0; e < 8; e++)
            v[e] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, TURN ? at[0] + e * step : at[TURN ? 0 : e], k_bytes, 0));
    }
    __device__ __forceinline__ void store(uint8_t *__restrict__ to) const
    {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            u32x4 o = v[i];
            if constexpr (TURN)
#pragma unroll
                for (int e = 0; e < 4; e++)
                    o[e] = __builtin_amdgcn_perm(v[2 * e + 1][i / 2], v[2 * e][i / 2], i % 2 ? 0x07060302 : 0x05040100);
            *reinterpret_cast<u32x4 *>(piece_at(to, TURN ? threadIdx.x / 8 * 8 + i : threadIdx.x / 8 + 32 * i, threadIdx.x % 8)) = o;
        }
    }
};

struct TileFrags {
    u32x4 a[4], b[4];
    __device__ __forceinline__ void read(const uint8_t *a_from, const uint8_t *b_from, int q, int ra, int rb, int half, int swz)
    {
        const int p = ((2 * q + half) ^ swz) * 16;
        // (in the order in which tile_multiply takes them)
        a[0] = *reinterpret_cast<const u32x4 *>(a_from + p + ra * kLine);
#pragma unroll
        for (int i = 0; i < 4; i++) b[i] = *reinterpret_cast<const u32x4 *>(b_from + p + (rb + 32 * i) * kLine);
#pragma unroll
        for (int i = 1; i < 4; i++) a[i] = *reinterpret_cast<const u32x4 *>(a_from + p + (ra + 32 * i) * kLine);
    }
};
__device__ __forceinline__ void tile_multiply(f32x16 (&acc)[4][4], const TileFrags &f)
{
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc[i][j] = multiply<u16>(f.b[j], f.a[i], acc[i][j]);
}
// Of the instructions up to the next sched_barrier: sixteen multiplications, an LDS read after
// every other one (all four waves' reads would wait for each other behind every one), between
// them V loads from memory and W LDS writes.
template <int V, int W> __device__ __forceinline__ void interleave()
{
#pragma unroll
    for (int i = 0; i < 8; i++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if constexpr (V) __builtin_amdgcn_sched_group_barrier(0x010, V, 0);
        if constexpr (W) __builtin_amdgcn_sched_group_barrier(0x200, W, 0);
    }
}

struct TilePlace {
    int ra, rb, half, swz;
};
// One chunk, which lies in a_from and b_from.  A's chunk after the next goes to a_to, W's next
// one from registers to b_to, and the one after it, at kb, is loaded there.  held: the last
// quarter of the chunk before (FIRST: there is none), on return this one's.
template <bool TURN, bool FIRST>
__device__ __forceinline__ void tile_chunk(uint8_t *__restrict__ a_to, uint8_t *__restrict__ b_to, const uint8_t *__restrict__ a_from,
                                           const uint8_t *__restrict__ b_from, const __amdgpu_buffer_rsrc_t &ga,
                                           const __amdgpu_buffer_rsrc_t &gb, const TileLoad &la, TileWeights<TURN> &lb, uint32_t ka,
                                           uint32_t kb, const TilePlace &at, f32x16 (&acc)[4][4], TileFrags &held)
{
    TileFrags f;
    f.read(a_from, b_from, 0, at.ra, at.rb, at.half, at.swz);
    la.go(ga, ka, a_to);
    if constexpr (!FIRST) {
        tile_multiply(acc, held);
        interleave<1, 0>();
    }
    __builtin_amdgcn_sched_barrier(0);
    held.read(a_from, b_from, 1, at.ra, at.rb, at.half, at.swz);
    tile_multiply(acc, f);
    interleave<0, 0>();
    __builtin_amdgcn_sched_barrier(0);
    f.read(a_from, b_from, 2, at.ra, at.rb, at.half, at.swz);
    lb.store(b_to);
    tile_multiply(acc, held);
    interleave<0, 1>();
    __builtin_amdgcn_sched_barrier(0);
    held.read(a_from, b_from, 3, at.ra, at.rb, at.half, at.swz);
    lb.load(gb, kb);
    tile_multiply(acc, f);
    interleave<1, 0>();
    __builtin_amdgcn_sched_barrier(0);
}
// A's chunk that is multiplied next has arrived (at most 16 loads are younger), this wave's LDS
// operations are done, and so are all others'.  Not __syncthreads: it would wait for the loads to
// LDS that are to be under way.
__device__ __forceinline__ void tile_meet()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x4070);  // vmcnt(16) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// kc: chunks of k.
template <bool TURN, class TO>
__global__ __launch_bounds__(256, 1) void k_grouped_large(const u16 *__restrict__ A, int64_t lda, const u16 *__restrict__ W, int64_t ldw,
                                                        int64_t w_step, Offsets off, int kc, int64_t n, bool fill, int tiles_n,
                                                        TO *__restrict__ C, int64_t ldc)
{
    constexpr int STAGE = 256 * kLine;
    __shared__ __align__(1024) uint8_t lds[5 * STAGE];  // three of A, two of W
    const Segment s = find_segment<false, true>(off, 256, tiles_n, fill, blockIdx.x);
    if (s.index < 0) return;
    int64_t r0, c0;
    place_tile(s, 256, tiles_n, r0, c0);
    if (s.index < 1 || s.index > off.groups) {
        zero_tile<256>(C, ldc, r0, s.r1, c0, n);
        return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const TilePlace at{wave / 2 * 128 + lane % 32, wave % 2 * 128 + lane % 32, lane / 32, lane >> 1 & 7};
    const u16 *B = W + (s.index - 1) * w_step;
    const __amdgpu_buffer_rsrc_t ga = buffer_of(A + r0 * lda), gb = buffer_of(TURN ? B + c0 : B + c0 * ldw);
    const uint32_t sb = TURN ? (uint32_t)ldw * 2 * 64 : kLine;
    auto chunk = [&](int c) { return (uint32_t)std::min(c, kc - 1); };  // (what is loaded past the last one is not used)
    TileLoad la;
    TileWeights<TURN> lb;
    TileFrags held;
    f32x16 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc[i][j] = f32x16{};
    la.set(s.r1 - r0, lda);
    lb.set(n - c0, ldw);
    uint8_t *a0 = lds, *a1 = lds + STAGE, *a2 = lds + 2 * STAGE, *b0 = lds + 3 * STAGE, *b1 = lds + 4 * STAGE;
    la.go(ga, 0, a0);
    lb.load(gb, 0);
    lb.store(b0);
    la.go(ga, chunk(1) * kLine, a1);
    lb.load(gb, chunk(1) * sb);
    tile_meet();
    tile_chunk<TURN, true>(a2, b1, a0, b0, ga, gb, la, lb, chunk(2) * kLine, chunk(2) * sb, at, acc, held);
#pragma unroll 1
    for (int c = 1; c < kc; c++) {
        uint8_t *t = a0;
        a0 = a1, a1 = a2, a2 = t;
        t = b0;
        b0 = b1, b1 = t;
        tile_meet();
        tile_chunk<TURN, false>(a2, b1, a0, b0, ga, gb, la, lb, chunk(c + 2) * kLine, chunk(c + 2) * sb, at, acc, held);
    }
    tile_multiply(acc, held);
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0): nothing is on its way to LDS any more
    __syncthreads();
    tile_store<TO, 4>(acc, lds, C, ldc, r0, s.r1, c0, n);
}

// ------------------------------------------------------------------ layers
//
// Many rows, up to 256 of k, bf16 on the matrix cores: bound by reading A and writing C (2,097,152 x 128
// x 128 bf16 218 us, 4.9 TB/s; 2,000,000 rows of 8 bits against fp32 matrices 295, 4.4).  A workgroup of eight
// waves keeps 32 NT columns of a group's matrix in LDS, as the fragments that the instructions
// take, and goes through a contiguous run of the rows; each wave takes 32 RB of them at a time
// straight from memory into fragments (a lane 16 neighbouring k of its row), the next ones
// loaded meanwhile.  A new matrix is put into LDS only where the run meets a new group.
//
// fp32 matrices (beside activations in 8 bits, whose values bf16 holds exactly) are cut into three
// bf16 parts, whose sum they are from 2^-110 on: three exact products for one in fp32 at 16 times
// its rate.

constexpr int kPanelWaves = 8;
constexpr int kPanelStage = 32 * (kLine + 16);  // bytes of a wave's way out through LDS

// k of element i of step ks (16 of k) in half h of a wave.
__device__ __forceinline__ int panel_k(int ks, int half) { return 32 * (ks / 2) + 16 * half + 8 * (ks % 2); }

// Rows of A on their way: 32 of k (step j) of a row, 16 of them in this lane.
struct SavedRows {
    const uint8_t *codes, *scales;
    int64_t code_pitch, scale_pitch;
    float zero;  // the code of 0: signed codes are taken 128 higher
    int k;
    struct Row {
        const uint8_t *codes, *scales;
    };
    struct Held {
        u32x4 c;
        int s;
    };
    __device__ __forceinline__ Row row(int64_t r, int half) const
    {
        return {codes + r * code_pitch + 16 * half, scales + r * scale_pitch};
    }
    __device__ __forceinline__ void load(Held &h, const Row &r, int j, int) const
    {
        h.c = u32x4{};
        h.s = 0;
        if (32 * j < k) {  // (the same for all lanes; codes behind the last column are 0)
            h.c = *reinterpret_cast<const u32x4 *>(r.codes + 32 * j);
            h.s = r.scales[j];
        }
    }
    __device__ __forceinline__ void fragments(const Held &h, int, int, u32x4 (&f)[2]) const
    {
        const float s = mx_scale(h.s);
        const uint32_t flip = zero != 0.0f ? 0x80808080u : 0u;
#pragma unroll
        for (int w = 0; w < 4; w++) {
            const uint32_t c = h.c[w] ^ flip;
            uint32_t v[4];
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = __float_as_uint(((float)(c >> (8 * e) & 255) - zero) * s);  // (exact)
#pragma unroll
            for (int e = 0; e < 2; e++) f[w / 2][w % 2 * 2 + e] = __builtin_amdgcn_perm(v[2 * e + 1], v[2 * e], 0x07060302);
        }
    }
};
struct Bf16Rows {
    const u16 *p;
    int64_t ld;
    int k;  // at least 8
    typedef const u16 *Row;
    struct Held {
        u32x4 v[2];
    };
    __device__ __forceinline__ Row row(int64_t r, int) const { return p + r * ld; }
    // (the row's last 16 bytes for those that go past it)
    __device__ __forceinline__ int at(int j, int half, int i) const { return std::min(32 * j + 16 * half + 8 * i, k - 8); }
    __device__ __forceinline__ void load(Held &h, const Row &r, int j, int half) const
    {
#pragma unroll
        for (int i = 0; i < 2; i++) h.v[i] = __builtin_bit_cast(u32x4, load_elems<u16, 8>(r + at(j, half, i), 8));
    }
    __device__ __forceinline__ void fragments(const Held &h, int j, int half, u32x4 (&f)[2]) const
    {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            f[i] = h.v[i];
            if (32 * j + 32 > k) {
                RowPiece<u16> q;
                q.v = __builtin_bit_cast(typename RowPiece<u16>::V, h.v[i]);
                q.shift = 32 * j + 16 * half + 8 * i - at(j, half, i);
                f[i] = __builtin_bit_cast(u32x4, q.get(0, k));
            }
        }
    }
};

// Columns c0 .. of a matrix of T (transpose: of its rows) as fragments: 1 KB for each of P
// parts of each 32 columns of each step of 16 k.
template <class T, int J, int NT, int P>
__device__ __forceinline__ void fill_panel(uint8_t *lds, const T *W, int64_t ld, bool transpose, int k, int64_t c0, int64_t n)
{
    for (int e = threadIdx.x; e < 2 * J * NT * kWave; e += kPanelWaves * kWave) {
        const int lane = e % kWave, t = e / kWave % NT, ks = e / kWave / NT;
        const int64_t c = c0 + 32 * t + lane % 32;
        const int k0 = panel_k(ks, lane / 32);
        uint32_t part[P][8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            T v = T(0);
            if (c < n && k0 + i < k) v = transpose ? W[c * ld + k0 + i] : W[(k0 + i) * ld + c];
            float rest = to_f32(v);
            const bool whole = fabsf(rest) == __builtin_inff();  // (infinity is all in the first part)
#pragma unroll
            for (int q = 0; q < P; q++) {
                part[q][i] = __float_as_uint(rest);
                rest -= __uint_as_float(part[q][i] & 0xffff0000u);
                if (whole) rest = 0.0f;
            }
        }
#pragma unroll
        for (int q = 0; q < P; q++) {
            u32x4 f;
#pragma unroll
            for (int i = 0; i < 4; i++) f[i] = __builtin_amdgcn_perm(part[q][2 * i + 1], part[q][2 * i], 0x07060302);
            *reinterpret_cast<u32x4 *>(lds + ((ks * NT + t) * P + q) * 1024 + lane * 16) = f;
        }
    }
}

template <class Rows, class TW, class TO, int J, int NT, int RB, int P>
__global__ __launch_bounds__(kPanelWaves * kWave, 2) void k_grouped_panel(Rows A, const TW *__restrict__ W, int64_t ldw, int64_t w_step,
                                                                        bool transpose, Offsets off, int k, int64_t n, bool fill,
                                                                        TO *__restrict__ C, int64_t ldc)
{
    constexpr int ROWS = kPanelWaves * 32 * RB, E = kPiece<TO>;
    __shared__ __align__(1024) uint8_t lds[2 * J * NT * P * 1024 + kPanelWaves * kPanelStage];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, half = lane / 32;
    uint8_t *mine = lds + 2 * J * NT * P * 1024 + wave * kPanelStage;
    const int64_t c0 = (int64_t)blockIdx.y * 32 * NT;
    const int64_t all = uniform(count_items<false>(off, ROWS, 1, fill));
    int64_t item = uniform(all * blockIdx.x / gridDim.x);
    const int64_t last = uniform(all * (blockIdx.x + 1) / gridDim.x);
    if (item >= last) return;
    // this wave's rows of an item
    struct Strip {
        int64_t r0, r1;
        int segment;
    };
    Segment seg = find_segment<false, false>(off, ROWS, 1, fill, item);
    int64_t base = seg.r0 + seg.local * ROWS;
    auto strip = [&] { return Strip{base + wave * 32 * RB, seg.r1, seg.index}; };
    typename Rows::Held held[RB][J];
    typename Rows::Row row[RB];
    auto set_rows = [&](const Strip &s) {  // (rows past the last one repeat it; a strip without rows takes any)
#pragma unroll
        for (int i = 0; i < RB; i++)
            row[i] = A.row(std::max<int64_t>(0, std::min(s.r0 + 32 * i + lane % 32, s.r1 - 1)), half);
    };
    auto load = [&](int j) {
#pragma unroll
        for (int i = 0; i < RB; i++) A.load(held[i][j], row[i], j, half);
    };
    Strip now = strip();
    set_rows(now);
#pragma unroll
    for (int j = 0; j < J; j++) load(j);
    int panel = -1;
    for (; item < last; item++) {
        const bool group = now.segment >= 1 && now.segment <= off.groups;
        if (group && now.segment != panel) {
            panel = now.segment;
            __syncthreads();
            fill_panel<TW, J, NT, P>(lds, W + (panel - 1) * w_step, ldw, transpose, k, c0, n);
            __syncthreads();
        }
        Strip next = now;
        if (item + 1 < last) {
            base += ROWS;
            if (base >= seg.r1) {
                seg = find_segment<false, false>(off, ROWS, 1, fill, item + 1);
                base = seg.r0 + seg.local * ROWS;
            }
            next = strip();
        }
        set_rows(next);
        f32x16 acc[RB][NT];
#pragma unroll
        for (int i = 0; i < RB; i++)
#pragma unroll
            for (int t = 0; t < NT; t++) acc[i][t] = f32x16{};
        if (group && now.r0 < now.r1) {
#pragma unroll
            for (int j = 0; j < J; j++) {
                u32x4 a[RB][2];
#pragma unroll
                for (int i = 0; i < RB; i++) A.fragments(held[i][j], j, half, a[i]);
                load(j);
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int t = 0; t < NT; t++)
#pragma unroll
                        for (int q = P - 1; q >= 0; q--) {
                            const u32x4 b = *reinterpret_cast<const u32x4 *>(lds + (((2 * j + h) * NT + t) * P + q) * 1024 + lane * 16);
#pragma unroll
                            for (int i = 0; i < RB; i++) acc[i][t] = multiply<u16>(b, a[i][h], acc[i][t]);
                        }
            }
        } else {
#pragma unroll
            for (int j = 0; j < J; j++) load(j);
        }
        if (now.r0 < now.r1) {
            // out through LDS, 128 bytes of a row at a time
            constexpr int TILES = sizeof(TO) == 4 ? 1 : 2, PITCH = kLine + 16;
#pragma unroll
            for (int i = 0; i < RB; i++)
#pragma unroll
                for (int t = 0; t < NT; t += TILES) {
#pragma unroll
                    for (int u = 0; u < TILES; u++)
#pragma unroll
                        for (int g = 0; g < 4; g++) {
                            typedef TO quad __attribute__((ext_vector_type(4)));
                            const f32x16 &v = acc[i][t + u];
                            *reinterpret_cast<quad *>(mine + lane % 32 * PITCH + (32 * u + 8 * g + 4 * half) * sizeof(TO)) =
                                quad{from_f32<TO>(v[4 * g]), from_f32<TO>(v[4 * g + 1]), from_f32<TO>(v[4 * g + 2]), from_f32<TO>(v[4 * g + 3])};
                        }
                    __builtin_amdgcn_wave_barrier();  // (a wave's LDS operations keep their order)
                    typename Elems<TO, E>::type out[4];
#pragma unroll
                    for (int q = 0; q < 4; q++)
                        out[q] = *reinterpret_cast<const typename Elems<TO, E>::type *>(mine + (8 * q + lane / 8) * PITCH + lane % 8 * 16);
                    __builtin_amdgcn_wave_barrier();
                    const int64_t c = c0 + 32 * t + lane % 8 * E;
#pragma unroll
                    for (int q = 0; q < 4; q++) {
                        const int64_t r = now.r0 + 32 * i + 8 * q + lane / 8;
                        if (r < now.r1 && c < n) store_elems<TO, E, true, false>(C + r * ldc + c, out[q], n - c);
                    }
                }
        }
        now = next;
    }
}

// ---------------------------------------------------------- weight gradients
//
// The summed index is the rows, along which neither operand is contiguous.  A workgroup of eight
// waves makes a tile of 128 WA x 64 WB (all of a layer's gradient, so that each operand is read
// once) from a run of a group's rows; a wave loads whole rows of a chunk, eight (fp32: four) of
// them, N columns a lane, which are 16 bytes along k for each column when they are put into LDS.
// Bound by the loads' way: two chunks are under way in registers (a third spills) while one is multiplied.
// Runs end in partial products, which a second launch adds in order.  204,800 rows of 256 codes and
// 128 bf16, 9 groups: 41 us and 9 for the 34 MB of partials; bytes alone would take 16.  16,384 rows of
// 4096 by 4096, 16 groups, bf16: 1,182 us, 465 TFLOP/s.

constexpr int kGradThreads = 512;
constexpr int64_t kGradChain = 8192;  // rows that are summed one after another

// Place of piece p of row r: writes of lanes whose rows are 1, 2 or 4 apart and reads of
// neighbouring rows both spread over LDS's banks.
__device__ __forceinline__ uint8_t *grad_piece(uint8_t *lds, int row, int piece)
{
    return lds + row * kLine + ((piece ^ ((row >> 1 ^ row >> 4) & 7)) << 4);
}

// Columns c0 .. c0 + 64 N - 1 of rows, N of a lane: those from column() on.  A row's address is the
// same for all lanes, but for a lane's own 32 bits.  NARROW: there are fewer than N columns.
template <class T, int N, bool NARROW = false> struct GradDense {
    typedef T type;
    const T *p;
    int64_t ld;
    int64_t width;
    struct Held {
        typename Elems<T, N>::type v[kPiece<T>];
    };
    struct Row {
        const T *p;
    };
    // (the last columns for lanes that would go past them: several lanes then hold the same)
    __device__ __forceinline__ int64_t column(int64_t c0) const
    {
        return std::max<int64_t>(0, std::min(c0 + threadIdx.x % kWave * N, width - N));
    }
    __device__ __forceinline__ Row row(int64_t r, int64_t c) const { return {p + r * ld + c}; }
    __device__ __forceinline__ void move(Row &r, bool on) const { r.p += on ? ld : 0; }
    __device__ __forceinline__ void load(Held &h, int e, const Row &r, uint32_t at, int64_t) const
    {
        h.v[e] = load_elems<T, N>(r.p + at, NARROW ? width - at : N);
    }
    __device__ __forceinline__ void none(Held &h, int e) const { h.v[e] = typename Elems<T, N>::type{}; }
    template <class F> __device__ __forceinline__ void columns(const Held &h, F put) const
    {
#pragma unroll
        for (int i = 0; i < N; i++) put(i, turned<T, N>(h.v, i));
    }
};
template <class T, int N> struct GradSaved {
    typedef T type;
    const uint8_t *codes, *scales;
    int64_t code_pitch, scale_pitch;
    uint32_t sign;  // 128 where codes have a sign, else 0
    typedef std::conditional_t<N == 1, uint8_t, std::conditional_t<N == 2, u16, uint32_t>> Word;
    struct Held {
        Word c[kPiece<T>];
        uint8_t s[kPiece<T>];
    };
    struct Row {
        const uint8_t *codes, *scales;
    };
    __device__ __forceinline__ int64_t column(int64_t c0) const
    {
        return std::min<int64_t>(c0 + threadIdx.x % kWave * N, code_pitch - N);
    }
    __device__ __forceinline__ Row row(int64_t r, int64_t c) const { return {codes + r * code_pitch + c, scales + r * scale_pitch}; }
    __device__ __forceinline__ void move(Row &r, bool on) const
    {
        r.codes += on ? code_pitch : 0;
        r.scales += on ? scale_pitch : 0;
    }
    __device__ __forceinline__ void load(Held &h, int e, const Row &r, uint32_t at, int64_t column) const
    {
        h.c[e] = *reinterpret_cast<const Word *>(r.codes + at);
        h.s[e] = r.scales[(uint32_t)(column / kMxBlock)];
    }
    __device__ __forceinline__ void none(Held &h, int e) const
    {
        h.c[e] = 0;
        h.s[e] = 0;
    }
    // (128 is added to a signed code by turning its highest bit, and taken from the number again)
    template <class F> __device__ __forceinline__ void columns(const Held &h, F put) const
    {
        float scale[kPiece<T>];
        const float less = (float)sign;
#pragma unroll
        for (int e = 0; e < kPiece<T>; e++) scale[e] = mx_scale(h.s[e]);
#pragma unroll
        for (int i = 0; i < N; i++) {
            typename Elems<T, kPiece<T>>::type v;
#pragma unroll
            for (int e = 0; e < kPiece<T>; e++) {
                const uint32_t word = h.c[e] ^ sign * 0x01010101u;
                v[e] = from_f32<T>(((float)(word >> (8 * i) & 255) - less) * scale[e]);
            }
            put(i, __builtin_bit_cast(u32x4, v));
        }
    }
};

// Chunks of `per` rows of a group, a tile of it each; out is the chunk's a x b (one chunk a
// group: the group's).  A's lanes hold 2 WA columns, G's WB.  LONG: `per` is more than a chain, chains are
// added in memory (code of its own: in the others it would take 3 to 28 registers).
template <class LA, class LG, int WA, int WB, bool LONG>
__global__ __launch_bounds__(kGradThreads, 2) void k_grouped_grad(LA A, LG G, Offsets off, int64_t a, int64_t b, int64_t per, int tiles_b,
                                                                 float *__restrict__ out)
{
    using T = typename LA::type;
    constexpr int SA = 128 * WA, SB = 64 * WB, STAGE = (SA + SB) * kLine, E = kPiece<T>;
    __shared__ __align__(1024) uint8_t lds[2 * STAGE];
    const Segment s = find_segment<true, false>(off, per, 1, false, blockIdx.x);
    if (s.index < 0) return;
    const int64_t k0 = uniform(s.r0 + s.local * per), k1 = uniform(std::min(s.r0 + (s.local + 1) * per, s.r1));
    const int64_t a0 = (int64_t)(blockIdx.y / tiles_b) * SA, b0 = (int64_t)(blockIdx.y % tiles_b) * SB;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, half = lane / 32;
    const int64_t ca = A.column(a0), cb = G.column(b0);
    // (a lane moved back from the end of the rows may hold columns before the tile's first)
    const int la = (int)(ca - a0), lb = (int)(cb - b0);
    const int64_t fa = std::max<int64_t>(0, a0 - 4), fb = std::max<int64_t>(0, b0 - 4), last = off.rows - 1;
    const uint32_t at_a = (uint32_t)(ca - fa), at_b = (uint32_t)(cb - fb);
    struct Held {
        typename LA::Held a;
        typename LG::Held b;
    } h0, h1;
    // (loads that are always made, from the last row where there are no more, so that the wait for one
    // chunk's need not be one for the next's)
    auto load = [&](Held &h, int64_t k) {
        k = std::min(k + wave * E, last);
        const int more = (int)std::min<int64_t>(last - k, E);
        auto ra = A.row(k, fa);
        auto rb = G.row(k, fb);
#pragma unroll
        for (int e = 0; e < E; e++) {
            A.load(h.a, e, ra, at_a, ca);
            G.load(h.b, e, rb, at_b, cb);
            A.move(ra, e < more);
            G.move(rb, e < more);
        }
    };
    // Rows `from` on, of the next chain, of other groups or none, as zeros.
    auto end = [&](Held &h, int64_t k, int64_t from) {
        k += wave * E;
        if (k + E > from)
#pragma unroll
            for (int e = 0; e < E; e++)
                if (k + e >= from) {
                    A.none(h.a, e);
                    G.none(h.b, e);
                }
    };
    auto store = [&](const Held &h, uint8_t *to) {
        A.columns(h.a, [&](int i, u32x4 v) {
            if (la + i >= 0) *reinterpret_cast<u32x4 *>(grad_piece(to, la + i, wave)) = v;
        });
        G.columns(h.b, [&](int i, u32x4 v) {
            if (lb + i >= 0) *reinterpret_cast<u32x4 *>(grad_piece(to + SA * kLine, lb + i, wave)) = v;
        });
    };
    f32x16 acc[WA][WB];
#pragma unroll
    for (int i = 0; i < WA; i++)
#pragma unroll
        for (int j = 0; j < WB; j++) acc[i][j] = f32x16{};
    const int ra = wave / 2 * 32 * WA + lane % 32, rb = wave % 2 * 32 * WB + lane % 32;
    // (waves past the gradient's last row or column multiply nothing)
    const bool mine = a0 + wave / 2 * 32 * WA < a && b0 + wave % 2 * 32 * WB < b;
    auto work = [&](uint8_t *from) {
        if (mine)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                u32x4 fa[WA], fb[WB];
#pragma unroll
                for (int i = 0; i < WA; i++) fa[i] = *reinterpret_cast<const u32x4 *>(grad_piece(from, ra + 32 * i, 2 * q + half));
#pragma unroll
                for (int j = 0; j < WB; j++) fb[j] = *reinterpret_cast<const u32x4 *>(grad_piece(from + SA * kLine, rb + 32 * j, 2 * q + half));
#pragma unroll
                for (int i = 0; i < WA; i++)
#pragma unroll
                    for (int j = 0; j < WB; j++) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j]);
            }
    };
    constexpr int64_t STEP = kChunk<T>;
    float *to = out + (int64_t)blockIdx.x * a * b;
    for (int64_t c0 = k0;; c0 += kGradChain) {
        const int64_t c1 = LONG ? std::min(c0 + kGradChain, k1) : k1;
        if (c0 < c1) {
            load(h0, c0);
            load(h1, c0 + STEP);
            end(h0, c0, c1);
            store(h0, lds);
            __syncthreads();
            for (int64_t k = c0; k < c1; k += 2 * STEP) {
                load(h0, k + 2 * STEP);
                work(lds);
                end(h1, k + STEP, c1);
                store(h1, lds + STAGE);
                __syncthreads();
                load(h1, k + 3 * STEP);
                if (k + STEP < c1) work(lds + STAGE);
                end(h0, k + 2 * STEP, c1);
                store(h0, lds);
                __syncthreads();
            }
        }
#pragma unroll
        for (int i = 0; i < WA; i++)
#pragma unroll
            for (int j = 0; j < WB; j++)
#pragma unroll
                for (int g = 0; g < 4; g++) {
                    const int64_t r = a0 + ra + 32 * i, c = b0 + wave % 2 * 32 * WB + 32 * j + 8 * g + 4 * half;
                    if (r < a && c < b) {
                        const f32x16 &v = acc[i][j];
                        typename Elems<float, 4>::type sum = {v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
                        if (LONG && c0 > k0) sum += load_elems<float, 4>(to + r * b + c, b - c);  // (this lane's own)
                        store_elems<float, 4>(to + r * b + c, sum, b - c);
                    }
                }
        if (!LONG || c1 >= k1) break;
#pragma unroll
        for (int i = 0; i < WA; i++)
#pragma unroll
            for (int j = 0; j < WB; j++) acc[i][j] = f32x16{};
    }
}
// The chunks of a group added in order, every eight of them in 64 bits: 256 threads, four elements each; blockIdx.y the group.
__global__ __launch_bounds__(256) void k_grouped_join(const float *__restrict__ part, Offsets off, int64_t ab, int64_t per,
                                                      int64_t all, float *__restrict__ out)
{
    // number of the group's first chunk: chunks of the groups before it
    int64_t first = 0, mine = 1;
    for (int j0 = 0; j0 <= (int)blockIdx.y; j0 += kWave) {
        const int j = j0 + lane_id();
        int64_t chunks = 0;
        if (j <= (int)blockIdx.y) {
            const int64_t r0 = off.at(j), r1 = off.at(j + 1);
            chunks = r1 > r0 ? (r1 - r0 + per - 1) / per : 1;
        }
        if ((int)blockIdx.y < j0 + kWave) mine = lane_value(chunks, blockIdx.y - j0);
        first += (int64_t)wave_sum_u64((unsigned long long)chunks);
    }
    first -= mine;
    const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (e >= ab) return;
    double s[4] = {};  // (a hundred thousand partials are possible)
    const int64_t end = std::min(first + mine, all);  // (offsets that descend: no more than there are)
    constexpr int U = 8;  // partials in flight
    for (int64_t c = first; c < end; c += U) {
        typename Elems<float, 4>::type v[U];
#pragma unroll
        for (int u = 0; u < U; u++) v[u] = load_elems<float, 4>(part + std::min(c + u, end - 1) * ab + e, ab - e);
        float some[4] = {};
#pragma unroll
        for (int u = 0; u < U; u++)
            if (c + u < end)
#pragma unroll
                for (int i = 0; i < 4; i++) some[i] += v[u][i];
#pragma unroll
        for (int i = 0; i < 4; i++) s[i] += some[i];
    }
    store_elems<float, 4>(out + blockIdx.y * ab + e, typename Elems<float, 4>::type{(float)s[0], (float)s[1], (float)s[2], (float)s[3]}, ab - e);
}

// ------------------------------------------------------------------- launch

Offsets check_offsets(const void *offsets, int bytes, int64_t groups, int64_t rows)
{
    if (bytes != 4 && bytes != 8) fail(GS_ERR_INVALID_ARG, "offsets have 4 or 8 bytes");
    if (groups < 1) fail(GS_ERR_INVALID_ARG, "there must be at least one group");
    if (groups > 65535) fail(GS_ERR_UNSUPPORTED, "at most 65535 groups");
    if (rows < 0 || rows > INT32_MAX) fail(GS_ERR_INVALID_ARG, "bad matrix size");
    if (!offsets) fail(GS_ERR_INVALID_ARG, "offsets are null");
    if ((uintptr_t)offsets % bytes) fail(GS_ERR_INVALID_ARG, "offsets are not aligned");
    return {offsets, bytes == 8, (int)groups, rows};
}

struct Operand {  // dense, or saved
    const void *p;
    int64_t ld;
    const gs_saved *saved;
};

// Rows of a run, and how many runs there can be: a workgroup for each compute unit, a run a chain
// at most, unless so many partial products would take too much.
struct GroupedGradPlan {
    int64_t per, chunks, tiles_a, tiles_b;
    bool direct;
    int wa, wb;
};
GroupedGradPlan grouped_grad_plan(int64_t rows, int64_t groups, int64_t a, int64_t b)
{
    GroupedGradPlan p;
    p.wa = a <= 128 ? 1 : 2;
    p.wb = b <= 64 ? 1 : 2;
    p.tiles_a = ceil_div(a, 128 * p.wa);
    p.tiles_b = ceil_div(b, 64 * p.wb);
    const int64_t tiles = p.tiles_a * p.tiles_b, want = std::max<int64_t>(1, 256 / tiles);
    p.per = std::min<int64_t>(kGradChain, std::max<int64_t>(256, ceil_div(ceil_div(rows, want), 64) * 64));
    // (what partial sums would take: at most 1 GB of them)
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 28) / (a * b));
    if (ceil_div(rows, p.per) + groups > most) p.per = ceil_div(ceil_div(rows, std::max<int64_t>(1, most - groups)), 64) * 64;
    p.direct = rows <= p.per || most <= groups;
    if (p.direct) p.per = std::max<int64_t>(1, rows);
    p.chunks = p.direct ? groups : ceil_div(rows, p.per) + groups;
    return p;
}

void check_product(int64_t k, int64_t n)
{
    if (k < 1 || n < 1) fail(GS_ERR_INVALID_ARG, "bad matrix size");
    if (k > kMxMaxCols || n > kMxMaxCols) fail(GS_ERR_UNSUPPORTED, "at most 2^24 columns");
}

}  // namespace
}  // namespace gs

using namespace gs;

static int grouped_matmul(const Operand &A, int a_dtype, int64_t rows, const void *W, int w_dtype, int64_t ldw, int64_t w_step,
                          int64_t groups, int64_t k, int64_t n, int transpose, const void *offsets, int offset_bytes, int fill,
                          void *C, int64_t ldc, int c_dtype, gs_stream stream)
{
    return guarded([&] {
        check_product(k, n);
        const Offsets off = check_offsets(offsets, offset_bytes, groups, rows);
        const int wsize = dtype_size(w_dtype), csize = dtype_size(c_dtype);
        const int64_t in = transpose ? n : k, outw = transpose ? k : n;
        if (A.saved) {
            check_saved(A.saved, false);
            if (A.saved->rows != rows || A.saved->cols != in) fail(GS_ERR_INVALID_ARG, "A has another shape");
        } else {
            check_operand("A", A.p, rows, in, A.ld, dtype_size(a_dtype));
            if (a_dtype != w_dtype) fail(GS_ERR_INVALID_ARG, "A and W have different types");
        }
        check_operand("W", W, k, n, ldw, wsize);
        if (w_step < 0) fail(GS_ERR_INVALID_ARG, "negative step from group to group");
        if (groups > 1 && w_step > (((int64_t)1 << 62) / wsize - k * ldw) / (groups - 1))
            fail(GS_ERR_INVALID_ARG, "W: span is not addressable");
        check_operand("C", C, rows, outw, ldc, csize);
        if (rows == 0) return;
        const Extent c{C, rows, outw * csize, ldc * csize};
        if (!A.saved) check_apart("C", c, "A", {A.p, rows, in * dtype_size(a_dtype), A.ld * dtype_size(a_dtype)});
        const int64_t matrix = ((k - 1) * ldw + n) * wsize;
        // (matrices nearer to each other than their size, or one for all groups: what they take together)
        const int64_t step = w_step * wsize;
        check_apart("C", c, "W", step < matrix ? Extent{W, 1, (groups - 1) * step + matrix, (groups - 1) * step + matrix}
                                               : Extent{W, groups, matrix, step});
        const hipStream_t s = (hipStream_t)stream;
        // Which kernel: all figures are us, groups of equal sizes, one set of operands after the other.
        //
        // Large tiles: rows of whole aligned pieces, k of whole chunks, offsets in a matrix of 32 bits; enough
        // of them to keep half of the chip (rows x 1024 x 1024: 64 tiles 37 and 32 in tiles of 128, 128 tiles
        // 38 and 41, 256 tiles 43 and 76) that are half full of rows (8192 x 2048 x 4096: 128 rows a group 323
        // and 315, 256 171 and 288) and of columns (262,144 x 128 x 128: 57 and 37).
        const bool pieces = !A.saved && w_dtype == GS_BF16 && in % 64 == 0 && in >= 128 && A.ld % 8 == 0 && (uintptr_t)A.p % 16 == 0 &&
                            ldw % 8 == 0 && w_step % 8 == 0 && (uintptr_t)W % 16 == 0 && (transpose || (n % 8 == 0 && n >= 8)) &&
                            256 * A.ld < (1 << 30) && (transpose ? 256 : k) * ldw < (1 << 30);
        const int64_t large_n = ceil_div(outw, 256), large = (ceil_div(rows, 256) + groups + 2) * large_n;
        // Layers: bf16 operands or 8-bit rows, k from 16 to 256 (262,144 x 8 x 64: 29 and 29 in tiles, x 16 x 64:
        // 12 and 29), many rows, 256 and more of a group.  Against fp32 matrices from 32,768 rows on (x 128 x
        // 128: 21 and 20, 16,384 rows 21 and 14, 65,536 rows 22 and 30), bf16 from 196,608 (131,072 rows 25 and
        // 21, 262,144 rows 33 and 37, 2,097,152 rows 218 and 319); 262,144 x 128 x 128 of fp32 with 256 rows
        // a group 107 and 183, with 128 302 and 292.  Large tiles are better where both k and n are
        // (131,072 x 256 x 256: 52 and 41).
        const bool layers = in >= 16 && in <= 256 && rows >= 256 * groups && (A.saved || w_dtype == GS_BF16) &&
                            rows >= (w_dtype == GS_F32 ? 32768 : 196608) && !(pieces && in > 128 && outw > 128);
        if (pieces && !layers && outw > 128 && rows >= 128 * groups && ceil_div(rows, 256) * large_n >= 128 && large <= INT32_MAX / 256) {
            auto run = [&](auto kernel, auto type) {
                kernel<<<(unsigned)large, 256, 0, s>>>((const u16 *)A.p, A.ld, (const u16 *)W, ldw, w_step, off, (int)(in / 64), outw,
                                                       fill != 0, (int)large_n, (decltype(type) *)C, ldc);
            };
            if (transpose)
                c_dtype == GS_F32 ? run(k_grouped_large<false, float>, 0.0f) : run(k_grouped_large<false, u16>, u16(0));
            else
                c_dtype == GS_F32 ? run(k_grouped_large<true, float>, 0.0f) : run(k_grouped_large<true, u16>, u16(0));
            GS_HIP(hipGetLastError());
            return;
        }
        if (layers) {
            const int j = (int)ceil_div(in, 32);
            auto run = [&](auto rows_of, auto w, auto out, auto jc, auto nt, auto rb, auto parts) {
                using TW = decltype(w);
                using TO = decltype(out);
                constexpr int J = decltype(jc)::value, NT = decltype(nt)::value, RB = decltype(rb)::value, P = decltype(parts)::value;
                const int64_t panels = ceil_div(outw, 32 * NT);
                const int64_t x = std::min<int64_t>(ceil_div(rows, kPanelWaves * 32 * RB) + groups + 2, std::max<int64_t>(32, 256 / panels));
                k_grouped_panel<decltype(rows_of), TW, TO, J, NT, RB, P><<<dim3((unsigned)x, (unsigned)panels), kPanelWaves * kWave, 0, s>>>(
                    rows_of, (const TW *)W, ldw, w_step, transpose != 0, off, (int)in, outw, fill != 0, (TO *)C, ldc);
            };
            auto with_j = [&](auto rows_of, auto w, auto out, auto parts) {
                using std::integral_constant;
                const integral_constant<int, 1> c1;
                const integral_constant<int, 2> c2;
                const integral_constant<int, 4> c4;
                const integral_constant<int, 8> c8;
                auto with_n = [&](auto jc, auto rb) {
                    // (what LDS and registers hold)
                    constexpr bool DENSE = std::is_same_v<decltype(rows_of), Bf16Rows>;
                    if constexpr (decltype(jc)::value * decltype(parts)::value > 12 || (DENSE && decltype(jc)::value > 4))
                        run(rows_of, w, out, jc, c2, rb, parts);
                    else
                        outw <= 64 ? run(rows_of, w, out, jc, c2, rb, parts) : run(rows_of, w, out, jc, c4, rb, parts);
                };
                constexpr bool DENSE = std::is_same_v<decltype(rows_of), Bf16Rows>;
                const integral_constant<int, DENSE ? 1 : 2> rb4;
                j <= 1 ? with_n(c1, c2) : j <= 2 ? with_n(c2, c2) : j <= 4 ? with_n(c4, rb4) : with_n(c8, c1);
            };
            auto with_out = [&](auto rows_of, auto w, auto parts) {
                c_dtype == GS_F32 ? with_j(rows_of, w, 0.0f, parts) : with_j(rows_of, w, u16(0), parts);
            };
            const std::integral_constant<int, 1> one;
            const std::integral_constant<int, 3> three;
            if (A.saved) {
                const SavedRows r{A.saved->codes, A.saved->scales, saved_code_pitch(in), saved_scale_pitch(in),
                                  A.saved->act == GS_ACT_RELU ? 0.0f : 128.0f, (int)in};
                w_dtype == GS_F32 ? with_out(r, 0.0f, three) : with_out(r, u16(0), one);
            } else {
                with_out(Bf16Rows{(const u16 *)A.p, A.ld, (int)in}, u16(0), one);
            }
            GS_HIP(hipGetLastError());
            return;
        }
        // Few rows: the matrices are what is read (64 groups, 1024 x 1024 bf16: 32 rows a group 35 and 47 in
        // tiles, 48 56 and 50; 512 x 512 fp32: 32 rows 22 and 32, 64 36 and 32).
        if (rows <= 32 * groups && in >= 64 && outw >= 4) {
            auto run = [&](auto la, auto type, auto out, auto turn, auto cols) {
                using T = decltype(type);
                using TO = decltype(out);
                constexpr int N = decltype(cols)::value;
                const int64_t tiles_n = ceil_div(outw, 32 * N), grid = (ceil_div(rows, 32) + groups + 2) * tiles_n;
                if (grid > INT32_MAX / 512) fail(GS_ERR_UNSUPPORTED, "the product has too many tiles");
                k_grouped_few<decltype(la), T, decltype(turn)::value, N, TO><<<(unsigned)grid, kFewWaves * kWave, 0, s>>>(
                    la, (const T *)W, ldw, w_step, off, in, outw, fill != 0, (int)tiles_n, (TO *)C, ldc);
            };
            // 128 columns a workgroup where there is one a compute unit, else 64 (2048 x 1024 bf16, 8 groups:
            // 20 and 17, 32 groups 25 and 29; 512 x 512 fp32, 64 groups 18 and 19)
            const bool wide = std::min(rows, groups) * ceil_div(outw, 128) >= 256;
            auto with_n = [&](auto la, auto type, auto out, auto turn) {
                wide ? run(la, type, out, turn, std::integral_constant<int, 4>{}) : run(la, type, out, turn, std::integral_constant<int, 2>{});
            };
            auto with_out = [&](auto la, auto type) {
                if (c_dtype == GS_F32)
                    transpose ? with_n(la, type, 0.0f, std::false_type{}) : with_n(la, type, 0.0f, std::true_type{});
                else
                    transpose ? with_n(la, type, u16(0), std::false_type{}) : with_n(la, type, u16(0), std::true_type{});
            };
            auto with_type = [&](auto type) {
                using T = decltype(type);
                if (A.saved)
                    with_out(SavedAlongRows<T>{A.saved->codes, A.saved->scales, saved_code_pitch(in), saved_scale_pitch(in),
                                               {A.saved->act == GS_ACT_RELU}},
                             type);
                else
                    with_out(AlongRows<T>{(const T *)A.p, A.ld}, type);
            };
            w_dtype == GS_F32 ? with_type(0.0f) : with_type(u16(0));
            GS_HIP(hipGetLastError());
            return;
        }
        // Tiles of 64 x 64 where ones of 128 x 128 would be half empty or too few (1024 x 1024 bf16, 256 rows a
        // group: 128 of them 25 and 31, 256 of them 42 and 32; 64 groups of 64 rows 49 and 51, of 96 85 and 52).
        const int wt = rows <= 64 * groups || outw <= 64 || ceil_div(rows, 128) * ceil_div(outw, 128) < 192 ? 1 : 2;
        const int64_t tiles_n = ceil_div(outw, 64 * wt), grid = (ceil_div(rows, 64 * wt) + groups + 2) * tiles_n;
        if (grid > INT32_MAX / 256) fail(GS_ERR_UNSUPPORTED, "the product has too many tiles");
        auto go = [&](auto la, auto lb, auto out) {
            using LA = decltype(la);
            using LB = decltype(lb);
            using TO = decltype(out);
            auto run = [&](auto kernel) {
                kernel<<<(unsigned)grid, 256, 0, s>>>(la, lb, w_step, off, in, outw, fill != 0, (int)tiles_n, (TO *)C, ldc);
            };
            wt == 1 ? run(k_grouped<LA, LB, TO, 1>) : run(k_grouped<LA, LB, TO, 2>);
        };
        auto with_out = [&](auto la, auto lb) { c_dtype == GS_F32 ? go(la, lb, 0.0f) : go(la, lb, u16(0)); };
        auto with_w = [&](auto la, auto type) {
            using T = decltype(type);
            transpose ? with_out(la, AlongRows<T>{(const T *)W, ldw}) : with_out(la, AcrossRows<T>{(const T *)W, ldw});
        };
        auto with_type = [&](auto type) {
            using T = decltype(type);
            if (A.saved)
                with_w(SavedAlongRows<T>{A.saved->codes, A.saved->scales, saved_code_pitch(in), saved_scale_pitch(in),
                                         {A.saved->act == GS_ACT_RELU}},
                       type);
            else
                with_w(AlongRows<T>{(const T *)A.p, A.ld}, type);
        };
        w_dtype == GS_F32 ? with_type(0.0f) : with_type(u16(0));
        GS_HIP(hipGetLastError());
    });
}

static int grouped_weight_grad(const Operand &A, int a_dtype, int64_t rows, int64_t a, const void *G, int64_t ldg, int dtype, int64_t b,
                               int64_t groups, const void *offsets, int offset_bytes, float *out, void *work, uint64_t work_bytes,
                               gs_stream stream)
{
    return guarded([&] {
        check_product(a, b);
        const Offsets off = check_offsets(offsets, offset_bytes, groups, rows);
        if (A.saved) {
            check_saved(A.saved, false);
            if (A.saved->rows != rows || A.saved->cols != a) fail(GS_ERR_INVALID_ARG, "A has another shape");
        } else {
            check_operand("A", A.p, rows, a, A.ld, dtype_size(a_dtype));
            if (a_dtype != dtype) fail(GS_ERR_INVALID_ARG, "A and G have different types");
        }
        check_operand("G", G, rows, b, ldg, dtype_size(dtype));
        if (!out) fail(GS_ERR_INVALID_ARG, "null output");
        const GroupedGradPlan p = grouped_grad_plan(rows, groups, a, b);
        const uint64_t need = p.direct ? 0 : (uint64_t)(p.chunks * a * b) * 4;
        if (work_bytes < need || (need && !work))
            fail(GS_ERR_INVALID_ARG, "workspace of %llu bytes is below the %llu needed",
                 (unsigned long long)(work ? work_bytes : 0), (unsigned long long)need);
        if (p.tiles_a * p.tiles_b > 65535) fail(GS_ERR_UNSUPPORTED, "the product has too many tiles");
        const auto whole = [](const void *p, int64_t bytes) { return Extent{p, 1, bytes, bytes}; };
        const Extent made = whole(out, groups * a * b * 4), partial = whole(need ? work : nullptr, (int64_t)need);
        const Extent g = {G, rows, b * dtype_size(dtype), ldg * dtype_size(dtype)};
        check_apart("out", made, "G", g), check_apart("work", partial, "G", g), check_apart("work", partial, "out", made);
        if (!A.saved) {
            const Extent dense = {A.p, rows, a * dtype_size(dtype), A.ld * dtype_size(dtype)};
            check_apart("out", made, "A", dense), check_apart("work", partial, "A", dense);
        }
        const hipStream_t s = (hipStream_t)stream;
        float *part = p.direct ? out : (float *)work;
        auto go = [&](auto la, auto lg, auto wa, auto wb) {
            constexpr int WA = decltype(wa)::value, WB = decltype(wb)::value;
            auto run = [&](auto kernel) {
                kernel<<<dim3((unsigned)p.chunks, (unsigned)(p.tiles_a * p.tiles_b)), kGradThreads, 0, s>>>(la, lg, off, a, b, p.per,
                                                                                                          (int)p.tiles_b, part);
            };
            p.per > kGradChain ? run(k_grouped_grad<decltype(la), decltype(lg), WA, WB, true>)
                               : run(k_grouped_grad<decltype(la), decltype(lg), WA, WB, false>);
        };
        auto with_tile = [&](auto type, auto wa, auto wb) {
            using T = decltype(type);
            constexpr int WA = decltype(wa)::value, WB = decltype(wb)::value;
            if (p.wa != WA || p.wb != WB) return;
            const GradDense<T, WB> g{(const T *)G, ldg, b};
            if (A.saved)
                go(GradSaved<T, 2 * WA>{A.saved->codes, A.saved->scales, saved_code_pitch(a), saved_scale_pitch(a),
                                        A.saved->act == GS_ACT_RELU ? 0u : 128u},
                   g, wa, wb);
            else if (WA == 1 && a < 2)
                go(GradDense<T, 2, true>{(const T *)A.p, A.ld, a}, g, std::integral_constant<int, 1>{}, wb);
            else
                go(GradDense<T, 2 * WA>{(const T *)A.p, A.ld, a}, g, wa, wb);
        };
        auto with_type = [&](auto type) {
            const std::integral_constant<int, 1> one;
            const std::integral_constant<int, 2> two;
            with_tile(type, one, one), with_tile(type, one, two), with_tile(type, two, one), with_tile(type, two, two);
        };
        dtype == GS_F32 ? with_type(0.0f) : with_type(u16(0));
        GS_HIP(hipGetLastError());
        if (!p.direct) {
            k_grouped_join<<<dim3((unsigned)ceil_div(a * b, 1024), (unsigned)groups), 256, 0, s>>>(part, off, a * b, p.per, p.chunks, out);
            GS_HIP(hipGetLastError());
        }
    });
}

extern "C" {

int gs_grouped_matmul(const void *A, int64_t lda, int dtype, int64_t rows, const void *W, int64_t ldw, int64_t w_step, int64_t groups,
                      int64_t k, int64_t n, int transpose, const void *offsets, int offset_bytes, int fill, void *C, int64_t ldc,
                      int c_dtype, gs_stream stream)
{
    return grouped_matmul({A, lda, nullptr}, dtype, rows, W, dtype, ldw, w_step, groups, k, n, transpose, offsets, offset_bytes, fill, C,
                          ldc, c_dtype, stream);
}

int gs_grouped_matmul_saved(const gs_saved *A, const void *W, int dtype, int64_t ldw, int64_t w_step, int64_t groups, int64_t k,
                            int64_t n, int transpose, const void *offsets, int offset_bytes, int fill, void *C, int64_t ldc,
                            int c_dtype, gs_stream stream)
{
    if (!A) return guarded([] { fail(GS_ERR_INVALID_ARG, "null saved activations"); });
    return grouped_matmul({nullptr, 0, A}, dtype, A->rows, W, dtype, ldw, w_step, groups, k, n, transpose, offsets, offset_bytes, fill,
                          C, ldc, c_dtype, stream);
}

int gs_grouped_weight_grad_workspace(int64_t rows, int64_t groups, int64_t a, int64_t b, uint64_t *bytes)
{
    return guarded([&] {
        if (!bytes) fail(GS_ERR_INVALID_ARG, "null output");
        check_product(a, b);
        if (rows < 0 || rows > INT32_MAX || groups < 1) fail(GS_ERR_INVALID_ARG, "bad matrix size");
        if (groups > 65535) fail(GS_ERR_UNSUPPORTED, "at most 65535 groups");
        const GroupedGradPlan p = grouped_grad_plan(rows, groups, a, b);
        *bytes = p.direct ? 0 : (uint64_t)(p.chunks * a * b) * 4;
    });
}

int gs_grouped_weight_grad(const void *A, int64_t lda, const void *G, int64_t ldg, int dtype, int64_t rows, int64_t a, int64_t b,
                           int64_t groups, const void *offsets, int offset_bytes, float *out, void *work, uint64_t work_bytes,
                           gs_stream stream)
{
    return grouped_weight_grad({A, lda, nullptr}, dtype, rows, a, G, ldg, dtype, b, groups, offsets, offset_bytes, out, work, work_bytes,
                               stream);
}

int gs_grouped_weight_grad_saved(const gs_saved *A, const void *G, int64_t ldg, int dtype, int64_t b, int64_t groups,
                                 const void *offsets, int offset_bytes, float *out, void *work, uint64_t work_bytes, gs_stream stream)
{
    if (!A) return guarded([] { fail(GS_ERR_INVALID_ARG, "null saved activations"); });
    return grouped_weight_grad({nullptr, 0, A}, dtype, A->rows, A->cols, G, ldg, dtype, b, groups, offsets, offset_bytes, out, work,
                               work_bytes, stream);
}

}  // extern "C"
