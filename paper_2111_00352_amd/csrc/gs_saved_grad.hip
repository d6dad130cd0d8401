// Weight gradient value(A)^T . G from activations saved in 8 bits: the
// contraction over the n rows of an n x a matrix of codes and an n x b matrix of
// gradients.
//
// A value is a code of at most 8 significant bits times a power of two, which
// bf16 holds exactly.  An fp32 gradient is the sum of three bf16 numbers of 8
// bits each (its significand cut twice), so three bf16 products with fp32 sums
// give the fp32 product's accuracy at several times the fp32 matrix rate
// (V_MFMA_F32_32X32X16_BF16: 2.5 PFLOP/s against 157 TFLOP/s), and a bf16 gradient
// needs one.  That leaves the kernel bound by reading A and G once.  Gradients below
// 2^-110 end under bf16's smallest subnormal, 2^-133 (the instruction takes subnormals
// as they are): what lies below it, less than 2^-133 of a gradient, is cut off.
//
// Both operands are wanted with their rows, the k index of the product, running
// inside a lane, and they lie in memory by rows.  A lane therefore loads CA
// neighbouring columns of A (one dword at CA = 4) and CB of G in each of eight rows:
// as many 8-deep fragments as it loads columns, without a trip through LDS, of columns
// CA (CB) apart.  A wave's tile is 32 CA x 32 CB of the product; a workgroup's eight
// waves share it and split the rows, 16 at a time each, with the loads of the next
// two steps in flight.
//
// 100,000 rows of 128 x 64 in 32 bits take 15.4 us and 3.9 us for joining the partials
// (16.9 us a call); the operands' 39 MB are 6 us of that at the rate of a copy.  The
// rest is the start of 250 workgroups whose waves take three or four steps each, so that
// two of them in flight never run steadily, the join of eight waves through LDS in eight
// rounds, and the partials (8 MB written and read); how much each takes is not measured.
// 30,011 rows of 255 x 47 in bf16 (one or two steps a wave) 10.5 us and 2.5 us.
#include <algorithm>
#include <type_traits>

#include "gs_device.h"
#include "gs_lowbit.h"

namespace gs {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kGradWaves = 8;   // of a workgroup
constexpr int kGradStep = 16;   // rows a wave takes at a time
constexpr int kGradRows = kGradWaves * kGradStep;
// Longest run of rows a wave sums before the partials are joined.
constexpr int64_t kGradChainRows = 8192;
// Rows up to which one workgroup sums them all.  128 x 64 in 32 bits, in a graph: 256
// rows 8.3 us in one workgroup, 512 11.4, 1024 17.7; in two launches 9.1 us each.
constexpr int64_t kGradOne = 256;
constexpr int64_t kGradMaxLd = 1 << 26;  // (a lane's offset from its step's row has 32 bits)

#define GLOBAL __attribute__((address_space(1)))

template <int C> struct CodeBytes;
template <> struct CodeBytes<1> {
    typedef uint8_t type;
};
template <> struct CodeBytes<2> {
    typedef u16 type;
};
template <> struct CodeBytes<4> {
    typedef uint32_t type;
};

// Upper halves of a (into the low half) and b.
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b)
{
    return __builtin_amdgcn_perm(b, a, 0x07060302);
}

template <class T, int CA, int CB> struct GradStage {
    typename CodeBytes<CA>::type code[8];
    uint8_t scale[8];
    typename Elems<T, CB>::type g[8];
};

// Workgroup (x, y): rows [x * per, (x + 1) * per), columns of tile y; its sums go to
// part + x * a * b.  RELU: codes are unsigned.
template <class T, int CA, int CB, bool RELU>
__global__ __launch_bounds__(kGradWaves * kWave, 2) void k_saved_grad(
    const uint8_t *__restrict__ codes, int64_t code_pitch, const uint8_t *__restrict__ scales, int64_t scale_pitch,
    const T *__restrict__ G, int64_t ldg, int64_t n, int a, int b, int64_t per, float *__restrict__ part)
{
    constexpr int NP = sizeof(T) == 4 ? 3 : 1;  // bf16 parts of a gradient
    __shared__ float red[2][kGradWaves][16][kWave];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int nbt = (b + 32 * CB - 1) / (32 * CB);
    const int a0 = (blockIdx.y / nbt) * 32 * CA, b0 = (blockIdx.y % nbt) * 32 * CB;
    // Columns of lane l's fragments.  Lanes past the padded codes repeat its last
    // columns, which are not stored if they are past a; a width b that is no
    // multiple of CB ends in columns that two lanes hold (and store alike).
    auto col_a = [&](int l) { const int c = a0 + CA * l; return c < (int)code_pitch - CA ? c : (int)code_pitch - CA; };
    auto col_b = [&](int l) { const int c = b0 + CB * l; return c < b - CB ? c : b - CB; };
    const int half = lane / 32;
    const int64_t r0 = (int64_t)blockIdx.x * per, r1 = r0 + per < n ? r0 + per : n;
    int64_t r = r0 + wave * kGradStep;
    // Addresses are a row's, the same for all lanes, and this lane's offset from it.
    const uint32_t oc = 8 * half * (uint32_t)code_pitch + col_a(lane % 32);
    const uint32_t os = 8 * half * (uint32_t)scale_pitch + col_a(lane % 32) / kMxBlock;
    const uint32_t og = (8 * half * (uint32_t)ldg + col_b(lane % 32)) * (uint32_t)sizeof(T);

    GradStage<T, CA, CB> st[2];
    auto load = [&](GradStage<T, CA, CB> &st, int64_t row) {  // rows row + 8 * half + 0..7
        uint64_t pc = (uint64_t)(codes + row * code_pitch), ps = (uint64_t)(scales + row * scale_pitch);
        uint64_t pg = (uint64_t)(G + row * ldg);
        asm("" : "+s"(pc), "+s"(ps), "+s"(pg));  // (or every load would keep a pointer of its own)
#pragma unroll
        for (int j = 0; j < 8; j++) {
            st.code[j] = *(const GLOBAL typename CodeBytes<CA>::type *)((const GLOBAL uint8_t *)(pc + j * code_pitch) + oc);
            st.scale[j] = *((const GLOBAL uint8_t *)(ps + j * scale_pitch) + os);
            st.g[j] = *(const GLOBAL typename Elems<T, CB>::type *)((const GLOBAL uint8_t *)(pg + j * ldg * sizeof(T)) + og);
        }
    };
    auto load_end = [&](GradStage<T, CA, CB> &st, int64_t row) {  // the same with zeros from r1 on
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int64_t at = row + 8 * half + j;
            st.code[j] = 0;
            st.scale[j] = 0;
            st.g[j] = typename Elems<T, CB>::type{};
            if (at < r1) {
                st.code[j] = *reinterpret_cast<const typename CodeBytes<CA>::type *>(codes + at * code_pitch + col_a(lane % 32));
                st.scale[j] = scales[at * scale_pitch + col_a(lane % 32) / kMxBlock];
                st.g[j] = *reinterpret_cast<const typename Elems<T, CB>::type *>(G + at * ldg + col_b(lane % 32));
            }
        }
    };
    f32x16 acc[CA][CB];
#pragma unroll
    for (int i = 0; i < CA; i++)
#pragma unroll
        for (int j = 0; j < CB; j++) acc[i][j] = f32x16{};
    auto pack = [](const uint32_t *v) {
        return make_uint4(high_halves(v[0], v[1]), high_halves(v[2], v[3]), high_halves(v[4], v[5]),
                          high_halves(v[6], v[7]));
    };
    // Multiplies the rows in st, then_load() once their registers are free.
    auto multiply = [&](const GradStage<T, CA, CB> &st, auto &&then_load) {
        uint4 fa[CA];
        {
            // 2^(E - 127), E > 0 here (0 beside codes of 0); E = 255 gives infinity, and z NaN
            float s[8], z[8];
#pragma unroll
            for (int j = 0; j < 8; j++) {
                s[j] = __uint_as_float((uint32_t)st.scale[j] << 23);
                z[j] = s[j] * 0.0f;
            }
#pragma unroll
            for (int i = 0; i < CA; i++) {
                uint32_t v[8];
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const int c = (int)(st.code[j] >> (8 * i) & 255);
                    v[j] = __float_as_uint(__builtin_fmaf((float)(RELU ? c : (int)(int8_t)c), s[j], z[j]));
                }
                fa[i] = pack(v);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int i = 0; i < CB; i++) {
            uint4 fb[NP];
            if constexpr (NP == 1) {
                fb[0] = make_uint4(st.g[0][i] | (uint32_t)st.g[1][i] << 16, st.g[2][i] | (uint32_t)st.g[3][i] << 16,
                                   st.g[4][i] | (uint32_t)st.g[5][i] << 16, st.g[6][i] | (uint32_t)st.g[7][i] << 16);
            } else {
                // g = hi + mid + lo, each the leading 8 bits of what is left
                float rest[8], top = 0.0f;
                uint32_t v[8];
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const float g = st.g[j][i];
                    v[j] = __float_as_uint(g);
                    top = fmaxf(top, fabsf(g));
                    rest[j] = g - __uint_as_float(v[j] & 0xffff0000u);
                }
                fb[0] = pack(v);
                if (__any(top == __builtin_inff())) {  // (infinity less itself: it is all in hi)
                    asm volatile("");                  // (rare: not worth selects in every step)
#pragma unroll
                    for (int j = 0; j < 8; j++)
                        if (fabsf((float)st.g[j][i]) == __builtin_inff()) rest[j] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    v[j] = __float_as_uint(rest[j]);
                    rest[j] -= __uint_as_float(v[j] & 0xffff0000u);
                }
                fb[NP > 1 ? 1 : 0] = pack(v);
#pragma unroll
                for (int j = 0; j < 8; j++) v[j] = __float_as_uint(rest[j]);
                fb[NP > 1 ? 2 : 0] = pack(v);
            }
            if (i == CB - 1) {
                __builtin_amdgcn_sched_barrier(0);
                then_load();
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int p = NP - 1; p >= 0; p--)
#pragma unroll
                for (int k = 0; k < CA; k++)
                    acc[k][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa[k]),
                                                                        __builtin_bit_cast(bf16x8, fb[p]), acc[k][i], 0, 0, 0);
        }
    };
    // Whole steps two at a time; the registers of one are loaded for the step after the
    // next as soon as its fragments are made.
    const int64_t whole = r1 - kGradStep;  // last row a whole step can start at
    if (r <= whole) {
        load(st[0], r);
        if (r + kGradRows <= whole) load(st[1], r + kGradRows);
#pragma unroll 1
        for (; r + kGradRows <= whole; r += 2 * kGradRows) {
            multiply(st[0], [&] { if (r + 2 * kGradRows <= whole) load(st[0], r + 2 * kGradRows); });
            multiply(st[1], [&] { if (r + 3 * kGradRows <= whole) load(st[1], r + 3 * kGradRows); });
        }
        if (r <= whole) {
            multiply(st[0], [] {});
            r += kGradRows;
        }
    }
    if (r < r1) {
        load_end(st[0], r);
        multiply(st[0], [] {});
    }

    // The waves' sums are added in LDS, one 32 x 32 tile at a time, and stored as the
    // workgroup's partial.  Accumulator: lane l, register e hold row
    // 8 (e / 4) + 4 (l / 32) + e % 4, column l % 32.
    float *out = part + (int64_t)blockIdx.x * a * b;
#pragma unroll
    for (int t = 0; t < CA * CB; t++) {
        const int i = t / CB, j = t % CB;
#pragma unroll
        for (int e = 0; e < 16; e++) red[t & 1][wave][e][lane] = acc[i][j][e];
        __syncthreads();
        // (the other buffer's readers are past this barrier before it is written again)
#pragma unroll
        for (int q = 0; q < 16 / kGradWaves; q++) {
            const int e = wave * (16 / kGradWaves) + q;
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < kGradWaves; w++) s += red[t & 1][w][e][lane];
            const int row = col_a(8 * (e / 4) + 4 * half + e % 4) + i, col = col_b(lane % 32) + j;
            if (row < a) out[(int64_t)row * b + col] = s;
        }
    }
}

struct GradPlan {
    int ca, cb;
    int64_t tiles, chunks, per;
};

// A compute unit's share of the workgroups is one, or two where a wave's tile is a
// single instruction's (its registers allow two).  Up to kGradOne rows one workgroup
// sums them all, which saves the launch that joins partials.
GradPlan grad_plan(int64_t n, int64_t a, int64_t b)
{
    GradPlan p;
    p.ca = a <= 32 ? 1 : a <= 64 ? 2 : 4;
    p.cb = b <= 32 ? 1 : 2;
    p.tiles = ceil_div(a, 32 * p.ca) * ceil_div(b, 32 * p.cb);
    const int64_t fill = (p.ca * p.cb == 1 ? 512 : 256) / p.tiles;
    const int64_t want = n <= kGradOne ? 1 : std::max(std::max<int64_t>(1, fill), ceil_div(n, kGradChainRows * kGradWaves));
    p.chunks = std::max<int64_t>(1, std::min(want, ceil_div(n, kGradRows)));
    p.per = ceil_div(ceil_div(std::max<int64_t>(n, 1), p.chunks), kGradStep) * kGradStep;
    p.chunks = std::max<int64_t>(1, ceil_div(n, p.per));
    return p;
}

void check_grad_sizes(int64_t n, int64_t a, int64_t b)
{
    if (n < 0 || a <= 0 || b <= 0) fail(GS_ERR_INVALID_ARG, "bad product size");
    if (a > 4096 || b > 4096 || n > INT32_MAX) fail(GS_ERR_UNSUPPORTED, "a and b are at most 4096");
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" {

int gs_saved_weight_grad_workspace(int64_t n, int64_t a, int64_t b, uint64_t *bytes)
{
    return guarded([&] {
        if (!bytes) fail(GS_ERR_INVALID_ARG, "null output");
        check_grad_sizes(n, a, b);
        const GradPlan p = grad_plan(n, a, b);
        *bytes = p.chunks > 1 ? (uint64_t)(p.chunks * a * b) * 4 : 0;
    });
}

int gs_saved_weight_grad(const gs_saved *A, const void *G, int64_t ldg, int dtype, int64_t b, float *out,
                         void *work, uint64_t work_bytes, gs_stream stream)
{
    return guarded([&] {
        check_saved(A, false);
        const int64_t n = A->rows, a = A->cols;
        check_grad_sizes(n, a, b);
        check_operand("G", G, n, b, ldg, dtype_size(dtype));
        if (n > 1 && ldg > kGradMaxLd) fail(GS_ERR_UNSUPPORTED, "G's leading dimension is at most 2^26");
        if (!out) fail(GS_ERR_INVALID_ARG, "null output");
        const GradPlan p = grad_plan(n, a, b);
        const uint64_t need = p.chunks > 1 ? (uint64_t)(p.chunks * a * b) * 4 : 0;
        if (work_bytes < need || (need && !work))
            fail(GS_ERR_INVALID_ARG, "workspace of %llu bytes is below the %llu needed",
                 (unsigned long long)(work ? work_bytes : 0), (unsigned long long)need);
        const hipStream_t s = (hipStream_t)stream;
        float *part = p.chunks > 1 ? (float *)work : out;
        const dim3 grid((unsigned)p.chunks, (unsigned)p.tiles);
        auto go = [&](auto ca, auto cb, auto type, auto relu) {
            using T = decltype(type);
            k_saved_grad<T, decltype(ca)::value, decltype(cb)::value, decltype(relu)::value>
                <<<grid, kGradWaves * kWave, 0, s>>>(A->codes, saved_code_pitch(a), A->scales, saved_scale_pitch(a),
                                                    (const T *)G, ldg, n, (int)a, (int)b, p.per, part);
        };
        auto typed = [&](auto ca, auto cb) {
            if (p.ca != decltype(ca)::value || p.cb != decltype(cb)::value) return;
            if (dtype == GS_F32)
                A->act == GS_ACT_RELU ? go(ca, cb, 0.0f, std::true_type{}) : go(ca, cb, 0.0f, std::false_type{});
            else
                A->act == GS_ACT_RELU ? go(ca, cb, u16(0), std::true_type{}) : go(ca, cb, u16(0), std::false_type{});
        };
        using C1 = std::integral_constant<int, 1>;
        using C2 = std::integral_constant<int, 2>;
        using C4 = std::integral_constant<int, 4>;
        typed(C1{}, C1{}), typed(C1{}, C2{}), typed(C2{}, C1{}), typed(C2{}, C2{}), typed(C4{}, C1{}), typed(C4{}, C2{});
        GS_HIP(hipGetLastError());
        if (p.chunks > 1) reduce_partials(part, (int)p.chunks, a * b, out, s);
    });
}

}  // extern "C"
