// y = a b^T on microscaled operands: activations in E2M1 or E4M3, weights in E2M1, a power-of-two scale for each 32 elements of
// a row, which the matrix instruction (v_mfma_scale_f32_16x16x128_f8f6f4) applies itself.
//
// Operands of the instruction, K = 128: lane l holds row l % 16 of its operand and the scale byte of the elements 32 q .. + 32,
// q = l / 16.  E2M1: those 32 elements, 16 bytes.  E4M3: elements 16 q .. + 16 and 64 + 16 q .. + 16, 16 bytes each.
//
// Rounding: sums are held in fp32.  Within an instruction on E4M3 the hardware drops what of a product lies below 2^-13 of its largest
// neighbour.  That is taken as it is: errors against 64 bits, 4096 x 11008 x 4096, of the fp32 sums 2.4e-5 in norm (sums of fp32
// products 3.6e-8), of y, after its rounding to bf16, 1.65722e-3 (1.65705e-3); 1.4 % of y are the next bf16 value.  To keep those bits
// takes the activations in two parts by magnitude, twice the matrix instructions.  (E2M1: no product is that small; sums are exact
// until fp32 rounds them.)
#include <algorithm>

#include "mx_formats.h"
#include "quest_internal.h"

namespace quest {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kUnit = 128;
constexpr int kF4 = 4, kF8 = 0;   // the instruction's codes for E2M1 and E4M3

template <int FORMAT>
struct MxOperand {
    static constexpr bool kE4M3 = FORMAT == QUEST_MX_E4M3;
    static constexpr int kUnitBytes = kE4M3 ? 128 : 64;   // of a row
    uint4 lo, hi;

    __device__ __forceinline__ void load(const uint8_t *codes, int unit, int quarter)
    {
        const uint8_t *p = codes + unit * kUnitBytes + 16 * quarter;
        lo = *reinterpret_cast<const uint4 *>(p);
        if constexpr (kE4M3)
            hi = *reinterpret_cast<const uint4 *>(p + 64);
    }
    __device__ __forceinline__ v8i operand() const
    {
        if constexpr (kE4M3)
            return v8i{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        else
            return v8i{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, 0, 0, 0, 0};
    }
};

// The scale dwords (of all four quarters) of GROUP consecutive units of a row, by one load
template <int GROUP>
struct MxScales {
    typedef uint32_t Words __attribute__((ext_vector_type(GROUP), aligned(4)));
    Words words;

    __device__ __forceinline__ void load(const uint8_t *scales, int unit) { words = *reinterpret_cast<const Words *>(scales + 4 * unit); }
    // as if loaded `by` units further on (what would lie beyond is not used)
    __device__ __forceinline__ void skip(int by)
    {
        for (; by > 0; --by)
#pragma unroll
            for (int s = 0; s + 1 < GROUP; ++s)
                words[s] = words[s + 1];
    }
};
template <>
struct MxScales<1> {
    uint32_t words[1];

    __device__ __forceinline__ void load(const uint8_t *scales, int unit) { words[0] = *reinterpret_cast<const uint32_t *>(scales + 4 * unit); }
    __device__ __forceinline__ void skip(int) {}
};

// blockIdx.x: weight rows 16 NT blockIdx.x .., blockIdx.y: activation rows 16 MT blockIdx.y ..; the waves share the contraction
// in groups of GROUP consecutive units of 128 (K / 128 >= GROUP) and meet in LDS.  The weights are the row operand, so a lane's four
// sums are consecutive outputs of a row.
template <int FORMAT, int MT, int NT, int GROUP, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mx_few_kernel(const uint8_t *__restrict__ a_codes,
                                                            const uint8_t *__restrict__ a_scales,
                                                            const uint8_t *__restrict__ b_codes,
                                                            const uint8_t *__restrict__ b_scales, int M, int N, int K,
                                                            uint16_t *__restrict__ y, int64_t ld_y, float *__restrict__ acc_out)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    typedef MxOperand<FORMAT> A;
    typedef MxOperand<QUEST_MX_E2M1> B;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row16 = lane & 15, quarter = lane >> 4;
    const int n0 = blockIdx.x * 16 * NT, m0 = blockIdx.y * 16 * MT;
    const int units = K / kUnit;

    const uint8_t *a_row[MT], *b_row[NT], *a_scale[MT], *b_scale[NT];   // rows beyond the edge read the last row, not stored
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t row = min(m0 + 16 * i + row16, M - 1);
        a_row[i] = a_codes + row * units * A::kUnitBytes;
        a_scale[i] = a_scales + row * units * 4;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t row = min(n0 + 16 * j + row16, N - 1);
        b_row[j] = b_codes + row * units * B::kUnitBytes;
        b_scale[j] = b_scales + row * units * 4;
    }
    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            acc[i][j] = v4f{0, 0, 0, 0};
    const int groups = (units + GROUP - 1) / GROUP;
    if (wave < groups) {
        A a[GROUP][MT];
        B b[GROUP][NT];
        MxScales<GROUP> sa[MT], sb[NT];
        auto fetch_scales = [&](int group) {   // (a group that is not whole ends where the row ends)
            const int from = min(group * GROUP, units - GROUP);
#pragma unroll
            for (int j = 0; j < NT; ++j)
                sb[j].load(b_scale[j], from);
#pragma unroll
            for (int i = 0; i < MT; ++i)
                sa[i].load(a_scale[i], from);
        };
        auto fetch = [&](int s, int unit) {   // past the end: the last unit again, not used
            unit = min(unit, units - 1);
#pragma unroll
            for (int j = 0; j < NT; ++j)
                b[s][j].load(b_row[j], unit, quarter);
#pragma unroll
            for (int i = 0; i < MT; ++i)
                a[s][i].load(a_row[i], unit, quarter);
        };
        auto multiply = [&](int s, const MxScales<GROUP> (&wa)[MT], const MxScales<GROUP> (&wb)[NT]) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        b[s][j].operand(), a[s][i].operand(), acc[i][j], kF4, A::kE4M3 ? kF8 : kF4, 0,
                        (int)(wb[j].words[s] >> (8 * quarter)), 0, (int)(wa[i].words[s] >> (8 * quarter)));
        };
        int g = wave;
        fetch_scales(g);
#pragma unroll
        for (int s = 0; s < GROUP; ++s)
            fetch(s, g * GROUP + s);
        for (; g + WAVES < groups; g += WAVES) {
            MxScales<GROUP> now_a[MT], now_b[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i)
                now_a[i] = sa[i];
#pragma unroll
            for (int j = 0; j < NT; ++j)
                now_b[j] = sb[j];
            fetch_scales(g + WAVES);
#pragma unroll
            for (int s = 0; s < GROUP; ++s) {
                multiply(s, now_a, now_b);
                fetch(s, (g + WAVES) * GROUP + s);
            }
        }
        const int beyond = g * GROUP - min(g * GROUP, units - GROUP);
#pragma unroll
        for (int i = 0; i < MT; ++i)
            sa[i].skip(beyond);
#pragma unroll
        for (int j = 0; j < NT; ++j)
            sb[j].skip(beyond);
#pragma unroll
        for (int s = 0; s < GROUP; ++s)
            if (g * GROUP + s < units)
                multiply(s, sa, sb);
    }
    // the waves' sums, added in their order: [wave][i][j][lane]
    v4f *park = reinterpret_cast<v4f *>(smem);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            park[((wave * MT + i) * NT + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    const bool quad_ok = (ld_y & 3) == 0 && (reinterpret_cast<uintptr_t>(y) & 7) == 0;
    for (int t = tid; t < MT * NT * 64; t += 64 * WAVES) {
        v4f sum = park[t];
#pragma unroll
        for (int v = 1; v < WAVES; ++v)
            sum += park[v * (MT * NT * 64) + t];
        const int tile = t >> 6, l = t & 63;
        const int m = m0 + 16 * (tile / NT) + (l & 15), n = n0 + 16 * (tile % NT) + 4 * (l >> 4);
        if (m >= M || n >= N)
            continue;
        if (acc_out) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < N)
                    acc_out[(int64_t)m * N + n + e] = sum[e];
        }
        if (!y)
            continue;
        uint16_t *dst = y + (int64_t)m * ld_y + n;
        if (quad_ok && n + 4 <= N) {
            *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < N)
                    dst[e] = (uint16_t)float_to_bf16_bits(sum[e]);
        }
    }
}

template <int FORMAT, int MT, int NT, int GROUP, int WAVES>
hipError_t launch_few(const MxGemmArgs &a, hipStream_t stream)
{
    constexpr int64_t kRows = 65535 * 16 * MT;   // of a launch
    const int64_t row_a = FORMAT == QUEST_MX_E4M3 ? a.K : a.K / 2;
    hipError_t err = hipSuccess;
    for (int64_t first = 0; first < a.M && err == hipSuccess; first += kRows) {
        const int64_t rows = std::min(a.M - first, kRows);
        const dim3 grid((unsigned)((a.N + 16 * NT - 1) / (16 * NT)), (unsigned)((rows + 16 * MT - 1) / (16 * MT)));
        hipLaunchKernelGGL((mx_few_kernel<FORMAT, MT, NT, GROUP, WAVES>), grid, dim3(64 * WAVES), WAVES * MT * NT * 1024, stream,
                           a.a_codes + first * row_a, a.a_scales + first * (a.K / 32), a.b_codes, a.b_scales, (int)rows, (int)a.N,
                           (int)a.K, a.y ? static_cast<uint16_t *>(a.y) + first * a.ld_y : nullptr, a.ld_y,
                           a.acc_out ? a.acc_out + first * a.N : nullptr);
        err = hipGetLastError();
    }
    return err;
}

constexpr int64_t kShortestTiled = 384;   // (a tile takes two stages at least)

}  // namespace

/*
 * The kernel and its block: the smallest block of few rows with which no compute unit has a second workgroup, tiles where there is
 * none.  Measured with operands that come from memory (us; a graph of calls):
 *   24 x 4096 x 4096 E4M3 16x32 6.5, 32x32 7.9; 48 x 4096 x 4096 32x32 8.7, 64x32 9.7; 64 x 5632 x 2048 E2M1 64x32 5.6, 32x32 6.2,
 *     64x64 7.7; 200 x 4096 x 2048 E4M3 64x64 9.8, 64x32 13.2, tiles of 128 13.6; 256 x 4096 x 4096 64x64 17.6, tiles 27.2
 *   with 16 rows or fewer 16x32 for all larger outputs (16 x 22016 x 4096 E4M3 16x16 22.0, 16x32 16.3; 1 x 11008 x 4096 8.1 and 8.6),
 *     up to 32 rows 32x32 (24 x 11008 x 4096 14.4, 64x32 17.0, 64x64 14.3; 32 x 22016 x 4096 22.7, 27.2, 28.4)
 *   more blocks: tiles (512 x 4096 x 4096 E4M3 29.9, 64x64 34.1; 400 x 5632 x 2048 15.0 and 25.7), of 256 where the compute unit
 *     with most of them has less to do: one takes 2.2 times as long as one of 128 (2048 x 2048 x 2048, 64 or 256 tiles, 18.7 / 9.8;
 *     2048 x 5632 x 2048, 176 or 704, 22.4 / 24.9; 1024 x 11008 x 4096, 172 or 688, 32.5 / 42.8); tiles of 256 x 128 were the
 *     best nowhere
 * Contractions of 128 and 256, which are a single stage of a tile, stay with the few-rows kernel.
 */
quest_plan plan_mx_gemm(int64_t M, int64_t N, int64_t K)
{
    constexpr int64_t kUnitsOfChip = 256;
    auto blocks = [&](int64_t rows, int64_t cols) { return ((M + rows - 1) / rows) * ((N + cols - 1) / cols); };
    if (blocks(16, 16) <= kUnitsOfChip)
        return {QUEST_PLAN_FEW, 16, 16, 0};
    if (M <= 16 || blocks(16, 32) <= kUnitsOfChip)
        return {QUEST_PLAN_FEW, 16, 32, 0};
    if (M <= 32 || blocks(32, 32) <= kUnitsOfChip)
        return {QUEST_PLAN_FEW, 32, 32, 0};
    if (blocks(64, 32) <= kUnitsOfChip)
        return {QUEST_PLAN_FEW, 64, 32, 0};
    if (K < kShortestTiled || blocks(64, 64) <= kUnitsOfChip)
        return {QUEST_PLAN_FEW, 64, 64, 0};
    auto rounds = [&](int64_t tiles) { return (tiles + kUnitsOfChip - 1) / kUnitsOfChip; };
    const int block = 2.2 * (double)rounds(blocks(256, 256)) <= (double)rounds(blocks(128, 128)) ? 256 : 128;
    return {QUEST_PLAN_TILES, block, block, 0};
}

namespace {

// Groups of four units where each of the four waves has one, else of two, else of one.  (16 x 22016 x 4096 E4M3 in groups of
// four 16.3 us, of two 18.4; 24 x 11008 x 4096 E2M1 12.1 and 13.1, in groups of one, with a scale load for each unit, 16.0)
template <int FORMAT, int MT, int NT>
hipError_t launch_few_groups(const MxGemmArgs &a, hipStream_t stream)
{
    const int64_t units = a.K / kUnit;
    return units >= 16  ? launch_few<FORMAT, MT, NT, 4, 4>(a, stream)
           : units >= 8 ? launch_few<FORMAT, MT, NT, 2, 4>(a, stream)
                        : launch_few<FORMAT, MT, NT, 1, 4>(a, stream);
}

template <int FORMAT>
hipError_t launch_format(const MxGemmArgs &a, hipStream_t stream)
{
    quest_plan p = plan_mx_gemm(a.M, a.N, a.K);
    if (p.kernel == QUEST_PLAN_TILES && a.y && a.ld_y >= (1 << 24))   // a tile's 32 rows of y are one buffer of less than 2 GiB
        p = {QUEST_PLAN_FEW, 64, 64, 0};
    if (p.kernel == QUEST_PLAN_TILES)
        return FORMAT == QUEST_MX_E4M3 ? launch_mx_tiles_e4m3(a, p.block_rows, stream) : launch_mx_tiles_e2m1(a, p.block_rows, stream);
    if (p.block_cols == 16)
        return launch_few_groups<FORMAT, 1, 1>(a, stream);
    if (p.block_rows == 16)
        return launch_few_groups<FORMAT, 1, 2>(a, stream);
    if (p.block_rows == 32)
        return launch_few_groups<FORMAT, 2, 2>(a, stream);
    return p.block_cols == 32 ? launch_few_groups<FORMAT, 4, 2>(a, stream) : launch_few_groups<FORMAT, 4, 4>(a, stream);
}

}  // namespace

namespace {

// (the largest block parks 64 KiB)
template <int FORMAT>
hipError_t prepare_largest()
{
    hipError_t err = hipSuccess;
    auto allow = [&](auto kernel) {
        if (err == hipSuccess)
            err = allow_dynamic_lds(reinterpret_cast<const void *>(kernel), 64 << 10);
    };
    allow(mx_few_kernel<FORMAT, 4, 4, 1, 4>);
    allow(mx_few_kernel<FORMAT, 4, 4, 2, 4>);
    allow(mx_few_kernel<FORMAT, 4, 4, 4, 4>);
    return err;
}

}  // namespace

hipError_t prepare_mx_gemm_kernels()
{
    static OncePerDevice once;
    return once([] {
        const hipError_t err = prepare_largest<QUEST_MX_E2M1>();
        return err != hipSuccess ? err : prepare_largest<QUEST_MX_E4M3>();
    });
}

hipError_t launch_mx_gemm(const MxGemmArgs &a, hipStream_t stream)
{
    if (a.M == 0 || a.N == 0)
        return hipSuccess;
    const hipError_t err = prepare_mx_gemm_kernels();
    if (err != hipSuccess)
        return err;
    return a.a_format == QUEST_MX_E4M3 ? launch_format<QUEST_MX_E4M3>(a, stream) : launch_format<QUEST_MX_E2M1>(a, stream);
}

}  // namespace quest

quest_plan quest_plan_mx_gemm(int64_t M, int64_t N, int64_t K)
{
    return quest::plan_mx_gemm(M, N, K);
}
