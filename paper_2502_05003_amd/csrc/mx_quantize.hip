// The quantizer for microscaled operands (block Hadamard transform, a power-of-two scale for each 32 elements, E2M1 or E4M3
// codes, trust mask) and the way back to what the codes stand for.  Both are passes over memory.
#include <algorithm>

#include "mx_formats.h"
#include "quest_internal.h"

namespace quest {
namespace {

constexpr int kThreads = 256;
constexpr int kUnit = 512;              // elements of a wave with eight to a lane
constexpr int kWaveBlock = 64 * 32;     // largest Hadamard block of a wave with 32 to a lane

template <int FORMAT>
__device__ __forceinline__ void store_encoded(const MxEncoded<FORMAT> &q, int64_t at, uint8_t *codes, uint8_t *scales,
                                              uint8_t *mask, bool first_of_group)
{
    if constexpr (MxFormat<FORMAT>::kE4M3)
        *reinterpret_cast<uint2 *>(codes + at) = make_uint2(q.words[0], q.words[1]);
    else
        *reinterpret_cast<uint32_t *>(codes + at / 2) = q.words[0];
    if (first_of_group)
        scales[at / kMxGroup] = (uint8_t)q.scale;
    if (mask)
        mask[at / 8] = (uint8_t)q.trust;
}

// Blocks of up to 512 elements: a wave takes 512 consecutive elements, of one row or several (blocks divide rows, so waves that
// start at multiples of 512 elements cut none), eight to a lane.
template <typename T, int FORMAT>
__global__ __launch_bounds__(kThreads) void mx_quantize_lanes_kernel(const T *__restrict__ x, int64_t elements, int cols,
                                                                     int64_t ld, int log2n, float norm,
                                                                     uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                                     uint8_t *__restrict__ mask)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t first = unit * kUnit, at = first + 8 * lane;
    float v[8] = {};
    if (at < elements) {
        int64_t from = at;
        if (ld != cols) {   // the row the wave starts in by one division, the lane's by another, of a small number
            const int64_t row = first / cols;
            const int column = (int)(first - row * cols) + 8 * lane, more = column / cols;
            from = (row + more) * ld + column - more * cols;
        }
        load8(x + from, v);
    }
    wave_hadamard(v, log2n, norm, lane);
    const MxEncoded<FORMAT> q = mx_encode<FORMAT>(v);
    if (at < elements)
        store_encoded<FORMAT>(q, at, codes, scales, mask, (lane & 3) == 0);
}

// Stages 1, 2, .. of the transform on 32 elements of a lane, then (blocks of 64 and more) across lanes; without the factor
__device__ __forceinline__ void group_butterflies(float (&v)[32], int log2n, int lane)
{
#pragma unroll
    for (int s = 0; s < 5; ++s) {
        if (s < log2n) {
            const int h = 1 << s;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                if ((i & h) == 0) {
                    const float a = v[i], b = v[i + h];
                    v[i] = a + b;
                    v[i + h] = a - b;
                }
            }
        }
    }
    lane_butterflies<32, 5>(v, log2n, lane);
}

/*
 * Blocks of up to 2048 elements.  A lane takes a group of 32 elements as a whole, so that the first five strides of the
 * transform, the group's maximum and its scale stay in the lane and are computed once: 10 vector instructions per element where
 * eight elements to a lane take 19, which bound the kernel above in bf16.  A wave takes 64 consecutive groups; a lane's loads are 64
 * (fp32: 128) bytes apart from its neighbour's, and each line is used up by them all, in the CU's cache.
 * us, eight elements to a lane / so: 16384 x 2048 in bf16, blocks of 32, E2M1 with mask 26 / 18 (17 at the rate of a large copy);
 * to E4M3 as it is 16.9 / 16.4; 24 x 5632, where the chip is empty, 2.1 / 2.8; 8192 x 4096 in fp32 29.5 / 34.  Blocks of 512 take
 * 26 us, blocks of 2048 29 (through LDS, as the larger ones below, 44).
 */
template <typename T, int FORMAT>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const T *__restrict__ x, int64_t groups, int row_groups, int64_t ld,
                                                               int log2n, float norm, uint8_t *__restrict__ codes,
                                                               uint8_t *__restrict__ scales, uint8_t *__restrict__ mask)
{
    typedef MxFormat<FORMAT> F;
    const int lane = threadIdx.x & 63;
    const int64_t first = ((int64_t)blockIdx.x * (kThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * kWave;
    const int64_t g = first + lane;
    float v[32] = {};
    if (g < groups) {
        int64_t from = g * kMxGroup;
        if (ld != (int64_t)row_groups * kMxGroup) {   // the row the wave starts in by one division, the lane's by another, of a small number
            const int64_t row = first / row_groups;
            const int column = (int)(first - row * row_groups) + lane, more = column / row_groups;
            from = (row + more) * ld + (int64_t)(column - more * row_groups) * kMxGroup;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float part[8];
            load8(x + from + 8 * i, part);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[8 * i + e] = part[e];
        }
    }
    group_butterflies(v, log2n, lane);

    // largest magnitude (a NaN stays one); of the values with their factor, since rounding keeps the order
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < 32; ++e)
        top = __builtin_elementwise_maximum(top, fabsf(v[e]));
    const uint32_t largest = __float_as_uint(top * norm);
    const int field = (int)(largest >> 23);
    const bool finite = field < 255;   // (a NaN may carry a sign, which is above the field)
    const uint32_t scale = finite ? (uint32_t)max(field - F::kMaxExponent, 0) : 255u;
    if (__any(!finite)) {
#pragma unroll
        for (int e = 0; e < 32; ++e)
            v[e] = finite ? v[e] : 0.0f;
    }
    // t = x_h 2^-e in one product with norm 2^-e, which rounds like x_h = v norm does, as long as neither is subnormal
    float factor = __uint_as_float((finite ? 254u - scale : 127u) << 23);
    if (__any(largest != 0 && (scale < 32u || scale > 192u))) {
#pragma unroll
        for (int e = 0; e < 32; ++e)
            v[e] *= norm;
    } else {
        factor *= norm;
    }
    uint32_t untrusted = 0, words[4 * F::kWords];
#pragma unroll
    for (int i = 3; i >= 0; --i) {
        float t[8];
#pragma unroll
        for (int e = 7; e >= 0; --e) {
            t[e] = __fmul_rn(v[8 * i + e], factor);
            // (the sign bit of what is left to the border, shifted in)
            untrusted = __builtin_amdgcn_alignbit(untrusted, __float_as_uint(F::kTrusted - fabsf(t[e])), 31);
        }
        uint32_t part[F::kWords];
        mx_convert<FORMAT>(t, part);
#pragma unroll
        for (int w = 0; w < F::kWords; ++w)
            words[F::kWords * i + w] = part[w];
    }
    if (g >= groups)
        return;
#pragma unroll
    for (int w = 0; w < F::kWords; ++w)
        reinterpret_cast<uint4 *>(codes + g * (kMxGroup * F::kBits / 8))[w] =
            make_uint4(words[4 * w], words[4 * w + 1], words[4 * w + 2], words[4 * w + 3]);
    scales[g] = (uint8_t)scale;
    if (mask)
        reinterpret_cast<uint32_t *>(mask)[g] = finite ? ~untrusted : 0u;
}

// Larger blocks: a workgroup holds a row in LDS for the transform's wider strides, three at a time.  Bound by those passes: 16384 x 4096
// in bf16, blocks of 4096, E2M1 with mask 88 us (blocks of 2048, without LDS, 55; 35 at the rate of a large copy).
template <typename T, int FORMAT>
__global__ __launch_bounds__(kThreads) void mx_quantize_row_kernel(const T *__restrict__ x, int cols, int64_t ld, int log2n,
                                                                   float norm, uint8_t *__restrict__ codes,
                                                                   uint8_t *__restrict__ scales, uint8_t *__restrict__ mask)
{
    extern __shared__ float row[];
    const T *source = x + (int64_t)blockIdx.x * ld;
    for (int i = threadIdx.x * 8; i < cols; i += kThreads * 8) {
        float v[8];
        load8(source + i, v);
        butterflies<3>(v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            row[lds_pad(i + e)] = v[e];
    }
    lds_butterfly_passes(row, cols, log2n);
    const int64_t first = (int64_t)blockIdx.x * cols;
    for (int i = threadIdx.x * 8; i < cols; i += kThreads * 8) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = row[lds_pad(i + e)] * norm;
        store_encoded<FORMAT>(mx_encode<FORMAT>(v), first + i, codes, scales, mask, (threadIdx.x & 3) == 0);
    }
}

template <int FORMAT, typename T>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(const uint8_t *__restrict__ codes,
                                                                 const uint8_t *__restrict__ scales, int64_t elements, int cols,
                                                                 T *__restrict__ out, int64_t ld)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t first = unit * kUnit, at = first + 8 * lane;
    if (at >= elements)
        return;
    uint32_t words[MxFormat<FORMAT>::kWords];
    if constexpr (MxFormat<FORMAT>::kE4M3) {
        const uint2 w = *reinterpret_cast<const uint2 *>(codes + at);
        words[0] = w.x;
        words[1] = w.y;
    } else {
        words[0] = *reinterpret_cast<const uint32_t *>(codes + at / 2);
    }
    float v[8];
    mx_decode<FORMAT>(words, scales[at / kMxGroup], v);
    int64_t to = at;
    if (ld != cols) {
        const int64_t row = first / cols;
        const int column = (int)(first - row * cols) + 8 * lane, more = column / cols;
        to = (row + more) * ld + column - more * cols;
    }
    store8(out + to, v);
}

unsigned blocks_for(int64_t elements)
{
    constexpr int64_t kPerBlock = kUnit * (kThreads / kWave);
    return (unsigned)((elements + kPerBlock - 1) / kPerBlock);
}

template <typename T, int FORMAT>
hipError_t launch(const MxQuantizeArgs &a, hipStream_t stream)
{
    const float norm = (float)(1.0 / sqrt((double)(int64_t(1) << a.log2n)));
    const T *x = static_cast<const T *>(a.x);
    const int64_t elements = a.rows * a.cols, groups = elements / kMxGroup;
    // groups to lanes: bf16, from four waves a compute unit on, and the blocks that only they hold
    const bool whole = (1 << a.log2n) > kUnit || (sizeof(T) == 2 && groups >= 4 * 256 * kWave);
    if ((1 << a.log2n) <= kWaveBlock && whole) {
        hipLaunchKernelGGL((mx_quantize_kernel<T, FORMAT>), dim3((unsigned)((groups + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                           stream, x, groups, (int)(a.cols / kMxGroup), a.ld, a.log2n, norm, a.codes, a.scales, a.mask);
    } else if ((1 << a.log2n) <= kUnit) {
        hipLaunchKernelGGL((mx_quantize_lanes_kernel<T, FORMAT>), dim3(blocks_for(elements)), dim3(kThreads), 0, stream, x, elements,
                           (int)a.cols, a.ld, a.log2n, norm, a.codes, a.scales, a.mask);
    } else {
        const hipError_t err = prepare_mx_quantize_kernels();
        if (err != hipSuccess)
            return err;
        hipLaunchKernelGGL((mx_quantize_row_kernel<T, FORMAT>), dim3((unsigned)a.rows), dim3(kThreads),
                           (a.cols + a.cols / 32) * sizeof(float), stream, x, (int)a.cols, a.ld, a.log2n, norm, a.codes, a.scales,
                           a.mask);
    }
    return hipGetLastError();
}

template <int FORMAT, typename T>
hipError_t launch_back(const MxDequantizeArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((mx_dequantize_kernel<FORMAT, T>), dim3(blocks_for(a.rows * a.cols)), dim3(kThreads), 0, stream, a.codes,
                       a.scales, a.rows * a.cols, (int)a.cols, static_cast<T *>(a.out), a.ld);
    return hipGetLastError();
}

}  // namespace

hipError_t prepare_mx_quantize_kernels()
{
    static OncePerDevice once;
    return once([] {
        constexpr int kBytes = (QUEST_MAX_COLS + QUEST_MAX_COLS / 32) * (int)sizeof(float);
        hipError_t err = hipSuccess;
        for (const void *kernel : {reinterpret_cast<const void *>(mx_quantize_row_kernel<float, QUEST_MX_E2M1>),
                                   reinterpret_cast<const void *>(mx_quantize_row_kernel<float, QUEST_MX_E4M3>),
                                   reinterpret_cast<const void *>(mx_quantize_row_kernel<uint16_t, QUEST_MX_E2M1>),
                                   reinterpret_cast<const void *>(mx_quantize_row_kernel<uint16_t, QUEST_MX_E4M3>)})
            if (err == hipSuccess)
                err = allow_dynamic_lds(kernel, kBytes);
        return err;
    });
}

hipError_t launch_mx_quantize(const MxQuantizeArgs &a, hipStream_t stream)
{
    if (a.rows == 0)
        return hipSuccess;
    if (a.dtype == QUEST_F32)
        return a.format == QUEST_MX_E4M3 ? launch<float, QUEST_MX_E4M3>(a, stream) : launch<float, QUEST_MX_E2M1>(a, stream);
    return a.format == QUEST_MX_E4M3 ? launch<uint16_t, QUEST_MX_E4M3>(a, stream) : launch<uint16_t, QUEST_MX_E2M1>(a, stream);
}

hipError_t launch_mx_dequantize(const MxDequantizeArgs &a, hipStream_t stream)
{
    if (a.rows == 0)
        return hipSuccess;
    if (a.out_dtype == QUEST_F32)
        return a.format == QUEST_MX_E4M3 ? launch_back<QUEST_MX_E4M3, float>(a, stream) : launch_back<QUEST_MX_E2M1, float>(a, stream);
    return a.format == QUEST_MX_E4M3 ? launch_back<QUEST_MX_E4M3, uint16_t>(a, stream)
                                     : launch_back<QUEST_MX_E2M1, uint16_t>(a, stream);
}

}  // namespace quest
