// The quantizer for microscaled operands (block Hadamard transform, a power-of-two scale for each 32 elements, E2M1 or E4M3
// codes, trust mask) and the way back to what the codes stand for.  Both are passes over memory.
#include <algorithm>

#include "mx_formats.h"
#include "quest_internal.h"

namespace quest {
namespace {

constexpr int kThreads = 256;
constexpr int kUnit = 512;   // elements of a wave: eight to a lane

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

// Blocks of up to 512 elements: a wave takes 512 consecutive elements, of one row or several (blocks divide rows, so units that
// start at multiples of 512 cut none), and nothing leaves its registers in between.
template <typename T, int FORMAT>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const T *__restrict__ x, int64_t elements, int cols, int64_t ld,
                                                               int log2n, float norm, uint8_t *__restrict__ codes,
                                                               uint8_t *__restrict__ scales, uint8_t *__restrict__ mask)
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

// Larger blocks: a workgroup holds a row in LDS for the transform's wider strides.
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
    if ((1 << a.log2n) <= kUnit) {
        hipLaunchKernelGGL((mx_quantize_kernel<T, FORMAT>), dim3(blocks_for(a.rows * a.cols)), dim3(kThreads), 0, stream, x,
                           a.rows * a.cols, (int)a.cols, a.ld, a.log2n, norm, a.codes, a.scales, a.mask);
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
