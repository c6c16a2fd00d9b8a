// Root-mean-square norm with the residual's addition in front and the microscaled quantizer behind, and its backward pass.
// Both read and write each matrix once: a workgroup holds a row in registers between its reduction and its use.
#include <algorithm>

#include "mx_formats.h"
#include "quest_internal.h"

namespace quest {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

__device__ __forceinline__ float block_sum(float v, float *park)
{
    v = wave_sum_dpp(v);
    __syncthreads();   // the numbers of the row before have been read
    if ((threadIdx.x & 63) == 0)
        park[threadIdx.x >> 6] = v;
    __syncthreads();
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        sum += park[w];
    return sum;
}

// rounded to the type and back
__device__ __forceinline__ float rounded(float v, const float *) { return v; }
__device__ __forceinline__ float rounded(float v, const uint16_t *) { return bf16_bits_to_float(float_to_bf16_bits(v)); }

// Thread t holds the elements 8 t + 2048 i .. + 8, i < CH: a wave's lanes hold 512 consecutive ones.
template <typename T, typename W, int CH, int FORMAT>
__global__ __launch_bounds__(kThreads) void rms_norm_kernel(const T *__restrict__ x, int64_t ld_x, const T *__restrict__ residual,
                                                            int64_t ld_residual, const W *__restrict__ weight, int cols, float eps,
                                                            T *__restrict__ h_out, T *__restrict__ y_out, int log2n, float norm,
                                                            uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                            uint8_t *__restrict__ mask, float *__restrict__ rstd_out)
{
    __shared__ float park[kWaves];
    const int64_t row = blockIdx.x, first = row * cols;
    const int lane = threadIdx.x & 63;
    float v[CH][8], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = (i * kThreads + threadIdx.x) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[i][e] = 0.0f;
        if (c >= cols)
            continue;
        load8(x + row * ld_x + c, v[i]);
        if (residual) {
            float r[8];
            load8(residual + row * ld_residual + c, r);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[i][e] = rounded(v[i][e] + r[e], x);
            store8(h_out + first + c, v[i]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum = __fmaf_rn(v[i][e], v[i][e], sum);
    }
    const float mean = block_sum(sum, park) / (float)cols + eps;
    const float rstd = mean == 0.0f ? 0.0f : mean < INFINITY ? 1.0f / sqrtf(mean) : NAN;
    if (rstd_out && threadIdx.x == 0)
        rstd_out[row] = rstd;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = (i * kThreads + threadIdx.x) * 8;
        if (c < cols) {
            float w[8];
            load8(weight + c, w);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[i][e] = __fmul_rn(__fmul_rn(v[i][e], rstd), w[e]);
            if (y_out)
                store8(y_out + first + c, v[i]);
        }
        if (codes) {
            wave_hadamard(v[i], log2n, norm, lane);
            const MxEncoded<FORMAT> q = mx_encode<FORMAT>(v[i]);
            if (c < cols) {
                const int64_t at = first + c;
                if constexpr (MxFormat<FORMAT>::kE4M3)
                    *reinterpret_cast<uint2 *>(codes + at) = make_uint2(q.words[0], q.words[1]);
                else
                    *reinterpret_cast<uint32_t *>(codes + at / 2) = q.words[0];
                if ((lane & 3) == 0)
                    scales[at / kMxGroup] = (uint8_t)q.scale;
                if (mask)
                    mask[at / 8] = (uint8_t)q.trust;
            }
        }
    }
}

// A workgroup takes the rows blockIdx.x, + gridDim.x, ..; its share of dweight stays in registers until it is done.
template <typename T, typename W, int CH>
__global__ __launch_bounds__(kThreads) void rms_norm_backward_kernel(const T *__restrict__ dy, const T *__restrict__ h,
                                                                     const W *__restrict__ weight, const float *__restrict__ rstd_in,
                                                                     const T *__restrict__ dh, int64_t rows, int cols,
                                                                     T *__restrict__ dx, float *__restrict__ partial)
{
    __shared__ float park[kWaves];
    float dw[CH][8] = {};
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int64_t first = row * cols;
        const float rstd = rstd_in[row];
        float xhat[CH][8], t[CH][8], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = (i * kThreads + threadIdx.x) * 8;
            if (c >= cols)
                continue;
            float g[8], w[8];
            load8(h + first + c, xhat[i]);
            load8(dy + first + c, g);
            load8(weight + c, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xhat[i][e] *= rstd;
                dw[i][e] = __fmaf_rn(g[e], xhat[i][e], dw[i][e]);
                t[i][e] = g[e] * w[e];
                sum = __fmaf_rn(t[i][e], xhat[i][e], sum);
            }
        }
        const float mean = block_sum(sum, park) / (float)cols;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = (i * kThreads + threadIdx.x) * 8;
            if (c >= cols)
                continue;
            float r[8];
            if (dh) {
                load8(dh + first + c, r);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    r[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                r[e] = __fmaf_rn(rstd, __fmaf_rn(-xhat[i][e], mean, t[i][e]), r[e]);
            store8(dx + first + c, r);
        }
    }
    if (!partial)
        return;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = (i * kThreads + threadIdx.x) * 8;
        if (c < cols)
            store8(partial + (int64_t)blockIdx.x * cols + c, dw[i]);
    }
}

// dweight[j] = the sum of `parts` partial rows, in their order
__global__ __launch_bounds__(kThreads) void rms_norm_dweight_kernel(const float *__restrict__ partial, int parts, int cols,
                                                                    float *__restrict__ dweight)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= cols)
        return;
    float sum = 0.0f;
    for (int p = 0; p < parts; ++p)
        sum += partial[(int64_t)p * cols + c];
    dweight[c] = sum;
}

int parts_of(int64_t rows)
{
    return (int)std::min<int64_t>(rows, 512);
}

// f(std::integral_constant<int, CH>) for the number of chunks of 2048 elements that a row has
template <typename F>
void with_chunks(int64_t cols, F &&f)
{
    if (cols <= 2048)
        f(std::integral_constant<int, 1>());
    else if (cols <= 4096)
        f(std::integral_constant<int, 2>());
    else if (cols <= 8192)
        f(std::integral_constant<int, 4>());
    else
        f(std::integral_constant<int, 8>());
}

template <typename T, typename W>
hipError_t launch_forward(const RmsNormArgs &a, hipStream_t stream)
{
    with_chunks(a.cols, [&](auto ch) {
        auto kernel = a.format == QUEST_MX_E4M3 ? rms_norm_kernel<T, W, decltype(ch)::value, QUEST_MX_E4M3>
                                                : rms_norm_kernel<T, W, decltype(ch)::value, QUEST_MX_E2M1>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.rows), dim3(kThreads), 0, stream, static_cast<const T *>(a.x), a.ld_x,
                           static_cast<const T *>(a.residual), a.ld_residual, static_cast<const W *>(a.weight), (int)a.cols, a.eps,
                           static_cast<T *>(a.h_out), static_cast<T *>(a.y_out), a.log2n,
                           (float)(1.0 / sqrt((double)(int64_t(1) << a.log2n))), a.codes, a.scales, a.mask, a.rstd);
    });
    return hipGetLastError();
}

template <typename T, typename W>
hipError_t launch_backward(const RmsNormBackwardArgs &a, hipStream_t stream)
{
    const int parts = parts_of(a.rows);
    float *partial = a.dweight ? static_cast<float *>(a.workspace) : nullptr;
    hipError_t err = hipSuccess;
    if (a.rows > 0) {
        // (without dweight nothing ties rows to a workgroup)
        const unsigned blocks = partial ? (unsigned)parts : (unsigned)std::min<int64_t>(a.rows, 1 << 20);
        with_chunks(a.cols, [&](auto ch) {
            hipLaunchKernelGGL((rms_norm_backward_kernel<T, W, decltype(ch)::value>), dim3(blocks), dim3(kThreads), 0, stream,
                               static_cast<const T *>(a.dy), static_cast<const T *>(a.h), static_cast<const W *>(a.weight), a.rstd,
                               static_cast<const T *>(a.dh), a.rows, (int)a.cols, static_cast<T *>(a.dx), partial);
        });
        err = hipGetLastError();
    }
    if (err == hipSuccess && a.dweight) {
        hipLaunchKernelGGL(rms_norm_dweight_kernel, dim3((unsigned)((a.cols + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream,
                           partial, parts, (int)a.cols, a.dweight);
        err = hipGetLastError();
    }
    return err;
}

}  // namespace

int64_t rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols)
{
    return (int64_t)parts_of(rows) * cols * (int64_t)sizeof(float);
}

// Makes the runtime load this file's code object
hipError_t prepare_rms_norm_kernels()
{
    hipFuncAttributes attr;
    return hipFuncGetAttributes(&attr, reinterpret_cast<const void *>(rms_norm_dweight_kernel));
}

hipError_t launch_rms_norm(const RmsNormArgs &a, hipStream_t stream)
{
    if (a.rows == 0)
        return hipSuccess;
    if (a.dtype == QUEST_F32)
        return a.weight_dtype == QUEST_F32 ? launch_forward<float, float>(a, stream) : launch_forward<float, uint16_t>(a, stream);
    return a.weight_dtype == QUEST_F32 ? launch_forward<uint16_t, float>(a, stream) : launch_forward<uint16_t, uint16_t>(a, stream);
}

hipError_t launch_rms_norm_backward(const RmsNormBackwardArgs &a, hipStream_t stream)
{
    if (a.dtype == QUEST_F32)
        return a.weight_dtype == QUEST_F32 ? launch_backward<float, float>(a, stream) : launch_backward<float, uint16_t>(a, stream);
    return a.weight_dtype == QUEST_F32 ? launch_backward<uint16_t, float>(a, stream) : launch_backward<uint16_t, uint16_t>(a, stream);
}

}  // namespace quest
