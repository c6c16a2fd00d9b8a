// Root-mean-square norm with the residual's addition in front and the microscaled quantizer behind, and its backward pass.
// Both read and write each matrix once: a workgroup holds a row in registers between its reduction and its use.
#include <algorithm>

#include "mx_formats.h"
#include "quest_internal.h"

namespace quest {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kRowThreads = 1024;   // most for a row's workgroup of the forward pass

template <bool AGAIN>
__device__ __forceinline__ float block_sum(float v, float *park, int waves)
{
    v = wave_sum_dpp(v);
    if constexpr (AGAIN)
        __syncthreads();   // the numbers of the row before have been read
    if ((threadIdx.x & 63) == 0)
        park[threadIdx.x >> 6] = v;
    __syncthreads();
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < waves; ++w)
        sum += park[w];
    return sum;
}

/*
 * 1 / sqrt(sum * share + eps), rounded once: a row's every element carries its error.  (16384 x 2048 against 64 bits, means of six
 * seeds: error of rstd in norm 4.8e-8 with four roundings in fp32, 3.5e-8 so; of 2^25 E4M3 codes behind blocks of 32, 133 and 127
 * are not those of 64 bits, which the two products and the transform in fp32 make, and 1.5e-4 and 0.8e-4 in norm.)  In 64 bits, from
 * the hardware's reciprocal root, good to some 24 bits, by one Newton step, which squares the error.  Nothing for 0, NaN for a sum
 * that fp32 does not hold.
 */
__device__ __forceinline__ float reciprocal_root(float sum, double share, float eps)
{
    const double m = __fma_rn((double)sum, share, (double)eps);
    if (m == 0.0)
        return 0.0f;
    if (!(sum < INFINITY))
        return NAN;
    const double r = __builtin_amdgcn_rsq(m);
    return (float)__fma_rn(0.5 * r, __fma_rn(-m * r, r, 1.0), r);
}

// eight elements rounded to the type (bf16: by the hardware's conversion)
__device__ __forceinline__ void store8_packed(float *p, const float (&v)[8]) { store8(p, v); }
__device__ __forceinline__ void store8_packed(uint16_t *p, const float (&v)[8])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// rounded to the type and back
__device__ __forceinline__ float rounded(float v, const float *) { return v; }
__device__ __forceinline__ float rounded(float v, const uint16_t *) { return bf16_bits_to_float(float_to_bf16_bits(v)); }

/*
 * Forward pass.  Bound by memory: x and residual are read, h, codes and scales written (16384 x 2048 in bf16, E4M3, 236 MB, 46 us at
 * the rate of a large copy; it takes 47).  A row has a workgroup of its own, with as many waves as it needs: thread t of n holds
 * the elements 8 (t + n i) .. + 8, i < CH, so that a wave's lanes hold 512 consecutive ones.  Two chunks to a lane where a row has
 * more than 512 elements.  (us for 2^25 elements in bf16 with four waves for each row / one chunk / two: rows of 512 109 / 49 / 50,
 * 640 97 / 65 / 58, 1024 65 / 49 / 47, 2048 47 / 48 / 48, 4608 61 / 55 / 52, 11008 71 / - / 56)
 */
template <typename T, typename W, int CH, int FORMAT>
__global__ __launch_bounds__(kRowThreads) void rms_norm_kernel(const T *__restrict__ x, int64_t ld_x, const T *__restrict__ residual,
                                                            int64_t ld_residual, const W *__restrict__ weight, int cols, float eps,
                                                            T *__restrict__ h_out, T *__restrict__ y_out, int log2n, float norm,
                                                            uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                            uint8_t *__restrict__ mask, float *__restrict__ rstd_out)
{
    __shared__ float park[kRowThreads / kWave];
    const int threads = blockDim.x;
    const int64_t row = blockIdx.x, first = row * cols;
    const int lane = threadIdx.x & 63;
    float v[CH][8], w[CH][8], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = (i * threads + threadIdx.x) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[i][e] = 0.0f;
        if (c >= cols)
            continue;
        load8(x + row * ld_x + c, v[i]);
        load8(weight + c, w[i]);   // here, so that the sum does not stand between the call's two trips to memory
        if (residual) {
            float r[8];
            load8(residual + row * ld_residual + c, r);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[i][e] = rounded(v[i][e] + r[e], x);
            store8_packed(h_out + first + c, v[i]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum = __fmaf_rn(v[i][e], v[i][e], sum);
    }
    const float rstd = reciprocal_root(block_sum<false>(sum, park, threads / kWave), 1.0 / cols, eps);
    if (rstd_out && threadIdx.x == 0)
        rstd_out[row] = rstd;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = (i * threads + threadIdx.x) * 8;
        if (c < cols) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[i][e] = __fmul_rn(__fmul_rn(v[i][e], rstd), w[i][e]);
            if (y_out)
                store8_packed(y_out + first + c, v[i]);
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

/*
 * Backward pass.  Bound by memory: h, dy and dh are read and dx is written once (16384 x 2048 in bf16 268 MB, 52 us at the 5.1 TB/s
 * of a large copy).  A row belongs to GROUP waves, CH chunks of eight elements to a lane; a group takes every (number of
 * groups)-th row, with the next row's loads in flight while it works on one, and keeps its share of dweight in registers.  One wave
 * to a row up to 2048 elements: no barrier then ties waves together.  The groups of a workgroup add up their shares
 * in LDS; the workgroups' go to the workspace, where rms_norm_dweight_kernel adds them in a fixed order.
 * (us, with a workgroup to a row, one row at a time and dweight's sum in a workgroup per 256 columns / so: 16384 x 2048 in bf16
 * 185 / 55; 777 x 640 in fp32 116 / 14, of which the call itself is most)
 */
template <typename T, int CH>
struct RowLoads {   // as they come from memory
    static constexpr int kQuads = CH * 8 * (int)sizeof(T) / 16;
    uint4 h[kQuads], dy[kQuads], dh[kQuads];
    float rstd;
};

__device__ __forceinline__ void widened(const uint4 *raw, float (&v)[8], const float *)
{
    const float4 a = __builtin_bit_cast(float4, raw[0]), b = __builtin_bit_cast(float4, raw[1]);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void widened(const uint4 *raw, float (&v)[8], const uint16_t *)
{
    const uint4 w = raw[0];
    v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
    v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
    v[4] = __uint_as_float(w.z << 16); v[5] = __uint_as_float(w.z & 0xffff0000u);
    v[6] = __uint_as_float(w.w << 16); v[7] = __uint_as_float(w.w & 0xffff0000u);
}

// threads of a workgroup: four rows of a wave each, or one row of GROUP waves
constexpr int backward_threads(int group)
{
    return group == 1 ? kThreads : kWave * group;
}

template <typename T, typename W, int GROUP, int CH, bool ALONG>
__global__ __launch_bounds__(backward_threads(GROUP)) void rms_norm_backward_kernel(const T *__restrict__ dy, const T *__restrict__ h,
                                                                     const W *__restrict__ weight, const float *__restrict__ rstd_in,
                                                                     const T *__restrict__ dh, int64_t rows, int cols,
                                                                     T *__restrict__ dx, float *__restrict__ partial)
{
    constexpr int kBlock = backward_threads(GROUP), kGroupThreads = kWave * GROUP, kGroups = kBlock / kGroupThreads;
    constexpr bool kAhead = CH * sizeof(T) <= 8;      // (else the next row's loads would not fit the registers)
    constexpr int kQuads = 8 * (int)sizeof(T) / 16;   // of a chunk
    extern __shared__ __attribute__((aligned(16))) float shares[];   // [groups][cols], where dweight is wanted
    __shared__ float park[GROUP];
    const int group = threadIdx.x / kGroupThreads, t = threadIdx.x % kGroupThreads;
    float dw[CH][8] = {}, w[CH][8];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = (i * kGroupThreads + t) * 8;
        if (c < cols)
            load8(weight + c, w[i]);
    }
    typedef RowLoads<T, CH> Loads;
    auto fetch = [&](Loads &l, int64_t row) {
        const int64_t first = row * cols;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = (i * kGroupThreads + t) * 8;
            if (c >= cols)
                continue;
#pragma unroll
            for (int k = 0; k < kQuads; ++k) {
                l.h[i * kQuads + k] = reinterpret_cast<const uint4 *>(h + first + c)[k];
                l.dy[i * kQuads + k] = reinterpret_cast<const uint4 *>(dy + first + c)[k];
                if constexpr (ALONG)
                    l.dh[i * kQuads + k] = reinterpret_cast<const uint4 *>(dh + first + c)[k];
            }
        }
        l.rstd = rstd_in[row];
    };
    // (the same number of rounds for every group of a workgroup: they meet at barriers)
    const int64_t stride = (int64_t)gridDim.x * kGroups;
    int64_t row = (int64_t)blockIdx.x * kGroups + group;
    Loads next;
    if (kAhead && row < rows)
        fetch(next, row);
    for (int64_t round = (int64_t)blockIdx.x * kGroups; round < rows; round += stride, row += stride) {
        const bool mine = row < rows;
        if (!kAhead && mine)
            fetch(next, row);
        const Loads now = next;
        if (kAhead && row + stride < rows)
            fetch(next, row + stride);
        float xhat[CH][8], g[CH][8], sum = 0.0f;
        if (mine) {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                if ((i * kGroupThreads + t) * 8 >= cols)
                    continue;
                widened(now.h + i * kQuads, xhat[i], h);
                widened(now.dy + i * kQuads, g[i], h);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    xhat[i][e] *= now.rstd;
                    dw[i][e] = __fmaf_rn(g[i][e], xhat[i][e], dw[i][e]);
                    g[i][e] *= w[i][e];
                    sum = __fmaf_rn(g[i][e], xhat[i][e], sum);
                }
            }
        }
        const float mean = (GROUP == 1 ? wave_sum_dpp(sum) : block_sum<true>(sum, park, GROUP)) / (float)cols;
        if (mine) {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int c = (i * kGroupThreads + t) * 8;
                if (c >= cols)
                    continue;
                float r[8] = {};
                if constexpr (ALONG)
                    widened(now.dh + i * kQuads, r, h);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    r[e] = __fmaf_rn(now.rstd, __fmaf_rn(-xhat[i][e], mean, g[i][e]), r[e]);
                store8_packed(dx + row * cols + c, r);
            }
        }
    }
    if (!partial)
        return;
    float *const mine = partial + (int64_t)blockIdx.x * cols;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = (i * kGroupThreads + t) * 8;
        if (c < cols)
            store8(kGroups == 1 ? mine + c : shares + group * cols + c, dw[i]);
    }
    if constexpr (kGroups > 1) {
        __syncthreads();
        for (int c = threadIdx.x * 4; c < cols; c += kBlock * 4) {
            float4 sum = *reinterpret_cast<const float4 *>(shares + c);
#pragma unroll
            for (int o = 1; o < kGroups; ++o) {
                const float4 v = *reinterpret_cast<const float4 *>(shares + o * cols + c);
                sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
            }
            *reinterpret_cast<float4 *>(mine + c) = sum;
        }
    }
}

// dweight[j] = the sum of `parts` partial rows, in a fixed order: 16 columns to a workgroup, so that many take part; 64 threads share
// a column's rows and meet by lane exchanges and in LDS.  (us with 64 columns / so: 195 rows of 640 3.8 / 3.1, 512 of 2048 4.7 / 4.7)
constexpr int kSumWaves = 16, kSumCols = 16;
__global__ __launch_bounds__(kWave *kSumWaves) void rms_norm_dweight_kernel(const float *__restrict__ partial, int parts, int cols,
                                                                            float *__restrict__ dweight)
{
    __shared__ float sums[kSumWaves][kSumCols];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * kSumCols + lane % kSumCols;
    auto over_lanes = [](float v) {   // of one column
        v += __shfl_xor(v, 16, kWave);
        return v + __shfl_xor(v, 32, kWave);
    };
    float sum = 0.0f;
#pragma unroll 8
    for (int p = threadIdx.x / kSumCols; p < parts; p += kWave * kSumWaves / kSumCols)
        sum += partial[(int64_t)p * cols + c];
    sum = over_lanes(sum);
    if (lane < kSumCols)
        sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0)
        return;
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kSumWaves; w += 4)
        sum += sums[w + lane / kSumCols][lane % kSumCols];
    sum = over_lanes(sum);
    if (lane < kSumCols)
        dweight[c] = sum;
}

constexpr int64_t kOneWave = 2048;   // row length up to which a wave has a row to itself in the backward pass

int groups_of(int64_t cols)
{
    return cols <= kOneWave ? kWaves : 1;
}

// Workgroups of the backward pass, each with a partial row of dweight: two for each compute unit, one where a workgroup has a row at
// a time, whose partial rows cost more than the second one hides (us with 512 / 256: 573 x 5632 17.9 / 15.6, 16384 x 4096 107 / 98.5,
// 8192 x 8192 113 / 105; rows of a wave: 4096 x 2048 19.1 / 20.0).
int parts_of(int64_t rows, int64_t cols)
{
    return (int)std::min<int64_t>((rows + groups_of(cols) - 1) / groups_of(cols), groups_of(cols) == 1 ? 256 : 512);
}

template <typename T, typename W>
hipError_t launch_forward(const RmsNormArgs &a, hipStream_t stream)
{
    auto launch = [&](auto ch) {
        constexpr int CH = decltype(ch)::value;
        auto kernel = a.format == QUEST_MX_E4M3 ? rms_norm_kernel<T, W, CH, QUEST_MX_E4M3> : rms_norm_kernel<T, W, CH, QUEST_MX_E2M1>;
        const unsigned threads = (unsigned)((a.cols + 8 * CH * kWave - 1) / (8 * CH * kWave) * kWave);
        hipLaunchKernelGGL(kernel, dim3((unsigned)a.rows), dim3(threads), 0, stream, static_cast<const T *>(a.x), a.ld_x,
                           static_cast<const T *>(a.residual), a.ld_residual, static_cast<const W *>(a.weight), (int)a.cols, a.eps,
                           static_cast<T *>(a.h_out), static_cast<T *>(a.y_out), a.log2n,
                           (float)(1.0 / sqrt((double)(int64_t(1) << a.log2n))), a.codes, a.scales, a.mask, a.rstd);
    };
    if (a.cols <= 8 * kWave)
        launch(std::integral_constant<int, 1>());
    else
        launch(std::integral_constant<int, 2>());
    return hipGetLastError();
}

template <typename T, typename W>
hipError_t launch_backward(const RmsNormBackwardArgs &a, hipStream_t stream)
{
    const int parts = parts_of(a.rows, a.cols), groups = groups_of(a.cols);
    float *partial = a.dweight ? static_cast<float *>(a.workspace) : nullptr;
    hipError_t err = hipSuccess;
    if (a.rows > 0) {
        auto launch = [&](auto group, auto ch) {
            constexpr int G = decltype(group)::value, CH = decltype(ch)::value;
            auto kernel = a.dh ? rms_norm_backward_kernel<T, W, G, CH, true> : rms_norm_backward_kernel<T, W, G, CH, false>;
            hipLaunchKernelGGL(kernel, dim3((unsigned)parts), dim3(backward_threads(G)), groups > 1 ? groups * a.cols * sizeof(float) : 0, stream,
                               static_cast<const T *>(a.dy), static_cast<const T *>(a.h), static_cast<const W *>(a.weight), a.rstd,
                               static_cast<const T *>(a.dh), a.rows, (int)a.cols, static_cast<T *>(a.dx), partial);
        };
        typedef std::integral_constant<int, 1> One;
        if (a.cols <= 512)
            launch(One(), One());
        else if (a.cols <= 1024)
            launch(One(), std::integral_constant<int, 2>());
        else if (a.cols <= kOneWave)
            launch(One(), std::integral_constant<int, 4>());
        else if (a.cols <= 4096)
            launch(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
        else if (a.cols <= 8192)
            launch(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
        else
            launch(std::integral_constant<int, 8>(), std::integral_constant<int, 4>());
        err = hipGetLastError();
    }
    if (err == hipSuccess && a.dweight) {
        hipLaunchKernelGGL(rms_norm_dweight_kernel, dim3((unsigned)(a.cols / kSumCols)), dim3(kWave * kSumWaves), 0, stream,
                           partial, parts, (int)a.cols, a.dweight);
        err = hipGetLastError();
    }
    return err;
}

}  // namespace

int64_t rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols)
{
    return (int64_t)parts_of(rows, cols) * cols * (int64_t)sizeof(float);
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
