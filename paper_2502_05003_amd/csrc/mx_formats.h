// Microscaled operands on the device: groups of 32 elements with a power-of-two scale, to and from E2M1 and E4M3 codes.
//
// A lane holds eight consecutive elements, four neighbouring lanes a group.
#pragma once

#include "../../include/quest.h"
#include "gemm_tile.h"

namespace quest {

constexpr int kMxGroup = 32;

template <int FORMAT>
struct MxFormat {
    static constexpr bool kE4M3 = FORMAT == QUEST_MX_E4M3;
    static constexpr int kBits = kE4M3 ? 8 : 4;
    static constexpr int kMaxExponent = kE4M3 ? 8 : 2;          // exponent of the largest element
    static constexpr float kLargest = kE4M3 ? 448.0f : 6.0f;
    static constexpr float kTrusted = kE4M3 ? 464.0f : 7.0f;    // and half the interval below it
    static constexpr int kWords = kBits / 4;                    // dwords of eight codes
};

// the value of a lane `CTRL` away in the data-parallel-primitive pattern (all lanes of a row of sixteen active or not together)
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_moved(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xF, 0xF, false);
}
template <int CTRL>
__device__ __forceinline__ float dpp_moved(float v)
{
    return __uint_as_float(dpp_moved<CTRL>(__float_as_uint(v)));
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E;   // quad_perm [1, 0, 3, 2] and [2, 3, 0, 1]

// the value of the lane whose number differs in bit BIT: within rows of sixteen by lane patterns, beyond through the crossbar
template <int BIT>
__device__ __forceinline__ float lane_xor(float v)
{
    if constexpr (BIT == 1)
        return dpp_moved<kDppXor1>(v);
    else if constexpr (BIT == 2)
        return dpp_moved<kDppXor2>(v);
    else if constexpr (BIT == 4)
        return dpp_moved<0x141>(dpp_moved<0x1B>(v));   // quad_perm [3, 2, 1, 0], then row_half_mirror
    else if constexpr (BIT == 8)
        return dpp_moved<0x128>(v);                     // row_ror:8
    else
        return __shfl_xor(v, BIT, kWave);
}

// The transform's strides that lie across lanes: N values to a lane, log2n of the block, FIRST = log2 N.  (An exact product:
// a + b in the lower lane, a - b in the upper one.)
template <int N, int FIRST>
__device__ __forceinline__ void lane_butterflies(float (&v)[N], int log2n, int lane)
{
    static_for<6>([&](auto s) {
        constexpr int bit = 1 << decltype(s)::value;
        if (log2n > FIRST + decltype(s)::value) {
            const float sign = (lane & bit) ? -1.0f : 1.0f;
#pragma unroll
            for (int e = 0; e < N; ++e)
                v[e] = __fmaf_rn(v[e], sign, lane_xor<bit>(v[e]));
        }
    });
}

// Block Hadamard transform of consecutive elements, eight to a lane, over 2^log2n elements (<= 512: 64 lanes), strides 1, 2, ..;
// then the factor 2^(-log2n / 2).  (Strides in this order everywhere: the sums round the same whatever kernel a call takes.)
__device__ __forceinline__ void wave_hadamard(float (&v)[8], int log2n, float norm, int lane)
{
    if (log2n == 0)
        return;
    butterflies8(v, log2n);
    lane_butterflies<8, 3>(v, log2n, lane);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] *= norm;
}

// Eight elements in units of their scale to codes: nearest, ties to the even code, clipped at the largest element
template <int FORMAT>
__device__ __forceinline__ void mx_convert(float (&t)[8], uint32_t (&words)[MxFormat<FORMAT>::kWords])
{
    typedef MxFormat<FORMAT> F;
    if constexpr (F::kE4M3) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            t[e] = __builtin_amdgcn_fmed3f(t[e], -F::kLargest, F::kLargest);   // (the conversion makes NaN of what lies beyond)
        words[0] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
        words[0] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], (int)words[0], true);
        words[1] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], 0, false);
        words[1] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], (int)words[1], true);
    } else {
        uint32_t w = 0;   // (the conversion clips)
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[0], t[1], 1.0f, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[2], t[3], 1.0f, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[4], t[5], 1.0f, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, t[6], t[7], 1.0f, 3);
        words[0] = w;
    }
}

// Eight elements of a group of 32 (the other 24 in the three neighbouring lanes) to codes, scale byte and trust bits
template <int FORMAT>
struct MxEncoded {
    uint32_t words[MxFormat<FORMAT>::kWords];
    uint32_t scale, trust;
};

template <int FORMAT>
__device__ __forceinline__ MxEncoded<FORMAT> mx_encode(const float (&v)[8])
{
    typedef MxFormat<FORMAT> F;
    MxEncoded<FORMAT> out;
    // largest magnitude as bits: integers order finite values, infinity and NaN
    uint32_t largest = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        largest = max(largest, __float_as_uint(v[e]) & 0x7fffffffu);
    largest = max(largest, dpp_moved<kDppXor1>(largest));
    largest = max(largest, dpp_moved<kDppXor2>(largest));
    const int field = (int)(largest >> 23);            // biased exponent; subnormal largest values: 0
    const bool finite = field != 255;
    out.scale = finite ? (uint32_t)max(field - F::kMaxExponent, 0) : 255u;
    const float inverse = __uint_as_float(finite ? (254u - out.scale) << 23 : 0u);   // 2^-e, e = scale - 127: a normal number
    float t[8];
    out.trust = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        t[e] = finite ? __fmul_rn(v[e], inverse) : 0.0f;
        out.trust |= (finite && fabsf(t[e]) <= F::kTrusted ? 1u : 0u) << e;
    }
    mx_convert<FORMAT>(t, out.words);
    return out;
}

// Eight codes of one group as fp32 values
template <int FORMAT>
__device__ __forceinline__ void mx_decode(const uint32_t (&words)[MxFormat<FORMAT>::kWords], uint32_t scale, float (&v)[8])
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    // 2^(scale - 127) in two factors: the smallest is no normal number (elements have few bits: only a subnormal result rounds)
    const float first = __uint_as_float(scale == 255 ? 0x7fc00000u : max(scale, 1u) << 23), second = scale == 0 ? 0.5f : 1.0f;
    static_for<4>([&](auto pair) {
        constexpr int p = decltype(pair)::value;
        v2f u;
        if constexpr (MxFormat<FORMAT>::kE4M3)
            u = __builtin_amdgcn_cvt_pk_f32_fp8((int)words[p / 2], p % 2 != 0);
        else
            u = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(words[0], 1.0f, p);
        v[2 * p] = __fmul_rn(__fmul_rn(u[0], second), first);
        v[2 * p + 1] = __fmul_rn(__fmul_rn(u[1], second), first);
    });
}

}  // namespace quest
