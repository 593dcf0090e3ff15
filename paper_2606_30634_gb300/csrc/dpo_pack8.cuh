// dpo_pack8.cuh -- activations in 8 bits: E4M3 codes, a power-of-two scale for
// each group of 32 elements along a row (include/dpo.h). The scale is formed
// from the bits of the group's largest magnitude and multiplying by it or its
// inverse is exact, so a code depends on its group's values alone and not on
// the kernel that formed it, and decoding rounds nothing.
#pragma once

#include "dpo_device.cuh"

#include <cuda_fp16.h>
#include <cuda_fp8.h>

namespace dpo {
namespace {

constexpr int kGroup = 32;
constexpr int64_t groups_of(int64_t cols) { return (cols + kGroup - 1) / kGroup; }

// Scale byte s of a group with this largest finite magnitude: the smallest with
// amax <= 448 * 2^(s - 127), at least 1. With amax = f 2^(E - 127), 448 =
// 1.75 * 2^8: E - 8, one more when f > 1.75.
__device__ __forceinline__ uint32_t scale_byte(float amax)
{
    const uint32_t b = __float_as_uint(amax);
    const int s = (int)(b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(s, 1);
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float inv_scale_of(uint32_t byte)
{
    return __uint_as_float((254u - byte) << 23);
}

// Magnitude that counts for the scale: 0 for infinities and NaN.
constexpr float kMaxFinite = 3.402823466e38f;
__device__ __forceinline__ float finite_abs(float v)
{
    const float a = fabsf(v);
    return a <= kMaxFinite ? a : 0.0f;
}

// What is encoded: an infinity, which E4M3 has no code for, as NaN.
__device__ __forceinline__ float inf_to_nan(float v)
{
    return fabsf(v) == __int_as_float(0x7f800000) ? __int_as_float(0x7fc00000) : v;
}

// Two codes, lo in the low byte.
__device__ __forceinline__ uint32_t encode2(float lo, float hi)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d)
{
    return encode2(a, b) | encode2(c, d) << 16;
}

__device__ __forceinline__ float2 decode2(uint32_t codes)
{
    const __half2_raw h =
        __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes & 0xFFFFu), __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

}  // namespace
}  // namespace dpo
