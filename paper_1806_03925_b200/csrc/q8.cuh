// The 8-bit form of values (gear.h): e4m3 with one fp32 scale for every block of GEAR_Q8_BLOCK columns.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace gear {

constexpr int Q8_BLOCK = GEAR_Q8_BLOCK;

// A block's largest magnitude as the bits of a non-negative float: in that form a NaN is larger than an infinity and every number
// in order, so that an integer maximum passes it on.
__device__ __forceinline__ uint32_t q8_magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// scale = max(largest, 2^-100) / 448 (a NaN stays one); `inv` is what values are multiplied by: one rounding more than a division by
// the scale, which moves only values within 2^-23 of the middle between two e4m3 values.
__device__ __forceinline__ float q8_scale(uint32_t largest, float& inv) {
    float m = __uint_as_float(largest);
    if (m < 0x1p-100f) m = 0x1p-100f;
    const float s = m / 448.0f;
    inv = 1.0f / s;
    return s;
}
__device__ __forceinline__ uint16_t q8_pair(float lo, float hi) { return (uint16_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ uint8_t q8_one(float v) { return (uint8_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }

}  // namespace gear
