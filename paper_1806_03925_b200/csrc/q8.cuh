// The 8-bit form of values (gear.h): e4m3 with one fp32 scale for every block of GEAR_Q8_BLOCK columns.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace gear {

constexpr int Q8_BLOCK = GEAR_Q8_BLOCK;

// Two fp32 values in one 64-bit register, and arithmetic on both at once (each half rounded as its fp32 instruction rounds): half as
// many instructions to issue, which is what bounds the row kernels next to memory.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float lo, float hi) { return (f32x2)__float_as_uint(lo) | (f32x2)__float_as_uint(hi) << 32; }
__device__ __forceinline__ f32x2 both(float v) { return pack2(v, v); }
__device__ __forceinline__ float low(f32x2 v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float high(f32x2 v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) { f32x2 d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ f32x2 from_bf16x2(uint32_t w) { return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t to_bf16x2(f32x2 v) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(low(v), high(v));
    return *reinterpret_cast<const uint32_t*>(&h);
}

// The largest of a magnitude and two more, a NaN if there is one.  Between lanes the largest goes as the bits of a non-negative float,
// where a NaN is larger than an infinity and every number in order: an integer maximum.
__device__ __forceinline__ float q8_larger(float a, float b, float c) {
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}

// The 8-bit form of the values r v of a block (r: the norm's factor of the row, or 1):
//     scale = max(r largest, 2^-100) / 448,   q = r v / scale.
// r cancels out of the quotient, so q is v / (largest / 448), for which nothing has to be known of r yet: values go out before the
// row's sum of squares is there.  The divisor is kept in two parts, and the quotient is rounded once, as a division is (the product with
// an approximate reciprocal, corrected by its remainder in a fused multiply-add: P. Markstein, IBM J. Res. Dev. 34, 1990), so that a value lands on the other side of the middle between two e4m3 values only where
// that rounding, or those of v and of the block's largest, have put it there.  Where that does not hold (largest infinite, a NaN, below 2^-90, or r largest below 2^-100: q8_usual) the
// block is written by the definition (Q8Plain).
// (Blocks of zeros are usual too: zeros, and the smallest scale.)
__device__ __forceinline__ bool q8_usual(float largest) { return (largest >= 0x1p-90f && largest <= FLT_MAX) || largest == 0.f; }
__device__ __forceinline__ bool q8_usual(float largest, float r) {
    const float h = largest * r;                 // (a NaN for zeros where r is infinite or NaN)
    return q8_usual(largest) && h <= FLT_MAX && (h >= 0x1p-100f || largest == 0.f);
}
__device__ __forceinline__ float q8_over_448(float v) {
    constexpr float C = 1.0f / 448.0f;
    const float s = v * C;
    return fmaf(fmaf(s, -448.0f, v), C, s);
}
struct Q8Quotient {
    float s, rest, inv;                          // largest / 448 = s + rest
    __device__ __forceinline__ explicit Q8Quotient(float largest) {
        s = q8_over_448(largest);
        rest = fmaf(s, -448.0f, largest) * (1.0f / 448.0f);
        asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(s));
        if (largest == 0.f) inv = 0.f;
    }
    __device__ __forceinline__ f32x2 operator()(f32x2 v) const {
        const f32x2 q = mul2(v, both(inv));
        return fma2(fma2(q, both(-rest), fma2(q, both(-s), v)), both(inv), q);
    }
};
__device__ __forceinline__ float q8_usual_scale(float largest, float r) { return largest == 0.f ? 0x1p-100f / 448.0f : q8_over_448(largest) * r; }
struct Q8Plain {
    float scale, r;
    __device__ __forceinline__ Q8Plain(float largest, float factor) : r(factor) {
        const float h = largest * factor;
        scale = (h < 0x1p-100f ? 0x1p-100f : h) / 448.0f;      // (a NaN stays one)
    }
    __device__ __forceinline__ f32x2 operator()(f32x2 v) const { return pack2(low(v) * r / scale, high(v) * r / scale); }
};
__device__ __forceinline__ uint16_t q8_pair(f32x2 v) { return (uint16_t)__nv_cvt_float2_to_fp8x2(make_float2(low(v), high(v)), __NV_SATFINITE, __NV_E4M3); }

}  // namespace gear
