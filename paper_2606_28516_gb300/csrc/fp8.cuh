// 8-bit blocks: value = e4m3(q) 2^(s - 127), one scale byte s per block of 128 columns (activations: of one
// row; weights: of 128 rows). Device helpers shared by the quantiser, the GEMM's epilogue and the few-token
// kernels.
#pragma once

#include "common.cuh"

namespace cm {

// Scale byte of a block whose largest |value| has the fp32 bits `amax` (largest as an unsigned integer, so that
// NaN > inf > every finite value): the least s with amax <= 448 2^(s - 127). 448 = 1.75 2^8 is e4m3's largest
// value, so s is amax's biased exponent less 8, one more when its significand is above 1.75; held at 0 below
// (2^-127), 255 (the scale format's NaN) for a block with an infinity or a NaN.
__device__ __forceinline__ uint32_t fp8_scale_byte(uint32_t amax) {
    if (amax >= 0x7F800000u) return 255u;
    const int s = (int)(amax >> 23) - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return s < 0 ? 0u : (uint32_t)s;
}
// 2^(127 - s) of a scale byte that fp8_scale_byte gave (at most 247), NaN for 255.
__device__ __forceinline__ float fp8_inverse_scale(uint32_t s) {
    return s == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float((254u - s) << 23);
}
// 2^(s - 127) of any scale byte, NaN for 255.
__device__ __forceinline__ float fp8_scale(uint32_t s) {
    return s == 255u ? __uint_as_float(0x7FC00000u) : s == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23);
}
// Two factors that stand for 2^(a - 127) 2^(b - 127), for a sum of products of e4m3 values: the product itself may lie
// outside fp32 where the scaled sum does not (a zero sum times an infinity is NaN). Each factor has half the exponent, so
// that scaling by one after the other rounds or overflows only where the result does. A factor of 2^-127 is taken as 0: the
// result, below 2^-220, is. Scale bytes of 255 are the caller's to look for.
__device__ __forceinline__ float2 fp8_scale_pair(uint32_t a, uint32_t b) {
    const uint32_t h = (a + b) >> 1;
    return make_float2(__uint_as_float(h << 23), __uint_as_float((a + b - h) << 23));
}
// Two values to e4m3, to nearest even; lo in the low byte. NaN becomes e4m3's NaN.
__device__ __forceinline__ uint32_t fp8_pack2(float lo, float hi) {
    uint16_t v;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(hi), "f"(lo));
    return v;
}
__device__ __forceinline__ uint32_t fp8_pack4(float a, float b, float c, float d) {
    return fp8_pack2(a, b) | fp8_pack2(c, d) << 16;
}
// 32 values times inv, to e4m3.
__device__ __forceinline__ void fp8_pack32(uint32_t (&o)[8], const float (&v)[32], float inv) {
    const float2 k = make_float2(inv, inv);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 a = __fmul2_rn(make_float2(v[4 * i], v[4 * i + 1]), k), b = __fmul2_rn(make_float2(v[4 * i + 2], v[4 * i + 3]), k);
        o[i] = fp8_pack4(a.x, a.y, b.x, b.y);
    }
}
// Two e4m3 values (the low byte first) as fp32, exactly.
__device__ __forceinline__ float2 fp8_unpack2(uint32_t v) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)v));
    float2 f;
    asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}"
        : "=f"(f.x), "=f"(f.y)
        : "r"(h));
    return f;
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The larger magnitude of two values, NaN if either is; its sign is either's.
__device__ __forceinline__ float max_abs(float a, float b) {
    float r;
    asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// The largest magnitude of three values, NaN if one of them is.
__device__ __forceinline__ float max_abs3(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

}  // namespace cm
