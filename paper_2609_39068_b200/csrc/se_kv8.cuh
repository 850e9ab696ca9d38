// The 8-bit cache: e4m3 codes (1 sign, 4 exponent, 3 mantissa bits, bias 7, largest finite value 448) with a scale 2^e for
// each (page, kv-head), one for K and one for V:  value = code * 2^e.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "se_device.cuh"

namespace se {

constexpr int kKv8LeastExponent = -64, kKv8MostExponent = 7;

// Smallest power of two that brings a magnitude (the bits of a bf16, sign cleared) to 448 = 1.75 * 2^8 or below, within the
// exponents' range.  Above 448 * 2^7 = 57344 codes saturate; with all exponents at most 7 the values' exponents stay within
// reach of one multiplication in bf16 (kv8_bf16x2).
__device__ __forceinline__ float kv8_scale(uint32_t magnitude) {
    const int e = (int)(magnitude >> 7) - 135 + ((magnitude & 127u) > 96u ? 1 : 0);
    return __uint_as_float((uint32_t)(min(max(e, kKv8LeastExponent), kKv8MostExponent) + 127) << 23);
}

// the larger magnitudes of eight bf16, even and odd ones apart
__device__ __forceinline__ uint32_t largest8(const uint4 &w) {
    const uint32_t m = 0x7fff7fffu;
    return bmax2(bmax2(w.x & m, w.y & m), bmax2(w.z & m, w.w & m));
}

__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
// four codes as four halves (lower two, upper two): exact
__device__ __forceinline__ void halves_of_e4m3x4(uint32_t codes, uint32_t &lo, uint32_t &hi) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(codes));
}
__device__ __forceinline__ float2 float2_of_e4m3x2(uint32_t codes) {
    return __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes, __NV_E4M3)));
}

// eight bf16 into codes, multiplied by 1/scale (exact) and rounded to the nearest code, ties to even
__device__ __forceinline__ uint2 kv8_codes(const uint4 &w, float inv) {
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = bf16x2_to_f2(a[i]);
        c[i] = e4m3x2(f.x * inv, f.y * inv);
    }
    return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
}
// eight codes times `f`, rounded again
__device__ __forceinline__ uint2 kv8_again(const uint2 &u, float f) {
    const uint32_t a[2] = {u.x, u.y};
    uint32_t c[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2 lo = float2_of_e4m3x2(a[i] & 0xffffu), hi = float2_of_e4m3x2(a[i] >> 16);
        c[i] = e4m3x2(lo.x * f, lo.y * f) | e4m3x2(hi.x * f, hi.y * f) << 16;
    }
    return make_uint2(c[0], c[1]);
}
// eight codes as the bf16 values that they stand for: exact
__device__ __forceinline__ uint4 kv8_values(const uint2 &u, float scale) {
    const uint32_t a[2] = {u.x, u.y};
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = float2_of_e4m3x2(a[i / 2] >> (i % 2 * 16) & 0xffffu);
        const __nv_bfloat162 b = __float22bfloat162_rn(make_float2(f.x * scale, f.y * scale));
        v[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// Four codes as four bf16 times `f`: exact where f = scale * kv8_bf16_step() is a power of two.  A code's exponent and mantissa, moved
// to the place of a bf16's, are its value times 2^-120 (the difference of the biases), subnormal codes included.  The NaN codes (0x7f,
// 0xff) come out as +-480 * scale: who turns codes with it has to look for them (kv8_nan).
__device__ __forceinline__ constexpr float kv8_bf16_step() { return 0x1p120f; }
__device__ __forceinline__ void kv8_bf16x4(uint32_t codes, __nv_bfloat162 f, uint32_t &lo, uint32_t &hi) {
    uint32_t x[2];                       // halves: a code, its sign in all bits above
    asm("prmt.b32 %0, %1, 0, 0x9180;" : "=r"(x[0]) : "r"(codes));
    asm("prmt.b32 %0, %1, 0, 0xb3a2;" : "=r"(x[1]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t y = x[i] << 4 & 0x87f087f0u;
        const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&y), f);
        x[i] = *reinterpret_cast<const uint32_t *>(&v);
    }
    lo = x[0], hi = x[1];
}

// `found`, with the top bit of some byte set if one of the four codes is a NaN's: adding one to a code changes its sign where the seven
// bits below are all set (and a carry out of 0xff can only make more of them change).
__device__ __forceinline__ uint32_t kv8_nan(uint32_t codes, uint32_t found) { return found | ((codes + 0x01010101u) ^ codes); }

}  // namespace se
