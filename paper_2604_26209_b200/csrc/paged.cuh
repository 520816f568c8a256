// The 8-bit page format: e4m3 codes and one power-of-two scale (an e8m0 byte) per page, kv head, and key or value.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

namespace hpd {

// value = code * 2^(byte - 127); byte 255 stands for NaN
__device__ __forceinline__ float e8m0_value(uint32_t byte)
{
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fffffffu : byte << 23);
}
// 2^(127 - byte), what a value is multiplied by to become a code
__device__ __forceinline__ float e8m0_inverse(uint32_t byte)
{
    return __uint_as_float(byte < 254 ? (254 - byte) << 23 : byte == 254 ? 0x00400000u : 0x7fffffffu);
}
// The smallest scale of at least 2^-126 whose 448-fold (the largest e4m3 value, 1.75 * 2^8) reaches a bf16 magnitude given by its bits:
// exponent - 8, one more where the fraction is above 0.75 (96 of 128; the sum carries into the exponent then).
__device__ __forceinline__ int e8m0_needed(int bf16_bits) { return max(1, ((bf16_bits + 31) >> 7) - 8); }

// largest finite magnitude (bits) of two packed bf16, and of what came before
__device__ __forceinline__ int max_finite(int top, uint32_t two)
{
    const int a = two & 0x7fff, b = (two >> 16) & 0x7fff;
    if (a < 0x7f80) top = max(top, a);
    if (b < 0x7f80) top = max(top, b);
    return top;
}

// four codes of four fp32 values: to the nearest (even on ties), beyond the largest value the largest value, NaN stays NaN
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d)
{
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}
// two codes (the low half of a word) as fp16, which holds every code exactly, and back (as above)
__device__ __forceinline__ uint32_t e4m3x2_half2(uint32_t two)
{
    uint32_t h;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(h) : "r"(two));
    return h;
}
__device__ __forceinline__ uint32_t half2_e4m3x2(__half2 h)
{
    uint16_t two;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(two) : "r"(*reinterpret_cast<const uint32_t*>(&h)));
    return two;
}
__device__ __forceinline__ float2 e4m3x2_value(uint32_t two)
{
    const uint32_t h = e4m3x2_half2(two);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// four codes times a power of two
__device__ __forceinline__ uint32_t e4m3x4_times(uint32_t w, float f)
{
    const float2 a = e4m3x2_value(w & 0xffff), b = e4m3x2_value(w >> 16);
    return e4m3x4(a.x * f, a.y * f, b.x * f, b.y * f);
}

}  // namespace hpd
