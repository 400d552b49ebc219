// Numbers of a cache held in 8 bits: e4m3 codes, and a scale per block that is a power of two.
#pragma once
#include <stdint.h>

namespace wpp {

constexpr int kKv8LeastExp = -56, kKv8MostExp = 40;        // of a scale, base 2

// Two codes (bytes 0 and 1 of a word's half) as f16 numbers, exact (NaN stays NaN)
__device__ __forceinline__ uint32_t codes_f16x2(uint16_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(two));
    return r;
}
__device__ __forceinline__ uint32_t codes_f16x2_low(uint32_t w) { return codes_f16x2((uint16_t)w); }
__device__ __forceinline__ uint32_t codes_f16x2_high(uint32_t w) { return codes_f16x2((uint16_t)(w >> 16)); }
// Two numbers rounded to codes (nearest, halves to even; beyond 448: 448; NaN 0x7f), `lo` in byte 0
__device__ __forceinline__ uint16_t codes_of(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float f16_low(uint32_t w) {
    float r;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.f32.f16 %0, a;\n\t}" : "=f"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ float f16_high(uint32_t w) {
    float r;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.f32.f16 %0, b;\n\t}" : "=f"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
__device__ __forceinline__ int exponent_of(float x) { return (int)(__float_as_uint(x) >> 23 & 0xffu) - 127; }

}  // namespace wpp
