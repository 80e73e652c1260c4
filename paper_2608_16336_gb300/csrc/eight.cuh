// eight.cuh -- numbers of 8 bits and the scales of the block cache that holds them.
#ifndef MTSIM_EIGHT_CUH
#define MTSIM_EIGHT_CUH

#include "ops.cuh"

namespace mtop {

constexpr float kSmallestScale = 0x1p-60f, kLargestScale = 0x1p60f;

// Two numbers as e4m3 (nearest, ties to even; beyond 448: 448; NaN: NaN).
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack_e4m3(__half2 x) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(*(uint32_t *)&x));
    return r;
}
__device__ __forceinline__ __half2 halves_of_e4m3(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return *(__half2 *)&h;
}
__device__ __forceinline__ float2 unpack_e4m3(uint32_t two) { return __half22float2(halves_of_e4m3(two)); }

// The smallest power of two in range with a <= 448 times it: 448 is 1.75 * 2^8.
__device__ __forceinline__ float scale_for(float a) {
    const uint32_t b = __float_as_uint(a);
    const int e = (int)(b >> 23) - 127 - ((b & 0x7FFFFF) > 0x600000 ? 7 : 8);
    return __uint_as_float((uint32_t)(min(max(e, -60), 60) + 127) << 23);
}
// A scale as it is used.
__device__ __forceinline__ float scale_used(float s) { return fminf(fmaxf(s, kSmallestScale), kLargestScale); }

}  // namespace mtop

#endif
