// e4m3 bytes with power-of-two scales: what the 8-bit cache and the 8-bit norm share.
//
// The scale of a group of values is s = 2^e with the least e >= -100 that holds the
// group's largest finite magnitude in 448 s: e4m3 is a floating type, so a finer
// scale would win nothing, and x / s is exact.
#pragma once

#include "device_common.h"

namespace clsa {

constexpr int kC8MinExp = -100;          // least scale 2^-100
constexpr float kC8Top = 0x1.ep+127f;    // 240 * 2^120: magnitudes above would round past fp32

// Two e4m3 bytes (low halfword) of two values that lie within +-448; NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3_pair(float x, float y) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false) & 0xffffu;
}

// The scale for a largest finite magnitude, given as its bits.
__device__ __forceinline__ float e4m3_scale(uint32_t top) {
    top = min(top, __float_as_uint(kC8Top));
    // 448 = 1.75 * 2^8: the exponent of top / 448, one more above 1.75
    int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = max(e, kC8MinExp);
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// A value over its scale (inv: the scale's inverse, a power of two), within +-448;
// not finite -> NaN (e4m3 has no infinity).
__device__ __forceinline__ float e4m3_scaled(float x, float inv) {
    return x - x == 0.0f ? fminf(fmaxf(x, -kC8Top), kC8Top) * inv : NAN;
}

}  // namespace clsa
