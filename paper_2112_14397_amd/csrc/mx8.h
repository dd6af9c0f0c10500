// 8-bit values: 32 neighbours of a row share one scale, a power of two held as a byte b that stands for 2^(b - 127); the
// elements are e4m3 (largest magnitude 448, no infinity).  Internal to the library.
#pragma once
#include "common.h"

namespace evomoe {

constexpr int kMxGroup = 32;

// The scale byte for a group whose largest finite magnitude is amax: the smallest power of two with amax / 2^(b - 127) <= 448.
// With amax = 1.f x 2^(x - 127) that is 2^(x - 127 - 8), or the next one where 1.f exceeds 1.75 (448 = 1.75 x 2^8).  The
// clamp below holds zeros and what is smaller than 2^-119 at the smallest scale.
__device__ __forceinline__ uint32_t mx_scale_byte(float amax) {
    const uint32_t bits = __float_as_uint(amax);
    const int b = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u);
    return (uint32_t)max(b, 0);
}
// 2^(127 - b), what values are multiplied by (exactly) before they are rounded; b <= 247 as amax is finite, so that the factor
// is 2^-120 at least; 2^127 at most
__device__ __forceinline__ float mx_inverse(uint32_t b) { return __uint_as_float((254u - b) << 23); }

// magnitude for the group's maximum: infinities and NaNs count as 0
__device__ __forceinline__ float mx_magnitude(float v) {
    const float m = fabsf(v);
    return m < INFINITY ? m : 0.f;
}
// Four values -> four e4m3 bytes, round to nearest even (an infinity times the factor stays one, and the conversion makes it
// and a NaN the NaN of e4m3, as nothing that is finite exceeds 448 here).
__device__ __forceinline__ uint32_t mx_pack4(float a, float b, float c, float d, float inv) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, v, true);
}

}  // namespace evomoe
