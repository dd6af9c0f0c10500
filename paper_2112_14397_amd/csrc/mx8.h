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
// The largest magnitude of N values (the instruction passes a NaN over), and the largest finite one (an infinity, which is rare,
// takes a second look).
template <int N> __device__ __forceinline__ float mx_max(const float (&v)[N]) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < N; i += 2) m = fmaxf(fmaxf(fabsf(v[i]), fabsf(v[i + 1])), m);
    return m;
}
template <int N> __device__ __forceinline__ float mx_largest(const float (&v)[N]) {
    float m = mx_max(v);
    if (m == INFINITY) {
        m = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.f);
    }
    return m;
}
// Four values -> four e4m3 bytes, round to nearest even.  The instruction divides by the power of two in its scale operand's exponent
// field, whose mantissa it does not look at; with the mantissa's first bit set a field of 0 is 2^-127 too.  What is finite stays
// within 448; infinities and NaNs become the NaN of e4m3.
__device__ __forceinline__ uint32_t mx_pack4(float a, float b, float c, float d, uint32_t scale_byte) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    const float scale = __uint_as_float(scale_byte << 23 | 0x400000u);
    s16x2 v = {0, 0};
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, a, b, scale, false);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, c, d, scale, true);
    return __builtin_bit_cast(uint32_t, v);
}

}  // namespace evomoe
