// e4m3 encoding shared by the quantiser and the block norm.
#pragma once
#include <stdint.h>

namespace lamp {

constexpr float FP8_AMAX_MIN = 7.88860905e-31f;              // 2^-100

// |v| of a finite v, 0 otherwise: a block's scale comes from its finite values
__device__ __forceinline__ float finite_abs(float v) { v = fabsf(v); return v <= 3.402823466e+38f ? v : 0.f; }

__device__ __forceinline__ float amax8(const float (&f)[8])
{
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(f[i]));
    return m;
}

// Two codes, `a` in the low byte.  The conversion saturates, so an infinity is turned into a NaN first (v * 0 is NaN for it).
__device__ __forceinline__ uint16_t encode2(float a, float b, float inv_a, float inv_b)
{
    const float x = a * inv_a + a * 0.f, y = b * inv_b + b * 0.f;
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y), "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float inv)
{
    return (uint32_t)encode2(a, b, inv, inv) | ((uint32_t)encode2(c, d, inv, inv) << 16);
}
__device__ __forceinline__ uint2 encode8(const float (&f)[8], float inv)
{
    return make_uint2(encode4(f[0], f[1], f[2], f[3], inv), encode4(f[4], f[5], f[6], f[7], inv));
}

}  // namespace lamp
