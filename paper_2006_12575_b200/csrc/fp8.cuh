// e4m3 encoding shared by the quantiser and the block norm.
#pragma once
#include <stdint.h>

namespace lamp {

constexpr float FP8_AMAX_MIN = 7.88860905e-31f;              // 2^-100

// |v| of a finite v, 0 otherwise: a block's scale comes from its finite values
__device__ __forceinline__ float finite_abs(float v) { v = fabsf(v); return v <= 3.402823466e+38f ? v : 0.f; }

// Largest |v|: NaN is passed over, an infinity is not - a block whose maximum comes out infinite is looked at again with
// finite_abs (rare, so that the common case is one instruction per element)
__device__ __forceinline__ float amax8(const float (&f)[8])
{
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(f[i]));
    return m;
}
__device__ __forceinline__ float finite_amax8(const float (&f)[8])
{
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(f[i]));
    return m;
}

// Two codes, `a` in the low byte.  The conversion saturates and keeps NaN; INF: there are infinities among the values, which
// become NaN too (v * 0 is NaN for them).
template <bool INF>
__device__ __forceinline__ uint16_t encode2(float a, float b, float inv_a, float inv_b)
{
    float x = a * inv_a, y = b * inv_b;
    if (INF) { x += a * 0.f; y += b * 0.f; }
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y), "f"(x));
    return r;
}
template <bool INF>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float inv)
{
    return (uint32_t)encode2<INF>(a, b, inv, inv) | ((uint32_t)encode2<INF>(c, d, inv, inv) << 16);
}
template <bool INF>
__device__ __forceinline__ uint2 encode8(const float (&f)[8], float inv)
{
    return make_uint2(encode4<INF>(f[0], f[1], f[2], f[3], inv), encode4<INF>(f[4], f[5], f[6], f[7], inv));
}

// The codes of a block of 128 that LANES threads of a warp hold, 8 values each (zeros where there is none), and its amax, at
// least FP8_AMAX_MIN.  Every lane of the warp takes part.
template <int LANES>
__device__ __forceinline__ uint2 encode_block(const float (&f)[8], float &m)
{
    m = amax8(f);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (__any_sync(0xffffffffu, m > 3.402823466e+38f)) {
        m = finite_amax8(f);
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        m = fmaxf(m, FP8_AMAX_MIN);
        return encode8<true>(f, __fdiv_rn(448.f, m));
    }
    m = fmaxf(m, FP8_AMAX_MIN);
    return encode8<false>(f, __fdiv_rn(448.f, m));
}

}  // namespace lamp
