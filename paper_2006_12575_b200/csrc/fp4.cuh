// 4-bit codes (e2m1) and their block scales: e8m0 per 32, or e4m3 per 16 times a tensor's scale.
#pragma once
#include <stdint.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include "block_norm.cuh"

namespace lamp {
namespace fp4 {

// Place of the scale of (row, block i) among an operand's scales: tiles of 128 rows x 4 blocks, `tiles` of them along k
__host__ __device__ __forceinline__ int64_t scale_at(int64_t row, int64_t i, int64_t tiles)
{
    return ((row >> 7) * tiles + (i >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (i & 3);
}
__host__ __device__ __forceinline__ int64_t blocks_of(int64_t k, int block) { return (k + block - 1) / block; }
__host__ __device__ __forceinline__ int64_t tiles_of(int64_t k, int block) { return (blocks_of(k, block) + 3) / 4; }

// bits of the largest |v|: infinities above every finite value, NaN above both
__device__ __forceinline__ uint32_t amax_bits(const float (&f)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7FFFFFFFu);
    return m;
}

// The tensor's scale g, with what divisions by 6 g need
struct Divisor {
    float g, six_g, inv;
    __device__ __forceinline__ explicit Divisor(float scale)
    {
        g = scale;
        six_g = __fmul_rn(6.f, scale);
        inv = __frcp_rn(six_g);
    }
};

// a / b correctly rounded for b > 0, with inv = 1 / b correctly rounded: one correction of a * inv by its exact remainder (Markstein's theorem).  Only
// where nothing leaves fp32's range - b within 2^-90 .. 2^90, a * inv finite (from an infinite one the correction makes NaN) - elsewhere the division itself.
__device__ __forceinline__ float quotient(float a, float b, float inv)
{
    const float q = a * inv;
    return fmaf(-fmaf(q, b, -a), inv, q);                        // the remainder's negative: so -0 keeps its sign
}
__device__ __forceinline__ ptx::f32x2 quotient2(ptx::f32x2 a, ptx::f32x2 b, ptx::f32x2 inv, ptx::f32x2 minus_inv)
{
    const ptx::f32x2 q = ptx::mul2(a, inv);
    return ptx::fma2(ptx::fma2(q, b, ptx::mul2(a, ptx::twice(-1.f))), minus_inv, q);
}
__device__ __forceinline__ bool plain_range(float b) { return b >= 8.0779357e-28f && b <= 1.2379400e27f; }

// A block's scale byte, and what its values are divided by: `inv` = 1 / scale, exactly, where the scale is a power of two (blocks of 32), else
// by = scale * g and inv = its reciprocal, 0 where the division itself has to be taken.  by = 0: the block has no codes (NaN scale).
struct Scale { uint32_t byte; float by, inv; };

// from the bits of the block's amax
template <int BLOCK> __device__ __forceinline__ Scale block_scale(uint32_t amax, const Divisor &d)
{
    Scale s;
    const bool nan = amax >= 0x7F800000u;
    if constexpr (BLOCK == 32) {
        // amax = 1.m 2^(E - 127) <= 6 2^e = 1.5 2^(e + 2)  <=>  e >= E - 129, one more where 1.m > 1.5
        const int e = (int)(amax >> 23) - 2 + ((amax & 0x7FFFFFu) > 0x400000u ? 1 : 0);
        s.byte = nan ? 255u : (uint32_t)max(e, 0);
        s.by = s.inv = nan ? 0.f : __uint_as_float((254u - s.byte) << 23);
    } else {
        const float a = __uint_as_float(amax);
        // at 2^20 and above the scale is the largest, whatever the last digits are
        const float v = fminf(fmaxf(plain_range(d.six_g) && a > 1e-25f && a * d.inv < 1048576.f ? quotient(a, d.six_g, d.inv) : __fdiv_rn(a, d.six_g), 0.001953125f), 448.f);
        uint16_t two;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(0.f), "f"(v));
        s.byte = nan ? 0x7Fu : (two & 0xFFu);
        uint32_t half2;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(half2) : "h"(two));
        s.by = nan ? 0.f : __fmul_rn(__half2float(__ushort_as_half((unsigned short)(half2 & 0xFFFFu))), d.g);
        s.inv = __frcp_rn(s.by);
        // values far above the largest scale: no |x| * inv is larger than amax * inv, so one look decides for the block
        if (!plain_range(s.by) || !(a * s.inv <= 3.4028235e38f)) s.inv = 0.f;
    }
    return s;
}

// Eight codes, the first in the low half of the low byte.  The conversion rounds to nearest even and saturates.
__device__ __forceinline__ uint32_t encode8(const float (&v)[8])
{
    uint32_t r;
    asm("{\n.reg .b8 b0, b1, b2, b3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
        "mov.b32 %0, {b0, b1, b2, b3};\n}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
template <int BLOCK> __device__ __forceinline__ uint32_t encode8(const float (&f)[8], const Scale &s)
{
    float v[8];
    if (BLOCK == 32) {
        const ptx::f32x2 inv = ptx::twice(s.inv);
#pragma unroll
        for (int i = 0; i < 8; i += 2) ptx::unpack2(ptx::mul2(ptx::pack2(__float_as_uint(f[i]), __float_as_uint(f[i + 1])), inv), v[i], v[i + 1]);
    } else if (s.inv != 0.f) {
#pragma unroll
        for (int i = 0; i < 8; i += 2)
            ptx::unpack2(quotient2(ptx::pack2(__float_as_uint(f[i]), __float_as_uint(f[i + 1])), ptx::twice(s.by), ptx::twice(s.inv), ptx::twice(-s.inv)), v[i], v[i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fdiv_rn(f[i], s.by);
    }
    const uint32_t r = encode8(v);
    return s.by == 0.f ? 0u : r;
}

__device__ __forceinline__ void decode8(uint32_t codes, float (&v)[8])
{
    uint32_t h[4];
    asm("{\n.reg .b8 b0, b1, b2, b3;\nmov.b32 {b0, b1, b2, b3}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\ncvt.rn.f16x2.e2m1x2 %1, b1;\ncvt.rn.f16x2.e2m1x2 %2, b2;\ncvt.rn.f16x2.e2m1x2 %3, b3;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}
// scale * g of a scale byte
template <int BLOCK> __device__ __forceinline__ float decode_scale(uint32_t byte, float g)
{
    if constexpr (BLOCK == 32) return __uint_as_float(byte == 255u ? 0x7FC00000u : byte == 0u ? 0x00400000u : byte << 23);
    uint32_t half2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(half2) : "h"((uint16_t)byte));
    return __fmul_rn(__half2float(__ushort_as_half((unsigned short)(half2 & 0xFFFFu))), g);
}

}  // namespace fp4

// fp4_quant.cu.  Argument check of a 4-bit operand.
lamp_status_t check_fp4_operand(const lamp_fp4_operand_t *o);

}  // namespace lamp
