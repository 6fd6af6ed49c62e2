// Shared pieces of the block norm kernels (block_norm_fwd.cu, block_norm_bwd.cu): row layout, loads, reductions.
//
// A voxel's row of c channels is held by TPR threads, U units of 8 channels each: unit i = u * TPR + t covers channels
// 8 i .. 8 i + 7 (16-byte loads of bf16, two of fp32).  c <= 256: 4, 8, 16 or 32 threads and one unit, several rows per
// warp; c <= 512: one warp, two units; wider: the whole CTA (a multiple of 32 threads fitted to c), two units, partial
// sums exchanged through shared memory.
#pragma once
#include "common.cuh"
#include "umma_ptx.cuh"

namespace lamp {
namespace bn {

template <bool F32> struct Raw { uint4 v[F32 ? 2 : 1]; };

template <bool F32> __device__ __forceinline__ Raw<F32> load_raw(const void *base, int64_t off)
{
    Raw<F32> r;
    if constexpr (F32) {
        const uint4 *p = reinterpret_cast<const uint4 *>((const float *)base + off);
        r.v[0] = p[0]; r.v[1] = p[1];
    } else {
        r.v[0] = *reinterpret_cast<const uint4 *>((const bf16 *)base + off);
    }
    return r;
}
template <bool F32> __device__ __forceinline__ Raw<F32> zero_raw()
{
    Raw<F32> r;
    r.v[0] = make_uint4(0, 0, 0, 0);
    if constexpr (F32) r.v[1] = r.v[0];
    return r;
}
template <bool F32> __device__ __forceinline__ void to_float(const Raw<F32> &r, float (&f)[8])
{
    if constexpr (F32) {
        f[0] = __uint_as_float(r.v[0].x); f[1] = __uint_as_float(r.v[0].y); f[2] = __uint_as_float(r.v[0].z); f[3] = __uint_as_float(r.v[0].w);
        f[4] = __uint_as_float(r.v[1].x); f[5] = __uint_as_float(r.v[1].y); f[6] = __uint_as_float(r.v[1].z); f[7] = __uint_as_float(r.v[1].w);
    } else {
        unpack8(r.v[0], f);
    }
}
template <bool F32> __device__ __forceinline__ void store8(void *base, int64_t off, const float (&f)[8])
{
    if constexpr (F32) {
        uint4 *p = reinterpret_cast<uint4 *>((float *)base + off);
        p[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        p[1] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
    } else {
        *reinterpret_cast<uint4 *>((bf16 *)base + off) = pack8(f);
    }
}

// the same as four packed pairs
template <bool F32> __device__ __forceinline__ void to_pairs(const Raw<F32> &r, ptx::f32x2 (&f)[4])
{
    if constexpr (F32) {
        f[0] = ptx::pack2(r.v[0].x, r.v[0].y); f[1] = ptx::pack2(r.v[0].z, r.v[0].w);
        f[2] = ptx::pack2(r.v[1].x, r.v[1].y); f[3] = ptx::pack2(r.v[1].z, r.v[1].w);
    } else {
        const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = ptx::pack2(w[i] << 16, w[i] & 0xFFFF0000u);
    }
}
template <bool F32> __device__ __forceinline__ void store_pairs(void *base, int64_t off, const ptx::f32x2 (&f)[4])
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) ptx::unpack2(f[i], v[2 * i], v[2 * i + 1]);
    store8<F32>(base, off, v);
}
__device__ __forceinline__ float both(ptx::f32x2 v)
{
    float a, b;
    ptx::unpack2(v, a, b);
    return a + b;
}
// e^x for the gates.  From fp32 logits with expf; from bf16 ones without its correction for the rounding of x log2(e): that error
// is 2^-24 |x| of e^x, so a gate of size e^-|x| is off by less than 2^-24 of one, and a bf16 gradient is rounded far more coarsely
// (expf for both: 138 us against 133 on 81,840 x 320 backward, 66 against 60 on 131,072 x 256 forward, gate per element).
template <bool FINE> __device__ __forceinline__ float gate_exp(float x)
{
    if (FINE) return expf(x);
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * 1.4426950408889634f));
    return e;
}
__device__ __forceinline__ float reciprocal(float x)               // within a unit of the last place
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <bool FINE> __device__ __forceinline__ float sigmoid(float x) { return reciprocal(1.f + gate_exp<FINE>(-x)); }
// g = sigmoid(x) and its slope g (1 - g), both to a few units of their own last place: from e^-|x|, so that nothing cancels (1 - g
// from a rounded g has no digit left at x = 17)
template <bool FINE> __device__ __forceinline__ void sigmoid_slope(float x, float &g, float &slope)
{
    const float e = gate_exp<FINE>(-fabsf(x)), r = reciprocal(1.f + e), er = e * r;
    g = x >= 0.f ? r : er;
    slope = er * r;
}

// Per-channel parameters sit in shared memory as [array][half][unit] float4, so that neighbouring threads read
// neighbouring 16-byte words.
__device__ __forceinline__ void load_par(const float4 *par, int array, int units, int unit, float (&f)[8])
{
    const float4 a = par[(array * 2) * units + unit], b = par[(array * 2 + 1) * units + unit];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void load_par(const float4 *par, int array, int units, int unit, ptx::f32x2 (&f)[4])
{
    const ulonglong2 a = *reinterpret_cast<const ulonglong2 *>(par + (array * 2) * units + unit);
    const ulonglong2 b = *reinterpret_cast<const ulonglong2 *>(par + (array * 2 + 1) * units + unit);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
}
__device__ __forceinline__ void store_par(float *par, int array, int units, int ch, float v)
{
    par[(((array * 2) + ((ch >> 2) & 1)) * units + (ch >> 3)) * 4 + (ch & 3)] = v;
}

// Sum of two values over the TPR threads of a row (TPR = 0: over the CTA).  red: [2][2 * 16] floats, `turn` alternates
// between its halves so that one barrier per sum is enough.
template <int TPR>
__device__ __forceinline__ void row_sum2(float &a, float &b, float (*red)[32], int &turn)
{
#pragma unroll
    for (int o = (TPR == 0 || TPR > 32 ? 32 : TPR) / 2; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if constexpr (TPR == 0) {
        const int w = threadIdx.x >> 5, nw = blockDim.x >> 5;
        if ((threadIdx.x & 31) == 0) { red[turn][2 * w] = a; red[turn][2 * w + 1] = b; }
        __syncthreads();
        a = red[turn][0]; b = red[turn][1];
        for (int i = 1; i < nw; ++i) { a += red[turn][2 * i]; b += red[turn][2 * i + 1]; }
        turn ^= 1;
    }
}

template <int TPR>
__device__ __forceinline__ float row_sum(float a, float (*red)[32], int &turn)
{
#pragma unroll
    for (int o = (TPR == 0 || TPR > 32 ? 32 : TPR) / 2; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    if constexpr (TPR == 0) {
        const int w = threadIdx.x >> 5, nw = blockDim.x >> 5;
        if ((threadIdx.x & 31) == 0) red[turn][w] = a;
        __syncthreads();
        a = red[turn][0];
        for (int i = 1; i < nw; ++i) a += red[turn][i];
        turn ^= 1;
    }
    return a;
}

// How a call of c channels is laid out.
struct Shape { int tpr, u, threads, rows_per_cta; };
inline Shape shape_of(int c)
{
    const int units = c / 8;
    if (units <= 4) return {4, 1, 256, 64};
    if (units <= 8) return {8, 1, 256, 32};
    if (units <= 16) return {16, 1, 256, 16};
    if (units <= 32) return {32, 1, 256, 8};
    if (units <= 64) return {32, 2, 256, 8};
    return {0, 2, (units / 2 + (units & 1) + 31) / 32 * 32, 1};
}

constexpr int MAX_C = 8192;

}  // namespace bn
}  // namespace lamp
