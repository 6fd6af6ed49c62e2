// Quantisation to e4m3 codes with one fp32 scale per block of 128 (the operands of fp8_gemm.cu).
// Bound by memory: x is read once, one byte per element is written.
//   amax  = largest finite |x| of the block, at least 2^-100 (so that neither scale nor its reciprocal leaves the normal range)
//   scale = amax * (1/448),  code = rn(x * (448 / amax)),  NaN for x not finite.
// x * (448 / amax) is at most 448 (1 + 2^-23), which rounds to 448: no code overflows.
#include "common.cuh"
#include "fp8.cuh"

namespace lamp {

namespace {

constexpr int QT = 256;

template <bool F32>
__device__ __forceinline__ void load8(const void *base, int64_t off, float (&f)[8])
{
    if constexpr (F32) {
        const float4 a = __ldg(reinterpret_cast<const float4 *>((const float *)base + off));
        const float4 b = __ldg(reinterpret_cast<const float4 *>((const float *)base + off) + 1);
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
        unpack8(__ldg(reinterpret_cast<const uint4 *>((const bf16 *)base + off)), f);
    }
}

// Row blocks: 16 lanes share one block of 128 channels of one voxel, 8 channels each (16-byte loads, 8-byte stores).
// Consecutive half-warps take consecutive blocks of a row, so a CTA reads whole rows.
constexpr int QR_UNROLL = 4;
template <bool F32>
__global__ void __launch_bounds__(QT)
quant_rows_kernel(const void *__restrict__ x, int64_t pitch, int c, uint32_t kb, uint32_t div_kb, int64_t blocks, uint8_t *__restrict__ q, int64_t q_pitch,
                  float *__restrict__ scale, int64_t scale_pitch)
{
    pdl_launch_dependents();
    pdl_wait();
    const int l16 = threadIdx.x & 15;
    // row and block of each of the CTA's blocks: one division for the first, then offsets below kb + 64 by a multiplication
    // (exact there: (kb + 64) (kb div_kb - 2^32) < 2^32).  A 64-bit division per block cost a third of the kernel's time (35 us against 23 on 131,072 x 256 bf16).
    const uint32_t first = blockIdx.x * (QT / 16 * QR_UNROLL), row0 = first / kb, rest = first - row0 * kb;
    float f[QR_UNROLL][8];
    int64_t row[QR_UNROLL];
    int blk[QR_UNROLL];
    bool in[QR_UNROLL];
#pragma unroll
    for (int u = 0; u < QR_UNROLL; ++u) {
        const uint32_t at = u * (QT / 16) + (threadIdx.x >> 4), l = rest + at;
        const uint32_t q_ = kb == 1 ? l : __umulhi(l, div_kb);
        row[u] = (int64_t)row0 + q_;
        blk[u] = (int)(l - q_ * kb);
        in[u] = first + (int64_t)at < blocks && blk[u] * 128 + l16 * 8 < c;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[u][j] = 0.f;
        if (in[u]) load8<F32>(x, row[u] * pitch + blk[u] * 128 + l16 * 8, f[u]);
    }
#pragma unroll
    for (int u = 0; u < QR_UNROLL; ++u) {
        float m;
        const uint2 codes = encode_block<16>(f[u], m);
        if (in[u]) {
            *reinterpret_cast<uint2 *>(q + row[u] * q_pitch + blk[u] * 128 + l16 * 8) = codes;
            if (l16 == 0) scale[blk[u] * scale_pitch + row[u]] = __fmul_rn(m, 1.0f / 448.0f);
        }
    }
}

// 128 x 128 tiles: the tile goes through shared memory once; a thread then owns two channels and 32 voxels of it.  With a
// scale per row of the transposed operand (= per channel and 128 voxels) four threads combine their maxima, with a scale per
// tile the whole CTA does.  Transposed codes leave as 32-byte runs along the voxels, untransposed ones as 2-byte pairs
// through shared memory again.
template <bool F32>
__global__ void __launch_bounds__(QT)
quant_tile_kernel(const void *__restrict__ x, int64_t pitch, int c, int64_t rows, int transpose, int tile_scale, uint8_t *__restrict__ q,
                  int64_t q_pitch, float *__restrict__ scale, int64_t scale_pitch)
{
    extern __shared__ __align__(16) uint8_t smem[];
    constexpr int ES = F32 ? 4 : 2, SP = 128 * ES + 16;                       // shared row pitch in bytes
    float *red = (float *)(smem + 128 * SP);                                  // [4][128] maxima
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x;
    const int64_t r0 = (int64_t)blockIdx.x * 128;
    const int c0 = blockIdx.y * 128;
    constexpr int UPR = 128 * ES / 16;                                        // 16-byte units per row
#pragma unroll 8
    for (int i = t; i < 128 * UPR; i += QT) {
        const int r = i / UPR, u = i % UPR;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r0 + r < rows && c0 + u * (16 / ES) < c)
            v = __ldg(reinterpret_cast<const uint4 *>((const uint8_t *)x + ((r0 + r) * pitch + c0) * ES + u * 16));
        *reinterpret_cast<uint4 *>(smem + r * SP + u * 16) = v;
    }
    __syncthreads();
    const int cp = t & 63, part = t >> 6;                                     // channel pair, 32-voxel part
    float a0 = 0.f, a1 = 0.f;
    float f0[32], f1[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const uint8_t *p = smem + (part * 32 + i) * SP + cp * 2 * ES;
        if constexpr (F32) {
            const float2 v = *reinterpret_cast<const float2 *>(p);
            f0[i] = v.x; f1[i] = v.y;
        } else {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(p);
            f0[i] = __uint_as_float(w << 16); f1[i] = __uint_as_float(w & 0xFFFF0000u);
        }
        a0 = fmaxf(a0, finite_abs(f0[i]));
        a1 = fmaxf(a1, finite_abs(f1[i]));
    }
    red[part * 128 + 2 * cp] = a0;
    red[part * 128 + 2 * cp + 1] = a1;
    __syncthreads();
    a0 = fmaxf(fmaxf(red[2 * cp], red[128 + 2 * cp]), fmaxf(red[256 + 2 * cp], red[384 + 2 * cp]));
    a1 = fmaxf(fmaxf(red[2 * cp + 1], red[128 + 2 * cp + 1]), fmaxf(red[256 + 2 * cp + 1], red[384 + 2 * cp + 1]));
    if (tile_scale) {
        float m = fmaxf(a0, a1);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        __syncthreads();
        if ((t & 31) == 0) red[t >> 5] = m;
        __syncthreads();
        a0 = a1 = fmaxf(red[0], red[1]);                                      // warps 0 and 1 hold all 64 channel pairs
    }
    a0 = fmaxf(a0, FP8_AMAX_MIN);
    a1 = fmaxf(a1, FP8_AMAX_MIN);
    const float i0 = __fdiv_rn(448.f, a0), i1 = __fdiv_rn(448.f, a1);
    if (tile_scale) {
        if (t == 0) {
            const float s = __fmul_rn(a0, 1.0f / 448.0f);
            if (transpose) scale[(r0 / 128) * scale_pitch + c0 / 128] = s;
            else scale[(int64_t)(c0 / 128) * scale_pitch + r0 / 128] = s;
        }
    } else if (part == 0) {                                                   // transposed, one scale per channel
        if (c0 + 2 * cp < c) {                                                // c is even: both channels exist
            float *o = scale + (r0 / 128) * scale_pitch + c0 + 2 * cp;
            o[0] = __fmul_rn(a0, 1.0f / 448.0f);
            o[1] = __fmul_rn(a1, 1.0f / 448.0f);
        }
    }
    if (transpose) {
        const int64_t v0 = r0 + part * 32;
        if (c0 + 2 * cp >= c || v0 >= rows) return;
        uint8_t *o0 = q + (int64_t)(c0 + 2 * cp) * q_pitch + v0, *o1 = o0 + q_pitch;
        uint32_t w0[8], w1[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w0[i] = encode4<true>(f0[4 * i], f0[4 * i + 1], f0[4 * i + 2], f0[4 * i + 3], i0);
            w1[i] = encode4<true>(f1[4 * i], f1[4 * i + 1], f1[4 * i + 2], f1[4 * i + 3], i1);
        }
        if (rows - v0 >= 32) {                                                // q_pitch and v0 are multiples of 16
            *reinterpret_cast<uint4 *>(o0) = make_uint4(w0[0], w0[1], w0[2], w0[3]);
            *reinterpret_cast<uint4 *>(o0 + 16) = make_uint4(w0[4], w0[5], w0[6], w0[7]);
            *reinterpret_cast<uint4 *>(o1) = make_uint4(w1[0], w1[1], w1[2], w1[3]);
            *reinterpret_cast<uint4 *>(o1 + 16) = make_uint4(w1[4], w1[5], w1[6], w1[7]);
        } else {
            const int n = (int)(rows - v0);                                   // bytes behind the last voxel stay as they were
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < n) { o0[i] = (uint8_t)(w0[i / 4] >> (8 * (i & 3))); o1[i] = (uint8_t)(w1[i / 4] >> (8 * (i & 3))); }
        }
    } else {
        __syncthreads();                                                      // the tile has been read by everybody
#pragma unroll
        for (int i = 0; i < 32; ++i)
            *reinterpret_cast<uint16_t *>(smem + (part * 32 + i) * 144 + cp * 2) = encode2<true>(f0[i], f1[i], i0, i1);
        __syncthreads();
        for (int i = t; i < 128 * 16; i += QT) {                              // 8-byte units: c is a multiple of 8
            const int r = i >> 4, u = i & 15;
            if (r0 + r < rows && c0 + u * 8 < c)
                *reinterpret_cast<uint2 *>(q + (r0 + r) * q_pitch + c0 + u * 8) = *reinterpret_cast<const uint2 *>(smem + r * 144 + u * 8);
        }
    }
}

}  // namespace

}  // namespace lamp

using namespace lamp;

extern "C" lamp_status_t lamp_fp8_quantize(const lamp_tensor_t *x, int32_t transpose, const lamp_fp8_operand_t *out, void *cuda_stream)
{
    lamp_status_t s;
    if ((s = check_view(x, false)) != LAMP_OK) return s;
    if ((x->c & 7) || (x->c_pitch & 7) || (x->c_offset & 7)) return LAMP_ERR_UNSUPPORTED;
    if ((s = check_fp8_operand(out)) != LAMP_OK) return s;
    if (transpose != 0 && transpose != 1) return LAMP_ERR_INVALID_ARG;
    const int64_t rows = voxels(x);
    if (out->rows != (transpose ? (int64_t)x->c : rows) || out->k != (transpose ? rows : (int64_t)x->c)) return LAMP_ERR_INVALID_ARG;
    if (rows == 0) return LAMP_OK;
    const TView v = make_view(x);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (!transpose && !out->tile_scale) {
        const int kb = (x->c + 127) / 128;
        const int64_t blocks = rows * kb, grid = (blocks + QT / 16 * QR_UNROLL - 1) / (QT / 16 * QR_UNROLL);
        if (blocks > 4294967295ll || kb > 60000) return LAMP_ERR_UNSUPPORTED;
        const uint32_t div_kb = (uint32_t)((0x100000000ull + kb - 1) / kb);
        return launch_pdl(grid <= 2048, v.f32 ? quant_rows_kernel<true> : quant_rows_kernel<false>, dim3((unsigned)grid), dim3(QT), 0, st, v.p, v.pitch, v.c,
                          (uint32_t)kb, div_kb, blocks, (uint8_t *)out->q, out->q_pitch, out->scale, out->scale_pitch);
    }
    const int64_t gx = (rows + 127) / 128;
    const int gy = (x->c + 127) / 128;
    if (gx > 2147483647ll || gy > 65535) return LAMP_ERR_UNSUPPORTED;
    const int smem = 128 * (128 * (v.f32 ? 4 : 2) + 16) + 512 * 4;
    static SmemAttrOnce attr;
    if (v.f32 && (s = attr.ensure(quant_tile_kernel<true>, smem)) != LAMP_OK) return s;
    return launch_pdl(gx * gy <= 2048, v.f32 ? quant_tile_kernel<true> : quant_tile_kernel<false>, dim3((unsigned)gx, (unsigned)gy), dim3(QT), (size_t)smem, st, v.p,
                      v.pitch, v.c, rows, (int)transpose, (int)out->tile_scale, (uint8_t *)out->q, out->q_pitch, out->scale, out->scale_pitch);
}
