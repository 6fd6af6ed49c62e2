// Quantisation to 4-bit codes with a scale per block of 32 or 16 along k (the operands of fp4_gemm.cu), and back.
// Bound by memory: x is read once, half a byte per element and a byte per block are written (and the other way round).
// The scales of four neighbouring blocks of a row are one 32-bit word of the tiled order: the lanes that hold them put it together.
#include "fp4.cuh"

namespace lamp {

namespace {

using namespace bn;
using namespace fp4;

constexpr int QT = 256, QR_UNROLL = 4;

// A segment is 128 channels of a voxel, 8 channels on each of 16 lanes.
struct RowParams {
    void *x;                                  // source, or destination of the values
    int64_t pitch, rows, items;               // items: segments of all rows, those that only fill up a tile of scales included
    int32_t c;
    uint32_t segs, div_segs;
    uint8_t *q;
    int64_t q_pitch;
    uint8_t *scale;
    int64_t tiles;
    const float *g;
};

// row and segment of an item of this CTA: one division for the first, then offsets below segs + 64 by a multiplication (exact
// there: (segs + 64) (segs div_segs - 2^32) < 2^32)
struct Item { int64_t row; int seg; bool in; };
__device__ __forceinline__ Item item(const RowParams &P, uint32_t row0, uint32_t rest, uint32_t first, int u)
{
    const uint32_t at = u * (QT / 16) + (threadIdx.x >> 4), l = rest + at, q = P.segs == 1 ? l : __umulhi(l, P.div_segs);
    return Item{(int64_t)row0 + q, (int)(l - q * P.segs), first + (int64_t)at < P.items};
}

template <bool F32, int BLOCK>
__global__ void __launch_bounds__(QT)
quant4_rows_kernel(const RowParams P)
{
    pdl_launch_dependents();
    pdl_wait();
    const int l16 = threadIdx.x & 15;
    const uint32_t first = blockIdx.x * (QT / 16 * QR_UNROLL), row0 = first / P.segs, rest = first - row0 * P.segs;
    const float g = BLOCK == 16 && P.g ? __ldg(P.g) : 1.f, six_g = __fmul_rn(6.f, g);
    Raw<F32> r[QR_UNROLL];
    Item it[QR_UNROLL];
#pragma unroll
    for (int u = 0; u < QR_UNROLL; ++u) {
        it[u] = item(P, row0, rest, first, u);
        const int ch = it[u].seg * 128 + l16 * 8;
        r[u] = it[u].in && it[u].row < P.rows && ch < P.c ? load_raw<F32>(P.x, it[u].row * P.pitch + ch) : zero_raw<F32>();
    }
#pragma unroll
    for (int u = 0; u < QR_UNROLL; ++u) {
        float f[8];
        to_float<F32>(r[u], f);
        uint32_t m = amax_bits(f);
#pragma unroll
        for (int o = BLOCK / 16; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const Scale s = block_scale<BLOCK>(m, g, six_g);
        const int ch = it[u].seg * 128 + l16 * 8;
        const bool there = it[u].row < P.rows && ch / BLOCK * BLOCK < P.c;      // blocks and rows that fill up a tile have scale 0
        uint32_t word = there ? s.byte << (8 * ((ch / BLOCK) & 3)) : 0u;
        constexpr int LANES = BLOCK / 8;                                        // of a block; 4 blocks to a word
        word |= __shfl_xor_sync(0xffffffffu, word, LANES);
        word |= __shfl_xor_sync(0xffffffffu, word, 2 * LANES);
        if (!it[u].in) continue;
        if (it[u].row < P.rows && ch < P.c) *reinterpret_cast<uint32_t *>(P.q + it[u].row * P.q_pitch + ch / 2) = encode8<BLOCK>(f, s);
        const int64_t blk = ch / BLOCK;
        if (l16 % (4 * LANES) == 0 && blk / 4 < P.tiles) *reinterpret_cast<uint32_t *>(P.scale + scale_at(it[u].row, blk, P.tiles)) = word;
    }
}

template <bool F32, int BLOCK>
__global__ void __launch_bounds__(QT)
dequant4_rows_kernel(const RowParams P)
{
    pdl_launch_dependents();
    pdl_wait();
    const int l16 = threadIdx.x & 15;
    const uint32_t first = blockIdx.x * (QT / 16 * QR_UNROLL), row0 = first / P.segs, rest = first - row0 * P.segs;
    const float g = BLOCK == 16 && P.g ? __ldg(P.g) : 1.f;
    uint32_t codes[QR_UNROLL], byte[QR_UNROLL];
    Item it[QR_UNROLL];
#pragma unroll
    for (int u = 0; u < QR_UNROLL; ++u) {
        it[u] = item(P, row0, rest, first, u);
        const int ch = it[u].seg * 128 + l16 * 8;
        codes[u] = byte[u] = 0;
        it[u].in = it[u].in && ch < P.c;
        if (it[u].in) {
            codes[u] = __ldg(reinterpret_cast<const uint32_t *>(P.q + it[u].row * P.q_pitch + ch / 2));
            byte[u] = __ldg(P.scale + scale_at(it[u].row, ch / BLOCK, P.tiles));
        }
    }
#pragma unroll
    for (int u = 0; u < QR_UNROLL; ++u) {
        if (!it[u].in) continue;
        float v[8];
        decode8(codes[u], v);
        const float s = decode_scale<BLOCK>(byte[u], g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], s);
        store8<F32>(P.x, it[u].row * P.pitch + it[u].seg * 128 + l16 * 8, v);
    }
}

// Transposed: tiles of 128 voxels x 128 channels through shared memory.  A thread owns two channels and 32 voxels of the tile, that is
// one block of 32 or two of 16 per channel, and writes 16 bytes of codes per channel.
struct TileParams {
    void *x;
    int64_t pitch, voxels;
    int32_t c;
    uint8_t *q;
    int64_t q_pitch;
    uint8_t *scale;
    int64_t tiles;
    const float *g;
};
template <bool F32> struct TileLayout { static constexpr int ES = F32 ? 4 : 2, SP = 128 * ES + 16, BYTES = 128 * SP, UNITS = 128 * ES / 16; };

template <bool F32, int BLOCK>
__global__ void __launch_bounds__(QT)
quant4_tile_kernel(const TileParams P)
{
    using L = TileLayout<F32>;
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x;
    const int64_t r0 = (int64_t)blockIdx.x * 128;
    const int c0 = blockIdx.y * 128;
#pragma unroll 8
    for (int i = t; i < 128 * L::UNITS; i += QT) {
        const int r = i / L::UNITS, u = i % L::UNITS;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r0 + r < P.voxels && c0 + u * (16 / L::ES) < P.c)
            v = __ldg(reinterpret_cast<const uint4 *>((const uint8_t *)P.x + ((r0 + r) * P.pitch + c0) * L::ES + u * 16));
        *reinterpret_cast<uint4 *>(smem + r * L::SP + u * 16) = v;
    }
    __syncthreads();
    const float g = BLOCK == 16 && P.g ? __ldg(P.g) : 1.f, six_g = __fmul_rn(6.f, g);
    const int cp = t & 63, part = t >> 6;                                     // channel pair, 32-voxel part
    const int64_t v0 = r0 + part * 32, blocks = blocks_of(P.voxels, BLOCK);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int ch = c0 + 2 * cp + h;
        uint32_t code[4], bytes = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) code[b] = 0;
#pragma unroll
        for (int b = 0; b < 32 / BLOCK; ++b) {
            float f[BLOCK / 8][8];
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < BLOCK; ++i) {
                const uint8_t *p = smem + (part * 32 + b * BLOCK + i) * L::SP + cp * 2 * L::ES;
                f[i / 8][i % 8] = F32 ? ((const float *)p)[h] : bf2f(((const bf16 *)p)[h]);
            }
#pragma unroll
            for (int i = 0; i < BLOCK / 8; ++i) m = max(m, amax_bits(f[i]));
            const Scale s = block_scale<BLOCK>(m, g, six_g);
            const int64_t blk = v0 / BLOCK + b;
            if (ch < P.c && blk < blocks) bytes |= s.byte << (8 * b);
#pragma unroll
            for (int i = 0; i < BLOCK / 8; ++i) code[b * (BLOCK / 8) + i] = encode8<BLOCK>(f[i], s);
        }
        // every block of the last tile along k and every row of a tile of rows gets its scale, 0 where there is none
        const int64_t blk = v0 / BLOCK;
        if (blk / 4 < P.tiles) {
            uint8_t *o = P.scale + scale_at(ch, blk, P.tiles);
            if constexpr (BLOCK == 32) *o = (uint8_t)bytes; else *reinterpret_cast<uint16_t *>(o) = (uint16_t)bytes;
        }
        if (ch >= P.c || v0 >= P.voxels) continue;
        uint8_t *o = P.q + (int64_t)ch * P.q_pitch + v0 / 2;
        if (P.voxels - v0 >= 32) *reinterpret_cast<uint4 *>(o) = make_uint4(code[0], code[1], code[2], code[3]);
        else {
            const int n = (int)(P.voxels - v0 + 1) / 2;                        // bytes behind the last voxel stay as they were
#pragma unroll
            for (int i = 0; i < 16; ++i) if (i < n) o[i] = (uint8_t)(code[i / 4] >> (8 * (i & 3)));
        }
    }
}

template <bool F32, int BLOCK>
__global__ void __launch_bounds__(QT)
dequant4_tile_kernel(const TileParams P)
{
    using L = TileLayout<F32>;
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x;
    const int64_t r0 = (int64_t)blockIdx.x * 128;
    const int c0 = blockIdx.y * 128;
    const float g = BLOCK == 16 && P.g ? __ldg(P.g) : 1.f;
    const int cp = t & 63, part = t >> 6;
    const int64_t v0 = r0 + part * 32;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int ch = c0 + 2 * cp + h;
        if (ch >= P.c || v0 >= P.voxels) continue;
        const uint8_t *o = P.q + (int64_t)ch * P.q_pitch + v0 / 2;
        uint32_t code[4] = {0, 0, 0, 0};
        if (P.voxels - v0 >= 32) {
            const uint4 u = __ldg(reinterpret_cast<const uint4 *>(o));
            code[0] = u.x; code[1] = u.y; code[2] = u.z; code[3] = u.w;
        } else {
            const int n = (int)(P.voxels - v0 + 1) / 2;
#pragma unroll
            for (int i = 0; i < 16; ++i) if (i < n) code[i / 4] |= (uint32_t)o[i] << (8 * (i & 3));
        }
        float s[32 / BLOCK];
#pragma unroll
        for (int b = 0; b < 32 / BLOCK; ++b) {
            const int64_t blk = v0 / BLOCK + b;
            s[b] = blk < blocks_of(P.voxels, BLOCK) ? decode_scale<BLOCK>(__ldg(P.scale + scale_at(ch, blk, P.tiles)), g) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v[8];
            decode8(code[i], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float y = __fmul_rn(v[j], s[i * 8 / BLOCK]);
                uint8_t *p = smem + (part * 32 + i * 8 + j) * L::SP + cp * 2 * L::ES;
                if (F32) ((float *)p)[h] = y; else ((bf16 *)p)[h] = f2bf(y);
            }
        }
    }
    __syncthreads();
#pragma unroll 4
    for (int i = t; i < 128 * L::UNITS; i += QT) {
        const int r = i / L::UNITS, u = i % L::UNITS;
        if (r0 + r < P.voxels && c0 + u * (16 / L::ES) < P.c)
            *reinterpret_cast<uint4 *>((uint8_t *)P.x + ((r0 + r) * P.pitch + c0) * L::ES + u * 16) = *reinterpret_cast<const uint4 *>(smem + r * L::SP + u * 16);
    }
}

template <bool F32, int BLOCK>
lamp_status_t launch_rows(bool back, const RowParams &P, cudaStream_t st)
{
    const int64_t grid = (P.items + QT / 16 * QR_UNROLL - 1) / (QT / 16 * QR_UNROLL);
    return launch_pdl(grid <= 2048, back ? dequant4_rows_kernel<F32, BLOCK> : quant4_rows_kernel<F32, BLOCK>, dim3((unsigned)grid), dim3(QT), 0, st, P);
}
template <bool F32, int BLOCK>
lamp_status_t launch_tiles(bool back, const TileParams &P, cudaStream_t st)
{
    lamp_status_t s;
    static SmemAttrOnce quant, dequant;
    if ((s = quant.ensure(quant4_tile_kernel<F32, BLOCK>, TileLayout<F32>::BYTES)) != LAMP_OK) return s;
    if ((s = dequant.ensure(dequant4_tile_kernel<F32, BLOCK>, TileLayout<F32>::BYTES)) != LAMP_OK) return s;
    const int64_t gx = (P.voxels + 127) / 128, gy = (P.c + 127) / 128;
    return launch_pdl(gx * gy <= 2048, back ? dequant4_tile_kernel<F32, BLOCK> : quant4_tile_kernel<F32, BLOCK>, dim3((unsigned)gx, (unsigned)gy), dim3(QT),
                      (size_t)TileLayout<F32>::BYTES, st, P);
}

lamp_status_t convert(const lamp_tensor_t *x, int32_t transpose, const lamp_fp4_operand_t *o, bool back, cudaStream_t st)
{
    lamp_status_t s;
    if ((s = check_view(x, false)) != LAMP_OK) return s;
    if ((x->c & 7) || (x->c_pitch & 7) || (x->c_offset & 7)) return LAMP_ERR_UNSUPPORTED;
    if ((s = check_fp4_operand(o)) != LAMP_OK) return s;
    if (transpose != 0 && transpose != 1) return LAMP_ERR_INVALID_ARG;
    const int64_t rows = voxels(x);
    if (o->rows != (transpose ? (int64_t)x->c : rows) || o->k != (transpose ? rows : (int64_t)x->c)) return LAMP_ERR_INVALID_ARG;
    if (rows == 0) return LAMP_OK;
    const TView v = make_view(x);
    if (transpose) {
        const TileParams P = {v.p, v.pitch, rows, v.c, (uint8_t *)o->q, o->q_pitch, o->scale, tiles_of(rows, o->block), o->tensor_scale};
        if ((v.c + 127) / 128 > 65535) return LAMP_ERR_UNSUPPORTED;
        if (o->block == 32) return v.f32 ? launch_tiles<true, 32>(back, P, st) : launch_tiles<false, 32>(back, P, st);
        return v.f32 ? launch_tiles<true, 16>(back, P, st) : launch_tiles<false, 16>(back, P, st);
    }
    RowParams P = {v.p, v.pitch, rows, 0, v.c, 0, 0, (uint8_t *)o->q, o->q_pitch, o->scale, tiles_of(v.c, o->block), o->tensor_scale};
    P.segs = (uint32_t)((v.c + 127) / 128);
    P.div_segs = (uint32_t)((0x100000000ull + P.segs - 1) / P.segs);
    P.items = (back ? rows : (rows + 127) / 128 * 128) * P.segs;
    if (P.items > 4294967295ll || P.segs > 60000) return LAMP_ERR_UNSUPPORTED;
    if (o->block == 32) return v.f32 ? launch_rows<true, 32>(back, P, st) : launch_rows<false, 32>(back, P, st);
    return v.f32 ? launch_rows<true, 16>(back, P, st) : launch_rows<false, 16>(back, P, st);
}

}  // namespace

lamp_status_t check_fp4_operand(const lamp_fp4_operand_t *o)
{
    if (!o || o->rows < 0 || o->k < 0 || (o->block != 16 && o->block != 32)) return LAMP_ERR_INVALID_ARG;
    if (o->rows > 2147483647ll - 256 || o->k > 2147483647ll - 256) return LAMP_ERR_UNSUPPORTED;
    if (o->q_pitch < (o->k + 1) / 2 || (o->q_pitch & 15)) return LAMP_ERR_INVALID_ARG;
    if (o->block == 32 && o->tensor_scale) return LAMP_ERR_INVALID_ARG;
    if ((double)o->rows * (double)o->q_pitch > 1099511627776.0) return LAMP_ERR_UNSUPPORTED;       // 2^40 B
    if (o->rows == 0 || o->k == 0) return LAMP_OK;
    if (!o->q || !o->scale || (((uintptr_t)o->q | (uintptr_t)o->scale) & 15) || ((uintptr_t)o->tensor_scale & 3)) return LAMP_ERR_INVALID_ARG;
    return LAMP_OK;
}

}  // namespace lamp

using namespace lamp;

extern "C" size_t lamp_fp4_scale_bytes(int64_t rows, int64_t k, int32_t block)
{
    if (rows < 0 || k < 0 || rows > 2147483647ll - 256 || k > 2147483647ll - 256 || (block != 16 && block != 32)) return 0;
    return (size_t)((rows + 127) / 128 * fp4::tiles_of(k, block) * 512);
}

extern "C" lamp_status_t lamp_fp4_quantize(const lamp_tensor_t *x, int32_t transpose, const lamp_fp4_operand_t *out, void *cuda_stream)
{
    return convert(x, transpose, out, false, (cudaStream_t)cuda_stream);
}

extern "C" lamp_status_t lamp_fp4_dequantize(const lamp_fp4_operand_t *in, int32_t transpose, lamp_tensor_t *y, void *cuda_stream)
{
    return convert(y, transpose, in, true, (cudaStream_t)cuda_stream);
}
