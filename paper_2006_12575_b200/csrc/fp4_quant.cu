// Quantisation to 4-bit codes with a scale per block of 32 or 16 along k (the operands of fp4_gemm.cu), and back.
// Bound by memory: x is read once, half a byte per element and a byte per block are written (and the other way round).
// The scales of four neighbouring blocks of a row are one 32-bit word of the tiled order: the lanes that hold them put it together.
#include "fp4.cuh"

namespace lamp {

namespace {

using namespace bn;
using namespace fp4;

constexpr int QT = 256, QU = 4;

// A segment is up to 128 channels of a voxel, 8 channels on each of LPS lanes (4, 8 or 16: as many as the channels need, at least a block of
// 32).  A thread takes QU rows QT / LPS apart at the same channels, so that addresses are formed once: formed for every row they were most of
// the kernel's instructions (28 us for 131,072 x 256 bf16 against 18;
// what is left is bound by the instructions of the conversion as much as by memory).
struct RowParams {
    void *x;                                  // source, or destination of the values
    int64_t pitch, rows;
    int32_t c;
    uint32_t segs;
    uint8_t *q;
    int64_t q_pitch;
    uint8_t *scale;
    int64_t tiles;
    const float *g;
};
template <int LPS> struct RowPlace {
    static constexpr int RPP = QT / LPS, ROWS = RPP * QU;          // rows per pass (16, 32, 64) and per CTA (64, 128, 256: whole parts of a tile of scales)
    int64_t row;                                                   // of the first pass
    int ch;
    __device__ __forceinline__ RowPlace(const RowParams &P)
    {
        const uint32_t block = blockIdx.x / P.segs, seg = blockIdx.x - block * P.segs;
        row = (int64_t)block * ROWS + threadIdx.x / LPS;
        ch = (int)seg * 128 + (threadIdx.x % LPS) * 8;
    }
    // scale byte of (row of pass u, block blk): the passes stay within a tile of 128 rows (LPS = 16, 8) or take two
    __device__ __forceinline__ static int64_t scale_off(int u, int64_t tiles)
    {
        constexpr int in_tile = RPP >= 32 ? 4 * (RPP / 32) : 0;    // 32 rows further: 4 bytes
        if (RPP == 16) return (u & 1) * 256 + (u >> 1) * 4;
        return (u * RPP / 128) * tiles * 512 + (u % (128 / RPP)) * in_tile;
    }
};

// Bits of the amax of each of the thread's units over the LANES lanes of its block.  bf16: two values, then two units, at a time.
template <bool F32, int LANES> __device__ __forceinline__ void block_amax(const Raw<F32> (&r)[QU], uint32_t (&m)[QU])
{
    if constexpr (F32) {
#pragma unroll
        for (int u = 0; u < QU; ++u) {
            float f[8];
            to_float<F32>(r[u], f);
            m[u] = amax_bits(f);
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) m[u] = max(m[u], __shfl_xor_sync(0xffffffffu, m[u], o));
        }
    } else {
        uint32_t both[QU / 2];
#pragma unroll
        for (int u = 0; u < QU; ++u) {
            const uint4 &v = r[u].v[0];
            m[u] = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
        }
#pragma unroll
        for (int u = 0; u < QU / 2; ++u) {                         // the halves of two units into one word
            both[u] = __vmaxu2(__byte_perm(m[2 * u], m[2 * u + 1], 0x5410), __byte_perm(m[2 * u], m[2 * u + 1], 0x7632));
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) both[u] = __vmaxu2(both[u], __shfl_xor_sync(0xffffffffu, both[u], o));
            m[2 * u] = both[u] << 16;
            m[2 * u + 1] = both[u] & 0xFFFF0000u;
        }
    }
}
static_assert(QU == 4, "");

template <bool F32, int BLOCK, int LPS>
__global__ void __launch_bounds__(QT)
quant4_rows_kernel(const RowParams P)
{
    using Place = RowPlace<LPS>;
    constexpr int LANES = BLOCK / 8;                               // of a block
    pdl_launch_dependents();
    pdl_wait();
    const Place at(P);
    const Divisor d(BLOCK == 16 && P.g ? __ldg(P.g) : 1.f);
    const int blk = at.ch / BLOCK;
    // rows of this thread (0 where its channels do not exist), and those that have a place among the scales: the last tile is filled up
    const int64_t left = P.rows - at.row, left128 = (P.rows + 127) / 128 * 128 - at.row;
    auto count = [](int64_t n) { return n <= 0 ? 0 : n > (QU - 1) * Place::RPP ? QU : (int)((n + Place::RPP - 1) / Place::RPP); };
    const int rows = at.ch < P.c ? count(left) : 0, places = blk / 4 < P.tiles ? count(left128) : 0;
    const int64_t step = Place::RPP * P.pitch, q_step = Place::RPP * P.q_pitch, x0 = at.row * P.pitch + at.ch;
    Raw<F32> r[QU];
#pragma unroll
    for (int u = 0; u < QU; ++u) r[u] = u < rows ? load_raw<F32>(P.x, x0 + u * step) : zero_raw<F32>();
    uint8_t *q = P.q + at.row * P.q_pitch + at.ch / 2, *scale = P.scale + scale_at(at.row, blk & ~3, P.tiles);
    uint32_t m[QU], bytes = 0;                                     // scale bytes of this thread's block, one per unit
    block_amax<F32, LANES>(r, m);
#pragma unroll
    for (int u = 0; u < QU; ++u) {
        const Scale s = block_scale<BLOCK>(m[u], d);
        bytes |= s.byte << (8 * u);
        float f[8];
        to_float<F32>(r[u], f);
        if (u < rows) *reinterpret_cast<uint32_t *>(q + u * q_step) = encode8<BLOCK>(f, s);
    }
    // scale 0 for rows that only fill up a tile, as for blocks behind the last
    const int have = blk * BLOCK < P.c ? count(left) : 0;
    bytes &= have >= 4 ? 0xFFFFFFFFu : (1u << (8 * have)) - 1u;
    if constexpr (LPS >= 4 * LANES) {
        // Four blocks have four units' bytes each; a word of scales is one unit's byte of the four.  A transposition of 4 x 4 bytes over the
        // lanes of the blocks: block j then holds the word of unit j.
        const int j = (threadIdx.x / LANES) & 3;
        uint32_t o = __shfl_xor_sync(0xffffffffu, bytes, LANES);
        bytes = __byte_perm(bytes, o, j & 1 ? 0x3715 : 0x6240);
        o = __shfl_xor_sync(0xffffffffu, bytes, 2 * LANES);
        bytes = __byte_perm(bytes, o, j & 2 ? 0x3276 : 0x5410);
        if (threadIdx.x % LANES == 0 && j < places) *reinterpret_cast<uint32_t *>(scale + Place::scale_off(j, P.tiles)) = bytes;
    } else {
        // fewer than four blocks in all: LPS / LANES of them, the rest of the word is 0
#pragma unroll
        for (int u = 0; u < QU; ++u) {
            uint32_t word = ((bytes >> (8 * u)) & 0xFFu) << (8 * blk);
            if (LPS > LANES) word |= __shfl_xor_sync(0xffffffffu, word, LANES);
            if (threadIdx.x % LPS == 0 && u < places) *reinterpret_cast<uint32_t *>(scale + Place::scale_off(u, P.tiles)) = word;
        }
    }
}

template <bool F32, int BLOCK, int LPS>
__global__ void __launch_bounds__(QT)
dequant4_rows_kernel(const RowParams P)
{
    using Place = RowPlace<LPS>;
    pdl_launch_dependents();
    pdl_wait();
    const Place at(P);
    const float g = BLOCK == 16 && P.g ? __ldg(P.g) : 1.f;
    if (at.ch >= P.c) return;
    const uint8_t *q = P.q + at.row * P.q_pitch + at.ch / 2, *scale = P.scale + scale_at(at.row, at.ch / BLOCK, P.tiles);
    uint32_t codes[QU], byte[QU];
#pragma unroll
    for (int u = 0; u < QU; ++u) {
        if (at.row + u * Place::RPP >= P.rows) break;
        codes[u] = __ldg(reinterpret_cast<const uint32_t *>(q + (int64_t)(u * Place::RPP) * P.q_pitch));
        byte[u] = __ldg(scale + Place::scale_off(u, P.tiles));
    }
#pragma unroll
    for (int u = 0; u < QU; ++u) {
        if (at.row + u * Place::RPP >= P.rows) break;
        float v[8];
        decode8(codes[u], v);
        const float s = decode_scale<BLOCK>(byte[u], g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], s);
        store8_whole<F32>(P.x, (at.row + u * Place::RPP) * P.pitch + at.ch, v);
    }
}

// Transposed: tiles of 128 voxels x 64 channels (256 x 32 where there are no more channels) through shared memory.  A thread owns one channel and
// 32 voxels of the tile, that is one block of 32 or two of 16, and writes 16 bytes of codes.
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
template <bool F32, int TC> struct TileLayout {
    static constexpr int VOX = QT / TC * 32, ES = F32 ? 4 : 2, SP = TC * ES + 16, BYTES = VOX * SP, UNITS = TC * ES / 16;
    static_assert(BYTES <= 48 * 1024, "");
};

template <bool F32, int BLOCK, int TC>
__global__ void __launch_bounds__(QT)
quant4_tile_kernel(const TileParams P)
{
    using L = TileLayout<F32, TC>;
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x;
    const int64_t r0 = (int64_t)blockIdx.x * L::VOX;
    const int c0 = blockIdx.y * TC;
#pragma unroll
    for (int i = t; i < L::VOX * L::UNITS; i += QT) {
        const int r = i / L::UNITS, u = i % L::UNITS;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r0 + r < P.voxels && c0 + u * (16 / L::ES) < P.c)
            v = __ldg(reinterpret_cast<const uint4 *>((const uint8_t *)P.x + ((r0 + r) * P.pitch + c0) * L::ES + u * 16));
        *reinterpret_cast<uint4 *>(smem + r * L::SP + u * 16) = v;
    }
    __syncthreads();
    const Divisor d(BLOCK == 16 && P.g ? __ldg(P.g) : 1.f);
    const int col = t % TC, part = t / TC, ch = c0 + col;                     // channel, 32-voxel part
    const int64_t v0 = r0 + part * 32, blocks = blocks_of(P.voxels, BLOCK), blk = v0 / BLOCK;
    uint32_t code[4], bytes = 0;
#pragma unroll
    for (int b = 0; b < 32 / BLOCK; ++b) {
        float f[BLOCK / 8][8];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < BLOCK; ++i) {
            const uint8_t *p = smem + (part * 32 + b * BLOCK + i) * L::SP + col * L::ES;
            f[i / 8][i % 8] = F32 ? *(const float *)p : bf2f(*(const bf16 *)p);
        }
#pragma unroll
        for (int i = 0; i < BLOCK / 8; ++i) m = max(m, amax_bits(f[i]));
        const Scale s = block_scale<BLOCK>(m, d);
        if (ch < P.c && blk + b < blocks) bytes |= s.byte << (8 * b);
#pragma unroll
        for (int i = 0; i < BLOCK / 8; ++i) code[b * (BLOCK / 8) + i] = encode8<BLOCK>(f[i], s);
    }
    // every block of the last tile along k and every row of a tile of rows gets its scale, 0 where there is none; the CTAs of the last channels
    // write those of the rows behind their own
    if (blk / 4 < P.tiles) {
        const int last = c0 + TC >= P.c ? (P.c + 127) / 128 * 128 : c0 + TC;
        for (int row = ch; row < last; row += TC) {
            uint8_t *o = P.scale + scale_at(row, blk, P.tiles);
            const uint32_t v = row == ch ? bytes : 0u;
            if constexpr (BLOCK == 32) *o = (uint8_t)v; else *reinterpret_cast<uint16_t *>(o) = (uint16_t)v;
        }
    }
    if (ch >= P.c || v0 >= P.voxels) return;
    uint8_t *o = P.q + (int64_t)ch * P.q_pitch + v0 / 2;
    if (P.voxels - v0 >= 32) *reinterpret_cast<uint4 *>(o) = make_uint4(code[0], code[1], code[2], code[3]);
    else {
        const int n = (int)(P.voxels - v0 + 1) / 2;                            // bytes behind the last voxel stay as they were
#pragma unroll
        for (int i = 0; i < 16; ++i) if (i < n) o[i] = (uint8_t)(code[i / 4] >> (8 * (i & 3)));
    }
}

template <bool F32, int BLOCK, int TC>
__global__ void __launch_bounds__(QT)
dequant4_tile_kernel(const TileParams P)
{
    using L = TileLayout<F32, TC>;
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x;
    const int64_t r0 = (int64_t)blockIdx.x * L::VOX;
    const int c0 = blockIdx.y * TC;
    const float g = BLOCK == 16 && P.g ? __ldg(P.g) : 1.f;
    const int col = t % TC, part = t / TC, ch = c0 + col;
    const int64_t v0 = r0 + part * 32;
    if (ch < P.c && v0 < P.voxels) {
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
                uint8_t *p = smem + (part * 32 + i * 8 + j) * L::SP + col * L::ES;
                if (F32) *(float *)p = y; else *(bf16 *)p = f2bf(y);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = t; i < L::VOX * L::UNITS; i += QT) {
        const int r = i / L::UNITS, u = i % L::UNITS;
        if (r0 + r < P.voxels && c0 + u * (16 / L::ES) < P.c)
            *reinterpret_cast<uint4 *>((uint8_t *)P.x + ((r0 + r) * P.pitch + c0) * L::ES + u * 16) = *reinterpret_cast<const uint4 *>(smem + r * L::SP + u * 16);
    }
}

template <bool F32, int BLOCK, int LPS>
lamp_status_t launch_rows_k(bool back, const RowParams &P, cudaStream_t st)
{
    const int64_t grid = (P.rows + RowPlace<LPS>::ROWS - 1) / RowPlace<LPS>::ROWS;
    // the quantiser also fills up the last tile of scales (LPS = 16: a CTA has half a tile)
    const int64_t all = (back ? grid : (P.rows + 127) / 128 * 128 > grid * RowPlace<LPS>::ROWS ? grid + 1 : grid) * P.segs;
    if (all > 2147483647ll) return LAMP_ERR_UNSUPPORTED;
    return launch_pdl(all <= 2048, back ? dequant4_rows_kernel<F32, BLOCK, LPS> : quant4_rows_kernel<F32, BLOCK, LPS>, dim3((unsigned)all), dim3(QT), 0, st, P);
}
template <bool F32, int BLOCK>
lamp_status_t launch_rows(bool back, const RowParams &P, cudaStream_t st)
{
    if (P.c <= 32) return launch_rows_k<F32, BLOCK, 4>(back, P, st);
    if (P.c <= 64) return launch_rows_k<F32, BLOCK, 8>(back, P, st);
    return launch_rows_k<F32, BLOCK, 16>(back, P, st);
}
template <bool F32, int BLOCK, int TC>
lamp_status_t launch_tiles_k(bool back, const TileParams &P, cudaStream_t st)
{
    using L = TileLayout<F32, TC>;
    const int64_t gx = (P.voxels + L::VOX - 1) / L::VOX, gy = (P.c + TC - 1) / TC;
    if (gy > 65535) return LAMP_ERR_UNSUPPORTED;
    return launch_pdl(gx * gy <= 2048, back ? dequant4_tile_kernel<F32, BLOCK, TC> : quant4_tile_kernel<F32, BLOCK, TC>, dim3((unsigned)gx, (unsigned)gy), dim3(QT),
                      (size_t)L::BYTES, st, P);
}
template <bool F32, int BLOCK>
lamp_status_t launch_tiles(bool back, const TileParams &P, cudaStream_t st)
{
    return P.c <= 32 ? launch_tiles_k<F32, BLOCK, 32>(back, P, st) : launch_tiles_k<F32, BLOCK, 64>(back, P, st);
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
        if (o->block == 32) return v.f32 ? launch_tiles<true, 32>(back, P, st) : launch_tiles<false, 32>(back, P, st);
        return v.f32 ? launch_tiles<true, 16>(back, P, st) : launch_tiles<false, 16>(back, P, st);
    }
    const RowParams P = {v.p, v.pitch, rows, v.c, (uint32_t)((v.c + 127) / 128), (uint8_t *)o->q, o->q_pitch, o->scale, tiles_of(v.c, o->block), o->tensor_scale};
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
