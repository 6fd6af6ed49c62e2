// Matrix product of two e4m3 operands with fp32 scales per block of 128 along k:
//   y[m][n] = bias[n] + sum_b ( sum_{k in block b} qa[m][k] qb[n][k] ) * sa[b][m] * sb[b][n or n/128]
//
// The scales are arbitrary fp32 numbers, so the tensor cores can only sum within a block of 128; the blocks are
// added in fp32 registers ("promotion").  One operand lies on the 128 lanes of the tensor memory, the other on BN columns.
// Two kernels: fp8_gemm_pair_kernel for products whose tiles of 256 x 256 or 256 x 128 fill three quarters of the GPU (with the
// k axis of a tile shared by two pairs where that fills it), fp8_gemm_kernel with tiles of 128 x BN for the rest.
// Per CTA, warp-specialised:
//   TMA warp      per block of k a [128 x 128 B] lane tile and a [BN x 128 B] (pair: half of it) column tile, 128-byte swizzle.
//                 Rows and bytes beyond the operand are zero-filled (code 0 = 0.0): no size has to be a multiple of the tile.
//   MMA warps     tcgen05.mma kind::f8f6f4, four instructions (K = 32 each) per block, always into a fresh accumulator; the
//                 accumulators rotate through tensor memory (NACC of them), so block b + 1 is multiplied while block b is promoted.
//   scale warp    the blocks' scales into a ring in shared memory.
//   others        promotion: tcgen05.ld of an accumulator, acc += part * scale in fp32, then the epilogue.
// A scale per column needs one more multiplication per element than a scalar one: COLVEC.
// Few rows of a (m <= 64) put b on the lanes (swap): 128 weight rows per tile, the tokens on 16..64 columns.
// Few tiles: the CTAs of a cluster share the k axis of a tile, leave their fp32 parts in their shared memory, and each adds
// a slice of the columns over all of them in rank order - no workspace, no second launch, the same order every time.
// Measured (16384 x 4096 x 4096 to bf16): 268 us in a burst (2.05 PFLOP/s), 315 us back to back under the power cap; the steps
// there are noted at the parts that made them.  512 x 2048 x 32808 to fp32, scales on both sides: 65 us.  One token through
// 4096 x 4096: 6.6 us, of which the 16.8 MB of weights are 2.6 us.
// Every mbarrier wait is bounded; on expiry the CTA records LAMP_ERR_TIMEOUT and winds down.
#include <cuda.h>
#include <cudaTypedefs.h>
#include "common.cuh"
#include "umma_ptx.cuh"

namespace lamp {

namespace {

using namespace ptx;

constexpr int KB = 128;                       // codes per scale block = bytes per shared-memory row
constexpr int MAX_STAGES = 10, MAX_ACC = 4;
constexpr int RING = 8;                       // blocks of scales in flight (Scales)
constexpr int STAGE_FLOATS = 32 * 17;         // a promotion warp's staging area for rows that are not 16-byte aligned

struct GemmParams {
    int32_t rows_l, rows_c;                   // rows of the lane operand and of the column operand
    int32_t kblocks;
    int32_t nl, nc;                           // tiles per axis
    int64_t tiles;
    int32_t splits;                           // CTAs (of one cluster) that share the blocks of a tile
    const float *sl, *sc;
    int64_t pl, pc;                           // scale pitches
    int32_t tile_l, tile_c;                   // scale per 128 rows
    const float *bias;
    void *y;
    int64_t y_pitch;
    int32_t y_f32, swap;
    int32_t vec;                              // alignment of every row's tile start: 2 = 32 bytes, 1 = 16 bytes, 0 = neither
    int *status;
};

template <int BN> struct GemmLayout {
    static constexpr int A_BYTES = 128 * KB, C_BYTES = BN * KB, STAGE_BYTES = A_BYTES + C_BYTES;
    static constexpr int STAGES = BN == 128 ? 6 : BN == 64 ? 8 : 9;
    static constexpr int NACC = 4;
    static constexpr int NEPI = BN >= 64 ? 8 : 4;                 // promotion warps
    static constexpr int CW = BN >= 64 ? BN / 2 : BN;             // columns per promotion warp
    static constexpr int ISSUERS = BN >= 64 ? 2 : 1;              // MMA-issuing threads; narrower tiles wait for memory
    static constexpr int THREADS = (2 + ISSUERS + NEPI) * 32;     // TMA, MMA, scales, promotion
    static constexpr int EPI0 = 2 + ISSUERS;                      // first promotion warp
    static constexpr int TMEM_COLS = NACC * BN;                   // 64 .. 512, a power of two
    static constexpr int SCALE_BYTES = RING * (128 + BN) * 4, OUT_BYTES = NEPI * STAGE_FLOATS * 4;
    static constexpr int BAR_BYTES = (2 * MAX_STAGES + 2 * MAX_ACC + 2 * RING) * 8 + 16;
    static constexpr int TOTAL = 1024 + STAGES * STAGE_BYTES + SCALE_BYTES + OUT_BYTES + BAR_BYTES;
    static_assert(BN * 128 * 4 <= STAGES * STAGE_BYTES, "the split-k parts reuse the stages");
    static_assert(TOTAL <= 227 * 1024 && STAGES <= MAX_STAGES && NACC <= MAX_ACC, "");
};

// Instruction descriptor: D fp32, A and B e4m3, both K-major, M = 128, N = n.
__host__ __device__ constexpr uint32_t idesc_e4m3(uint32_t n) { return (1u << 4) | ((n >> 3) << 17) | ((128u >> 4) << 24); }

__device__ __forceinline__ void umma_fp8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
// 32 lanes x 16 columns into 16 registers
__device__ __forceinline__ void tmem_ld_x16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ float ld_peer_f32(uint32_t addr, uint32_t rank)
{
    uint32_t a;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

// NV consecutive outputs of one row (columns col .. col + NV - 1, of which `left` exist)
template <int NV>
__device__ __forceinline__ void store_row(const GemmParams &P, int64_t row, int col, const float (&v)[NV])
{
    const int left = P.rows_c - col;
    if (left <= 0) return;
    if (P.y_f32) {
        float *o = (float *)P.y + row * P.y_pitch + col;
        if (NV % 4 == 0 && left >= NV && P.vec >= 1) {
            if (NV % 8 == 0 && P.vec == 2) {
#pragma unroll
                for (int j = 0; j + 8 <= NV; j += 8) {
                    uint32_t u[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(v[j + i]);
                    st_global_32B(o + j, u);
                }
            } else {
#pragma unroll
                for (int j = 0; j + 4 <= NV; j += 4) *reinterpret_cast<float4 *>(o + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j) if (j < left) o[j] = v[j];
        }
    } else {
        bf16 *o = (bf16 *)P.y + row * P.y_pitch + col;
        if (NV % 8 == 0 && left >= NV && P.vec >= 1) {
            uint32_t u[(NV + 1) / 2];
#pragma unroll
            for (int j = 0; j + 2 <= NV; j += 2) {
                __nv_bfloat162 h = __floats2bfloat162_rn(v[j], v[j + 1]);
                u[j / 2] = *reinterpret_cast<uint32_t *>(&h);
            }
            if (NV % 16 == 0 && P.vec == 2) {
#pragma unroll
                for (int j = 0; j + 16 <= NV; j += 16) {
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = u[(j / 2 + i) % ((NV + 1) / 2)];
                    st_global_32B(o + j, w);
                }
            } else {
#pragma unroll
                for (int j = 0; j + 8 <= NV; j += 8)
                    *reinterpret_cast<uint4 *>(o + j) = make_uint4(u[j / 2], u[(j / 2 + 1) % ((NV + 1) / 2)], u[(j / 2 + 2) % ((NV + 1) / 2)],
                                                                   u[(j / 2 + 3) % ((NV + 1) / 2)]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j) if (j < left) o[j] = f2bf(v[j]);
        }
    }
}

// The finished sums of NV columns of a lane row: bias, rounding, store.  Every lane of the warp takes part; row = the lane's own.
// ODD (rows that are not 16-byte aligned, or a width that is no multiple of 16): through `stage`, 32 x 17 floats of the warp, so that
// neighbouring lanes write neighbouring columns: stored by the lanes that hold them, every 4-byte store is a sector of its
// own (1407 x 2805 fp32: 29 us against 12; 16384 x 4095 bf16, k = 512: 609 against 151).  A kernel of its own: the code
// alone cost the aligned products 5 %.
template <bool ODD, int NV>
__device__ __forceinline__ void finish(const GemmParams &P, int64_t row, int col, float (&v)[NV], float *stage)
{
    if ((!ODD || P.swap) && row >= P.rows_l) return;
    if (P.swap) {                              // lanes = channels of y, columns = its voxels
        const float b = P.bias ? __ldg(P.bias + row) : 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (col + j >= P.rows_c) break;
            const int64_t at = (int64_t)(col + j) * P.y_pitch + row;
            if (P.y_f32) ((float *)P.y)[at] = v[j] + b; else ((bf16 *)P.y)[at] = f2bf(v[j] + b);
        }
        return;
    }
    if (P.bias) {
#pragma unroll
        for (int j = 0; j < NV; ++j) if (col + j < P.rows_c) v[j] += __ldg(P.bias + col + j);
    }
    if (!ODD || NV < 16) {
        if (row < P.rows_l) store_row<NV>(P, row, col, v);
        return;
    }
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < NV; ++j) stage[lane * 17 + j] = v[j];
    __syncwarp();
    const int64_t row0 = row - lane;
    const int j = lane & 15;
    if (col + j < P.rows_c) {
#pragma unroll 4
        for (int i = 0; i < 32; i += 2) {
            const int r = i + (lane >> 4);
            if (row0 + r >= P.rows_l) break;
            const int64_t at = (row0 + r) * P.y_pitch + col + j;
            const float x = stage[r * 17 + j];
            if (P.y_f32) ((float *)P.y)[at] = x; else ((bf16 *)P.y)[at] = f2bf(x);
        }
    }
    __syncwarp();
}

// Sum over the S parts of a tile (in CTAs first, first + stride, ... of the cluster) of the `mine`-th CW / S columns of this
// thread's lane row, and their store.
template <bool ODD, int CW, int S>
__device__ __forceinline__ void reduce_parts(const GemmParams &P, uint32_t part_base, int lane_row, int64_t row, int col_local, int col0, uint32_t mine,
                                             uint32_t first, uint32_t stride, float *stage)
{
    constexpr int CWS = CW / S, CH = CWS < 16 ? CWS : 16;
#pragma unroll 1
    for (int j0 = 0; j0 < CWS; j0 += CH) {
        const int cl = col_local + (int)mine * CWS + j0;
        float v[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) v[j] = 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int j = 0; j < CH; ++j) v[j] += ld_peer_f32(part_base + ((cl + j) * 128 + lane_row) * 4, first + s * stride);
        finish<ODD, CH>(P, row, col0 + cl, v, stage);
    }
}

// The scales of a block - one per lane row, and one per column (COLVEC) or one per 128 columns - come through a ring of RING
// slots in shared memory that one warp fills with asynchronous copies, ahead and across tiles; the promotion warps wait
// for a slot as they wait for an accumulator.  (Loaded by the promotion warps themselves a block ahead they cost an L2
// round trip under load, about 1300 cycles, per block of 512 tensor cycles; copied by them 480 cycles of their issue.)
template <int BN, bool COLVEC> struct Scales {
    static constexpr int SLOT = 128 + (COLVEC ? BN : 4);           // floats
    __device__ __forceinline__ static void copy4(float *dst, const float *src, bool in)
    {
        // not there: zeros, without reading
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(in ? 4 : 0) : "memory");
    }
    // every lane of one warp; row0 = first lane row of the tile in this CTA, col0 = its first column
    __device__ __forceinline__ static void fill(const GemmParams &P, float *s, int kb, int64_t row0, int64_t col0, int lane)
    {
        const float *sl = P.sl + (int64_t)kb * P.pl, *sc = P.sc + (int64_t)kb * P.pc;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t row = row0 + i * 32 + lane;
            const bool in = row < P.rows_l;
            copy4(s + i * 32 + lane, in ? sl + (P.tile_l ? row / 128 : row) : P.sl, in);
        }
        if constexpr (COLVEC) {
#pragma unroll
            for (int i = 0; i < (BN + 31) / 32; ++i) {
                const int j = i * 32 + lane;
                const bool in = col0 + j < P.rows_c;
                if (j < BN) copy4(s + 128 + j, in ? sc + col0 + j : P.sc, in);
            }
        } else if (lane < (BN + 127) / 128) {
            const int64_t col = col0 + lane * 128;
            const bool in = col < P.rows_c;
            copy4(s + 128 + lane, in ? sc + col / 128 : P.sc, in);
        }
    }
    // arrives on `bar` (count 32) once this lane's copies have landed
    __device__ __forceinline__ static void arrive(uint32_t bar)
    {
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
    }
};

// CW columns of an accumulator row (this thread's lane), times the block's scales, added to `sum`.  `done` is called once
// everything is in registers.
template <int CW, bool COLVEC, typename Done>
__device__ __forceinline__ void promote(float (&sum)[CW], uint32_t taddr, float s, const float *sc, Done done)
{
    uint32_t r[2][16];
    tmem_ld_x16(taddr, r[0]);
#pragma unroll
    for (int c = 0; c < CW / 16; ++c) {
        tmem_ld_wait();
        if (c + 1 < CW / 16) tmem_ld_x16(taddr + (c + 1) * 16, r[(c + 1) & 1]);
        else done();
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
            float w[4] = {s, s, s, s};
            if constexpr (COLVEC) {                                // products of scales two at a time (61 us on the 512 x 2048 weight gradient, 64 one by one)
                const ulonglong2 cs = *reinterpret_cast<const ulonglong2 *>(sc + c * 16 + j);
                unpack2(mul2(cs.x, twice(s)), w[0], w[1]);
                unpack2(mul2(cs.y, twice(s)), w[2], w[3]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[c * 16 + j + i] = fmaf(__uint_as_float(r[c & 1][j + i]), w[i], sum[c * 16 + j + i]);
        }
    }
}

template <int BN, bool COLVEC, bool ODD>
__global__ void __launch_bounds__(GemmLayout<BN>::THREADS, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap map_l, const __grid_constant__ CUtensorMap map_c, const GemmParams P)
{
    using L = GemmLayout<BN>;
    constexpr int STAGES = L::STAGES, NACC = L::NACC, CW = L::CW;
    constexpr uint32_t IDESC = idesc_e4m3(BN);

    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    float *scale_buf = (float *)(smem + STAGES * L::STAGE_BYTES);
    float *out_stage = (float *)(smem + STAGES * L::STAGE_BYTES + L::SCALE_BYTES);
    uint64_t *bars = (uint64_t *)(smem + STAGES * L::STAGE_BYTES + L::SCALE_BYTES + L::OUT_BYTES);
    uint32_t *tmem_slot = (uint32_t *)(bars + 2 * MAX_STAGES + 2 * MAX_ACC + 2 * RING);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + MAX_STAGES);
    const uint32_t tfull0 = smem_u32(bars + 2 * MAX_STAGES), tempty0 = smem_u32(bars + 2 * MAX_STAGES + MAX_ACC);
    const uint32_t sfull0 = smem_u32(bars + 2 * MAX_STAGES + 2 * MAX_ACC), sempty0 = sfull0 + 8 * RING;

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
        for (int a = 0; a < NACC; ++a) { mbar_init(tfull0 + 8 * a, 1); mbar_init(tempty0 + 8 * a, L::NEPI); }
        for (int a = 0; a < RING; ++a) { mbar_init(sfull0 + 8 * a, 32); mbar_init(sempty0 + 8 * a, L::NEPI); }
        *abort_flag = 0;
        mbar_init_fence();
    }
    if (warp == 1) tmem_alloc(smem_u32(tmem_slot), L::TMEM_COLS);
    pdl_wait();                 // everything above touched shared and tensor memory only
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    // with splits > 1 the grid is tiles * splits CTAs and each has one (tile, split); otherwise it walks over tiles
    const int S = P.splits;
    const uint32_t rank = S > 1 ? cluster_rank() : 0u;
    const int64_t tile0 = S > 1 ? blockIdx.x / S : blockIdx.x;
    const int64_t tile_step = S > 1 ? P.tiles : gridDim.x;
    const int kb0 = (int)((int64_t)P.kblocks * rank / S), kb1 = (int)((int64_t)P.kblocks * (rank + 1) / S);

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
                const int l0 = (int)(tile / P.nc) * 128, c0 = (int)(tile % P.nc) * BN;
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!mbar_wait(empty0 + 8 * stage, phase ^ 1, abort_flag)) { ok = false; break; }
                    const uint32_t fb = full0 + 8 * stage;
                    mbar_expect_tx(fb, L::STAGE_BYTES);
                    const uint32_t sa = smem_u32(smem + stage * L::STAGE_BYTES);
                    tma_load_2d(sa, &map_l, fb, kb * KB, l0);
                    tma_load_2d(sa + L::A_BYTES, &map_c, fb, kb * KB, c0);
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
            }
        }
        __syncwarp();
    } else if (warp <= L::ISSUERS) {
        // ------------------------------------------------------------------ MMA issuers, for every ISSUERS-th block
        if (lane == 0) {
            constexpr int NI = L::ISSUERS;
            const int64_t mine = tile0 < P.tiles ? (P.tiles - tile0 + tile_step - 1) / tile_step * (kb1 - kb0) : 0;
            int stage = (warp - 1) % STAGES;
            uint32_t phase = 0, acc = warp - 1, acc_phase = 0;
            for (int64_t n = warp - 1; n < mine; n += NI) {
                if (!mbar_wait(tempty0 + 8 * acc, acc_phase ^ 1, abort_flag)) break;
                if (!mbar_wait(full0 + 8 * stage, phase, abort_flag)) break;
                tc_fence_after();
                const uint32_t sa = smem_u32(smem + stage * L::STAGE_BYTES);
                const uint64_t da = make_desc(sa, 0, 8 * KB, 2), dc = make_desc(sa + L::A_BYTES, 0, 8 * KB, 2);
#pragma unroll
                for (int k = 0; k < KB / 32; ++k)            // 32 codes = 32 bytes = 2 descriptor address units
                    umma_fp8(tmem_base + acc * BN, da + 2 * k, dc + 2 * k, IDESC, k ? 1u : 0u);
                umma_commit(empty0 + 8 * stage);             // frees the stage once these MMAs have read it
                umma_commit(tfull0 + 8 * acc);               // the block's sums are complete
                if ((stage += NI) >= STAGES) { stage -= STAGES; phase ^= 1; }
                if ((acc += NI) >= NACC) { acc -= NACC; acc_phase ^= 1; }
            }
        }
        __syncwarp();
    } else if (warp == L::ISSUERS + 1) {
        // ------------------------------------------------------------------ scales
        uint32_t n = 0;
        bool ok = true;
        for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
            const int64_t row0 = (tile / P.nc) * 128, col0 = (tile % P.nc) * BN;
            for (int kb = kb0; kb < kb1; ++kb, ++n) {
                const uint32_t slot = n % RING;
                ok = __all_sync(0xffffffffu, mbar_wait(sempty0 + 8 * slot, ((n / RING) & 1) ^ 1, abort_flag));
                if (!ok) break;
                Scales<BN, COLVEC>::fill(P, scale_buf + slot * Scales<BN, COLVEC>::SLOT, kb, row0, col0, lane);
                Scales<BN, COLVEC>::arrive(sfull0 + 8 * slot);
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        // ------------------------------------------------------------------ promotion
        const int q = warp & 3, half = (warp - L::EPI0) >> 2;              // lane quarter and column part of this warp
        float *stage = out_stage + (warp - L::EPI0) * STAGE_FLOATS;
        const int lane_row = q * 32 + lane;
        uint32_t acc = 0, acc_phase = 0, n = 0;
        bool ok = true;
        for (int64_t tile = tile0; tile < P.tiles; tile += tile_step) {
            const int64_t row = (tile / P.nc) * 128 + lane_row;
            const int cbase = (int)(tile % P.nc) * BN + half * CW;
            float sum[CW];
#pragma unroll
            for (int i = 0; i < CW; ++i) sum[i] = 0.f;
            for (int kb = kb0; kb < kb1; ++kb, ++n) {
                const uint32_t slot = n % RING;
                const float *sv = scale_buf + slot * Scales<BN, COLVEC>::SLOT, *sc = sv + 128 + (COLVEC ? half * CW : half * CW / 128);
                ok = ok && __all_sync(0xffffffffu, mbar_wait(sfull0 + 8 * slot, (n / RING) & 1, abort_flag));
                ok = ok && __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * acc, acc_phase, abort_flag));
                if (!ok) break;
                tc_fence_after();
                promote<CW, COLVEC>(sum, tmem_base + ((uint32_t)(q * 32) << 16) + acc * BN + half * CW, COLVEC ? sv[lane_row] : sv[lane_row] * sc[0], sc, [&]() {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(tempty0 + 8 * acc);
                });
                __syncwarp();
                if (lane == 0) mbar_arrive(sempty0 + 8 * slot);
                if (++acc == NACC) { acc = 0; acc_phase ^= 1; }
            }
            if (S == 1) {
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < CW / 16; ++c) {
                    float v[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = sum[c * 16 + j];
                    finish<ODD, 16>(P, row, cbase + c * 16, v, stage);
                }
            } else {
                // every stage of this CTA has been read: its memory takes the parts, [column][lane row]
                float *part = (float *)smem;
#pragma unroll
                for (int j = 0; j < CW; ++j) part[(half * CW + j) * 128 + lane_row] = sum[j];
            }
        }
        if (!ok) {
            if (lane == 0 && P.status) atomicExch(P.status, (int)LAMP_ERR_TIMEOUT);
            settle();                                           // copies in flight
        }
    }
    __syncwarp();
    if (S > 1) {
        cluster_sync_all();
        if (warp >= L::EPI0) {
            const int q = warp & 3, half = (warp - L::EPI0) >> 2, lane_row = q * 32 + lane;
            float *stage = out_stage + (warp - L::EPI0) * STAGE_FLOATS;
            const int64_t row = (tile0 / P.nc) * 128 + lane_row;
            const int col0 = (int)(tile0 % P.nc) * BN;
            const uint32_t base = smem_u32(smem);
            if (S == 2) reduce_parts<ODD, CW, 2>(P, base, lane_row, row, half * CW, col0, rank, 0, 1, stage);
            else if (S == 4) reduce_parts<ODD, CW, 4>(P, base, lane_row, row, half * CW, col0, rank, 0, 1, stage);
            else reduce_parts<ODD, CW, 8>(P, base, lane_row, row, half * CW, col0, rank, 0, 1, stage);
        }
        cluster_sync_all();      // no CTA leaves while a peer still reads its parts
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem_base, L::TMEM_COLS);
}

bool encode_operand(const lamp_fp8_operand_t *o, int box_rows, CUtensorMap *map)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = (PFN_cuTensorMapEncodeTiled_v12000)tensor_map_encoder();
    if (!enc) return false;
    const cuuint64_t gdim[2] = {(cuuint64_t)o->k, (cuuint64_t)o->rows};
    const cuuint64_t gstride[1] = {(cuuint64_t)o->q_pitch};
    const cuuint32_t box[2] = {(cuuint32_t)KB, (cuuint32_t)box_rows};
    const cuuint32_t es[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, o->q, gdim, gstride, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// ----------------------------------------------------------------------------------------------------------------------
// CTA pairs: tiles of 256 x BN, each CTA of the pair 128 lane rows (its tensor memory) and half of the columns' operand
// ----------------------------------------------------------------------------------------------------------------------
// What bounds the product of large operands is the path from L2 to shared memory: a 128 x 256 tile of one CTA takes 48 KB per
// block of k, and 148 SMs took 11 TB/s at most (16384 x 4096 x 4096: 284 us with the promotion left out).  A pair shares the column
// operand: 32 KB per CTA for the same work.  The leader (rank 0) issues the MMAs of both CTAs; full barriers live in the
// leader (both CTAs' copies complete there), empty and accumulator-full barriers in each CTA (the commits arrive in both),
// accumulator-empty barriers in the leader (the promotion warps of both CTAs arrive).
// Warps 4 .. 11 promote: 128 sums per thread, 32 loaded values and their addresses need 216 registers, which the other four warps
// give up (384 x 168 at launch = 128 x 72 + 256 x 216).
template <int BN> struct PairLayout {
    static constexpr int A_BYTES = 128 * KB, C_BYTES = BN / 2 * KB, STAGE_BYTES = A_BYTES + C_BYTES;
    static constexpr int STAGES = BN == 256 ? 6 : 8;
    static constexpr int NACC = BN == 256 ? 2 : 4;
    static constexpr int CW = BN / 2;                             // columns per promotion warp
    static constexpr int THREADS = 384, TMEM_COLS = 512;
    static constexpr int SCALE_BYTES = RING * (128 + BN) * 4, OUT_BYTES = 8 * STAGE_FLOATS * 4;
    static constexpr int BAR_BYTES = (2 * MAX_STAGES + 2 * MAX_ACC + 2 * RING) * 8 + 16;
    static constexpr int TOTAL = 1024 + STAGES * STAGE_BYTES + SCALE_BYTES + OUT_BYTES + BAR_BYTES;
    static_assert(BN * 128 * 4 <= STAGES * STAGE_BYTES, "the split-k parts reuse the stages");
    static_assert(TOTAL <= 227 * 1024 && STAGES <= MAX_STAGES && NACC <= MAX_ACC && NACC * BN <= TMEM_COLS, "");
};

__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap *map, uint32_t leader_bar, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(leader_bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void umma_fp8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives on the barrier of this offset in the CTAs of the mask once the MMAs issued so far have completed
__device__ __forceinline__ void umma_commit_pair(uint32_t bar, uint32_t ctas)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)ctas) : "memory");
}
// Arrival on a barrier of either CTA.  No release at cluster scope: what it hands over is tensor memory that has been read,
// not memory that was written, and that release is a fence that waits for everything the thread has in flight - it took
// 1200 cycles per block of k, three quarters of the kernel's time.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

template <int BN, bool COLVEC, bool ODD>
__global__ void __launch_bounds__(PairLayout<BN>::THREADS, 1)
fp8_gemm_pair_kernel(const __grid_constant__ CUtensorMap map_l, const __grid_constant__ CUtensorMap map_c, const GemmParams P)
{
    using L = PairLayout<BN>;
    constexpr int STAGES = L::STAGES, NACC = L::NACC, CW = L::CW;
    constexpr uint32_t IDESC = (1u << 4) | ((uint32_t)(BN >> 3) << 17) | ((256u >> 4) << 24);

    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    float *scale_buf = (float *)(smem + STAGES * L::STAGE_BYTES);
    float *out_stage = (float *)(smem + STAGES * L::STAGE_BYTES + L::SCALE_BYTES);
    uint64_t *bars = (uint64_t *)(smem + STAGES * L::STAGE_BYTES + L::SCALE_BYTES + L::OUT_BYTES);
    uint32_t *tmem_slot = (uint32_t *)(bars + 2 * MAX_STAGES + 2 * MAX_ACC + 2 * RING);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // a cluster is S (1 or 2) pairs that share the blocks of k of one tile; the even CTA of a pair leads it
    const uint32_t cta = cluster_rank(), rank = cta & 1, leader = cta & ~1u;
    const int S = P.splits;
    const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + MAX_STAGES);
    const uint32_t tfull0 = smem_u32(bars + 2 * MAX_STAGES), tempty0 = smem_u32(bars + 2 * MAX_STAGES + MAX_ACC);
    const uint32_t sfull0 = smem_u32(bars + 2 * MAX_STAGES + 2 * MAX_ACC), sempty0 = sfull0 + 8 * RING;

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
        for (int a = 0; a < NACC; ++a) { mbar_init(tfull0 + 8 * a, 1); mbar_init(tempty0 + 8 * a, 16); }
        for (int a = 0; a < RING; ++a) { mbar_init(sfull0 + 8 * a, 32); mbar_init(sempty0 + 8 * a, 8); }
        *abort_flag = 0;
        mbar_init_fence();
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(L::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    cluster_sync_all();          // the peer's barriers exist
    pdl_wait();                  // everything above touched shared and tensor memory only
    const uint32_t tmem_base = *tmem_slot;
    const int64_t tile0 = S > 1 ? blockIdx.x / (2 * S) : blockIdx.x >> 1, tile_step = S > 1 ? P.tiles : gridDim.x >> 1;
    const int split = (int)(cta >> 1), kb0 = (int)((int64_t)P.kblocks * split / S), kb1 = (int)((int64_t)P.kblocks * (split + 1) / S);
    bool ok = true;

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 0 && lane == 0) {
            // -------------------------------------------------------------- TMA producer, one per CTA
            int stage = 0;
            uint32_t phase = 0;
            for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
                const int l0 = (int)(tile / P.nc) * 256 + (int)rank * 128, c0 = (int)(tile % P.nc) * BN + (int)rank * (BN / 2);
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!mbar_wait(empty0 + 8 * stage, phase ^ 1, abort_flag)) { ok = false; break; }
                    const uint32_t fb = map_to_rank(full0 + 8 * stage, leader);
                    if (rank == 0) mbar_expect_tx(full0 + 8 * stage, 2 * L::STAGE_BYTES);
                    const uint32_t sa = smem_u32(smem + stage * L::STAGE_BYTES);
                    tma_load_2d_pair(sa, &map_l, fb, kb * KB, l0);
                    tma_load_2d_pair(sa + L::A_BYTES, &map_c, fb, kb * KB, c0);
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
            }
        } else if ((warp == 1 || warp == 2) && lane == 0 && rank == 0) {
            // -------------------------------------------------------------- MMA issuers, in the leader
            // Two, for alternate blocks: one thread takes about 120 cycles per MMA to issue and 300 for the two waits of a
            // block, 780 together where the tensor cores need 512.
            const int64_t mine = tile0 < P.tiles ? (P.tiles - tile0 + tile_step - 1) / tile_step * (kb1 - kb0) : 0;
            int stage = warp - 1;
            uint32_t phase = 0, acc = warp - 1, acc_phase = 0;
            for (int64_t n = warp - 1; n < mine; n += 2) {
                if (!mbar_wait(tempty0 + 8 * acc, acc_phase ^ 1, abort_flag)) { ok = false; break; }
                if (!mbar_wait(full0 + 8 * stage, phase, abort_flag)) { ok = false; break; }
                tc_fence_after();
                const uint32_t sa = smem_u32(smem + stage * L::STAGE_BYTES);
                const uint64_t da = make_desc(sa, 0, 8 * KB, 2), dc = make_desc(sa + L::A_BYTES, 0, 8 * KB, 2);
#pragma unroll
                for (int k = 0; k < KB / 32; ++k)
                    umma_fp8_pair(tmem_base + acc * BN, da + 2 * k, dc + 2 * k, IDESC, k ? 1u : 0u);
                // nobody waits for the last arrivals of the empty barriers in the other CTA; the accumulator's commit behind them,
                // which its promotion warps do wait for, completes after them, so they land before that CTA leaves
                umma_commit_pair(empty0 + 8 * stage, 3u << leader);
                umma_commit_pair(tfull0 + 8 * acc, 3u << leader);
                if ((stage += 2) >= STAGES) { stage -= STAGES; phase ^= 1; }
                if ((acc += 2) >= NACC) { acc -= NACC; acc_phase ^= 1; }
            }
        }
        else if (warp == 3) {
            // -------------------------------------------------------------- scales
            uint32_t n = 0;
            for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
                const int64_t row0 = (tile / P.nc) * 256 + rank * 128, col0 = (tile % P.nc) * BN;
                for (int kb = kb0; kb < kb1; ++kb, ++n) {
                    const uint32_t slot = n % RING;
                    ok = __all_sync(0xffffffffu, mbar_wait(sempty0 + 8 * slot, ((n / RING) & 1) ^ 1, abort_flag));
                    if (!ok) break;
                    Scales<BN, COLVEC>::fill(P, scale_buf + slot * Scales<BN, COLVEC>::SLOT, kb, row0, col0, lane);
                    Scales<BN, COLVEC>::arrive(sfull0 + 8 * slot);
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ promotion
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int q = warp & 3, half = (warp - 4) >> 2;
        const int lane_row = q * 32 + lane;
        float *stage = out_stage + (warp - 4) * STAGE_FLOATS;
        uint32_t acc = 0, acc_phase = 0, n = 0;
        const uint32_t tempty_leader = map_to_rank(tempty0, leader);
        for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
            const int64_t row = (tile / P.nc) * 256 + rank * 128 + lane_row;
            const int cbase = (int)(tile % P.nc) * BN + half * CW;
            float sum[CW];
#pragma unroll
            for (int i = 0; i < CW; ++i) sum[i] = 0.f;
            for (int kb = kb0; kb < kb1; ++kb, ++n) {
                const uint32_t slot = n % RING;
                const float *sv = scale_buf + slot * Scales<BN, COLVEC>::SLOT, *sc = sv + 128 + (COLVEC ? half * CW : half * CW / 128);
                ok = __all_sync(0xffffffffu, mbar_wait(sfull0 + 8 * slot, (n / RING) & 1, abort_flag));
                ok = ok && __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * acc, acc_phase, abort_flag));
                if (!ok) break;
                tc_fence_after();
                promote<CW, COLVEC>(sum, tmem_base + ((uint32_t)(q * 32) << 16) + acc * BN + half * CW, COLVEC ? sv[lane_row] : sv[lane_row] * sc[0], sc, [&]() {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(tempty_leader + 8 * acc);
                });
                __syncwarp();
                if (lane == 0) mbar_arrive(sempty0 + 8 * slot);
                if (++acc == NACC) { acc = 0; acc_phase ^= 1; }
            }
            if (S > 1) {
                // every stage has been read: its memory takes the parts, [column][lane row]
                float *part = (float *)smem;
#pragma unroll
                for (int j = 0; j < CW; ++j) part[(half * CW + j) * 128 + lane_row] = sum[j];
                break;
            }
            if (!ok) break;
#pragma unroll
            for (int c = 0; c < CW / 16; ++c) {
                float v[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = sum[c * 16 + j];
                finish<ODD, 16>(P, row, cbase + c * 16, v, stage);
            }
        }
    }
    if (!ok) {
        if (P.status) atomicExch(P.status, (int)LAMP_ERR_TIMEOUT);
        settle();                                                  // copies in flight
    }
    if (S > 1) {
        cluster_sync_all();
        if (warp >= 4) {
            const int q = warp & 3, half = (warp - 4) >> 2, lane_row = q * 32 + lane;
            float *stage = out_stage + (warp - 4) * STAGE_FLOATS;
            const int64_t row = (tile0 / P.nc) * 256 + rank * 128 + lane_row;
            const int col0 = (int)(tile0 % P.nc) * BN;
            const uint32_t base = smem_u32(smem);
            reduce_parts<ODD, CW, 2>(P, base, lane_row, row, half * CW, col0, split, rank, 2, stage);
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();          // no CTA leaves, or frees tensor memory, while the other still uses what is its own
    tc_fence_after();
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(L::TMEM_COLS) : "memory");
}

template <int BN, bool COLVEC, bool ODD>
lamp_status_t launch_pair_k(const lamp_fp8_operand_t *l, const lamp_fp8_operand_t *c, const GemmParams &P, cudaStream_t st)
{
    using L = PairLayout<BN>;
    CUtensorMap ml, mc;
    if (!encode_operand(l, 128, &ml) || !encode_operand(c, BN / 2, &mc)) return LAMP_ERR_CUDA;
    static SmemAttrOnce attr;
    { const lamp_status_t as = attr.ensure(fp8_gemm_pair_kernel<BN, COLVEC, ODD>, (int)L::TOTAL); if (as != LAMP_OK) return as; }
    const int64_t pairs = sm_count() / 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (unsigned)(P.splits > 1 ? P.tiles * P.splits : P.tiles < pairs ? P.tiles : pairs));
    cfg.blockDim = dim3(L::THREADS);
    cfg.dynamicSmemBytes = L::TOTAL;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2 * P.splits; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = P.tiles <= 4 * pairs ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, fp8_gemm_pair_kernel<BN, COLVEC, ODD>, ml, mc, P) == cudaSuccess ? LAMP_OK : LAMP_ERR_CUDA;
}

template <int BN, bool COLVEC, bool ODD>
lamp_status_t launch(const lamp_fp8_operand_t *l, const lamp_fp8_operand_t *c, const GemmParams &P, cudaStream_t st)
{
    using L = GemmLayout<BN>;
    CUtensorMap ml, mc;
    if (!encode_operand(l, 128, &ml) || !encode_operand(c, BN, &mc)) return LAMP_ERR_CUDA;
    static SmemAttrOnce attr;
    { const lamp_status_t as = attr.ensure(fp8_gemm_kernel<BN, COLVEC, ODD>, (int)L::TOTAL); if (as != LAMP_OK) return as; }
    const int sms = sm_count();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(P.splits > 1 ? (unsigned)(P.tiles * P.splits) : (unsigned)(P.tiles < sms ? P.tiles : sms));
    cfg.blockDim = dim3(L::THREADS);
    cfg.dynamicSmemBytes = L::TOTAL;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    int na = 0;
    if (P.tiles <= 4 * (int64_t)sms) {
        at[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[na++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (P.splits > 1) {
        at[na].id = cudaLaunchAttributeClusterDimension;
        at[na].val.clusterDim.x = P.splits;
        at[na].val.clusterDim.y = 1;
        at[na++].val.clusterDim.z = 1;
    }
    cfg.attrs = at;
    cfg.numAttrs = na;
    return cudaLaunchKernelEx(&cfg, fp8_gemm_kernel<BN, COLVEC, ODD>, ml, mc, P) == cudaSuccess ? LAMP_OK : LAMP_ERR_CUDA;
}

bool odd_rows(const GemmParams &P) { return !P.swap && (P.vec == 0 || P.rows_c % 16 != 0); }
template <int BN>
lamp_status_t launch_cv(const lamp_fp8_operand_t *l, const lamp_fp8_operand_t *c, const GemmParams &P, cudaStream_t st)
{
    if (odd_rows(P)) return c->tile_scale ? launch<BN, false, true>(l, c, P, st) : launch<BN, true, true>(l, c, P, st);
    return c->tile_scale ? launch<BN, false, false>(l, c, P, st) : launch<BN, true, false>(l, c, P, st);
}
template <int BN>
lamp_status_t launch_pair(const lamp_fp8_operand_t *l, const lamp_fp8_operand_t *c, const GemmParams &P, cudaStream_t st)
{
    if (odd_rows(P)) return c->tile_scale ? launch_pair_k<BN, false, true>(l, c, P, st) : launch_pair_k<BN, true, true>(l, c, P, st);
    return c->tile_scale ? launch_pair_k<BN, false, false>(l, c, P, st) : launch_pair_k<BN, true, false>(l, c, P, st);
}

// Clusters of `ctas` CTAs, one CTA per SM, that run at once: the SMs of a cluster belong to one GPC, so not every SM finds a
// place.  (148 SMs: 74 clusters of 2, 33 of 4, 15 of 8; one cluster more than that is a second wave - 141 us against 71 for a
// weight gradient of 512 x 2048 outputs.)
int64_t cluster_room(int sms, int ctas) { return ctas <= 2 ? sms / ctas : ctas == 4 ? sms * 2 / 9 : sms / 10; }

}  // namespace

lamp_status_t check_fp8_operand(const lamp_fp8_operand_t *o)
{
    if (!o || o->rows < 0 || o->k < 0) return LAMP_ERR_INVALID_ARG;
    if (o->tile_scale != 0 && o->tile_scale != 1) return LAMP_ERR_INVALID_ARG;
    if (o->rows > 2147483647ll - 256 || o->k > 2147483647ll - 256) return LAMP_ERR_UNSUPPORTED;
    if (o->q_pitch < o->k || (o->q_pitch & 15) || o->scale_pitch < (o->tile_scale ? (o->rows + 127) / 128 : o->rows)) return LAMP_ERR_INVALID_ARG;
    if ((double)o->rows * (double)o->q_pitch > 1099511627776.0) return LAMP_ERR_UNSUPPORTED;       // 2^40 B
    if ((double)o->scale_pitch * (double)((o->k + 127) / 128) > 1099511627776.0 / 4) return LAMP_ERR_UNSUPPORTED;
    if (o->rows == 0 || o->k == 0) return LAMP_OK;
    if (!o->q || !o->scale || ((uintptr_t)o->q & 15) || ((uintptr_t)o->scale & 3)) return LAMP_ERR_INVALID_ARG;
    return LAMP_OK;
}

}  // namespace lamp

using namespace lamp;

extern "C" lamp_status_t lamp_gemm_fp8(const lamp_fp8_operand_t *a, const lamp_fp8_operand_t *b, const float *bias, lamp_tensor_t *y,
                                       void *cuda_stream)
{
    lamp_status_t s;
    if ((s = check_fp8_operand(a)) != LAMP_OK || (s = check_fp8_operand(b)) != LAMP_OK) return s;
    if ((s = check_view(y, true)) != LAMP_OK) return s;
    if (a->k != b->k || a->k == 0 || voxels(y) != a->rows || (int64_t)y->c != b->rows || ((uintptr_t)bias & 3)) return LAMP_ERR_INVALID_ARG;
    if (a->rows == 0) return LAMP_OK;
    const TView v = make_view(y);

    GemmParams P = {};
    const bool swap = a->rows <= 64 && b->rows > a->rows;
    const lamp_fp8_operand_t *l = swap ? b : a, *c = swap ? a : b;
    P.rows_l = (int32_t)l->rows; P.rows_c = (int32_t)c->rows;
    P.kblocks = (int32_t)((a->k + KB - 1) / KB);
    P.sl = l->scale; P.sc = c->scale; P.pl = l->scale_pitch; P.pc = c->scale_pitch;
    P.tile_l = l->tile_scale; P.tile_c = c->tile_scale;
    P.bias = bias; P.y = v.p; P.y_pitch = v.pitch; P.y_f32 = v.f32; P.swap = swap;
    const size_t es = v.f32 ? 4 : 2;
    const uintptr_t mis = (uintptr_t)v.p | (uintptr_t)(v.pitch * es);
    P.vec = (mis & 31) == 0 ? 2 : (mis & 15) == 0 ? 1 : 0;
    P.status = status_word_ptr();
    const int sms = sm_count();
    P.nl = (P.rows_l + 127) / 128;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    P.splits = 1;
    // pairs where their tiles fill the GPU
    for (int bn = 256; bn >= 128; bn /= 2) {
        const int64_t nl = (P.rows_l + 255) / 256, nc = (P.rows_c + bn - 1) / bn;
        if (swap || P.rows_c < bn) continue;
        int splits = 1;
        if (nl * nc <= cluster_room(sms, 4) && P.kblocks >= 16) splits = 2;
        if (nl * nc * splits * 2 < sms * 3 / 4) continue;
        P.splits = splits;
        P.nl = (int32_t)nl; P.nc = (int32_t)nc; P.tiles = nl * nc;
        return bn == 256 ? launch_pair<256>(l, c, P, st) : launch_pair<128>(l, c, P, st);
    }
    const int bn = P.rows_c <= 16 ? 16 : P.rows_c <= 32 ? 32 : P.rows_c <= 64 ? 64 : 128;
    P.nc = (P.rows_c + bn - 1) / bn;
    P.tiles = (int64_t)P.nl * P.nc;
    while (P.splits < 8 && P.tiles <= cluster_room(sms, 2 * P.splits) && P.kblocks >= 4 * P.splits) P.splits *= 2;
    switch (bn) {
    case 16: return launch_cv<16>(l, c, P, st);
    case 32: return launch_cv<32>(l, c, P, st);
    case 64: return launch_cv<64>(l, c, P, st);
    default: return launch_cv<128>(l, c, P, st);
    }
}
