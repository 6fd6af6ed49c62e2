// Matrix product of two 4-bit operands with a scale per block of 32 or 16 along k, applied by the tensor cores:
//   y[m][n] = bias[n] + ga gb sum_k qa[m][k] sa[m][k / block] qb[n][k] sb[n][k / block]
//
// tcgen05.mma kind::mxf4 (blocks of 32, e8m0) or kind::mxf4nvf4 (blocks of 16, e4m3) multiplies 64 codes per instruction and takes the scales from
// tensor memory; the sum over all of k stays in one fp32 accumulator there.  The scales lie in memory as tensor memory takes
// them: 128 rows x 4 blocks are 512 bytes, [row % 32][row / 32][block]; tcgen05.cp puts them on 4 columns (row % 32 = lane, repeated for
// the four lane quarters).  One operand lies on the 128 lanes of the accumulator, the other on BN columns.
// Two kernels: fp4_gemm_pair_kernel for products whose tiles of 256 x 256 or 256 x 128 fill three quarters of the GPU,
// fp4_gemm_kernel with tiles of 128 x BN for the rest (the CTAs of a cluster share the k axis of a tile where tiles are few).
// Per CTA, warp-specialised:
//   TMA warp   per 256 codes of k: [128 x 128 B] of the lane operand, [BN x 128 B] of the column operand (pair: half of it), 128-byte swizzle, and
//              the scales of both.  What lies beyond an operand is zero-filled: no size has to be a multiple of the tile.
//   MMA warp   one thread: scales to tensor memory (a place per stage, so that nothing is overwritten that an MMA may still read),
//              four MMAs of 64 codes, commit.
//   others     epilogue.
// Few rows of a (m <= 64) put b on the lanes (swap): 128 weight rows per tile, the tokens on 16..64 columns.
// Measured (blocks of 16, to bf16): 16384 x 4096 x 4096 107 us in a burst (5.1 PFLOP/s), 127 back to back under the power cap; its main loop, 256 codes
// of a tile of 256 x 256 in 0.39 us, is bound by the path from L2 (38 KB per CTA and stage: 15 TB/s for the GPU; without the loads 96 us, without the
// scale copies no faster), and each tile waits 1.7 us for its accumulator to be emptied, of which the scales leave room for one.  One token
// through 4096 x 4096: 5.0 us; 512 x 2048 x 32808 to fp32 27 us.
// Every mbarrier wait is bounded; on expiry the CTA records LAMP_ERR_TIMEOUT and winds down.
#include <cuda.h>
#include <cudaTypedefs.h>
#include "fp4.cuh"
#include "gemm_out.cuh"

namespace lamp {

namespace {

using namespace ptx;
using namespace gemm;

constexpr int KB = 128;                       // bytes of a shared-memory row: 256 codes, a stage of k
constexpr int KCODES = 256, STEPS = KCODES / 64;
constexpr int MAX_STAGES = 8;

struct GemmParams : OutParams {
    int32_t kblocks;
    int32_t nl, nc;                           // tiles per axis
    int64_t tiles;
    int32_t splits;                           // CTAs (of one cluster) that share the blocks of a tile
    const float *ga, *gb;
    int *status;
};

template <int BLOCK> struct Kind {
    static constexpr int ATOMS = KCODES / (4 * BLOCK);             // scale tiles of a stage: 4 columns each per 128 rows
    static constexpr int BYTES = ATOMS * 512;                      // per 128 rows
    static constexpr int COLS = ATOMS * 4;
};

// Instruction descriptor: D fp32, A and B e2m1, both K-major; scale type e8m0 (bit 23) or e4m3; ids of the scales within a 32-bit column.
template <int BLOCK> __host__ __device__ constexpr uint32_t idesc_e2m1(uint32_t m, uint32_t n, uint32_t id)
{
    return (id << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | ((BLOCK == 32 ? 1u : 0u) << 23) | ((m >> 7) << 27) | (id << 29);
}

#define LAMP_FP4_MMA(GROUP, KIND, VEC)                                                                                                     \
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"                                                                               \
                 "tcgen05.mma.cta_group::" GROUP ".kind::" KIND ".block_scale.scale_vec::" VEC " [%0], %1, %2, %3, [%4], [%5], p;\n}"      \
                 ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory")
template <int GROUP, int BLOCK>
__device__ __forceinline__ void umma_fp4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate)
{
    if constexpr (GROUP == 1 && BLOCK == 32) LAMP_FP4_MMA("1", "mxf4", "2X");
    if constexpr (GROUP == 1 && BLOCK == 16) LAMP_FP4_MMA("1", "mxf4nvf4", "4X");
    if constexpr (GROUP == 2 && BLOCK == 32) LAMP_FP4_MMA("2", "mxf4", "2X");
    if constexpr (GROUP == 2 && BLOCK == 16) LAMP_FP4_MMA("2", "mxf4nvf4", "4X");
}
// True in one lane of the warp.  The issuing loops run in the whole warp and only the tcgen05 instructions under this predicate: their
// descriptors then stay in uniform registers.
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(p));
    return p != 0;
}
// 512 bytes of scales from shared memory to 4 columns
template <int GROUP> __device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint64_t sdesc)
{
    if constexpr (GROUP == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
}
__device__ __forceinline__ uint64_t scale_desc(uint32_t saddr) { return make_desc(saddr, 0, 128, 0); }

// One stage: scales of `a_addr` (one tile of rows) and `c_addr` (CT tiles of rows, [row tile][atom][512]) to their columns, then the MMAs.
// Columns of the column operand: for each atom the row tiles side by side, as one instruction reads them.
template <int GROUP, int BLOCK, int M, int BN>
__device__ __forceinline__ void stage_mmas(uint32_t acc, uint32_t sf, uint32_t sa, uint32_t sc, uint32_t ssa, uint32_t ssc, bool first)
{
    using K = Kind<BLOCK>;
    constexpr int CT = (BN + 127) / 128;
#pragma unroll
    for (int a = 0; a < K::ATOMS; ++a) {
        scales_to_tmem<GROUP>(sf + a * 4, scale_desc(ssa + a * 512));
#pragma unroll
        for (int t = 0; t < CT; ++t) scales_to_tmem<GROUP>(sf + K::COLS + (a * CT + t) * 4, scale_desc(ssc + (t * K::ATOMS + a) * 512));
    }
    const uint64_t da = make_desc(sa, 0, 8 * KB, 2), dc = make_desc(sc, 0, 8 * KB, 2);
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {                             // 64 codes = 32 bytes = 2 descriptor address units
        const int a = BLOCK == 32 ? k / 2 : k;
        const uint32_t id = BLOCK == 32 ? (k & 1) * 2 : 0;        // blocks of 32: two of a column's four scales per instruction
        umma_fp4<GROUP, BLOCK>(acc, da + 2 * k, dc + 2 * k, idesc_e2m1<BLOCK>(M, BN, id), sf + a * 4, sf + K::COLS + a * CT * 4, (first && k == 0) ? 0u : 1u);
    }
}

// ----------------------------------------------------------------------------------------------------------------------
// one CTA per tile of 128 x BN
// ----------------------------------------------------------------------------------------------------------------------
template <int BN, int BLOCK> struct GemmLayout {
    static constexpr int A_BYTES = 128 * KB, C_BYTES = BN * KB, S_BYTES = Kind<BLOCK>::BYTES;
    static constexpr int STAGE_BYTES = A_BYTES + C_BYTES + 2 * S_BYTES;
    static constexpr int STAGES = BN == 128 ? 5 : 7;
    static constexpr int NACC = 2;
    static constexpr int NEPI = BN >= 64 ? 8 : 4;                 // epilogue warps
    static constexpr int CW = BN >= 64 ? BN / 2 : BN;             // columns per epilogue warp
    static constexpr int THREADS = (2 + NEPI) * 32;
    static constexpr int SF0 = NACC * BN, SFC = 2 * Kind<BLOCK>::COLS;
    static constexpr int TMEM_COLS = 512;
    static constexpr int STAGE_WORDS = BN == 128 ? BOX_WORDS : STAGE_FLOATS;
    static constexpr int OUT_BYTES = NEPI * STAGE_WORDS * 4;
    static constexpr int BAR_BYTES = (2 * MAX_STAGES + 2 * NACC) * 8 + 16;
    static constexpr int TOTAL = 1024 + STAGES * STAGE_BYTES + OUT_BYTES + BAR_BYTES;
    static_assert(BN * 128 * 4 <= STAGES * STAGE_BYTES, "the split-k parts reuse the stages");
    static_assert(STAGE_BYTES % 1024 == 0, "128-byte swizzle");
    static_assert(SF0 + STAGES * SFC <= TMEM_COLS, "");
    static_assert(TOTAL <= 227 * 1024 && STAGES <= MAX_STAGES, "");
};

template <int BN, int BLOCK, bool ODD>
__global__ void __launch_bounds__(GemmLayout<BN, BLOCK>::THREADS, 1)
fp4_gemm_kernel(const __grid_constant__ CUtensorMap map_l, const __grid_constant__ CUtensorMap map_c, const __grid_constant__ CUtensorMap map_sl,
                const __grid_constant__ CUtensorMap map_sc, const GemmParams P)
{
    using L = GemmLayout<BN, BLOCK>;
    constexpr int STAGES = L::STAGES, NACC = L::NACC, CW = L::CW;

    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    float *out_stage = (float *)(smem + STAGES * L::STAGE_BYTES);
    uint64_t *bars = (uint64_t *)(smem + STAGES * L::STAGE_BYTES + L::OUT_BYTES);
    uint32_t *tmem_slot = (uint32_t *)(bars + 2 * MAX_STAGES + 2 * NACC);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + MAX_STAGES);
    const uint32_t tfull0 = smem_u32(bars + 2 * MAX_STAGES), tempty0 = smem_u32(bars + 2 * MAX_STAGES + NACC);

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
        for (int a = 0; a < NACC; ++a) { mbar_init(tfull0 + 8 * a, 1); mbar_init(tempty0 + 8 * a, L::NEPI); }
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
    bool ok = true;

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
                const int tl = (int)(tile / P.nc), tc = (int)(tile % P.nc);
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!mbar_wait(empty0 + 8 * stage, phase ^ 1, abort_flag)) { ok = false; break; }
                    const uint32_t fb = full0 + 8 * stage;
                    mbar_expect_tx(fb, L::STAGE_BYTES);
                    const uint32_t sa = smem_u32(smem + stage * L::STAGE_BYTES), sc = sa + L::A_BYTES, ss = sc + L::C_BYTES;
                    tma_load_2d(sa, &map_l, fb, kb * KB, tl * 128);
                    tma_load_2d(sc, &map_c, fb, kb * KB, tc * BN);
                    tma_load_3d(ss, &map_sl, fb, 0, kb * Kind<BLOCK>::ATOMS, tl);
                    tma_load_3d(ss + L::S_BYTES, &map_sc, fb, 0, kb * Kind<BLOCK>::ATOMS, tc * BN / 128);
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        int stage = 0;
        uint32_t phase = 0, acc = 0, acc_phase = 0;
        for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
            ok = __all_sync(0xffffffffu, mbar_wait(tempty0 + 8 * acc, acc_phase ^ 1, abort_flag));
            if (!ok) break;
            tc_fence_after();
            for (int kb = kb0; kb < kb1; ++kb) {
                ok = __all_sync(0xffffffffu, mbar_wait(full0 + 8 * stage, phase, abort_flag));
                if (!ok) break;
                tc_fence_after();
                const uint32_t sa = smem_u32(smem + stage * L::STAGE_BYTES), sc = sa + L::A_BYTES, ss = sc + L::C_BYTES;
                if (elect_one()) {
                    stage_mmas<1, BLOCK, 128, BN>(tmem_base + acc * BN, tmem_base + L::SF0 + stage * L::SFC, sa, sc, ss, ss + L::S_BYTES, kb == kb0);
                    umma_commit(empty0 + 8 * stage);     // frees the stage, and its scales, once these MMAs have read them
                }
                __syncwarp();
                if (++stage == STAGES) { stage = 0; phase ^= 1; }
            }
            if (elect_one()) umma_commit(tfull0 + 8 * acc);
            __syncwarp();
            if (++acc == NACC) { acc = 0; acc_phase ^= 1; }
        }
    } else {
        // ------------------------------------------------------------------ epilogue
        const int q = warp & 3, half = (warp - 2) >> 2;                    // lane quarter and column part of this warp
        float *stage = out_stage + (warp - 2) * L::STAGE_WORDS;
        const int lane_row = q * 32 + lane;
        const Alpha alpha = alpha_of(P.ga ? __ldg(P.ga) : 1.f, P.gb ? __ldg(P.gb) : 1.f);
        uint32_t acc = 0, acc_phase = 0;
        for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
            ok = __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * acc, acc_phase, abort_flag));
            if (!ok) break;
            tc_fence_after();
            const int64_t row = (tile / P.nc) * 128 + lane_row;
            const int cbase = (int)(tile % P.nc) * BN + half * CW;
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + acc * BN + half * CW;
            if constexpr (ODD && BN == 128) {
                if (S == 1) {                                              // rows that start anywhere: 128 bytes of each at a time
                    uint32_t all[4][16], w[32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld_x16(taddr + c * 16, all[c]);
                    tmem_ld_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(tempty0 + 8 * acc);
                    if (++acc == NACC) { acc = 0; acc_phase ^= 1; }
                    const int64_t row0 = row - lane;
                    if (row0 >= P.rows_l) continue;
                    scale_bias<4>(P, all, alpha, cbase);
                    if (P.y_f32) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            if (cbase + b * 32 >= P.rows_c) break;
                            box_words<true, 4>(all, b, w);
                            store_box_odd(P, w, row0, cbase + b * 32, (uint32_t *)stage, lane);
                        }
                    } else if (cbase < P.rows_c) {
                        box_words<false, 4>(all, 0, w);
                        store_box_odd(P, w, row0, cbase, (uint32_t *)stage, lane);
                    }
                    continue;
                }
            }
            uint32_t r[2][16];
            tmem_ld_x16(taddr, r[0]);
#pragma unroll
            for (int c = 0; c < CW / 16; ++c) {
                tmem_ld_wait();
                if (c + 1 < CW / 16) tmem_ld_x16(taddr + (c + 1) * 16, r[(c + 1) & 1]);
                else {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(tempty0 + 8 * acc);
                }
                float v[16];
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    uint32_t x = r[c & 1][j], y = r[c & 1][j + 1];
                    mul_twice(x, y, twice(alpha.first), twice(alpha.rest));
                    v[j] = __uint_as_float(x); v[j + 1] = __uint_as_float(y);
                }
                if (S == 1) finish<ODD, 16>(P, row, cbase + c * 16, v, stage);
                else {
                    // every stage of this CTA has been read: its memory takes the parts, [column][lane row]
                    float *part = (float *)smem;
#pragma unroll
                    for (int j = 0; j < 16; ++j) part[(half * CW + c * 16 + j) * 128 + lane_row] = v[j];
                }
            }
            if (++acc == NACC) { acc = 0; acc_phase ^= 1; }
        }
    }
    if (!ok) {
        if (P.status) atomicExch(P.status, (int)LAMP_ERR_TIMEOUT);
        settle();                                                  // copies in flight
    }
    __syncwarp();
    if (S > 1) {
        cluster_sync_all();
        if (warp >= 2) {
            const int q = warp & 3, half = (warp - 2) >> 2, lane_row = q * 32 + lane;
            float *stage = out_stage + (warp - 2) * L::STAGE_WORDS;
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

// ----------------------------------------------------------------------------------------------------------------------
// CTA pairs: tiles of 256 x BN, each CTA of the pair 128 lane rows (its tensor memory) and half of the columns' operand
// ----------------------------------------------------------------------------------------------------------------------
// The leader (rank 0) issues the MMAs of both CTAs; full barriers live in the leader (both CTAs' copies complete there), empty and
// accumulator-full barriers in each CTA (the commits arrive in both), accumulator-empty barriers in the leader (the epilogue
// warps of both CTAs arrive).  Each CTA holds the scales of its own lane rows and of all columns.
// 256 columns: one accumulator (the scales need the rest of tensor memory), which the epilogue warps empty into registers before they
// store; 128 columns: two.
template <int BN, int BLOCK> struct PairLayout {
    static constexpr int CT = BN / 128;
    static constexpr int A_BYTES = 128 * KB, C_BYTES = BN / 2 * KB, S_BYTES = Kind<BLOCK>::BYTES;
    static constexpr int STAGE_BYTES = A_BYTES + C_BYTES + (1 + CT) * S_BYTES;
    static constexpr int STAGES = BN == 256 ? 5 : 6;
    static constexpr int NACC = BN == 256 ? 1 : 2;
    static constexpr int CW = BN / 2;                             // columns per epilogue warp
    static constexpr int THREADS = 384, TMEM_COLS = 512;
    static constexpr int SF0 = NACC * BN, SFC = (1 + CT) * Kind<BLOCK>::COLS;
    static constexpr int OUT_BYTES = 8 * BOX_WORDS * 4;           // per epilogue warp 32 rows x 128 bytes, or those with a pitch of 33 words
    static constexpr int BAR_BYTES = (2 * MAX_STAGES + 2 * NACC) * 8 + 16;
    static constexpr int TOTAL = 1024 + STAGES * STAGE_BYTES + OUT_BYTES + BAR_BYTES;
    static_assert(STAGE_BYTES % 1024 == 0 && OUT_BYTES >= 8 * 4096, "128-byte swizzle");
    static_assert(SF0 + STAGES * SFC <= TMEM_COLS, "");
    static_assert(TOTAL <= 227 * 1024 && STAGES <= MAX_STAGES, "");
};

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap *map, uint32_t leader_bar, int c0, int c1, int c2)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(leader_bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t src, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(c0), "r"(c1) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// 32 rows x 128 bytes of y from a warp's registers (lane = row, NW words) through its 4 KB of shared memory, by a bulk store that clips
// what lies beyond y.  Whole 128-byte lines leave, and nothing waits for them (stored by the lanes that hold them, 32 bytes of 32 rows at a
// time, 16384 x 4096 x 512 took 70 us).
__device__ __forceinline__ void store_box(const CUtensorMap *map, uint32_t buf, const uint32_t (&w)[32], int col, int row, int lane)
{
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");       // the store before has read the buffer
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 8; ++c)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 128 + ((c ^ (lane & 7)) * 16)), "r"(w[4 * c]), "r"(w[4 * c + 1]), "r"(w[4 * c + 2]),
                     "r"(w[4 * c + 3]) : "memory");
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) tma_store_2d(map, buf, col, row);
}

// ODD: rows of y that are not 16-byte aligned.
template <int BN, int BLOCK, bool ODD>
__global__ void __launch_bounds__(PairLayout<BN, BLOCK>::THREADS, 1)
fp4_gemm_pair_kernel(const __grid_constant__ CUtensorMap map_l, const __grid_constant__ CUtensorMap map_c, const __grid_constant__ CUtensorMap map_sl,
                     const __grid_constant__ CUtensorMap map_sc, const __grid_constant__ CUtensorMap map_y, const GemmParams P)
{
    using L = PairLayout<BN, BLOCK>;
    constexpr int STAGES = L::STAGES, NACC = L::NACC, CW = L::CW;

    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    float *out_stage = (float *)(smem + STAGES * L::STAGE_BYTES);
    uint64_t *bars = (uint64_t *)(smem + STAGES * L::STAGE_BYTES + L::OUT_BYTES);
    uint32_t *tmem_slot = (uint32_t *)(bars + 2 * MAX_STAGES + 2 * NACC);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + MAX_STAGES);
    const uint32_t tfull0 = smem_u32(bars + 2 * MAX_STAGES), tempty0 = smem_u32(bars + 2 * MAX_STAGES + NACC);

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
        for (int a = 0; a < NACC; ++a) { mbar_init(tfull0 + 8 * a, 1); mbar_init(tempty0 + 8 * a, 16); }
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
    const int64_t tile0 = blockIdx.x >> 1, tile_step = gridDim.x >> 1;
    bool ok = true;

    if (warp < 4) {
        if (warp == 0 && lane == 0) {
            // -------------------------------------------------------------- TMA producer, one per CTA
            int stage = 0;
            uint32_t phase = 0;
            for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
                const int tl = (int)(tile / P.nc) * 2 + (int)rank, tc = (int)(tile % P.nc);
                for (int kb = 0; kb < P.kblocks; ++kb) {
                    if (!mbar_wait(empty0 + 8 * stage, phase ^ 1, abort_flag)) { ok = false; break; }
                    const uint32_t fb = map_to_rank(full0 + 8 * stage, 0);
                    if (rank == 0) mbar_expect_tx(full0 + 8 * stage, 2 * L::STAGE_BYTES);
                    const uint32_t sa = smem_u32(smem + stage * L::STAGE_BYTES), sc = sa + L::A_BYTES, ss = sc + L::C_BYTES;
                    tma_load_2d_pair(sa, &map_l, fb, kb * KB, tl * 128);
                    tma_load_2d_pair(sc, &map_c, fb, kb * KB, tc * BN + (int)rank * (BN / 2));
                    tma_load_3d_pair(ss, &map_sl, fb, 0, kb * Kind<BLOCK>::ATOMS, tl);
                    tma_load_3d_pair(ss + L::S_BYTES, &map_sc, fb, 0, kb * Kind<BLOCK>::ATOMS, tc * L::CT);
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
            }
        } else if (warp == 1 && rank == 0) {
            // -------------------------------------------------------------- MMA issuer, in the leader
            int stage = 0;
            uint32_t phase = 0, acc = 0, acc_phase = 0;
            for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
                ok = __all_sync(0xffffffffu, mbar_wait(tempty0 + 8 * acc, acc_phase ^ 1, abort_flag));
                if (!ok) break;
                tc_fence_after();
                for (int kb = 0; kb < P.kblocks; ++kb) {
                    ok = __all_sync(0xffffffffu, mbar_wait(full0 + 8 * stage, phase, abort_flag));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sa = smem_u32(smem + stage * L::STAGE_BYTES), sc = sa + L::A_BYTES, ss = sc + L::C_BYTES;
                    if (elect_one()) {
                        stage_mmas<2, BLOCK, 256, BN>(tmem_base + acc * BN, tmem_base + L::SF0 + stage * L::SFC, sa, sc, ss, ss + L::S_BYTES, kb == 0);
                        // nobody waits for the last arrivals of the empty barriers in the other CTA; the accumulator's commit behind them,
                        // which its epilogue warps do wait for, completes after them, so they land before that CTA leaves
                        umma_commit_pair(empty0 + 8 * stage, 3u);
                    }
                    __syncwarp();
                    if (++stage == STAGES) { stage = 0; phase ^= 1; }
                }
                if (elect_one()) umma_commit_pair(tfull0 + 8 * acc, 3u);
                __syncwarp();
                if (++acc == NACC) { acc = 0; acc_phase ^= 1; }
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ epilogue
        const int q = warp & 3, half = (warp - 4) >> 2;
        const int lane_row = q * 32 + lane;
        uint32_t *odd_stage = (uint32_t *)out_stage + (warp - 4) * BOX_WORDS;
        const uint32_t box_stage = smem_u32(out_stage) + (warp - 4) * 4096;        // 1024-byte boundaries, as the swizzle wants
        uint32_t acc = 0, acc_phase = 0;
        const uint32_t tempty_leader = map_to_rank(tempty0, 0);
        const Alpha alpha = alpha_of(P.ga ? __ldg(P.ga) : 1.f, P.gb ? __ldg(P.gb) : 1.f);
        for (int64_t tile = tile0; tile < P.tiles && ok; tile += tile_step) {
            ok = __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * acc, acc_phase, abort_flag));
            if (!ok) break;
            tc_fence_after();
            const int64_t row = (tile / P.nc) * 256 + rank * 128 + lane_row;
            const int cbase = (int)(tile % P.nc) * BN + half * CW;
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + acc * BN + half * CW;
            uint32_t r[CW / 16][16];
#pragma unroll
            for (int c = 0; c < CW / 16; ++c) tmem_ld_x16(taddr + c * 16, r[c]);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(tempty_leader + 8 * acc);
            const int row0 = (int)(row - lane);
            if (row0 < P.rows_l) {
                scale_bias<CW / 16>(P, r, alpha, cbase);
                auto store = [&](const uint32_t (&w)[32], int col) {
                    if constexpr (ODD) store_box_odd(P, w, row0, col, odd_stage, lane);
                    else store_box(&map_y, box_stage, w, col, row0, lane);
                };
                uint32_t w[32];
                if (P.y_f32) {
#pragma unroll
                    for (int b = 0; b < CW / 32; ++b) {
                        if (cbase + b * 32 >= P.rows_c) break;
                        box_words<true, CW / 16>(r, b, w);
                        store(w, cbase + b * 32);
                    }
                } else {
#pragma unroll
                    for (int b = 0; b < CW / 64; ++b) {
                        if (cbase + b * 64 >= P.rows_c) break;
                        box_words<false, CW / 16>(r, b, w);
                        store(w, cbase + b * 64);
                    }
                }
            }
            if (++acc == NACC) { acc = 0; acc_phase ^= 1; }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");       // stores still read shared memory
    }
    if (!ok) {
        if (P.status) atomicExch(P.status, (int)LAMP_ERR_TIMEOUT);
        settle();                                                  // copies in flight
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();          // no CTA leaves, or frees tensor memory, while the other still uses what is its own
    tc_fence_after();
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(L::TMEM_COLS) : "memory");
}

// ----------------------------------------------------------------------------------------------------------------------
// host
// ----------------------------------------------------------------------------------------------------------------------
bool encode_codes(const lamp_fp4_operand_t *o, int box_rows, CUtensorMap *map)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = (PFN_cuTensorMapEncodeTiled_v12000)tensor_map_encoder();
    if (!enc) return false;
    const cuuint64_t gdim[2] = {(cuuint64_t)((o->k + 1) / 2), (cuuint64_t)o->rows};
    const cuuint64_t gstride[1] = {(cuuint64_t)o->q_pitch};
    const cuuint32_t box[2] = {(cuuint32_t)KB, (cuuint32_t)box_rows};
    const cuuint32_t es[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, o->q, gdim, gstride, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// [tiles of rows][tiles along k][128 words]
bool encode_scales(const lamp_fp4_operand_t *o, int box_tiles, CUtensorMap *map)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = (PFN_cuTensorMapEncodeTiled_v12000)tensor_map_encoder();
    if (!enc) return false;
    const int64_t tiles = fp4::tiles_of(o->k, o->block);
    const cuuint64_t gdim[3] = {128, (cuuint64_t)tiles, (cuuint64_t)((o->rows + 127) / 128)};
    const cuuint64_t gstride[2] = {512, (cuuint64_t)tiles * 512};
    const cuuint32_t box[3] = {128, (cuuint32_t)(KCODES / (4 * o->block)), (cuuint32_t)box_tiles};
    const cuuint32_t es[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, o->scale, gdim, gstride, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// y as [rows][columns], boxes of 32 rows x 128 bytes
bool encode_output(const GemmParams &P, CUtensorMap *map)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = (PFN_cuTensorMapEncodeTiled_v12000)tensor_map_encoder();
    if (!enc) return false;
    const int es = P.y_f32 ? 4 : 2;
    const cuuint64_t gdim[2] = {(cuuint64_t)P.rows_c, (cuuint64_t)P.rows_l};
    const cuuint64_t gstride[1] = {(cuuint64_t)P.y_pitch * es};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / es), 32};
    const cuuint32_t one[2] = {1, 1};
    return enc(map, P.y_f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, P.y, gdim, gstride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename... KArgs, typename... Args>
lamp_status_t launch_tiles(void (*kernel)(KArgs...), SmemAttrOnce &attr, int smem, int threads, unsigned grid, int cluster, bool early, cudaStream_t st, const Args &...args)
{
    { const lamp_status_t as = attr.ensure(kernel, smem); if (as != LAMP_OK) return as; }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    int na = 0;
    if (early) {
        at[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[na++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        at[na].id = cudaLaunchAttributeClusterDimension;
        at[na].val.clusterDim.x = (unsigned)cluster;
        at[na].val.clusterDim.y = 1;
        at[na++].val.clusterDim.z = 1;
    }
    cfg.attrs = at;
    cfg.numAttrs = na;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? LAMP_OK : LAMP_ERR_CUDA;
}

template <int BN, int BLOCK, bool ODD>
lamp_status_t launch_pair(const lamp_fp4_operand_t *l, const lamp_fp4_operand_t *c, const GemmParams &P, cudaStream_t st)
{
    using L = PairLayout<BN, BLOCK>;
    static SmemAttrOnce attr;
    CUtensorMap ml, mc, msl, msc, my = {};
    if (!encode_codes(l, 128, &ml) || !encode_codes(c, BN / 2, &mc) || !encode_scales(l, 1, &msl) || !encode_scales(c, L::CT, &msc)) return LAMP_ERR_CUDA;
    if (!ODD && !encode_output(P, &my)) return LAMP_ERR_CUDA;
    const int64_t pairs = sm_count() / 2;
    return launch_tiles(fp4_gemm_pair_kernel<BN, BLOCK, ODD>, attr, L::TOTAL, L::THREADS, 2 * (unsigned)(P.tiles < pairs ? P.tiles : pairs), 2, P.tiles <= 4 * pairs, st,
                        ml, mc, msl, msc, my, P);
}
template <int BN, int BLOCK, bool ODD>
lamp_status_t launch_one(const lamp_fp4_operand_t *l, const lamp_fp4_operand_t *c, const GemmParams &P, cudaStream_t st)
{
    using L = GemmLayout<BN, BLOCK>;
    static SmemAttrOnce attr;
    CUtensorMap ml, mc, msl, msc;
    if (!encode_codes(l, 128, &ml) || !encode_codes(c, BN, &mc) || !encode_scales(l, 1, &msl) || !encode_scales(c, 1, &msc)) return LAMP_ERR_CUDA;
    const int sms = sm_count();
    return launch_tiles(fp4_gemm_kernel<BN, BLOCK, ODD>, attr, L::TOTAL, L::THREADS, (unsigned)(P.splits > 1 ? P.tiles * P.splits : P.tiles < sms ? P.tiles : sms), P.splits,
                        P.tiles <= 4 * (int64_t)sms, st, ml, mc, msl, msc, P);
}

template <int BLOCK>
lamp_status_t product(const lamp_fp4_operand_t *l, const lamp_fp4_operand_t *c, GemmParams &P, cudaStream_t st)
{
    const int sms = sm_count();
    P.splits = 1;
    const bool odd = odd_rows(P);
    // pairs where their tiles fill the GPU
    for (int bn = 256; bn >= 128; bn /= 2) {
        const int64_t nl = (P.rows_l + 255) / 256, nc = (P.rows_c + bn - 1) / bn;
        if (P.swap || P.rows_c < bn || nl * nc * 2 < sms * 3 / 4) continue;
        P.nl = (int32_t)nl; P.nc = (int32_t)nc; P.tiles = nl * nc;
        const bool unaligned = P.vec == 0;
        if (bn == 256) return unaligned ? launch_pair<256, BLOCK, true>(l, c, P, st) : launch_pair<256, BLOCK, false>(l, c, P, st);
        return unaligned ? launch_pair<128, BLOCK, true>(l, c, P, st) : launch_pair<128, BLOCK, false>(l, c, P, st);
    }
    const int bn = P.rows_c <= 16 ? 16 : P.rows_c <= 32 ? 32 : P.rows_c <= 64 ? 64 : 128;
    P.nl = (P.rows_l + 127) / 128;
    P.nc = (P.rows_c + bn - 1) / bn;
    P.tiles = (int64_t)P.nl * P.nc;
    while (P.splits < 8 && P.tiles <= cluster_room(sms, 2 * P.splits) && P.kblocks >= 4 * P.splits) P.splits *= 2;
    switch (bn) {
    case 16: return odd ? launch_one<16, BLOCK, true>(l, c, P, st) : launch_one<16, BLOCK, false>(l, c, P, st);
    case 32: return odd ? launch_one<32, BLOCK, true>(l, c, P, st) : launch_one<32, BLOCK, false>(l, c, P, st);
    case 64: return odd ? launch_one<64, BLOCK, true>(l, c, P, st) : launch_one<64, BLOCK, false>(l, c, P, st);
    default: return odd ? launch_one<128, BLOCK, true>(l, c, P, st) : launch_one<128, BLOCK, false>(l, c, P, st);
    }
}

}  // namespace

}  // namespace lamp

using namespace lamp;

extern "C" lamp_status_t lamp_gemm_fp4(const lamp_fp4_operand_t *a, const lamp_fp4_operand_t *b, const float *bias, lamp_tensor_t *y,
                                       void *cuda_stream)
{
    lamp_status_t s;
    if ((s = check_fp4_operand(a)) != LAMP_OK || (s = check_fp4_operand(b)) != LAMP_OK) return s;
    if ((s = check_view(y, true)) != LAMP_OK) return s;
    if (a->k != b->k || a->k == 0 || a->block != b->block || voxels(y) != a->rows || (int64_t)y->c != b->rows || ((uintptr_t)bias & 3))
        return LAMP_ERR_INVALID_ARG;
    if (a->rows == 0) return LAMP_OK;
    GemmParams P = {};
    const bool swap = a->rows <= 64 && b->rows > a->rows;
    const lamp_fp4_operand_t *l = swap ? b : a, *c = swap ? a : b;
    P.rows_l = (int32_t)l->rows; P.rows_c = (int32_t)c->rows;
    P.kblocks = (int32_t)((a->k + KCODES - 1) / KCODES);
    P.ga = a->tensor_scale; P.gb = b->tensor_scale;
    set_output(P, make_view(y), bias, swap);
    P.status = status_word_ptr();
    return a->block == 32 ? product<32>(l, c, P, (cudaStream_t)cuda_stream) : product<16>(l, c, P, (cudaStream_t)cuda_stream);
}
