// What the 8-bit and the 4-bit matrix products share: the way of a finished tile from registers to y, the sum over the CTAs of a
// cluster that share the k axis of a tile, cluster helpers, and how many clusters run at once.
#pragma once
#include <cuda.h>
#include "common.cuh"
#include "umma_ptx.cuh"

namespace lamp {
namespace gemm {

using namespace ptx;

constexpr int STAGE_FLOATS = 32 * 17;         // a storing warp's staging area for rows that are not 16-byte aligned

struct OutParams {
    int32_t rows_l, rows_c;                   // rows of the lane operand and of the column operand
    const float *bias;
    void *y;
    int64_t y_pitch;
    int32_t y_f32, swap;                      // swap: lanes = channels of y, columns = its voxels
    int32_t vec;                              // alignment of every row's tile start: 2 = 32 bytes, 1 = 16 bytes, 0 = neither
};
inline void set_output(OutParams &P, const TView &v, const float *bias, bool swap)
{
    P.bias = bias; P.y = v.p; P.y_pitch = v.pitch; P.y_f32 = v.f32; P.swap = swap;
    const uintptr_t mis = (uintptr_t)v.p | (uintptr_t)(v.pitch * (v.f32 ? 4 : 2));
    P.vec = (mis & 31) == 0 ? 2 : (mis & 15) == 0 ? 1 : 0;
}
inline bool odd_rows(const OutParams &P) { return !P.swap && (P.vec == 0 || P.rows_c % 16 != 0); }

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
__device__ __forceinline__ void store_row(const OutParams &P, int64_t row, int col, const float (&v)[NV])
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
__device__ __forceinline__ void finish(const OutParams &P, int64_t row, int col, float (&v)[NV], float *stage)
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

// 32 rows x 128 bytes of y (lane = row, `w` its words: 32 columns of fp32 or 64 of bf16) to rows that start anywhere, through `stage`, BOX_WORDS words of
// the warp: a row at a time, a word per lane, so that 128 bytes in a row leave together (16 columns of two rows at a time, as finish() does it,
// wrote most sectors in two pieces: 16384 x 4095 bf16, k = 512 took 122 us, this 81; 28 with aligned rows - the sectors that two stores share cost).  bf16 rows that start between two words are shifted by one
// element.  Every lane takes part.
constexpr int BOX_WORDS = 32 * 33;
__device__ __forceinline__ void store_box_odd(const OutParams &P, const uint32_t (&w)[32], int64_t row0, int col, uint32_t *stage, int lane)
{
#pragma unroll
    for (int j = 0; j < 32; ++j) stage[lane * 33 + j] = w[j];
    __syncwarp();
    const int rows = P.rows_l - row0 < 32 ? (int)(P.rows_l - row0) : 32, left = P.rows_c - col;      // rows and columns that exist
    if (P.y_f32) {
        float *o = (float *)P.y + row0 * P.y_pitch + col + lane;
        if (left >= 32 && rows == 32) {
            float v[32];                                           // all of them first: the compiler does not move a load past a store
#pragma unroll
            for (int r = 0; r < 32; ++r) v[r] = __uint_as_float(stage[r * 33 + lane]);
#pragma unroll
            for (int r = 0; r < 32; ++r, o += P.y_pitch) *o = v[r];
        } else if (lane < left) {
            for (int r = 0; r < rows; ++r, o += P.y_pitch) *o = __uint_as_float(stage[r * 33 + lane]);
        }
    } else {
        // every second row starts alike
        for (int p = 0; p < 2; ++p) {
            bf16 *o = (bf16 *)P.y + (row0 + p) * P.y_pitch + col;
            const uint32_t *s = stage + p * 33 + lane;
            const bool between = (uintptr_t)o & 2;
            const int64_t step = 2 * P.y_pitch;
            if (left >= 64 && rows == 32) {
                uint32_t v[16];                                    // all of them first: the compiler does not move a load past a store
#pragma unroll
                for (int r = 0; r < 16; ++r) v[r] = s[r * 66];
                if (!between) {
                    o += 2 * lane;
#pragma unroll
                    for (int r = 0; r < 16; ++r, o += step) *reinterpret_cast<uint32_t *>(o) = v[r];
                } else {
                    // lane l has elements 2 l + 1 and 2 l + 2; the first and the last one go by themselves
                    bf16 *e = o + (lane == 0 ? 0 : 63);
                    const bool edge = lane == 0 || lane == 31;
                    const int next = lane < 31 ? 1 : 0;
                    o += 2 * lane + 1;
#pragma unroll
                    for (int r = 0; r < 16; ++r, o += step, e += step) {
                        if (lane < 31) *reinterpret_cast<uint32_t *>(o) = __byte_perm(v[r], s[r * 66 + next], 0x5432);
                        if (edge) *reinterpret_cast<uint16_t *>(e) = (uint16_t)(lane == 0 ? v[r] : v[r] >> 16);
                    }
                }
            } else {
                const int e = 2 * lane + (between ? 1 : 0);        // first element of this lane's word
                for (int r = p; r < rows; r += 2, o += step, s += 66) {
                    const uint32_t a = s[0], b = between && lane < 31 ? s[1] : 0u, v = between ? __byte_perm(a, b, 0x5432) : a;
                    if (e + 1 < left && e + 1 < 64) *reinterpret_cast<uint32_t *>(o + e) = v;
                    else if (e < left) *reinterpret_cast<uint16_t *>(o + e) = (uint16_t)v;
                    if (between && lane == 0) *reinterpret_cast<uint16_t *>(o) = (uint16_t)a;
                }
            }
        }
    }
    __syncwarp();
}
// ga gb of two tensors' scales as factors to be applied in turn.  Their product alone (rest = 1) where it is well inside fp32's range, else
// the one nearer to 1 first: what lies between is then never further from 1 than the result or the sum is, so nothing is lost or infinite that the result is not.
struct Alpha { float first, rest; };
__device__ __forceinline__ Alpha alpha_of(float ga, float gb)
{
    const float both = ga * gb, low = fminf(ga, gb), high = fmaxf(ga, gb);
    if (!(both < 7.8886091e-31f) && !(both > 1.2676506e30f)) return {both, 1.f};           // 2^-100 .. 2^100, and NaN
    if (both < 1.f) return {high, low};
    return {low, high};
}
// both factors, two values per instruction: as many instructions as one factor took a value at a time, and no branch
__device__ __forceinline__ void mul_twice(uint32_t &x, uint32_t &y, f32x2 first, f32x2 rest)
{
    float u, v;
    unpack2(mul2(mul2(pack2(x, y), first), rest), u, v);
    x = __float_as_uint(u);
    y = __float_as_uint(v);
}
// alpha * (16 * N accumulator columns) + bias, and the words of 128 bytes of a row from them
template <int N> __device__ __forceinline__ void scale_bias(const OutParams &P, uint32_t (&r)[N][16], Alpha a, int col0)
{
    const f32x2 first = twice(a.first), rest = twice(a.rest);
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
        for (int j = 0; j < 16; j += 2) mul_twice(r[c][j], r[c][j + 1], first, rest);
    if (!P.bias) return;
    const int last = P.rows_c - 1;
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) r[c][j] = __float_as_uint(__uint_as_float(r[c][j]) + __ldg(P.bias + min(col0 + c * 16 + j, last)));      // columns behind the last are not stored
}
template <bool F32, int N> __device__ __forceinline__ void box_words(const uint32_t (&r)[N][16], int b, uint32_t (&w)[32])
{
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        if constexpr (F32) w[j] = r[2 * b + j / 16][j % 16];
        else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(r[4 * b + j / 8][2 * j % 16]), __uint_as_float(r[4 * b + j / 8][2 * j % 16 + 1]));
            w[j] = *reinterpret_cast<const uint32_t *>(&h);
        }
    }
}

// Sum over the S parts of a tile (in CTAs first, first + stride, ... of the cluster) of the `mine`-th CW / S columns of this
// thread's lane row, and their store.
template <bool ODD, int CW, int S>
__device__ __forceinline__ void reduce_parts(const OutParams &P, uint32_t part_base, int lane_row, int64_t row, int col_local, int col0, uint32_t mine,
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

// Clusters of `ctas` CTAs, one CTA per SM, that run at once: the SMs of a cluster belong to one GPC, so not every SM finds a
// place.  (148 SMs: 74 clusters of 2, 33 of 4, 15 of 8; one cluster more than that is a second wave - 141 us against 71 for a
// weight gradient of 512 x 2048 outputs.)
inline int64_t cluster_room(int sms, int ctas) { return ctas <= 2 ? sms / ctas : ctas == 4 ? sms * 2 / 9 : sms / 10; }

}  // namespace gemm
}  // namespace lamp
