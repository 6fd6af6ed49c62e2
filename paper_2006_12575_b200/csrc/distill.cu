// Distillation loss from a teacher's top logits, and its gradient:
//   loss_r = T^2 sum_j p_j (log p_j - log q_{idx_j}),   dloss_r/dz_i = T (q_i S - sum_{j: idx_j = i} p_j),   S = sum_j p_j.
// Bound by memory: a row of c logits is read once and its gradient written once.  The exponentials are taken relative to
// the row's maximum, with the difference formed first in every form, so q is as exact as fp32 allows whatever the size of the
// logits (2^(z c - m c) with one rounded product m c is not: it carries half a unit of m c, a factor of 2^18 at logits of
// -1e9, and infinity where one thread's first classes are all masked with -1e10).  Only the gradient alone starts from the
// stored log-sum, whose rounding it carries.
// The gradient of a listed class is the difference of two numbers that training makes nearly equal, so it is formed in
// fp32 and rounded once: the dense pass writes q_i S everywhere, then the owner of each listed class overwrites it.
// A class listed twice subtracts both probabilities (each of its entries writes the same value).
//
// Rows of odd length start at any element, so a row is walked in 16-byte units aligned in memory; a unit that is not
// wholly inside the row is handled element by element.
//   c <= 128, k <= 32:  one thread per row, many rows at a time through shared memory.
//   c <= 1272 bf16 or 636 fp32, k <= 128:  one warp per row, the row in registers, the next row on its way (held so, rows of
//           3000 classes took 389 us where the CTA form takes 251: too few warps fit).
//   c <= 1024, longer lists:  one warp per row.
//   wider:  one CTA per row, or a cluster of up to 8 CTAs where a row does not fit in the shared memory of one or rows are
//           few; they exchange maximum and sum through distributed shared memory.
#include <cuda.h>
#include <float.h>
#include "common.cuh"
#include "umma_ptx.cuh"

namespace lamp {

namespace {

constexpr int FWD = 1, BWD = 2;
constexpr int MAX_PARTS = 4096;                     // partial losses, one per CTA (or cluster)
constexpr int MAX_K = 1024;
constexpr float LOG2E = 1.4426950408889634f;
constexpr int WR_WARPS = 8, WR_MAX_C = 1024;
constexpr int RW_MAX_UNITS = 5;                     // 16-byte units per lane of a row held by one warp

struct DistillParams {
    const void *z;
    void *dz;
    int64_t pz, pdz, rows;
    int32_t c, k;
    const int32_t *idx;
    const float *t, *tlse;
    float temp, w_all;                              // w_all: the weight of every row where `w` is NULL
    const float *w;
    const float *lse_in;
    float *loss_rows, *lse_out;
    double *part;                                   // one partial loss per CTA or cluster, or NULL
    int32_t stash;                                  // 16-byte units of a buffer (CTA form)
    int *status;
};

template <bool F32> struct Elem {
    static constexpr int E = F32 ? 4 : 8;           // elements of a 16-byte unit
    static constexpr int SHIFT = F32 ? 2 : 1;       // log2 of the element size
};

template <bool F32> __device__ __forceinline__ float elem(const void *p, int64_t i)
{
    if constexpr (F32) return ((const float *)p)[i]; else return bf2f(((const bf16 *)p)[i]);
}
template <bool F32> __device__ __forceinline__ void put(void *p, int64_t i, float v)
{
    if constexpr (F32) ((float *)p)[i] = v; else ((bf16 *)p)[i] = f2bf(v);
}

// elements of the row's first 16-byte unit that lie in front of the row
template <bool F32> __device__ __forceinline__ int misalign(const void *p, int64_t at)
{
    return (int)((((uintptr_t)p >> Elem<F32>::SHIFT) + (uintptr_t)at) & (Elem<F32>::E - 1));
}

template <bool F32> __device__ __forceinline__ void unit_values(const uint4 &r, float (&v)[Elem<F32>::E])
{
    if constexpr (F32) {
        v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
    } else {
        unpack8(r, v);
    }
}
template <bool F32> __device__ __forceinline__ uint4 unit_raw(const float (&v)[Elem<F32>::E])
{
    if constexpr (F32) return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    else return pack8(v);
}

// Unit u of the row that starts at element `at`: elements lo = u E - off .. lo + E - 1 of the row; -inf outside it.
template <bool F32>
__device__ __forceinline__ uint4 load_unit(const void *z, int64_t at, int off, int u, int c)
{
    constexpr int E = Elem<F32>::E;
    const int lo = u * E - off;
    if (lo >= 0 && lo + E <= c) return *reinterpret_cast<const uint4 *>((const char *)z + ((at + lo) << Elem<F32>::SHIFT));
    float v[E];
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = lo + j >= 0 && lo + j < c ? elem<F32>(z, at + lo + j) : -INFINITY;
    return unit_raw<F32>(v);
}
template <bool F32>
__device__ __forceinline__ void store_unit(void *dz, int64_t at, int off, bool same, int u, int c, const float (&v)[Elem<F32>::E])
{
    constexpr int E = Elem<F32>::E;
    const int lo = u * E - off;
    if (same && lo >= 0 && lo + E <= c) {
        *reinterpret_cast<uint4 *>((char *)dz + ((at + lo) << Elem<F32>::SHIFT)) = unit_raw<F32>(v);
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j) if (lo + j >= 0 && lo + j < c) put<F32>(dz, at + lo + j, v[j]);
    }
}

// 2^x; results below the normal range become 0
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// (m, s) = maximum of z and sum of e^((z - m) / T) of two parts.  m starts at -FLT_MAX, not -inf, so that no difference of
// infinities arises; the difference is taken before the change of base, which also holds where z log2(e) would overflow
// (rows masked with the type's lowest value).
__device__ __forceinline__ void join(float &m, float &s, float m2, float s2, float c2)
{
    const float n = fmaxf(m, m2);
    s = s * ex2((m - n) * c2) + s2 * ex2((m2 - n) * c2);
    m = n;
}
// e^(z / T) relative to the reference m: the row's maximum of z, or, where only the gradient is asked for, the log-sum of z / T
template <int MODE> __device__ __forceinline__ float power(float z, float c2, float inv_t, float m)
{
    return (MODE & FWD) ? ex2((z - m) * c2) : ex2(fmaf(z, inv_t, -m) * LOG2E);
}
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// largest value of the warp, none of them NaN: floats ordered as integers, one instruction for the warp
__device__ __forceinline__ float warp_max_fast(float v)
{
    int i = __float_as_int(v);
    i ^= (i >> 31) & 0x7fffffff;
    i = __reduce_max_sync(0xffffffffu, i);
    return __int_as_float(i ^ ((i >> 31) & 0x7fffffff));
}
// One warp reads the teacher's entries of a row: ids (-1: absent) and log p to shared memory; returns S (0: no entry left).
// As for the student, the difference to the largest entry is formed before anything is divided by T.
__device__ __forceinline__ float teacher_row(const DistillParams &P, int64_t row, int lane, int *ids, float *logp)
{
    const float inv_t = 1.f / P.temp, tlse = P.tlse ? P.tlse[row] : 0.f;
    float m = -FLT_MAX, S = 0.f;
    bool some = false;
    for (int j = lane; j < P.k; j += 32) {
        int id = P.idx[row * P.k + j];
        if (id < 0 || id >= P.c) id = -1;
        const float v = id >= 0 ? P.t[row * P.k + j] : -INFINITY;
        ids[j] = id;
        logp[j] = v;
        some |= v != -INFINITY;                                     // NaN counts
        m = fmaxf(m, v);
    }
    if (!__any_sync(0xffffffffu, some)) return 0.f;
    if (P.tlse) {
        for (int j = lane; j < P.k; j += 32) {
            logp[j] = fmaf(logp[j], inv_t, -tlse);
            S += ids[j] >= 0 ? expf(logp[j]) : 0.f;
        }
        S = warp_sum(S);
        __syncwarp();
        return S;
    }
    m = warp_max_fast(m);
    for (int j = lane; j < P.k; j += 32) {
        logp[j] = (logp[j] - m) * inv_t;
        S += expf(logp[j]);
    }
    S = warp_sum(S);
    const float ls = logf(S);
    for (int j = lane; j < P.k; j += 32) logp[j] -= ls;
    __syncwarp();
    return S == S ? 1.f : NAN;
}

// A row's teacher entries in the registers of a warp (k <= 32 KE), lane + 32 i, so that they can be loaded a row ahead.
constexpr int SHORT_K = 128;
template <int KE> struct Entries {
    int id[KE];
    float t[KE];
    __device__ __forceinline__ void load(const DistillParams &P, int64_t row, int lane)
    {
#pragma unroll
        for (int i = 0; i < KE; ++i) {
            const int j = lane + 32 * i;
            id[i] = j < P.k ? P.idx[row * P.k + j] : -1;
            t[i] = j < P.k ? P.t[row * P.k + j] : 0.f;
        }
    }
    // ids of absent entries become -1; p and log p of the others.  Returns S (0: no entry left).
    __device__ __forceinline__ float prepare(const DistillParams &P, float tlse, float (&p)[KE], float (&logp)[KE])
    {
        const float inv_t = 1.f / P.temp, c2 = LOG2E / P.temp;
        float m = -FLT_MAX;
        bool some = false;
#pragma unroll
        for (int i = 0; i < KE; ++i) {
            if ((uint32_t)id[i] >= (uint32_t)P.c) id[i] = -1;
            p[i] = logp[i] = 0.f;
            if (id[i] < 0) continue;
            some |= t[i] != -INFINITY;                              // NaN counts
            m = fmaxf(m, t[i]);
        }
        if (!__any_sync(0xffffffffu, some)) return 0.f;
        float S = 0.f;
        if (P.tlse) {
#pragma unroll
            for (int i = 0; i < KE; ++i) {
                logp[i] = fmaf(t[i], inv_t, -tlse);
                p[i] = id[i] >= 0 ? expf(logp[i]) : 0.f;
                S += p[i];
            }
            return warp_sum(S);
        }
        m = warp_max_fast(m);
#pragma unroll
        for (int i = 0; i < KE; ++i) { p[i] = id[i] >= 0 ? ex2((t[i] - m) * c2) : 0.f; S += p[i]; }
        S = warp_sum(S);
        const float ls = logf(S), inv = 1.f / S;
#pragma unroll
        for (int i = 0; i < KE; ++i) { p[i] *= inv; logp[i] = (t[i] - m) * inv_t - ls; }
        return S == S ? 1.f : NAN;
    }
    // pm = p summed over the entries that name the same class.  ids, pr: 32 KE words of shared memory of this warp, which
    // then hold ids and p (k4: k up to a multiple of 4).
    __device__ __forceinline__ void merge(int k, int k4, int lane, const float (&p)[KE], float (&pm)[KE], int *ids, float *pr) const
    {
        bool twice = false;
#pragma unroll
        for (int i = 0; i < KE; ++i) {
            const int j = lane + 32 * i;
            if (j < k4) { ids[j] = id[i]; pr[j] = p[i]; }
            pm[i] = p[i];
        }
        __syncwarp();
        if (k <= 32) {
            const uint32_t same = __match_any_sync(0xffffffffu, id[0]);      // by every lane, also those without an entry
            twice = id[0] >= 0 && same != 1u << lane;
        } else {
            int n = 0;                                              // entries equal to one of this lane's, but for itself
            for (int q = 0; q < k4; q += 4) {
                const int4 v = *reinterpret_cast<const int4 *>(ids + q);
#pragma unroll
                for (int i = 0; i < KE; ++i)
                    if (id[i] >= 0) n += (v.x == id[i]) + (v.y == id[i]) + (v.z == id[i]) + (v.w == id[i]) - (q == ((lane + 32 * i) & ~3));
            }
            twice = n != 0;
        }
        if (__any_sync(0xffffffffu, twice)) {
#pragma unroll
            for (int i = 0; i < KE; ++i) {
                float s = 0.f;
                for (int q = 0; q < k; ++q) s += ids[q] == id[i] ? pr[q] : 0.f;
                pm[i] = s;
            }
        }
    }
};

// ----------------------------------------------------------------------------------------------------------------------
// one warp per row, lists of any length
// ----------------------------------------------------------------------------------------------------------------------
template <bool F32, int MODE>
__global__ void __launch_bounds__(WR_WARPS * 32)
distill_warp_kernel(const DistillParams P)
{
    constexpr int E = Elem<F32>::E, NU = WR_MAX_C / (32 * E) + 1;
    extern __shared__ int smem_i[];
    __shared__ double wl[WR_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int *ids = smem_i + warp * 3 * P.k;
    float *logp = (float *)(ids + P.k), *zt = logp + P.k;
    const float c2 = LOG2E / P.temp, inv_t = 1.f / P.temp;
    double total = 0;
    pdl_launch_dependents();
    pdl_wait();
    for (int64_t row = (int64_t)blockIdx.x * WR_WARPS + warp; row < P.rows; row += (int64_t)gridDim.x * WR_WARPS) {
        const int64_t at = row * P.pz, dat = row * P.pdz;
        const float w = P.w ? P.w[row] : P.w_all;
        const int off = misalign<F32>(P.z, at);
        const bool same = (MODE & BWD) && off == misalign<F32>(P.dz, dat);
        const int nu = (P.c + off + E - 1) / E;
        float S = 0.f;
        __syncwarp();
        if (w != 0.f) S = teacher_row(P, row, lane, ids, logp);
        if (S != 0.f)                                               // before anything is written: dz may be z
            for (int j = lane; j < P.k; j += 32) zt[j] = ids[j] >= 0 ? elem<F32>(P.z, at + ids[j]) : 0.f;
        float loss = 0.f, lse = 0.f;
        if (S != 0.f) {
            uint4 raw[NU];
            float m = -FLT_MAX, s = 0.f;
#pragma unroll
            for (int i = 0; i < NU; ++i) if (lane + 32 * i < nu) raw[i] = load_unit<F32>(P.z, at, off, lane + 32 * i, P.c);
            __syncwarp();                                           // the listed logits lie in other lanes' units: read before any is written
            float scale;                                            // 1 / sum, relative to the maximum
            if constexpr (MODE & FWD) {
#pragma unroll
                for (int i = 0; i < NU; ++i) if (lane + 32 * i < nu) {
                    float v[E];
                    unit_values<F32>(raw[i], v);
#pragma unroll
                    for (int j = 0; j < E; ++j) m = fmaxf(m, v[j]);
                }
                m = warp_max(m);
#pragma unroll
                for (int i = 0; i < NU; ++i) if (lane + 32 * i < nu) {
                    float v[E];
                    unit_values<F32>(raw[i], v);
#pragma unroll
                    for (int j = 0; j < E; ++j) s += ex2((v[j] - m) * c2);
                }
                s = warp_sum(s);
                if (s == 0.f) s = NAN;                              // no logit above -inf: there is no softmax
                const float ls = logf(s);
                lse = m * inv_t + ls;
                scale = 1.f / s;
                for (int j = lane; j < P.k; j += 32) {
                    const float p = ids[j] >= 0 ? expf(logp[j]) : 0.f;
                    if (p != 0.f) loss += p * (logp[j] - ((zt[j] - m) * inv_t - ls));
                }
                loss = warp_sum(loss) * P.temp * P.temp;
            } else {
                m = P.lse_in[row];
                scale = 1.f;
            }
            if constexpr (MODE & BWD) {
                const float gT = w * P.temp, gq = gT * S * scale;
#pragma unroll
                for (int i = 0; i < NU; ++i) if (lane + 32 * i < nu) {
                    float v[E];
                    unit_values<F32>(raw[i], v);
#pragma unroll
                    for (int j = 0; j < E; ++j) v[j] = gq * power<MODE>(v[j], c2, inv_t, m);
                    store_unit<F32>(P.dz, dat, off, same, lane + 32 * i, P.c, v);
                }
                __syncwarp();
                for (int j = lane; j < P.k; j += 32) {
                    if (ids[j] < 0) continue;
                    float p = 0.f;
                    for (int i = 0; i < P.k; ++i) if (ids[i] == ids[j]) p += expf(logp[i]);
                    put<F32>(P.dz, dat + ids[j], gT * (S * (scale * power<MODE>(zt[j], c2, inv_t, m)) - p));
                }
            }
        } else if constexpr (MODE & BWD) {
            float v[E];
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = 0.f;
            for (int u = lane; u < nu; u += 32) store_unit<F32>(P.dz, dat, off, same, u, P.c, v);
        }
        if constexpr (MODE & FWD) {
            if (lane == 0) {
                if (P.loss_rows) P.loss_rows[row] = loss;
                if (P.lse_out) P.lse_out[row] = lse;
                if (w != 0.f) total += (double)w * loss;
            }
        }
    }
    if ((MODE & FWD) && P.part) {
        if (lane == 0) wl[warp] = total;
        __syncthreads();
        if (threadIdx.x == 0) {
            double a = 0;
            for (int i = 0; i < WR_WARPS; ++i) a += wl[i];
            P.part[blockIdx.x] = a;
        }
    }
}

// largest element of a unit
template <bool F32> __device__ __forceinline__ float unit_max(const uint4 &r)
{
    if constexpr (F32) {
        return fmaxf(fmaxf(__uint_as_float(r.x), __uint_as_float(r.y)), fmaxf(__uint_as_float(r.z), __uint_as_float(r.w)));
    } else {
        const __nv_bfloat162 *h = reinterpret_cast<const __nv_bfloat162 *>(&r);
        const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
}
// pair i of a unit as two packed fp32 values
template <bool F32> __device__ __forceinline__ ptx::f32x2 unit_pair(const uint4 &r, int i)
{
    if constexpr (F32) return i == 0 ? ptx::pack2(r.x, r.y) : ptx::pack2(r.z, r.w);
    const uint32_t w = i == 0 ? r.x : i == 1 ? r.y : i == 2 ? r.z : r.w;
    return ptx::pack2(w << 16, w & 0xFFFF0000u);
}
// e^((z - m) / T) of a packed pair, c = log2(e) / T
__device__ __forceinline__ ptx::f32x2 pair_exp(ptx::f32x2 z, float c, float m)
{
    float a, b;
    ptx::unpack2(ptx::mul2(ptx::add2(z, ptx::twice(-m)), ptx::twice(c)), a, b);
    return ptx::pack2(__float_as_uint(ex2(a)), __float_as_uint(ex2(b)));
}

template <bool F32>
__device__ __forceinline__ float unit_sum(const uint4 &raw, float c, float m)
{
    ptx::f32x2 s = 0;
#pragma unroll
    for (int j = 0; j < Elem<F32>::E / 2; ++j) s = ptx::add2(s, pair_exp(unit_pair<F32>(raw, j), c, m));
    float a, b;
    ptx::unpack2(s, a, b);
    return a + b;
}

// gradient of a unit before the listed classes are taken off.  FWD in MODE: from the maximum m (c = log2(e) / T); else from a
// given log-sum m: e^(z / T - m), the difference before the change of base (c = 1 / T)
template <bool F32, int MODE>
__device__ __forceinline__ uint4 unit_grad(const uint4 &raw, float c, float m, float gq)
{
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < Elem<F32>::E / 2; ++j) {
        ptx::f32x2 e = unit_pair<F32>(raw, j);
        float x, y;
        if constexpr (MODE & FWD) {
            e = pair_exp(e, c, m);
        } else {
            ptx::unpack2(ptx::mul2(ptx::fma2(e, ptx::twice(c), ptx::twice(-m)), ptx::twice(LOG2E)), x, y);
            e = ptx::pack2(__float_as_uint(ex2(x)), __float_as_uint(ex2(y)));
        }
        ptx::unpack2(ptx::mul2(e, ptx::twice(gq)), x, y);
        if constexpr (F32) {
            o[2 * j] = __float_as_uint(x); o[2 * j + 1] = __float_as_uint(y);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
            o[j] = *reinterpret_cast<const uint32_t *>(&h);
        }
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// a unit of the gradient, already in its type
template <bool F32>
__device__ __forceinline__ void put_unit(void *dz, int64_t at, int off, bool same, int u, int c, const uint4 &o)
{
    constexpr int E = Elem<F32>::E;
    const int lo = u * E - off;
    if (same && lo >= 0 && lo + E <= c) {
        *reinterpret_cast<uint4 *>((char *)dz + ((at + lo) << Elem<F32>::SHIFT)) = o;
    } else {
        float v[E];
        unit_values<F32>(o, v);
#pragma unroll
        for (int j = 0; j < E; ++j) if (lo + j >= 0 && lo + j < c) put<F32>(dz, at + lo + j, v[j]);
    }
}

// ----------------------------------------------------------------------------------------------------------------------
// one warp per row, short lists
// ----------------------------------------------------------------------------------------------------------------------
// A warp has few instructions per row and long latencies in front of them (weight -> entries -> listed logits), so they are
// taken out of the chain: entries and weight are loaded two rows ahead, the row and its listed logits one row ahead, all in
// registers.  NU units of 16 bytes per lane.
template <bool F32, int MODE, int NU, int KE>
__global__ void __launch_bounds__(WR_WARPS * 32)
distill_row_kernel(const DistillParams P)
{
    constexpr int E = Elem<F32>::E;
    __shared__ __align__(16) int sh_ids[WR_WARPS][32 * KE];
    __shared__ __align__(16) float sh_p[WR_WARPS][32 * KE];
    __shared__ double wl[WR_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, k4 = (P.k + 3) & ~3;
    const float c2 = LOG2E / P.temp, inv_t = 1.f / P.temp;
    const uint32_t low = F32 ? 0xFF800000u : 0xFF80FF80u;                   // -inf
    double total = 0;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t first = (int64_t)blockIdx.x * WR_WARPS + warp, step = (int64_t)gridDim.x * WR_WARPS;
    // one row ahead (b_) and two rows ahead (a_)
    Entries<KE> a_e, b_e;
    float a_w = 0.f, b_w = 0.f, a_tl = 0.f, b_tl = 0.f, b_lse = 0.f, b_z[KE];
    uint4 b_raw[NU];
    auto far = [&](int64_t row) {
        a_w = 0.f;
        if (row >= P.rows) return;
        a_e.load(P, row, lane);
        a_w = P.w ? P.w[row] : P.w_all;
        if (P.tlse) a_tl = P.tlse[row];
    };
    auto near = [&](int64_t row) {                                          // what far() loaded, and the row itself
        b_e = a_e; b_w = a_w; b_tl = a_tl;
        if (b_w == 0.f) return;
        const int64_t at = row * P.pz;
        const int off = misalign<F32>(P.z, at), nu = (P.c + off + E - 1) / E;
#pragma unroll
        for (int i = 0; i < NU; ++i) b_raw[i] = lane + 32 * i < nu ? load_unit<F32>(P.z, at, off, lane + 32 * i, P.c) : make_uint4(low, low, low, low);
#pragma unroll
        for (int i = 0; i < KE; ++i) b_z[i] = (uint32_t)b_e.id[i] < (uint32_t)P.c ? elem<F32>(P.z, at + b_e.id[i]) : 0.f;
        if (!(MODE & FWD)) b_lse = P.lse_in[row];
    };
    far(first);
    near(first);
    far(first + step);
    for (int64_t row = first; row < P.rows; row += step) {
        const float w = b_w, tl = b_tl, lse_in = b_lse;
        Entries<KE> e = b_e;
        float zt[KE];
        uint4 raw[NU];
#pragma unroll
        for (int i = 0; i < KE; ++i) zt[i] = b_z[i];
#pragma unroll
        for (int i = 0; i < NU; ++i) raw[i] = b_raw[i];
        if (row + step < P.rows) {
            near(row + step);
            far(row + 2 * step);
        }
        const int64_t dat = row * P.pdz;
        const int off = misalign<F32>(P.z, row * P.pz), nu = (P.c + off + E - 1) / E;
        const bool same = (MODE & BWD) && off == misalign<F32>(P.dz, dat);
        float p[KE], logp[KE], S = 0.f, loss = 0.f, lse = 0.f;
        if (w != 0.f) S = e.prepare(P, tl, p, logp);
        if (S != 0.f) {
            float m, scale = 1.f;
            if constexpr (MODE & FWD) {
                m = -FLT_MAX;
#pragma unroll
                for (int i = 0; i < NU; ++i) m = fmaxf(m, unit_max<F32>(raw[i]));
                m = warp_max_fast(m);
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < NU; ++i) s += unit_sum<F32>(raw[i], c2, m);
                s = warp_sum(s);
                if (s == 0.f) s = NAN;                                      // no logit above -inf: there is no softmax
                const float ls = logf(s);
                lse = m * inv_t + ls;
                scale = 1.f / s;
#pragma unroll
                for (int i = 0; i < KE; ++i) if (p[i] != 0.f) loss += p[i] * (logp[i] - ((zt[i] - m) * inv_t - ls));
                loss = warp_sum(loss) * P.temp * P.temp;
            } else {
                m = lse_in;
            }
            if constexpr (MODE & BWD) {
                const float gT = w * P.temp, gq = gT * S * scale;
                __syncwarp();                                               // every lane has the listed logits of its entries
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    const int u = lane + 32 * i;
                    if (u >= nu) break;
                    put_unit<F32>(P.dz, dat, off, same, u, P.c, unit_grad<F32, MODE>(raw[i], (MODE & FWD) ? c2 : inv_t, m, gq));
                }
                float pm[KE];
                e.merge(P.k, k4, lane, p, pm, sh_ids[warp], sh_p[warp]);
                __syncwarp();                                               // the listed classes go over what the dense pass wrote
#pragma unroll
                for (int i = 0; i < KE; ++i)
                    if (e.id[i] >= 0) put<F32>(P.dz, dat + e.id[i], gT * (S * (scale * power<MODE>(zt[i], c2, inv_t, m)) - pm[i]));
            }
        } else if constexpr (MODE & BWD) {
            for (int u = lane; u < nu; u += 32) put_unit<F32>(P.dz, dat, off, same, u, P.c, make_uint4(0, 0, 0, 0));
        }
        if constexpr (MODE & FWD) {
            if (lane == 0) {
                if (P.loss_rows) P.loss_rows[row] = loss;
                if (P.lse_out) P.lse_out[row] = lse;
                if (w != 0.f) total += (double)w * loss;
            }
        }
        __syncwarp();                                                       // sh_ids, sh_p are free again
    }
    if ((MODE & FWD) && P.part) {
        if (lane == 0) wl[warp] = total;
        __syncthreads();
        if (threadIdx.x == 0) {
            double a = 0;
            for (int i = 0; i < WR_WARPS; ++i) a += wl[i];
            P.part[blockIdx.x] = a;
        }
    }
}

// ----------------------------------------------------------------------------------------------------------------------
// one CTA, or a cluster of CTAs, per row
// ----------------------------------------------------------------------------------------------------------------------
// Warp-specialised, two or more CTAs per SM, so that the phases of one row (sum: bound by the exponential unit; gradient: by
// stores) overlap with other phases of another.  The helper warp prepares the next row's teacher entries and has the next row
// (or this CTA's slice of it) copied into shared memory, a half at a time as the consumers' last pass over the current row
// gives the halves up (short slices whole: a wait costs about 100 cycles, four chunks 205 us where two take 191): bulk asynchronous copies of the whole 16-byte units, the ragged first and last unit by hand, filled
// up with -inf.  The consumers' first pass takes the halves as they land, so it runs while the rest is on its way.
// A row is read from HBM exactly once.
// The first pass keeps maximum and sum per thread, moved on once per four units.
// Measured (4096 x 50001 bf16, loss and gradient, us): loads by the threads that use them 348; one CTA per SM with two row
// buffers 327; the same with the row held in registers and packed fp32 arithmetic 240 (loss alone 112, gradient alone 131:
// the phases of a row simply add up when all warps of an SM share it); two CTAs per SM with passes for maximum, sum and
// gradient over a row that has landed 189 (loss alone 148, gradient alone 151); this form 192 (117, 151).
struct RowSlot {                                    // what the helper prepares for a row
    float S, w;
};

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
// Barrier of the consumer warps.  An mbarrier with a bounded wait, not a hardware barrier: a warp that gave up must not leave
// the others waiting for it.
__device__ __forceinline__ bool consumer_sync(uint32_t bar, uint32_t &phase, int lane, volatile int *abort_flag)
{
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(bar);
    const bool ok = __all_sync(0xffffffffu, ptx::mbar_wait(bar, phase, abort_flag));
    phase ^= 1;
    return ok;
}
__device__ __forceinline__ void st_async_v4(uint32_t addr, uint32_t bar, float a, float b, float c, float d)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%2, %3, %4, %5}, [%1];"
                 ::"r"(addr), "r"(bar), "r"(__float_as_uint(a)), "r"(__float_as_uint(b)), "r"(__float_as_uint(c)), "r"(__float_as_uint(d)) : "memory");
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

__host__ __device__ constexpr int lists_of(int k) { return k <= SHORT_K ? 5 : 3; }
constexpr int CR_MAX_THREADS = 1024, CR_CHUNKS = 2, CR_WHOLE = 2048;      // slices below CR_WHOLE units are one chunk

template <bool F32, int MODE>
__global__ void __launch_bounds__(CR_MAX_THREADS, 1)
distill_cta_kernel(const DistillParams P, const int S_CTAS)
{
    constexpr int E = Elem<F32>::E;
    extern __shared__ __align__(16) uint4 buf[];                       // [P.stash] units, then the lists [2][LISTS][k4]
    __shared__ __align__(16) float4 msg[2][8];                         // per row parity: (maximum, sum, D, P) of every CTA of the cluster
    __shared__ __align__(8) uint64_t bars[7 + 2 * CR_CHUNKS];          // consumers, exchange[2], lists ready[2], lists free[2], chunk full[], empty[]
    __shared__ float red[2][2][32];
    __shared__ RowSlot slot[2];
    __shared__ int abort_s;
    volatile int *abort_flag = &abort_s;
    // per row: ids, log p, z of the listed classes, and for short lists p and its sum over equal ids (long ones use exp(log p))
    const int k4 = (P.k + 3) & ~3, nl = lists_of(P.k);
    const bool brief = P.k <= SHORT_K;
    int *ids0 = (int *)(buf + P.stash);
    const int nthr = blockDim.x - 32, nwarp = nthr >> 5;               // consumers; the last warp is the helper
    const int sweeps = (P.stash + nthr - 1) / nthr, chunk = (P.stash < CR_WHOLE ? sweeps : (sweeps + CR_CHUNKS - 1) / CR_CHUNKS) * nthr;   // units of a chunk
    const int nch = (P.stash + chunk - 1) / chunk;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const float c2 = LOG2E / P.temp, inv_t = 1.f / P.temp;
    const uint32_t rank = S_CTAS > 1 ? blockIdx.x % S_CTAS : 0;
    const int64_t first = blockIdx.x / S_CTAS, step = gridDim.x / S_CTAS;
    const uint32_t cons = ptx::smem_u32(bars), exch0 = cons + 8, ready0 = cons + 24, lists0 = cons + 40, full0 = cons + 56, empty0 = full0 + 8 * CR_CHUNKS;
    pdl_launch_dependents();
    if (tid == 0) {
        ptx::mbar_init(cons, nwarp);
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(exch0 + 8 * b, 1);
            ptx::mbar_init(ready0 + 8 * b, 1);
            ptx::mbar_init(lists0 + 8 * b, nwarp);
        }
        for (int i = 0; i < CR_CHUNKS; ++i) { ptx::mbar_init(full0 + 8 * i, 1); ptx::mbar_init(empty0 + 8 * i, nwarp); }
        abort_s = 0;
        ptx::mbar_init_fence();
    }
    __syncthreads();
    if (S_CTAS > 1) cluster_barrier();                                 // every peer's barriers exist
    pdl_wait();
    // a row's units, and the slice of them that this CTA has
    auto geometry = [&](int64_t row, int &off, int &nu, int &u0, int &u1) {
        off = misalign<F32>(P.z, row * P.pz);
        nu = (P.c + off + E - 1) / E;
        u0 = S_CTAS == 1 ? 0 : (int)((int64_t)nu * rank / S_CTAS);
        u1 = S_CTAS == 1 ? nu : (int)((int64_t)nu * (rank + 1) / S_CTAS);
    };
    bool ok = true;
    double total = 0;
    if (warp == nwarp) {
        // ------------------------------------------------------------------ helper
        int i = 0;
        uint32_t loads = 0;                                            // rows copied so far: the phase of the chunk barriers
        float w_next = first < P.rows ? (P.w ? P.w[first] : P.w_all) : 0.f;
        float tl = P.tlse && first < P.rows ? P.tlse[first] : 0.f;
        Entries<SHORT_K / 32> ahead;
        if (brief && first < P.rows) ahead.load(P, first, lane);
        for (int64_t row = first; row < P.rows; row += step, ++i) {
            const int b = i & 1;
            const float w = w_next;
            if (row + step < P.rows && P.w) w_next = P.w[row + step];
            int *ids = ids0 + b * nl * k4;
            float *logp = (float *)(ids + k4), *zt = logp + k4, *pr = zt + k4, *pm = pr + k4;
            int off, nu, u0, u1;
            geometry(row, off, nu, u0, u1);
            const int64_t at = row * P.pz;
            const int e0 = u0 * E - off, e1 = u1 * E - off;            // elements of the slice
            ok = __all_sync(0xffffffffu, ptx::mbar_wait(lists0 + 8 * b, ((uint32_t)(i >> 1) & 1) ^ 1, abort_flag));
            if (!ok) break;
            float S = 0.f;
            if (w != 0.f) {
                if (brief) {
                    float p[SHORT_K / 32], lp[SHORT_K / 32], q[SHORT_K / 32];
                    S = ahead.prepare(P, tl, p, lp);
                    if (S != 0.f) {
                        ahead.merge(P.k, k4, lane, p, q, ids, pr);
#pragma unroll
                        for (int e = 0; e < SHORT_K / 32; ++e)
                            if (lane + 32 * e < k4) { logp[lane + 32 * e] = lp[e]; pm[lane + 32 * e] = q[e]; }
                    }
                } else {
                    S = teacher_row(P, row, lane, ids, logp);
                }
                // the listed logits of the slice, before anything of the row is written (dz may be z)
                if (S != 0.f)
                    for (int j = lane; j < P.k; j += 32) {
                        const int id = ids[j];
                        zt[j] = id >= 0 && id >= e0 && id < e1 ? elem<F32>(P.z, at + id) : 0.f;
                    }
            }
            if (brief && row + step < P.rows) ahead.load(P, row + step, lane);
            if (P.tlse && row + step < P.rows) tl = P.tlse[row + step];
            if (lane == 0) { slot[b].S = S; slot[b].w = w; }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ready0 + 8 * b);
            if (S == 0.f) continue;                                    // nothing of this row is read
            // whole units of the slice: not the first if it starts in front of the row, not the last if it ends behind it
            const int f0 = u0 == 0 && off ? 1 : u0, f1 = u1 == nu && (P.c + off) % E ? nu - 1 : u1;
            for (int ch = 0; ch < nch; ++ch) {
                ok = __all_sync(0xffffffffu, ptx::mbar_wait(empty0 + 8 * ch, (loads & 1) ^ 1, abort_flag));
                if (!ok) break;
                const int c0 = u0 + ch * chunk, c1 = c0 + chunk, g0 = c0 > f0 ? c0 : f0, g1 = c1 < f1 ? c1 : f1;
                if (lane == 1 && f0 > u0 && u1 > u0 && ch == 0) buf[0] = load_unit<F32>(P.z, at, off, u0, P.c);
                if (lane == 2 && f1 < u1 && f1 >= f0 && f1 >= c0 && f1 < c1) buf[f1 - u0] = load_unit<F32>(P.z, at, off, f1, P.c);
                __syncwarp();
                if (lane == 0) {
                    if (g1 > g0) {
                        ptx::fence_proxy_async();                      // the chunk's last readers, then the copy
                        ptx::mbar_expect_tx(full0 + 8 * ch, (uint32_t)(g1 - g0) * 16);
                        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                     ::"r"(ptx::smem_u32(buf + (g0 - u0))), "l"((const char *)P.z + ((at + (int64_t)g0 * E - off) << Elem<F32>::SHIFT)),
                                       "r"((uint32_t)(g1 - g0) * 16), "r"(full0 + 8 * ch) : "memory");
                    } else {
                        ptx::mbar_arrive(full0 + 8 * ch);
                    }
                }
            }
            if (!ok) break;
            ++loads;
        }
    } else {
        // ------------------------------------------------------------------ consumers
        int i = 0;
        uint32_t cphase = 0, loads = 0;
        for (int64_t row = first; row < P.rows; row += step, ++i) {
            const int b = i & 1;
            const int64_t dat = row * P.pdz;
            int off, nu, u0, u1;
            geometry(row, off, nu, u0, u1);
            const int n = u1 - u0;
            const bool same = (MODE & BWD) && off == misalign<F32>(P.dz, dat);
            const int e0 = u0 * E - off, e1 = u1 * E - off;            // elements of the slice
            const int *ids = ids0 + b * nl * k4;
            const float *logp = (const float *)(ids + k4), *zt = logp + k4, *pr = zt + k4, *pm = pr + k4;
            ok = __all_sync(0xffffffffu, ptx::mbar_wait(ready0 + 8 * b, (uint32_t)(i >> 1) & 1, abort_flag));
            if (!ok) break;
            const float S = slot[b].S, w = slot[b].w;
            float loss = 0.f, lse = 0.f;
            auto landed = [&](int ch) { return __all_sync(0xffffffffu, ptx::mbar_wait(full0 + 8 * ch, loads & 1, abort_flag)); };
            auto give_back = [&](int ch) {
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(empty0 + 8 * ch);
            };
            if (S != 0.f) {
                float m, s = 1.f, scale = 1.f;                         // maximum of z, sum of e^((z - m) / T)
                if constexpr (MODE & FWD) {
                    s = 0.f;
                    m = -FLT_MAX;                                      // with -inf alone the sum stays 0
                    for (int ch = 0; ch < nch; ++ch) {
                        if (!(ok = landed(ch))) break;
                        const int end = (ch + 1) * chunk < n ? (ch + 1) * chunk : n;
                        for (int u = ch * chunk + tid; u < end; u += 4 * nthr) {       // four units at a time
                            uint4 raw[4];
                            float top = -FLT_MAX;
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                if (u + q * nthr < end) { raw[q] = buf[u + q * nthr]; top = fmaxf(top, unit_max<F32>(raw[q])); }
                            if (top > m) { s *= ex2((m - top) * c2); m = top; }
#pragma unroll
                            for (int q = 0; q < 4; ++q) if (u + q * nthr < end) s += unit_sum<F32>(raw[q], c2, m);
                        }
                        if (!(MODE & BWD)) give_back(ch);              // the last pass
                    }
                    if (!ok) break;
                    const float mt = m;
                    m = warp_max_fast(m);
                    s = warp_sum(s * ex2((mt - m) * c2));
                    if (lane == 0) { red[i & 1][0][warp] = m; red[i & 1][1][warp] = s; }
                    if (!(ok = consumer_sync(cons, cphase, lane, abort_flag))) break;
                    const float mw = lane < nwarp ? red[i & 1][0][lane] : -FLT_MAX;
                    m = warp_max_fast(mw);
                    s = warp_sum(lane < nwarp ? red[i & 1][1][lane] * ex2((mw - m) * c2) : 0.f);
                    float D = 0.f, PS = 0.f;                           // sum_j p_j (log p_j - (z_j - m) / T), sum_j p_j over the slice's entries
                    if (warp == 0) {
                        for (int j = lane; j < P.k; j += 32) {
                            const int id = ids[j];
                            if (id < 0 || id < e0 || id >= e1) continue;
                            const float p = brief ? pr[j] : expf(logp[j]);
                            if (p != 0.f) { D += p * (logp[j] - (zt[j] - m) * inv_t); PS += p; }
                        }
                        D = warp_sum(D); PS = warp_sum(PS);
                    }
                    if (S_CTAS > 1) {
                        const int x = loads & 1;
                        if (warp == 0) {
                            if (lane == 0) ptx::mbar_expect_tx(exch0 + 8 * x, 16 * S_CTAS);
                            __syncwarp();
                            if (lane < S_CTAS)
                                st_async_v4(peer_addr(ptx::smem_u32(&msg[x][rank]), lane), peer_addr(exch0 + 8 * x, lane), m, s, D, PS);
                        }
                        ok = __all_sync(0xffffffffu, ptx::mbar_wait(exch0 + 8 * x, (loads >> 1) & 1, abort_flag));
                        if (!ok) break;
                        m = -FLT_MAX; s = 0.f;
                        for (int r = 0; r < S_CTAS; ++r) join(m, s, msg[x][r].x, msg[x][r].y, c2);
                        D = 0.f; PS = 0.f;
                        for (int r = 0; r < S_CTAS; ++r) {
                            D += msg[x][r].z + (msg[x][r].w != 0.f ? msg[x][r].w * ((m - msg[x][r].x) * inv_t) : 0.f);
                            PS += msg[x][r].w;
                        }
                    }
                    if (s == 0.f) s = NAN;                             // no logit above -inf: there is no softmax
                    scale = 1.f / s;
                    if (rank == 0 && warp == 0) {
                        const float ls = logf(s);
                        lse = m * inv_t + ls;
                        loss = (D + PS * ls) * P.temp * P.temp;
                    }
                } else {
                    m = P.lse_in[row];
                }
                if constexpr (MODE & BWD) {
                    const float gT = w * P.temp, gq = gT * S * scale;
                    for (int ch = 0; ch < nch; ++ch) {
                        if (!(MODE & FWD) && !(ok = landed(ch))) break;
                        const int end = (ch + 1) * chunk < n ? (ch + 1) * chunk : n;
#pragma unroll 2
                        for (int u = ch * chunk + tid; u < end; u += nthr) {
                            put_unit<F32>(P.dz, dat, off, same, u0 + u, P.c, unit_grad<F32, MODE>(buf[u], (MODE & FWD) ? c2 : inv_t, m, gq));
                        }
                        give_back(ch);
                    }
                    if (!ok) break;
                    if (!(ok = consumer_sync(cons, cphase, lane, abort_flag))) break;    // the listed classes go over what the dense pass wrote
                    for (int j = tid; j < P.k; j += nthr) {
                        const int id = ids[j];
                        if (id < 0 || id < e0 || id >= e1) continue;
                        float p = 0.f;
                        if (brief) p = pm[j];
                        else for (int q = 0; q < P.k; ++q) if (ids[q] == id) p += expf(logp[q]);
                        put<F32>(P.dz, dat + id, gT * (S * (scale * power<MODE>(zt[j], c2, inv_t, m)) - p));
                    }
                }
                ++loads;
            } else if constexpr (MODE & BWD) {
                float v[E];
#pragma unroll
                for (int j = 0; j < E; ++j) v[j] = 0.f;
                for (int u = u0 + tid; u < u1; u += nthr) store_unit<F32>(P.dz, dat, off, same, u, P.c, v);
            }
            if ((MODE & FWD) && rank == 0 && tid == 0) {
                if (P.loss_rows) P.loss_rows[row] = loss;
                if (P.lse_out) P.lse_out[row] = lse;
                if (w != 0.f) total += (double)w * loss;
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(lists0 + 8 * b);           // ... and the lists
        }
        if ((MODE & FWD) && P.part && rank == 0 && tid == 0) P.part[blockIdx.x / S_CTAS] = total;
    }
    if (!ok) {
        if (lane == 0 && P.status) atomicExch(P.status, (int)LAMP_ERR_TIMEOUT);
        ptx::settle();                                                 // copies in flight
    }
    __syncthreads();
    if (S_CTAS > 1) cluster_barrier();                                 // no CTA leaves while a peer may still write to it
}

// ----------------------------------------------------------------------------------------------------------------------
// one thread per row: few classes (a segmentation network's), many rows
// ----------------------------------------------------------------------------------------------------------------------
// 256 rows (128 of more than 32 classes) per turn go through shared memory, so that global memory sees whole lines although
// a row is only a few words; the next turn's rows and entries are copied there asynchronously meanwhile (up to 32 classes).
// A thread then works on its own row.  fp32 rows whose stride hits each bank at most twice are worked on where they landed;
// others are first spread out to fp32 rows of odd pitch.  A thread adds its gradient up in its own row, listed classes after
// the dense part, so a class listed twice is simply met twice.  Up to 4 entries per row (SHORT) stay in registers.
// Measured (2,097,152 x 10 fp32, k = 4, loss and gradient, us): loads by the threads, no copies ahead 86; this form 66, of
// which most is instruction issue (2.9 per cycle).
constexpr int TR_MAX_C = 128, TR_REG_C = 32, TR_MAX_K = 32;
__host__ __device__ constexpr int tr_rows(int cp) { return cp ? 256 : 128; }      // CP = 0: more than TR_REG_C classes
struct ThreadPlan {
    int32_t vec;                                    // rows are back to back and 16-byte aligned
    int32_t ahead;                                  // copies run a turn ahead (two stages)
    int32_t direct;                                 // rows are worked on in the stage
    int32_t stage_bytes, pitch;                     // of one stage; floats between the rows that are worked on
};

__device__ __forceinline__ void copy_async16(void *dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(dst)), "l"(src) : "memory");
}

template <bool F32, int MODE, int CP, bool SHORT>
__global__ void __launch_bounds__(tr_rows(CP))
distill_thread_kernel(const DistillParams P, const ThreadPlan G)
{
    constexpr int E = Elem<F32>::E, TR_ROWS = tr_rows(CP), ES = F32 ? 4 : 2;
    extern __shared__ __align__(16) char stage_s[];                    // stages: rows [rows][c], ids [rows][k], logits [rows][k]; then the spread rows
    __shared__ double wl[TR_ROWS / 32];
    const int tid = threadIdx.x, c = P.c, k = P.k;
    float *spread = (float *)(stage_s + (G.ahead ? 2 : 1) * G.stage_bytes);
    const int zb = G.ahead ? (TR_ROWS * c * ES + 15) & ~15 : 0, kbytes = (TR_ROWS * k * 4 + 15) & ~15;
    const float c2 = LOG2E / P.temp, inv_t = 1.f / P.temp;
    // x / c = umulhi(x, ceil(2^32 / c)) for x < 2^14, c in 2 .. 128 (the error x (div c - 2^32) stays below 2^32)
    const uint32_t div_c = (uint32_t)((0x100000000ull + c - 1) / c);
    auto over_c = [&](int x) { return c == 1 ? (uint32_t)x : __umulhi((uint32_t)x, div_c); };
    double total = 0;
    pdl_launch_dependents();
    pdl_wait();
    auto spread_unit = [&](const uint4 &raw, int i0, int n) {          // elements i0 .. of the turn to the rows of odd pitch
        float v[E];
        unit_values<F32>(raw, v);
        uint32_t r = over_c(i0), col = i0 - r * c;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (i0 + j < n) spread[r * G.pitch + col] = v[j];
            if (++col == (uint32_t)c) { col = 0; ++r; }
        }
    };
    // a turn's rows and entries into a stage: asynchronously where all of them are there in whole 16-byte units
    auto fill = [&](int64_t r0, char *st) {
        const int nr = (int)(P.rows - r0 < TR_ROWS ? P.rows - r0 : TR_ROWS);
        if (G.ahead && nr == TR_ROWS) {
            const char *z = (const char *)P.z + r0 * c * ES, *id = (const char *)(P.idx + r0 * k), *tt = (const char *)(P.t + r0 * k);
            for (int i = tid; i < TR_ROWS * c * ES / 16; i += TR_ROWS) copy_async16(st + i * 16, z + i * 16);
            for (int i = tid; i < TR_ROWS * k * 4 / 16; i += TR_ROWS) {
                copy_async16(st + zb + i * 16, id + i * 16);
                copy_async16(st + zb + kbytes + i * 16, tt + i * 16);
            }
        } else {
            const int n = nr * c;
            if (!G.ahead && G.vec) {                                   // straight to where the rows are worked on
                const uint4 *src = reinterpret_cast<const uint4 *>((const char *)P.z + r0 * c * ES);
                for (int i = tid; i < n / E; i += TR_ROWS) spread_unit(src[i], i * E, n);
                for (int i = n / E * E + tid; i < n; i += TR_ROWS) spread[over_c(i) * G.pitch + i - over_c(i) * c] = elem<F32>(P.z, r0 * c + i);
            } else {
                for (int i = tid; i < n; i += TR_ROWS) {
                    const uint32_t r = over_c(i), col = i - r * c;
                    if (!G.ahead) spread[r * G.pitch + col] = elem<F32>(P.z, (r0 + r) * P.pz + col);
                    else if constexpr (F32) ((float *)st)[i] = elem<F32>(P.z, (r0 + r) * P.pz + col);
                    else ((bf16 *)st)[i] = ((const bf16 *)P.z)[(r0 + r) * P.pz + col];
                }
            }
            for (int i = tid; i < nr * k; i += TR_ROWS) {
                ((int *)(st + zb))[i] = P.idx[r0 * k + i];
                ((float *)(st + zb + kbytes))[i] = P.t[r0 * k + i];
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const int64_t first = (int64_t)blockIdx.x * TR_ROWS, step = (int64_t)gridDim.x * TR_ROWS;
    float w_n = 0.f, tl_n = 0.f, lin_n = 0.f;
    auto scalars = [&](int64_t r) {
        w_n = r < P.rows ? (P.w ? P.w[r] : P.w_all) : 0.f;
        if (P.tlse) tl_n = r < P.rows ? P.tlse[r] : 0.f;
        if (!(MODE & FWD)) lin_n = r < P.rows ? P.lse_in[r] : 0.f;
    };
    if (first < P.rows && G.ahead) fill(first, stage_s);
    scalars(first + tid);
    int s_at = 0;
    for (int64_t r0 = first; r0 < P.rows; r0 += step) {
        const int nr = (int)(P.rows - r0 < TR_ROWS ? P.rows - r0 : TR_ROWS);
        char *st = stage_s + s_at * G.stage_bytes;
        if (!G.ahead) fill(r0, st);
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();                                               // the stage is filled; the other one has been read
        const float w = w_n, tl = tl_n, lin = lin_n;
        if (G.ahead && r0 + step < P.rows) { s_at ^= 1; fill(r0 + step, stage_s + s_at * G.stage_bytes); }
        scalars(r0 + step + tid);
        float *zr = (G.direct ? (float *)st : spread) + tid * G.pitch;
        if (G.ahead && !G.direct) {
            for (int i = tid; i < (nr * c + E - 1) / E; i += TR_ROWS) spread_unit(reinterpret_cast<const uint4 *>(st)[i], i * E, nr * c);
            __syncthreads();
        }
        const int *id_s = (const int *)(st + zb) + tid * k;
        const float *t_s = (const float *)(st + zb + kbytes) + tid * k;
        // the teacher: S and, for every entry of a listed class, log p and p.  Short lists keep them in registers.
        int id4[SHORT ? 4 : 1];
        float lp4[SHORT ? 4 : 1], p4[SHORT ? 4 : 1];
        float S = 0.f, mt = 0.f, lt = tl;                              // log p = (t - mt) / T - lt
        if constexpr (SHORT) {
            mt = -INFINITY;
            bool nan = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                id4[j] = -1; lp4[j] = -INFINITY;
                if (j < k && w != 0.f) {
                    id4[j] = id_s[j];
                    if ((uint32_t)id4[j] < (uint32_t)c) lp4[j] = t_s[j]; else id4[j] = -1;
                    nan |= lp4[j] != lp4[j];
                    mt = fmaxf(mt, lp4[j]);
                }
            }
            if (!P.tlse) {
                if (mt != -INFINITY || nan) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) { lp4[j] -= mt; p4[j] = ex2(lp4[j] * c2); S += p4[j]; }
                    const float inv = 1.f / S, l = logf(S);
#pragma unroll
                    for (int j = 0; j < 4; ++j) { p4[j] *= inv; lp4[j] = fmaf(lp4[j], inv_t, -l); }
                    S = S == S ? 1.f : NAN;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) { lp4[j] = fmaf(lp4[j], inv_t, -lt); p4[j] = id4[j] >= 0 ? expf(lp4[j]) : 0.f; S += p4[j]; }
            }
        } else if (w != 0.f) {
            if (P.tlse) {
                for (int j = 0; j < k; ++j) if ((uint32_t)id_s[j] < (uint32_t)c) S += expf(fmaf(t_s[j], inv_t, -lt));
            } else {
                float top = -INFINITY;
                bool nan = false;
                for (int j = 0; j < k; ++j) {
                    if ((uint32_t)id_s[j] >= (uint32_t)c) continue;
                    nan |= t_s[j] != t_s[j];
                    top = fmaxf(top, t_s[j]);
                }
                if (top != -INFINITY || nan) {
                    float s = 0.f;
                    for (int j = 0; j < k; ++j) if ((uint32_t)id_s[j] < (uint32_t)c) s += ex2((t_s[j] - top) * c2);
                    mt = top;
                    lt = logf(s);
                    S = s == s ? 1.f : NAN;
                }
            }
        }
        auto entries = [&](auto f) {                                   // f(class, log p, p)
            if constexpr (SHORT) {
#pragma unroll
                for (int j = 0; j < 4; ++j) if (id4[j] >= 0) f(id4[j], lp4[j], p4[j]);
            } else {
                for (int j = 0; j < k; ++j) {
                    const int id = id_s[j];
                    if ((uint32_t)id < (uint32_t)c) { const float lp = fmaf(t_s[j] - mt, inv_t, -lt); f(id, lp, expf(lp)); }
                }
            }
        };
        float loss = 0.f, lse = 0.f;
        if (S != 0.f) {
            // CP > 0: the row in registers; otherwise it is walked in shared memory, where the exponentials replace the logits
            float v[CP ? CP : 1];
            if constexpr (CP > 0) {
#pragma unroll
                for (int i = 0; i < CP; ++i) v[i] = i < c ? zr[i] : -INFINITY;
            }
            float m, scale = 1.f, ls = 0.f;
            if constexpr (MODE & FWD) {
                m = -FLT_MAX;
                float s = 0.f;
                if constexpr (CP > 0) {
#pragma unroll
                    for (int i = 0; i < CP; ++i) m = fmaxf(m, v[i]);
#pragma unroll
                    for (int i = 0; i < CP; ++i) { v[i] = ex2((v[i] - m) * c2); s += v[i]; }
                } else {
#pragma unroll 4
                    for (int i = 0; i < c; ++i) m = fmaxf(m, zr[i]);
                }
                // the listed logits, before their exponentials take their place
                float ps = 0.f;
                entries([&](int id, float lp, float p) {
                    if (p != 0.f) { loss += p * (lp - (zr[id] - m) * inv_t); ps += p; }
                });
                if constexpr (CP == 0) {
#pragma unroll 4
                    for (int i = 0; i < c; ++i) { const float e = ex2((zr[i] - m) * c2); s += e; if (MODE & BWD) zr[i] = e; }
                }
                if (s == 0.f) s = NAN;
                scale = 1.f / s;
                ls = logf(s);
                lse = m * inv_t + ls;
                loss = (loss + ps * ls) * P.temp * P.temp;
            } else {
                m = lin;
                if constexpr (CP > 0) {
#pragma unroll
                    for (int i = 0; i < CP; ++i) v[i] = ex2(fmaf(v[i], inv_t, -m) * LOG2E);
                }
            }
            const float gT = w * P.temp, gq = gT * S * scale;
            if constexpr (MODE & BWD) {
                if constexpr (CP > 0) {
#pragma unroll
                    for (int i = 0; i < CP; ++i) if (i < c) zr[i] = gq * v[i];
                } else {
#pragma unroll 4
                    for (int i = 0; i < c; ++i) zr[i] = gq * ((MODE & FWD) ? zr[i] : ex2(fmaf(zr[i], inv_t, -m) * LOG2E));
                }
                entries([&](int id, float, float p) { zr[id] -= gT * p; });
            }
        } else if ((MODE & BWD) && tid < nr) {
            for (int i = 0; i < c; ++i) zr[i] = 0.f;
        }
        if ((MODE & FWD) && tid < nr) {
            if (P.loss_rows) P.loss_rows[r0 + tid] = loss;
            if (P.lse_out) P.lse_out[r0 + tid] = lse;
            if (w != 0.f) total += (double)w * loss;
        }
        if constexpr (MODE & BWD) {
            __syncthreads();
            const int n = nr * c;
            if (G.vec) {
                uint4 *dst = reinterpret_cast<uint4 *>((char *)P.dz + r0 * c * ES);
                for (int i = tid; i < n / E; i += TR_ROWS) {
                    if (G.direct) { dst[i] = reinterpret_cast<const uint4 *>(st)[i]; continue; }
                    float v[E];
                    uint32_t r = over_c(i * E), col = i * E - r * c;
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        v[j] = spread[r * G.pitch + col];
                        if (++col == (uint32_t)c) { col = 0; ++r; }
                    }
                    dst[i] = unit_raw<F32>(v);
                }
                for (int i = n / E * E + tid; i < n; i += TR_ROWS) {
                    const uint32_t r = over_c(i);
                    put<F32>(P.dz, r0 * c + i, (G.direct ? (float *)st : spread)[r * G.pitch + i - r * c]);
                }
            } else {
                for (int i = tid; i < n; i += TR_ROWS) {
                    const uint32_t r = over_c(i), col = i - r * c;
                    put<F32>(P.dz, (r0 + r) * P.pdz + col, (G.direct ? (float *)st : spread)[r * G.pitch + col]);
                }
            }
        }
        if (!G.ahead) __syncthreads();                                 // the stage and the spread rows are free again
    }
    if ((MODE & FWD) && P.part) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        if ((tid & 31) == 0) wl[tid >> 5] = total;
        __syncthreads();
        if (tid == 0) {
            double a = 0;
            for (int i = 0; i < TR_ROWS / 32; ++i) a += wl[i];
            P.part[blockIdx.x] = a;
        }
    }
}

__global__ void __launch_bounds__(256)
distill_sum_kernel(const double *__restrict__ part, int n, float *__restrict__ loss)
{
    __shared__ double sm[256];
    pdl_launch_dependents();
    pdl_wait();
    double a = 0;
    for (int i = threadIdx.x; i < n; i += 256) a += part[i];
    sm[threadIdx.x] = a;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
        if (threadIdx.x < o) sm[threadIdx.x] += sm[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) *loss = (float)sm[0];
}

template <bool F32, int MODE>
lamp_status_t launch_warp(const DistillParams &P, int grid, cudaStream_t st)
{
    const int smem = WR_WARPS * 3 * P.k * 4;
    if (smem > 32 * 1024) {                                  // static shared memory counts too: well below the 48 KB default
        static SmemAttrOnce attr;
        const lamp_status_t s = attr.ensure(distill_warp_kernel<F32, MODE>, WR_WARPS * 3 * MAX_K * 4);
        if (s != LAMP_OK) return s;
    }
    return launch_pdl(true, distill_warp_kernel<F32, MODE>, dim3(grid), dim3(WR_WARPS * 32), (size_t)smem, st, P);
}

template <bool F32, int MODE, int NU>
lamp_status_t launch_row(const DistillParams &P, int grid, cudaStream_t st)
{
    if (P.k <= 32) return launch_pdl(true, distill_row_kernel<F32, MODE, NU, 1>, dim3(grid), dim3(WR_WARPS * 32), (size_t)0, st, P);
    return launch_pdl(true, distill_row_kernel<F32, MODE, NU, SHORT_K / 32>, dim3(grid), dim3(WR_WARPS * 32), (size_t)0, st, P);
}
template <bool F32, int MODE>
lamp_status_t launch_row_u(const DistillParams &P, int nu, int grid, cudaStream_t st)
{
    if (nu == 2) return launch_row<F32, MODE, 2>(P, grid, st);
    return launch_row<F32, MODE, RW_MAX_UNITS>(P, grid, st);
}

template <bool F32, int MODE, int CP>
lamp_status_t launch_thread(const DistillParams &P, int grid, bool vec, cudaStream_t st)
{
    constexpr int R = tr_rows(CP), ES = F32 ? 4 : 2;
    ThreadPlan G = {};
    G.vec = vec;
    G.ahead = CP > 0 && vec && (((uintptr_t)P.idx | (uintptr_t)P.t) & 15) == 0;
    G.direct = G.ahead && F32 && P.c % 4 != 0;                               // stride c: each bank is hit by c's power of two, at most 2
    G.pitch = G.direct ? P.c : P.c | 1;
    G.stage_bytes = (G.ahead ? (R * P.c * ES + 15) & ~15 : 0) + 2 * ((R * P.k * 4 + 15) & ~15);
    const int smem = (G.ahead ? 2 : 1) * G.stage_bytes + (G.direct ? 0 : R * G.pitch * 4);
    const bool brief = P.k <= 4;
    auto kernel = brief ? distill_thread_kernel<F32, MODE, CP, true> : distill_thread_kernel<F32, MODE, CP, false>;
    if (smem > 32 * 1024) {
        static SmemAttrOnce attr[2];
        const lamp_status_t s = attr[brief].ensure(kernel, 226 * 1024);
        if (s != LAMP_OK) return s;
    }
    return launch_pdl(true, kernel, dim3(grid), dim3(R), (size_t)smem, st, P, G);
}
template <bool F32, int MODE>
lamp_status_t launch_thread_c(const DistillParams &P, int grid, bool vec, cudaStream_t st)
{
    if (P.c <= 4) return launch_thread<F32, MODE, 4>(P, grid, vec, st);
    if (P.c <= 12) return launch_thread<F32, MODE, 12>(P, grid, vec, st);
    if (P.c <= 20) return launch_thread<F32, MODE, 20>(P, grid, vec, st);
    if (P.c <= TR_REG_C) return launch_thread<F32, MODE, 32>(P, grid, vec, st);
    return launch_thread<F32, MODE, 0>(P, grid, vec, st);
}

template <bool F32, int MODE>
lamp_status_t launch_cta(const DistillParams &P, int grid, int splits, int threads, int smem, cudaStream_t st)
{
    static SmemAttrOnce attr;
    const lamp_status_t s = attr.ensure(distill_cta_kernel<F32, MODE>, 226 * 1024);
    if (s != LAMP_OK) return s;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = splits; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = splits > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, distill_cta_kernel<F32, MODE>, P, splits) == cudaSuccess ? LAMP_OK : LAMP_ERR_CUDA;
}

template <int MODE>
lamp_status_t run(DistillParams &P, bool f32, float *loss, void *ws, cudaStream_t st)
{
    const int sms = sm_count();
    int parts;
    lamp_status_t s;
    P.part = loss ? (double *)ws : nullptr;
    P.status = status_word_ptr();
    if (P.c <= TR_MAX_C && P.k <= TR_MAX_K) {
        const int turn = tr_rows(P.c <= TR_REG_C), room = MAX_PARTS / sms * sms;     // as many turns at a time as there are partial losses
        const int64_t need = (P.rows + turn - 1) / turn;
        parts = (int)(need < room ? need : room);
        const bool vec = P.pz == P.c && ((uintptr_t)P.z & 15) == 0 && (!(MODE & BWD) || (P.pdz == P.c && ((uintptr_t)P.dz & 15) == 0));
        s = f32 ? launch_thread_c<true, MODE>(P, parts, vec, st) : launch_thread_c<false, MODE>(P, parts, vec, st);
    } else if (P.k <= SHORT_K && P.c <= (f32 ? 4 : 8) * (32 * RW_MAX_UNITS - 1)) {
        const int units = (P.c + (f32 ? 3 : 7)) / (f32 ? 4 : 8) + 1, nu = units <= 64 ? 2 : RW_MAX_UNITS;
        const int64_t need = (P.rows + WR_WARPS - 1) / WR_WARPS, room = (int64_t)sms * (nu == 2 && P.k <= 32 ? 3 : 2);
        parts = (int)(need < room ? need : room);
        s = f32 ? launch_row_u<true, MODE>(P, nu, parts, st) : launch_row_u<false, MODE>(P, nu, parts, st);
    } else if (P.c <= WR_MAX_C) {
        const int64_t need = (P.rows + WR_WARPS - 1) / WR_WARPS;
        parts = (int)(need < 8ll * sms ? need : 8ll * sms);
        if (parts > MAX_PARTS) parts = MAX_PARTS;
        s = f32 ? launch_warp<true, MODE>(P, parts, st) : launch_warp<false, MODE>(P, parts, st);
    } else {
        const int units = (P.c + (f32 ? 3 : 7)) / (f32 ? 4 : 8) + 1;
        const int lists = 2 * lists_of(P.k) * ((P.k + 3) & ~3) * 4;
        const int room1 = (224 * 1024 - lists) / 16, room2 = (111 * 1024 - lists) / 16;      // units of a slice with one or two CTAs per SM
        // a cluster per row where a slice would not fit otherwise, or where rows alone would leave SMs idle and every CTA still
        // has about two units a thread
        int splits = 1;
        while (splits < 8 && ((units + splits - 1) / splits + 1 > room2 || (P.rows * splits * 2 <= sms && units >= 2048 * splits))) splits *= 2;
        const int slice = (units + splits - 1) / splits + 1;
        if (slice > room1) return LAMP_ERR_UNSUPPORTED;
        P.stash = slice;
        // about a dozen units per consumer thread; 1024 threads per SM (64 registers), shared between as many CTAs as fit
        int threads = (slice / 12 + 31) / 32 * 32;
        const int most = slice > room2 ? CR_MAX_THREADS - 32 : CR_MAX_THREADS / 2 - 32;
        threads = 32 + (threads < 96 ? 96 : threads > most ? most : threads);
        const int smem = slice * 16 + lists;
        int per_sm = CR_MAX_THREADS / threads;
        if (per_sm > 226 * 1024 / (smem + 2048)) per_sm = 226 * 1024 / (smem + 2048);
        if (per_sm < 1) per_sm = 1;
        int64_t groups = (int64_t)per_sm * sms / splits;
        if (groups > P.rows) groups = P.rows;
        parts = (int)groups;
        s = f32 ? launch_cta<true, MODE>(P, parts * splits, splits, threads, smem, st) : launch_cta<false, MODE>(P, parts * splits, splits, threads, smem, st);
    }
    if (s != LAMP_OK || !loss) return s;
    return launch_pdl(true, distill_sum_kernel, dim3(1), dim3(256), 0, st, (const double *)ws, parts, loss);
}

lamp_status_t check_teacher(const lamp_teacher_topk_t *t)
{
    if (!t || t->k < 1 || !(t->temperature > 0.f) || t->temperature > 3.402823466e+38f) return LAMP_ERR_INVALID_ARG;
    if (t->k > MAX_K) return LAMP_ERR_UNSUPPORTED;
    if (t->temperature < 0x1p-60f || t->temperature > 0x1p60f) return LAMP_ERR_UNSUPPORTED;     // T^2 and log2(e) / T stay well inside fp32
    if (((uintptr_t)t->idx | (uintptr_t)t->logits | (uintptr_t)t->lse) & 3) return LAMP_ERR_INVALID_ARG;
    return LAMP_OK;
}

lamp_status_t fill(DistillParams *P, const lamp_tensor_t *z, const lamp_teacher_topk_t *t, const float *w, const lamp_tensor_t *dz)
{
    lamp_status_t s;
    if ((s = check_view(z, true)) != LAMP_OK || (s = check_teacher(t)) != LAMP_OK) return s;
    if (z->c > (z->dtype == LAMP_F32 ? 200000 : 400000)) return LAMP_ERR_UNSUPPORTED;       // a row in the shared memory of 8 CTAs
    const TView v = make_view(z);
    *P = DistillParams{};
    P->z = v.p; P->pz = v.pitch; P->rows = voxels(z); P->c = z->c; P->k = t->k;
    P->idx = t->idx; P->t = t->logits; P->tlse = t->lse; P->temp = t->temperature;
    P->w = w; P->w_all = P->rows > 0 ? (float)(1.0 / (double)P->rows) : 0.f;
    if (P->rows > 0 && (!t->idx || !t->logits)) return LAMP_ERR_INVALID_ARG;
    if ((uintptr_t)w & 3) return LAMP_ERR_INVALID_ARG;
    if (dz) {
        if ((s = check_view(dz, true)) != LAMP_OK) return s;
        if (dz->n != z->n || dz->d != z->d || dz->h != z->h || dz->w != z->w || dz->c != z->c) return LAMP_ERR_INVALID_ARG;
        if (dz->dtype != z->dtype) return LAMP_ERR_UNSUPPORTED;
        const TView d = make_view(dz);
        P->dz = d.p; P->pdz = d.pitch;
    }
    return LAMP_OK;
}

}  // namespace

}  // namespace lamp

using namespace lamp;

extern "C" size_t lamp_distill_topk_workspace_bytes(const lamp_tensor_t *z)
{
    return z && check_view(z, true) == LAMP_OK ? (size_t)MAX_PARTS * sizeof(double) : 0;
}

static lamp_status_t check_loss(const float *loss_rows, const float *lse, const float *loss, const void *ws, size_t ws_bytes)
{
    if (((uintptr_t)loss_rows | (uintptr_t)lse | (uintptr_t)loss) & 3) return LAMP_ERR_INVALID_ARG;
    if (loss && (!ws || ((uintptr_t)ws & 15) || ws_bytes < (size_t)MAX_PARTS * sizeof(double))) return LAMP_ERR_WORKSPACE;
    return LAMP_OK;
}

extern "C" lamp_status_t lamp_distill_topk_fwd(const lamp_tensor_t *z, const lamp_teacher_topk_t *teacher, const float *row_weight,
                                               float *loss_rows, float *lse, float *loss, void *ws, size_t ws_bytes, void *cuda_stream)
{
    DistillParams P;
    lamp_status_t s = fill(&P, z, teacher, row_weight, nullptr);
    if (s != LAMP_OK || (s = check_loss(loss_rows, lse, loss, ws, ws_bytes)) != LAMP_OK) return s;
    if (!loss_rows && !lse && !loss) return LAMP_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (P.rows == 0) {
        if (loss) LAMP_CUDA_OK(cudaMemsetAsync(loss, 0, 4, st));
        return LAMP_OK;
    }
    P.loss_rows = loss_rows; P.lse_out = lse;
    return run<FWD>(P, z->dtype == LAMP_F32, loss, ws, st);
}

extern "C" lamp_status_t lamp_distill_topk_bwd(const lamp_tensor_t *z, const lamp_teacher_topk_t *teacher, const float *row_grad,
                                               const float *lse, lamp_tensor_t *dz, void *cuda_stream)
{
    DistillParams P;
    if (!dz) return LAMP_ERR_INVALID_ARG;
    const lamp_status_t s = fill(&P, z, teacher, row_grad, dz);
    if (s != LAMP_OK) return s;
    if (P.rows == 0) return LAMP_OK;
    if (!lse || ((uintptr_t)lse & 3)) return LAMP_ERR_INVALID_ARG;
    P.lse_in = lse;
    return run<BWD>(P, z->dtype == LAMP_F32, nullptr, nullptr, (cudaStream_t)cuda_stream);
}

extern "C" lamp_status_t lamp_distill_topk_fwd_bwd(const lamp_tensor_t *z, const lamp_teacher_topk_t *teacher, const float *row_weight,
                                                   float *loss_rows, float *loss, lamp_tensor_t *dz, void *ws, size_t ws_bytes,
                                                   void *cuda_stream)
{
    DistillParams P;
    if (!dz) return LAMP_ERR_INVALID_ARG;
    lamp_status_t s = fill(&P, z, teacher, row_weight, dz);
    if (s != LAMP_OK || (s = check_loss(loss_rows, nullptr, loss, ws, ws_bytes)) != LAMP_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (P.rows == 0) {
        if (loss) LAMP_CUDA_OK(cudaMemsetAsync(loss, 0, 4, st));
        return LAMP_OK;
    }
    P.loss_rows = loss_rows;
    return run<FWD | BWD>(P, z->dtype == LAMP_F32, loss, ws, st);
}
