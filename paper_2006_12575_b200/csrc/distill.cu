// Distillation loss from a teacher's top logits, and its gradient:
//   loss_r = T^2 sum_j p_j (log p_j - log q_{idx_j}),   dloss_r/dz_i = T (q_i S - sum_{j: idx_j = i} p_j),   S = sum_j p_j.
// Bound by memory: a row of c logits is read once (running maximum and sum of the softmax in one pass) and its gradient
// written once.  The exponentials are taken in base 2 relative to the row's maximum m: e_i = 2^(z_i log2(e) / T - m), so
// that q_i = e_i / sum e is as exact as fp32 allows whatever the size of the logits.
// The gradient of a listed class is the difference of two numbers that training makes nearly equal, so it is formed in
// fp32 and rounded once: the dense pass writes q_i S everywhere, then the owner of each listed class overwrites it.
// A class listed twice subtracts both probabilities (each of its entries writes the same value).
//
// Rows of odd length start at any element, so a row is walked in 16-byte units aligned in memory; a unit that is not
// wholly inside the row is handled element by element.
//   c <= 1024: one warp per row, the row stays in registers.
//   wider:     one CTA per row, or, where rows are few, a cluster of up to 8 CTAs that share the row and exchange maximum and
//              sum through distributed shared memory.  The row is kept in shared memory as far as it fits and read again
//              (from L2) beyond that.
#include "common.cuh"

namespace lamp {

namespace {

constexpr int FWD = 1, BWD = 2;
constexpr int MAX_PARTS = 4096;                     // partial losses, one per CTA (or cluster)
constexpr int MAX_K = 1024;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int WR_WARPS = 8, WR_MAX_C = 1024;
constexpr int CR_THREADS = 512;

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
    int32_t stash;                                  // 16-byte units of a row slice kept in shared memory (CTA form)
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

// running maximum m (base 2 exponent) and sum s of 2^(x - m)
__device__ __forceinline__ void join(float &m, float &s, float m2, float s2)
{
    const float n = fmaxf(m, m2);
    // a side that is empty (-inf) contributes nothing; its exponent would be -inf - -inf
    s = (m == -INFINITY ? 0.f : s * exp2f(m - n)) + (m2 == -INFINITY ? 0.f : s2 * exp2f(m2 - n));
    // NaN anywhere makes the row NaN
    if (m != m || m2 != m2) s = NAN;
    m = n;
}
// e^(z / T) relative to the reference m: 2^(z c - m) with c = log2(e) / T and m the row's maximum in base 2, or, from a given
// log-sum m, e^(z c - m) with c = 1 / T (the difference is formed before the change of base, which keeps its digits)
template <int MODE> __device__ __forceinline__ float power(float z, float c, float m)
{
    return (MODE & FWD) ? exp2f(fmaf(z, c, -m)) : exp2f(fmaf(z, c, -m) * LOG2E);
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
__device__ __forceinline__ void warp_join(float &m, float &s)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
        join(m, s, m2, s2);
    }
}

// One warp reads the teacher's entries of a row: ids (-1: absent), log p and z / T's numerator to shared memory; returns S
// (0: no entry left).
template <bool F32>
__device__ __forceinline__ float teacher_row(const DistillParams &P, int64_t row, int64_t at, int lane, int lo, int hi, int *ids, float *logp, float *zt)
{
    const float inv_t = 1.f / P.temp;
    float m = -INFINITY;
    bool nan = false;
    for (int j = lane; j < P.k; j += 32) {
        int id = P.idx[row * P.k + j];
        if (id < 0 || id >= P.c) id = -1;
        const float v = id >= 0 ? P.t[row * P.k + j] * inv_t : -INFINITY;
        ids[j] = id;
        logp[j] = v;
        zt[j] = id >= lo && id < hi ? elem<F32>(P.z, at + id) : 0.f;      // before anything is written (dz may be z)
        nan |= v != v;
        m = fmaxf(m, v);
    }
    nan = __any_sync(0xffffffffu, nan);
    float lse;
    if (P.tlse) {
        lse = P.tlse[row];
    } else {
        float mm = warp_max(m);
        if (mm == -INFINITY && !nan) return 0.f;
        float s = 0.f;
        for (int j = lane; j < P.k; j += 32) s += expf(logp[j] - mm);
        lse = mm + logf(warp_sum(s));
    }
    float S = 0.f;
    for (int j = lane; j < P.k; j += 32) {
        logp[j] -= lse;
        S += expf(logp[j]);
    }
    S = warp_sum(S);
    __syncwarp();
    return P.tlse || S != S ? S : 1.f;
}

// ----------------------------------------------------------------------------------------------------------------------
// one warp per row
// ----------------------------------------------------------------------------------------------------------------------
template <bool F32, int MODE>
__global__ void __launch_bounds__(WR_WARPS * 32)
distill_warp_kernel(const DistillParams P)
{
    constexpr int E = Elem<F32>::E, NU = WR_MAX_C / (32 * E) + (F32 ? 1 : 1);
    extern __shared__ int smem_i[];
    __shared__ double wl[WR_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int *ids = smem_i + warp * 3 * P.k;
    float *logp = (float *)(ids + P.k), *zt = logp + P.k;
    const float c2 = (MODE & FWD) ? LOG2E / P.temp : 1.f / P.temp;
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
        if (w != 0.f) S = teacher_row<F32>(P, row, at, lane, 0, P.c, ids, logp, zt);
        float loss = 0.f, lse = 0.f;
        if (S != 0.f) {
            uint4 raw[NU];
            float m = -INFINITY, s = 0.f;
#pragma unroll
            for (int i = 0; i < NU; ++i) if (lane + 32 * i < nu) raw[i] = load_unit<F32>(P.z, at, off, lane + 32 * i, P.c);
            float scale;                                            // 1 / sum, relative to 2^m
            if constexpr (MODE & FWD) {
#pragma unroll
                for (int i = 0; i < NU; ++i) if (lane + 32 * i < nu) {
                    float v[E];
                    unit_values<F32>(raw[i], v);
#pragma unroll
                    for (int j = 0; j < E; ++j) m = v[j] != v[j] || m != m ? NAN : fmaxf(m, v[j]);
                }
                // maximum over the warp, NaN kept
                const bool bad = __any_sync(0xffffffffu, m != m);
                m = bad ? NAN : warp_max(m);
                m *= c2;
#pragma unroll
                for (int i = 0; i < NU; ++i) if (lane + 32 * i < nu) {
                    float v[E];
                    unit_values<F32>(raw[i], v);
#pragma unroll
                    for (int j = 0; j < E; ++j) s += exp2f(fmaf(v[j], c2, -m));
                }
                s = warp_sum(s);
                const float l2 = log2f(s);
                lse = (m + l2) * LN2;
                scale = 1.f / s;
                for (int j = lane; j < P.k; j += 32) {
                    const float p = ids[j] >= 0 ? expf(logp[j]) : 0.f;
                    if (p != 0.f) loss += p * (logp[j] - LN2 * (fmaf(zt[j], c2, -m) - l2));
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
                    for (int j = 0; j < E; ++j) v[j] = gq * power<MODE>(v[j], c2, m);
                    store_unit<F32>(P.dz, dat, off, same, lane + 32 * i, P.c, v);
                }
                __syncwarp();
                for (int j = lane; j < P.k; j += 32) {
                    if (ids[j] < 0) continue;
                    float p = 0.f;
                    for (int i = 0; i < P.k; ++i) if (ids[i] == ids[j]) p += expf(logp[i]);
                    put<F32>(P.dz, dat + ids[j], gT * (S * (scale * power<MODE>(zt[j], c2, m)) - p));
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

// ----------------------------------------------------------------------------------------------------------------------
// one CTA, or a cluster of CTAs, per row
// ----------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ float peer_f32(const float *p, uint32_t rank)
{
    uint32_t a = (uint32_t)__cvta_generic_to_shared(p), b;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(a), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(b) : "memory");
    return v;
}

template <bool F32, int MODE>
__global__ void __launch_bounds__(CR_THREADS)
distill_cta_kernel(const DistillParams P, int S_CTAS)
{
    constexpr int E = Elem<F32>::E, NW = CR_THREADS / 32;
    extern __shared__ uint4 stash[];
    int *ids = (int *)(stash + P.stash);
    float *logp = (float *)(ids + P.k), *zt = logp + P.k;
    __shared__ float red[2][NW], sh_S, sh_ms[2], sh_loss;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const float c2 = (MODE & FWD) ? LOG2E / P.temp : 1.f / P.temp;
    const int rank = S_CTAS > 1 ? (int)(blockIdx.x % S_CTAS) : 0;
    const int64_t first = blockIdx.x / S_CTAS, step = gridDim.x / S_CTAS;
    double total = 0;
    pdl_launch_dependents();
    pdl_wait();
    for (int64_t row = first; row < P.rows; row += step) {
        const int64_t at = row * P.pz, dat = row * P.pdz;
        const float w = P.w ? P.w[row] : P.w_all;                  // the same for the whole cluster: so are all branches on it
        const int off = misalign<F32>(P.z, at);
        const bool same = (MODE & BWD) && off == misalign<F32>(P.dz, dat);
        const int nu_all = (P.c + off + E - 1) / E;
        const int u0 = (int)((int64_t)nu_all * rank / S_CTAS), u1 = (int)((int64_t)nu_all * (rank + 1) / S_CTAS);
        const int e0 = u0 * E - off, e1 = u1 * E - off;            // elements of this CTA's slice (clipped to the row below)
        float S = 0.f, loss = 0.f, lse = 0.f;
        if (w != 0.f) {
            if (warp == 0) {
                const float v = teacher_row<F32>(P, row, at, lane, e0 < 0 ? 0 : e0, e1 > P.c ? P.c : e1, ids, logp, zt);
                if (lane == 0) sh_S = v;
            }
            float m = -INFINITY, s = 0.f;
            if constexpr (MODE & FWD) {
                for (int u = u0 + tid; u < u1; u += CR_THREADS) {
                    const uint4 raw = load_unit<F32>(P.z, at, off, u, P.c);
                    if (u - u0 < P.stash) stash[u - u0] = raw;
                    float v[E], n;
                    unit_values<F32>(raw, v);
                    n = v[0];
#pragma unroll
                    for (int j = 1; j < E; ++j) n = fmaxf(n, v[j]);
                    n *= c2;
                    if (n > m) { s *= exp2f(m - n); m = n; }        // m = -inf: s is 0
                    if (m != -INFINITY) {
#pragma unroll
                        for (int j = 0; j < E; ++j) s += exp2f(fmaf(v[j], c2, -m));
                    } else {
#pragma unroll
                        for (int j = 0; j < E; ++j) if (v[j] != v[j]) s = NAN;
                    }
                }
                warp_join(m, s);
                if (lane == 0) { red[0][warp] = m; red[1][warp] = s; }
            }
            __syncthreads();
            S = sh_S;
            float scale;
            if constexpr (MODE & FWD) {
                m = red[0][0]; s = red[1][0];
                for (int i = 1; i < NW; ++i) join(m, s, red[0][i], red[1][i]);
                if (S_CTAS > 1) {
                    if (tid == 0) { sh_ms[0] = m; sh_ms[1] = s; }
                    cluster_barrier();
                    m = peer_f32(&sh_ms[0], 0); s = peer_f32(&sh_ms[1], 0);
                    for (int r = 1; r < S_CTAS; ++r) join(m, s, peer_f32(&sh_ms[0], r), peer_f32(&sh_ms[1], r));
                }
                if (m == -INFINITY) s = NAN;                        // no logit above -inf: there is no softmax
                scale = 1.f / s;
                if (warp == 0 && S != 0.f) {
                    const float l2 = log2f(s);
                    lse = (m + l2) * LN2;
                    for (int j = lane; j < P.k; j += 32) {
                        const bool mine = ids[j] >= 0 && ids[j] >= e0 && ids[j] < e1;
                        const float p = mine ? expf(logp[j]) : 0.f;
                        if (p != 0.f) loss += p * (logp[j] - LN2 * (fmaf(zt[j], c2, -m) - l2));
                    }
                    loss = warp_sum(loss) * P.temp * P.temp;
                }
                if (S_CTAS > 1) {
                    if (tid == 0) sh_loss = loss;
                    cluster_barrier();                             // also: every peer has read sh_ms
                    if (rank == 0 && tid == 0)
                        for (int r = 1; r < S_CTAS; ++r) loss += peer_f32(&sh_loss, r);
                }
            } else {
                m = P.lse_in[row];
                scale = 1.f;
            }
            if ((MODE & BWD) && S != 0.f) {
                const float gT = w * P.temp, gq = gT * S * scale;
                for (int u = u0 + tid; u < u1; u += CR_THREADS) {
                    const uint4 raw = (MODE & FWD) && u - u0 < P.stash ? stash[u - u0] : load_unit<F32>(P.z, at, off, u, P.c);
                    float v[E];
                    unit_values<F32>(raw, v);
#pragma unroll
                    for (int j = 0; j < E; ++j) v[j] = gq * power<MODE>(v[j], c2, m);
                    store_unit<F32>(P.dz, dat, off, same, u, P.c, v);
                }
                __syncthreads();                                   // the listed classes go over what the dense pass wrote
                for (int j = tid; j < P.k; j += CR_THREADS) {
                    const int id = ids[j];
                    if (id < 0 || id < e0 || id >= e1) continue;
                    float p = 0.f;
                    for (int i = 0; i < P.k; ++i) if (ids[i] == id) p += expf(logp[i]);
                    put<F32>(P.dz, dat + id, gT * (S * (scale * power<MODE>(zt[j], c2, m)) - p));
                }
            }
        }
        if ((MODE & BWD) && S == 0.f) {
            float v[E];
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = 0.f;
            for (int u = u0 + tid; u < u1; u += CR_THREADS) store_unit<F32>(P.dz, dat, off, same, u, P.c, v);
        }
        if ((MODE & FWD) && rank == 0 && tid == 0) {
            if (P.loss_rows) P.loss_rows[row] = loss;
            if (P.lse_out) P.lse_out[row] = lse;
            if (w != 0.f) total += (double)w * loss;
        }
        if (w != 0.f) __syncthreads();                             // ids, logp, zt, red are free again
        if ((MODE & FWD) && S_CTAS > 1 && w != 0.f) cluster_barrier();   // sh_loss has been read
    }
    if ((MODE & FWD) && P.part && rank == 0 && tid == 0) P.part[blockIdx.x / S_CTAS] = total;
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

template <bool F32, int MODE>
lamp_status_t launch_cta(const DistillParams &P, int grid, int splits, int smem, cudaStream_t st)
{
    static SmemAttrOnce attr;
    const lamp_status_t s = attr.ensure(distill_cta_kernel<F32, MODE>, 226 * 1024);
    if (s != LAMP_OK) return s;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(CR_THREADS);
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
    if (P.c <= WR_MAX_C) {
        const int64_t need = (P.rows + WR_WARPS - 1) / WR_WARPS;
        parts = (int)(need < 8ll * sms ? need : 8ll * sms);
        if (parts > MAX_PARTS) parts = MAX_PARTS;
        s = f32 ? launch_warp<true, MODE>(P, parts, st) : launch_warp<false, MODE>(P, parts, st);
    } else {
        const int units = (P.c + (f32 ? 3 : 7)) / (f32 ? 4 : 8) + 1;
        // a cluster per row where rows alone would leave SMs idle and every CTA still has two units a thread
        int splits = 1;
        while (splits < 8 && P.rows * splits * 2 <= sms && units >= 4 * CR_THREADS * splits) splits *= 2;
        const int slice = (units + splits - 1) / splits + 1, lists = 3 * P.k * 4;
        // two CTAs per SM, so that one loads while the other computes or writes
        const int room = ((MODE & FWD) && (MODE & BWD)) ? (112 * 1024 - lists) / 16 : 0;
        P.stash = slice < room ? slice : room > 0 ? room : 0;
        int64_t groups = 2ll * sms / splits;
        if (groups > P.rows) groups = P.rows;
        parts = (int)groups;
        const int smem = P.stash * 16 + lists;
        s = f32 ? launch_cta<true, MODE>(P, parts * splits, splits, smem, st) : launch_cta<false, MODE>(P, parts * splits, splits, smem, st);
    }
    if (s != LAMP_OK || !loss) return s;
    return launch_pdl(true, distill_sum_kernel, dim3(1), dim3(256), 0, st, (const double *)ws, parts, loss);
}

lamp_status_t check_teacher(const lamp_teacher_topk_t *t)
{
    if (!t || t->k < 1 || !(t->temperature > 0.f) || t->temperature > 3.0e38f) return LAMP_ERR_INVALID_ARG;
    if (t->k > MAX_K) return LAMP_ERR_UNSUPPORTED;
    if (((uintptr_t)t->idx | (uintptr_t)t->logits | (uintptr_t)t->lse) & 3) return LAMP_ERR_INVALID_ARG;
    return LAMP_OK;
}

lamp_status_t fill(DistillParams *P, const lamp_tensor_t *z, const lamp_teacher_topk_t *t, const float *w, const lamp_tensor_t *dz)
{
    lamp_status_t s;
    if ((s = check_view(z, true)) != LAMP_OK || (s = check_teacher(t)) != LAMP_OK) return s;
    if (z->c > 1 << 28) return LAMP_ERR_UNSUPPORTED;
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
