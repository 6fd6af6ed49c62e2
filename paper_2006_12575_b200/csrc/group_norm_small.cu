// Group norm of samples that a thread-block cluster holds in its registers: one launch, every tensor read once.
// A cluster of up to 8 CTAs takes the channels c0 .. c0 + cc of a sample (whole groups, whole units), each CTA a run of its voxels, at most U per
// thread.  The values are loaded all at once and stay in registers while the sums go through shared memory, over the cluster's
// distributed shared memory (added in rank order in every CTA), and back.
// Bound by latency: the deepest level of a U-Net (2 x 512 voxels x 512 channels) took 11 us as three kernels of the streaming form;
// 6.2 here, of which bank conflicts of the fp64 sums and integer divisions had been 1.9 more.
#include "group_norm.cuh"
#include <algorithm>
#include <numeric>

namespace lamp {

namespace {

using namespace gn;

constexpr int MAX_CC = 512, MAX_GROUPS = GT, MAX_CL = 8;
// Units per thread: a few where that is enough, else as many as 64 registers of values hold.
constexpr int few(bool back) { return back ? 2 : 4; }
constexpr int most(bool xf, bool back) { return (xf ? 8 : 16) / (back ? 2 : 1); }

struct SmallParams : GnParams {
    int32_t cc, cl;                           // channels of a cluster, CTAs of a cluster
    int64_t vc;                               // voxels of a CTA
};

__device__ __forceinline__ uint32_t rank_in_cluster()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ double peer_f64(const double *p, uint32_t rank)
{
    uint32_t a;
    double v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(ptx::smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(a) : "memory");
    return v;
}

// s = sum of *a over the cluster's CTAs, t of *b, in rank order
__device__ __forceinline__ void over_cluster(int cl, const double *a, const double *b, double &s, double &t)
{
    if (cl == 1) { s = *a; t = *b; return; }
    double ps[MAX_CL], pt[MAX_CL];                               // all of them on their way at once
#pragma unroll
    for (int i = 0; i < MAX_CL; ++i) { ps[i] = i < cl ? peer_f64(a, i) : 0.0; pt[i] = i < cl ? peer_f64(b, i) : 0.0; }
    s = t = 0.0;
#pragma unroll
    for (int i = 0; i < MAX_CL; ++i) { s += ps[i]; t += pt[i]; }
}

struct Spot {
    int64_t sample, v0;                       // first voxel of this thread
    int c0, ch, unit, line, have;             // have: of this thread's voxels, `ty` apart
    uint32_t rank;
};
__device__ __forceinline__ Spot spot(const SmallParams &P)
{
    Spot q;
    q.rank = P.cl > 1 ? rank_in_cluster() : 0u;
    const int64_t cluster = blockIdx.x / P.cl;
    q.sample = cluster / P.chunks;
    q.c0 = (int)(cluster - q.sample * P.chunks) * P.cc;
    q.line = threadIdx.x / P.uc;
    q.unit = threadIdx.x - q.line * P.uc;
    q.ch = q.c0 + q.unit * 8;
    const int64_t first = q.rank * P.vc + q.line, end = min(P.v, (q.rank + 1) * P.vc);
    q.v0 = first;
    q.have = q.line < P.ty && q.ch < P.c && first < end ? (int)((end - first + P.ty - 1) / P.ty) : 0;
    return q;
}

template <bool XF> __device__ __noinline__ void sums_exact(const SmallParams &P, uint32_t again, double *sa, double *sb)
{
    const Spot q = spot(P);
    sums_again<XF>(P, again, (q.sample * P.v + q.v0) * P.px + q.ch, P.ty * P.px, q.have, q.sample * P.v * P.px, q.ch, sa, sb);
}

template <bool XF, bool ZF, int ACT, int U>
__global__ void __launch_bounds__(GT)
gn_small_kernel(const __grid_constant__ SmallParams P)
{
    extern __shared__ __align__(16) double sm[];
    __shared__ double gs[MAX_GROUPS], gt[MAX_GROUPS];
    __shared__ float2 mr[MAX_GROUPS];
    pdl_launch_dependents();
    pdl_wait();
    const Spot q = spot(P);
    const int64_t line = P.ty * P.px, at = (q.sample * P.v + q.v0) * P.px + q.ch;
    const int g0 = q.c0 / P.cg, c1 = min(P.c, q.c0 + P.cc), g1 = (c1 - 1) / P.cg;
    Raw<XF> r[U];
    float ref[8];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = u < q.have ? load_raw<XF>(P.x, at + u * line) : zero_raw<XF>();
#pragma unroll
    for (int j = 0; j < 8; ++j) ref[j] = q.have ? value_at<XF>(P.x, q.sample * P.v * P.px + group_of(P, q.ch + j) * P.cg) : 0.f;
    const int mine = g0 + threadIdx.x;                           // the group whose sums this thread finishes: no more groups than threads
    const float own_first = mine <= g1 ? value_at<XF>(P.x, q.sample * P.v * P.px + (int64_t)mine * P.cg) : 0.f;
    double a[8], b[8];
    uint32_t again = 0;                                         // channels whose squares left fp32
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = b[j] = 0.0;
    if (q.have) {
        f32x2 k[4], s1[4], s2[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = s1[j] = s2[j] = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {                            // what is not there is 0 and adds nothing
            f32x2 t[4];
            to_pairs<XF>(r[u], t);
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = add2(k[j], t[j]);
        }
        const float inv = -1.f / (float)q.have;
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = mul2(k[j], twice(inv));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= q.have) break;
            f32x2 t[4];
            to_pairs<XF>(r[u], t);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x2 d = add2(t[j], k[j]);
                s1[j] = add2(s1[j], d);
                s2[j] = fma2(d, d, s2[j]);
            }
        }
        float nk[8], f1[8], f2[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            unpack2(k[j], nk[2 * j], nk[2 * j + 1]);
            unpack2(s1[j], f1[2 * j], f1[2 * j + 1]);
            unpack2(s2[j], f2[2 * j], f2[2 * j + 1]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            about(nk[j], f1[j], f2[j], q.have, ref[j], a[j], b[j]);
            again |= squares_hold(f2[j], P.eps) ? 0u : 1u << j;
        }
    }
    const Totals tot = sum_lines(P.ty, P.uc, q.line, q.unit, a, b, sm, [&](double *sa, double *sb) {
        if (again) sums_exact<XF>(P, again, sa, sb);
    });
    sum_groups(g0, g1, P.cg,
               [&](int g, int l, int lanes, double &s, double &t) {
                   for (int ch = g * P.cg - q.c0 + l; ch < (g + 1) * P.cg - q.c0; ch += lanes) { s += tot.a(ch); t += tot.b(ch); }
               },
               [&](int g, double s, double t) { gs[g - g0] = s; gt[g - g0] = t; });
    if (P.cl > 1) { cluster_arrive(); cluster_wait(); }
    else __syncthreads();
    if (mine <= g1) {
        double s, t;
        over_cluster(P.cl, &gs[mine - g0], &gt[mine - g0], s, t);
        const float2 v = mean_rstd_of(s, t, own_first, P.inv_count, P.eps);
        mr[mine - g0] = v;
        if (q.rank == 0) P.mean_rstd[q.sample * P.groups + mine] = v;
    }
    __syncthreads();
    if (P.cl > 1) cluster_arrive();                              // this CTA has read its peers' sums, and x for the last time but from registers
    float zs[8];
    if (P.cl > 1) cluster_wait();                                // nobody still reads a sum here, or a first value that z may overwrite
    if (!q.have) return;
    const Affine f = affine(P, q.ch, [&](int g) { return mr[g - g0]; });
    const int64_t out_line = P.ty * P.po, to = (q.sample * P.v + q.v0) * P.po + q.ch;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (u >= q.have) break;
        apply<XF, ZF, ACT>(P, f, r[u], zs);
        store8_whole<ZF>(P.out, to + u * out_line, zs);
    }
}

// The calls for channels whose rstd is far from 1
__device__ __forceinline__ Run run_of(const SmallParams &P, const Spot &q)
{
    const int64_t line = q.sample * P.v + q.v0;
    return Run{line * P.px + q.ch, P.ty * P.px, line * P.pdz + q.ch, P.ty * P.pdz, line * P.po + q.ch, P.ty * P.po, q.have};
}
template <bool XF, bool ZF, int ACT> __device__ __noinline__ void sums_far(const SmallParams &P, uint32_t far, double *sa, double *sb)
{
    const Spot q = spot(P);
    far_sums<XF, ZF, ACT>(far_of(P, q.sample), run_of(P, q), far, q.ch, sa, sb);
}
template <bool XF, bool ZF, int ACT> __device__ __noinline__ void apply_far(const SmallParams &P, const float2 *means, int g0)
{
    const Spot q = spot(P);
    far_apply<XF, ZF, ACT>(far_of(P, q.sample), run_of(P, q), q.ch, means, g0);
}

template <bool XF, bool ZF, int ACT, int U>
__global__ void __launch_bounds__(GT, U == few(true) ? 2 : 1)         // 2 x 512 x 512 fp32 with 150 registers: a second wave, 12.5 us for 9
gn_small_bwd_kernel(const __grid_constant__ SmallParams P)
{
    extern __shared__ __align__(16) double sm[];
    __shared__ double gs[MAX_GROUPS], gt[MAX_GROUPS];
    __shared__ float2 means[MAX_GROUPS];
    pdl_launch_dependents();
    pdl_wait();
    const Spot q = spot(P);
    const int64_t xl = P.ty * P.px, zl = P.ty * P.pdz, at = (q.sample * P.v + q.v0) * P.px + q.ch, dz_at = (q.sample * P.v + q.v0) * P.pdz + q.ch;
    const int g0 = q.c0 / P.cg, c1 = min(P.c, q.c0 + P.cc), g1 = (c1 - 1) / P.cg;
    const float2 *mr = P.mean_rstd + q.sample * P.groups;
    Raw<XF> rx[U];
    Raw<ZF> rz[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        rx[u] = u < q.have ? load_raw<XF>(P.x, at + u * xl) : zero_raw<XF>();
        rz[u] = u < q.have ? load_raw<ZF>(P.dz, dz_at + u * zl) : zero_raw<ZF>();
    }
    Affine f = {};
    double a[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = b[j] = 0.0;
    uint32_t far = 0;                                           // channels whose sums left fp32
    if (q.have) {
        f = affine(P, q.ch, [&](int g) { return mr[g]; });
        f32x2 s1[4] = {0, 0, 0, 0}, s2[4] = {0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= q.have) break;
            f32x2 d[4], dt[4];
            slopes<XF, ZF, ACT>(P, f, rx[u], rz[u], d, dt);
#pragma unroll
            for (int j = 0; j < 4; ++j) { s1[j] = add2(s1[j], dt[j]); s2[j] = fma2(dt[j], d[j], s2[j]); }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float f1[2], f2[2];
            unpack2(s1[j], f1[0], f1[1]);
            unpack2(s2[j], f2[0], f2[1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                a[2 * j + i] = f1[i];
                const float rstd = mr[group_of(P, q.ch + 2 * j + i)].y;
                b[2 * j + i] = (double)f2[i] * rstd;
                far |= sum_is_far(rstd, f2[i]) ? 1u << (2 * j + i) : 0u;
            }
        }
    }
    // The cluster exchanges the groups' sums, which every CTA needs; of the channels' sums each CTA adds a slice.  (All of them in every CTA: 32 x 64 x 512
    // channels took 21.7 us.)
    const Totals tot = sum_lines(P.ty, P.uc, q.line, q.unit, a, b, sm, [&](double *sa, double *sb) {
        if (far) sums_far<XF, ZF, ACT>(P, far, sa, sb);
    });
    sum_groups(g0, g1, P.cg,
               [&](int g, int l, int lanes, double &s, double &t) {
                   for (int ch = g * P.cg + l; ch < (g + 1) * P.cg; ch += lanes) {
                       const double w = P.w ? P.w[ch] : 1.f;
                       s += w * tot.a(ch - q.c0);
                       t += w * tot.b(ch - q.c0);
                   }
               },
               [&](int g, double s, double t) { gs[g - g0] = s; gt[g - g0] = t; });
    if (P.cl > 1) { cluster_arrive(); cluster_wait(); }
    else __syncthreads();
    const int mine = g0 + threadIdx.x;                           // the group whose sums this thread finishes: no more groups than threads
    if (mine <= g1) {
        double s, t;
        over_cluster(P.cl, &gs[mine - g0], &gt[mine - g0], s, t);
        means[mine - g0] = make_float2((float)(s * P.inv_count), (float)(t * P.inv_count));
    }
    if (P.chan || P.dw || P.db) {
        const int slice = (c1 - q.c0 + P.cl - 1) / P.cl, end = min(c1 - q.c0, (int)(q.rank + 1) * slice);
        for (int i = q.rank * slice + (GT - 1 - threadIdx.x); i < end; i += GT) {        // the warps that have no group first
            const int ch = q.c0 + i;
            double s, t;
            over_cluster(P.cl, tot.sa + padded(i), tot.sb + padded(i), s, t);
            if (P.chan) P.chan[q.sample * P.c + ch] = make_double2(s, t);
            else {                                               // one sample: its sums are the parameters' gradients
                if (P.db) P.db[ch] = (float)s;
                if (P.dw) P.dw[ch] = (float)t;
            }
        }
    }
    __syncthreads();
    if (P.cl > 1) cluster_arrive();                              // this CTA has read its peers' sums; waited for at the end
    if (q.have) {
        const auto mr_of = [&](int g) { return mr[g]; };
        const auto means_of = [&](int g) { return means[g - g0]; };
        const Back k = back_terms(P, q.ch, mr_of, means_of);
        if (terms_are_far(P, q.ch, k, mr_of, means_of)) apply_far<XF, ZF, ACT>(P, means, g0);
        else {
            const int64_t ol = P.ty * P.po, to = (q.sample * P.v + q.v0) * P.po + q.ch;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= q.have) break;
                float o[8];
                back_apply<XF, ZF, ACT>(P, f, k, rx[u], rz[u], o);
                store8_whole<XF>(P.out, to + u * ol, o);
            }
        }
    }
    if (P.cl > 1) cluster_wait();                                // no CTA leaves while a peer still reads its sums
}

// dw and db from the sums of all samples: a warp per channel, the lanes over the samples
__global__ void __launch_bounds__(GT)
gn_small_params_kernel(const double2 *chan, int n, int c, float *dw, float *db)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, ch = blockIdx.x * (GT / 32) + (threadIdx.x >> 5);
    if (ch >= c) return;
    double s = 0.0, t = 0.0;
    for (int i = lane; i < n; i += 32) { const double2 v = chan[(int64_t)i * c + ch]; s += v.x; t += v.y; }
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        t += __shfl_xor_sync(0xffffffffu, t, o);
    }
    if (lane == 0 && db) db[ch] = (float)s;
    if (lane == 0 && dw) dw[ch] = (float)t;
}

struct Plan { int cc, cl, u; };
bool plan(const GnParams &P, bool xf, bool back, Plan &out)
{
    const int base = std::lcm(8, P.cg), es = xf ? 4 : 2;
    auto fits = [&](int cc, int cl, int u) { return (P.v + cl - 1) / cl <= (int64_t)(GT / (cc / 8)) * u; };
    // the widest piece: its units leave room for the lines that MAX_CL CTAs need
    const int64_t lines = ((P.v + MAX_CL - 1) / MAX_CL + most(xf, back) - 1) / most(xf, back);
    if (lines > GT) return false;
    const int widest = std::min({P.c, MAX_CC, (int)(GT / lines) * 8, MAX_GROUPS * P.cg});
    int m = widest / base;
    if (m == 0) return false;
    if (base * m * es < 32 && base * m < P.c) return false;      // pieces of rows shorter than a sector of memory: twice the traffic
    const int sms = sm_count();
    auto chunks = [&](int k) { return (int64_t)P.n * ((P.c + base * k - 1) / (base * k)); };
    // narrower pieces, of 64 bytes at least, until clusters of MAX_CL fill the GPU
    const int want = P.n < sms ? (sms + MAX_CL * P.n - 1) / (MAX_CL * P.n) : 1;
    if (want > 1 && chunks(m) < (int64_t)want * P.n) m = std::min(m, std::max({1, (64 / es + base - 1) / base, (P.c - 1) / ((want - 1) * base)}));
    out.cc = base * m;
    out.cl = 1;
    while (out.cl < MAX_CL && (!fits(out.cc, out.cl, few(back)) || chunks(m) * out.cl * 2 <= sms)) {
        if (fits(out.cc, out.cl, few(back)) && P.v <= (int64_t)out.cl * (GT / (out.cc / 8))) break;     // a voxel per thread already
        out.cl *= 2;
    }
    out.u = fits(out.cc, out.cl, few(back)) ? few(back) : most(xf, back);
    // With as many values as the registers hold an SM has one CTA, and one wave of them waits for memory, works and stores in step: behind one and a half
    // waves the streaming form is ahead (16 x 512 x 512 forward 25.6 here, 20.6 there; 64 x 1,500 x 128 42.6 and 22.5; 8 x 1,024 x 512, 1.3 waves, 18.1 and 21.4).
    if (out.u != few(back) && chunks(m) * out.cl * 2 > 3ll * sms) return false;
    // With few values the same holds behind four CTAs per SM (512 x 64 x 512 forward 59.2 here, 30.0 there, backward 141 and 47), but forward without a cluster
    // (1,000 x 64 x 64: 16.4 and 19.8).
    if ((back || out.cl > 1) && chunks(m) * out.cl > 4ll * sms) return false;
    return chunks(m) * out.cl <= 2147483647ll;
}

template <typename Kernel>
lamp_status_t launch(Kernel kernel, const SmallParams &P, int64_t clusters, size_t smem, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(clusters * P.cl));
    cfg.blockDim = dim3(GT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)P.cl;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = P.cl > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, P) == cudaSuccess ? LAMP_OK : LAMP_ERR_CUDA;
}

template <bool XF, bool ZF, int ACT>
lamp_status_t run(SmallParams &P, bool back, int u, int64_t clusters, cudaStream_t st)
{
    const size_t lines = lines_bytes(P.ty, P.uc);
    if (!back)
        return u == few(false) ? launch(gn_small_kernel<XF, ZF, ACT, few(false)>, P, clusters, lines, st)
                               : launch(gn_small_kernel<XF, ZF, ACT, most(XF, false)>, P, clusters, lines, st);
    const lamp_status_t s = u == few(true) ? launch(gn_small_bwd_kernel<XF, ZF, ACT, few(true)>, P, clusters, lines, st)
                                           : launch(gn_small_bwd_kernel<XF, ZF, ACT, most(XF, true)>, P, clusters, lines, st);
    if (s != LAMP_OK || !P.chan) return s;
    return launch_pdl(true, gn_small_params_kernel, dim3((unsigned)((P.c + GT / 32 - 1) / (GT / 32))), dim3(GT), 0, st, (const double2 *)P.chan, (int)P.n, (int)P.c, P.dw, P.db);
}

template <bool XF, bool ZF>
lamp_status_t by_act(SmallParams &P, bool back, int u, int64_t clusters, cudaStream_t st)
{
    switch (P.act) {
    case LAMP_ACT_NONE: return run<XF, ZF, LAMP_ACT_NONE>(P, back, u, clusters, st);
    case LAMP_ACT_LEAKY_RELU: return run<XF, ZF, LAMP_ACT_LEAKY_RELU>(P, back, u, clusters, st);
    case LAMP_ACT_SILU: return run<XF, ZF, LAMP_ACT_SILU>(P, back, u, clusters, st);
    default: return run<XF, ZF, LAMP_ACT_GELU>(P, back, u, clusters, st);
    }
}

}  // namespace

lamp_status_t gn_small(const gn::GnParams &G, bool xf, bool zf, bool back, cudaStream_t st)
{
    Plan p;
    if (!plan(G, xf, back, p)) return LAMP_ERR_UNSUPPORTED;
    SmallParams P = {};
    static_cast<GnParams &>(P) = G;
    P.cc = p.cc; P.cl = p.cl;
    P.chunks = (G.c + p.cc - 1) / p.cc;
    P.uc = p.cc / 8;
    P.ty = GT / P.uc;
    P.vc = (G.v + p.cl - 1) / p.cl;
    P.chan = back && G.n > 1 && (G.dw || G.db) ? G.part : nullptr;
    const int64_t clusters = (int64_t)G.n * P.chunks;
    if (!xf) return by_act<false, false>(P, back, p.u, clusters, st);
    return zf ? by_act<true, true>(P, back, p.u, clusters, st) : by_act<true, false>(P, back, p.u, clusters, st);
}

}  // namespace lamp
