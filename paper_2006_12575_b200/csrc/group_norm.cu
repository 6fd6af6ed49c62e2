// Group norm with an activation, channels last:  t = (x - mean_g) rstd_g w[c] + b[c],  z = act(t),  and its backward pass.
//
// The statistics of a group need all of its values before the first output: a pass that sums, a kernel that finishes the few
// sums, a pass that applies.  Forward both passes read x, backward both read x and dz; the second runs against the direction of the
// first, so that it starts with what the first left in L2 (126 MB).  Bound by memory.
// A voxel's channels are taken in units of 8 (16 bytes of bf16, 32 of fp32), a thread keeps its unit for all of its voxels, so
// everything per channel stays in registers; a CTA holds TY voxels of one sample side by side and takes every parts-th TY of them.
// Each thread copies its values asynchronously into a ring of its own in shared memory, D units ahead of the one it works on (nobody else reads
// them, so no barrier): as many bytes in flight as with registers, all the time, and the first are on their way while the constants are
// formed.  With U units loaded into registers, worked on, and the next ones loaded, 128^3 x 32 bf16 backward took 129 us (now 114), 81,840 x 320
// fp32 101 (87, with a GELU that keeps its digits 89); 128^3 x 64 bf16 forward takes the same either way.
// Sums: a thread adds d = x - k and d^2 of at most RUN voxels in fp32, k the mean of the first values it loads - without it the squares of
// data far from 0 lose the variance; where the squares leave fp32's range the thread adds its values again in fp64.  Between threads, CTAs and channels of a group the sums are fp64, taken about r, the group's first
// value, and added in a fixed order.
#include "group_norm.cuh"
#include <algorithm>

namespace lamp {

namespace {

using namespace gn;

// CTAs per SM that the streaming kernels are compiled and sized for
constexpr int resident(bool xf, bool back) { return (xf ? 3 : 4) - (back ? 1 : 0); }
constexpr int RUN = 256;                      // voxels that a thread sums at most
// units ahead: 32 KB of rings per CTA forward, 48 KB (36 KB for fp32 with bf16) backward; deeper ones leave the L1 cache too little for fp32 (six
// units: 105 us on 81,840 x 320 fp32 backward, three: 89)
__host__ __device__ constexpr int depth(bool xf, bool back) { return back ? (xf ? 3 : 6) : (xf ? 4 : 8); }

// ----------------------------------------------------------------------------------------------------------- places
struct Place {
    int64_t sample, v0;                       // this thread's first voxel
    int part, ch, unit, ty;                   // this thread's first channel, its unit in the chunk, its voxel line
    int count;                                // of this thread's voxels, P.apart apart
};
// `back`: samples and parts in the opposite order
__device__ __forceinline__ Place place(const GnParams &P, bool back)
{
    Place q;
    const int64_t at = back ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
    q.sample = at / P.parts;
    q.part = (int)(at - q.sample * P.parts);
    q.ty = threadIdx.x / P.uc;
    q.unit = threadIdx.x - q.ty * P.uc;
    const int u = blockIdx.y * P.uc + q.unit;
    q.ch = u * 8;
    q.v0 = q.part * P.lead + q.ty;
    const int64_t end = min(P.v, q.part * P.lead + P.span);
    q.count = q.ty < P.ty && q.ch < P.c && q.v0 < end ? (int)((end - q.v0 + P.apart - 1) / P.apart) : 0;
    return q;
}

// This thread's D units in shared memory
template <bool F32, int D> struct Ring {
    static constexpr int PLANE = GT * 16, SLOT = PLANE * (F32 ? 2 : 1), BYTES = D * SLOT;
    uint32_t at;
    __device__ __forceinline__ explicit Ring(void *smem) { at = ptx::smem_u32(smem) + threadIdx.x * 16; }
    __device__ __forceinline__ void load(int slot, const void *base, int64_t off) const
    {
        const char *p = (const char *)base + off * (F32 ? 4 : 2);
        if (F32) {                                                // the two halves of a sector come one after the other: through L1
            asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(at + slot * SLOT), "l"(p) : "memory");
            asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(at + slot * SLOT + PLANE), "l"(p + 16) : "memory");
        } else asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + slot * SLOT), "l"(p) : "memory");
    }
    __device__ __forceinline__ Raw<F32> get(int slot) const
    {
        Raw<F32> r;
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.v[i].x), "=r"(r.v[i].y), "=r"(r.v[i].z), "=r"(r.v[i].w) : "r"(at + slot * SLOT + i * PLANE) : "memory");
        return r;
    }
};
// One group per unit, empty ones behind the last: the group D - N units ahead has landed when at most N are outstanding.
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void landed() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// start(i, slot) sends for unit i, take(slot) reads it out of its slot, work(i, unit) does the rest; all of the `count` units in turn.
template <int D, typename S> __device__ __forceinline__ void begin(int count, S start)
{
#pragma unroll
    for (int i = 0; i < D; ++i) {
        if (i < count) start(i, i);
        commit();
    }
}
template <int D, typename S, typename T, typename W> __device__ __forceinline__ void stream(int count, S start, T take, W work)
{
    int slot = 0;
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
        landed<D - 1>();
        const auto unit = take(slot);
        if (i + D < count) start(i + D, slot);                   // the slot has been read
        commit();
        work(i, unit);
        slot = slot + 1 == D ? 0 : slot + 1;
    }
}

// ----------------------------------------------------------------------------------------------------------- forward
template <bool XF> __device__ __noinline__ void sums_exact(const GnParams &P, uint32_t again, double *sa, double *sb)
{
    const Place q = place(P, false);
    const int64_t base = q.sample * P.v;
    sums_again<XF>(P, again, (base + q.v0) * P.px + q.ch, P.apart * P.px, q.count, base * P.px, q.ch, sa, sb);
}

template <bool XF>
__global__ void __launch_bounds__(GT, resident(XF, false))
gn_sums_kernel(const __grid_constant__ GnParams P)
{
    extern __shared__ __align__(16) double sm[];                // the rings, then the sums over the lines
    constexpr int D = depth(XF, false);
    pdl_launch_dependents();
    pdl_wait();
    const Place q = place(P, false);
    const int64_t base = q.sample * P.v, step = P.apart * P.px, x0 = (base + q.v0) * P.px + q.ch;
    const int mine = q.count;
    const Ring<XF, D> ring(sm);
    const auto start = [&](int i, int slot) { ring.load(slot, P.x, x0 + i * step); };
    f32x2 k[4], s1[4], s2[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = s1[j] = s2[j] = 0;
    begin<D>(mine, start);
    float ref[8];                                               // its groups' first values
#pragma unroll
    for (int j = 0; j < 8; ++j) ref[j] = mine > 0 ? value_at<XF>(P.x, base * P.px + group_of(P, q.ch + j) * P.cg) : 0.f;
    if (mine > 0) {
        constexpr int FIRST = D < 4 ? D : 4;
        const int first = mine < FIRST ? mine : FIRST;
        landed<D - FIRST>();
#pragma unroll
        for (int u = 0; u < FIRST; ++u) {
            if (u >= first) break;
            f32x2 t[4];
            to_pairs<XF>(ring.get(u), t);
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = add2(k[j], t[j]);
        }
        const float inv = -1.f / (float)first;
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = mul2(k[j], twice(inv));              // -k
    }
    stream<D>(mine, start, [&](int slot) { return ring.get(slot); },
              [&](int, const Raw<XF> &r) {
                  f32x2 t[4];
                  to_pairs<XF>(r, t);
#pragma unroll
                  for (int j = 0; j < 4; ++j) {
                      const f32x2 d = add2(t[j], k[j]);
                      s1[j] = add2(s1[j], d);
                      s2[j] = fma2(d, d, s2[j]);
                  }
              });
    landed<0>();
    __syncthreads();                                            // the rings make room
    double a[8], b[8];
    uint32_t again = 0;                                         // channels whose squares left fp32
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = b[j] = 0.0;
    if (mine > 0) {
        float nk[8], f1[8], f2[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            unpack2(k[j], nk[2 * j], nk[2 * j + 1]);
            unpack2(s1[j], f1[2 * j], f1[2 * j + 1]);
            unpack2(s2[j], f2[2 * j], f2[2 * j + 1]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            about(nk[j], f1[j], f2[j], mine, ref[j], a[j], b[j]);
            again |= squares_hold(f2[j], P.eps) ? 0u : 1u << j;
        }
    }
    const Totals tot = sum_lines(P.ty, P.uc, q.ty, q.unit, a, b, sm, [&](double *sa, double *sb) {
        if (again) sums_exact<XF>(P, again, sa, sb);
    });
    const int cc = P.uc * 8, c0 = blockIdx.y * cc, c1 = min(P.c, c0 + cc);
    sum_groups(c0 / P.cg, (c1 - 1) / P.cg, P.cg,
               [&](int g, int l, int lanes, double &s, double &t) {
                   for (int ch = max(c0, g * P.cg) + l; ch < min(c1, (g + 1) * P.cg); ch += lanes) { s += tot.a(ch - c0); t += tot.b(ch - c0); }
               },
               [&](int g, double s, double t) {
                   P.part[((q.sample * P.groups + g) * P.parts + q.part) * P.chunks + blockIdx.y] = make_double2(s, t);
                   if (q.part == 0 && g * P.cg >= c0) P.ref[q.sample * P.groups + g] = value_at<XF>(P.x, base * P.px + g * P.cg);
               });
}

// Adds a group's sums about its first value: the partial sums first, first + step, .., or given sums per channel about 0
__device__ __forceinline__ void add_sums(const GnParams &P, int64_t sample, int g, int first, int step, double &s, double &t)
{
    if (P.stats) {
        const double2 *p = reinterpret_cast<const double2 *>(P.stats) + sample * P.c + g * P.cg;
#pragma unroll 4
        for (int i = first; i < P.cg; i += step) { const double2 v = p[i]; s += v.x; t += v.y; }
        return;
    }
    const double2 *p = P.part + (sample * P.groups + g) * P.parts * P.chunks;
    if (P.chunks == 1) {
#pragma unroll 4
        for (int i = first; i < P.parts; i += step) { const double2 v = p[i]; s += v.x; t += v.y; }
        return;
    }
    const int cc = P.uc * 8, k0 = g * P.cg / cc, ks = ((g + 1) * P.cg - 1) / cc - k0 + 1;
#pragma unroll 4
    for (int i = first; i < P.parts * ks; i += step) { const double2 v = p[i / ks * P.chunks + k0 + i % ks]; s += v.x; t += v.y; }
}
__device__ __forceinline__ float2 finish(const GnParams &P, int64_t at, double s, double t)
{
    return mean_rstd_of(s, t, P.stats ? 0.0 : P.ref[at], P.inv_count, P.eps);
}

// mean and rstd of a group; W warps per group: one where the sums are few (a CTA has 8 groups), all where they are many
template <int W>
__global__ void __launch_bounds__(GT)
gn_finish_kernel(const GnParams P)
{
    __shared__ double red[2][GT / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = W == 1 ? lane : threadIdx.x;
    const int64_t at = W == 1 ? (int64_t)blockIdx.x * (GT / 32) + warp : blockIdx.x;
    if (at >= (int64_t)P.n * P.groups) return;
    const int64_t sample = at / P.groups;
    double s = 0.0, t = 0.0;
    add_sums(P, sample, (int)(at - sample * P.groups), first, 32 * W, s, t);
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        t += __shfl_xor_sync(0xffffffffu, t, o);
    }
    if (W > 1) {
        if (lane == 0) { red[0][warp] = s; red[1][warp] = t; }
        __syncthreads();
        s = t = 0.0;
        for (int i = 0; i < W; ++i) { s += red[0][i]; t += red[1][i]; }
    }
    if (first == 0) P.mean_rstd[at] = finish(P, at, s, t);
}

// (mean, rstd) of a group of the sample
__device__ __forceinline__ auto stats_of(const GnParams &P, const Place &q)
{
    return [mr = P.mean_rstd + q.sample * P.groups](int g) { return mr[g]; };
}

template <bool XF, bool ZF, int ACT>
__global__ void __launch_bounds__(GT, resident(XF, false))
gn_apply_kernel(const GnParams P)
{
    extern __shared__ __align__(16) double sm[];
    constexpr int D = depth(XF, false);
    pdl_launch_dependents();
    pdl_wait();
    const Place q = place(P, true);
    const int mine = q.count;
    if (mine == 0 && !P.fused) return;
    const int64_t line = q.sample * P.v + q.v0 + (mine - 1) * P.apart;             // backwards from the last voxel
    const int64_t step = P.apart * P.px, x0 = line * P.px + q.ch, out_step = P.apart * P.po, o0 = line * P.po + q.ch;
    const Ring<XF, D> ring(sm);
    const auto start = [&](int i, int slot) { ring.load(slot, P.x, x0 - i * step); };
    begin<D>(mine, start);
    Affine f;
    if (P.fused) {                                              // every CTA finishes the sums of its groups
        float2 *mr = (float2 *)((char *)sm + Ring<XF, D>::BYTES);
        const int cc = P.uc * 8, c0 = blockIdx.y * cc, g0 = c0 / P.cg, g1 = (min(P.c, c0 + cc) - 1) / P.cg;
        sum_groups(g0, g1, P.stats ? P.cg : P.parts, [&](int g, int l, int lanes, double &s, double &t) { add_sums(P, q.sample, g, l, lanes, s, t); },
                   [&](int g, double s, double t) {
                       const int64_t at = q.sample * P.groups + g;
                       const float2 v = finish(P, at, s, t);
                       mr[g - g0] = v;
                       if (q.part == 0 && g * P.cg >= c0) P.mean_rstd[at] = v;
                   });
        __syncthreads();
        if (mine == 0) return;
        f = affine(P, q.ch, [&](int g) { return mr[g - g0]; });
    } else f = affine(P, q.ch, stats_of(P, q));
    stream<D>(mine, start, [&](int slot) { return ring.get(slot); },
              [&](int i, const Raw<XF> &r) {
                  float z[8];
                  apply<XF, ZF, ACT>(P, f, r, z);
                  store8_whole<ZF>(P.out, o0 - i * out_step, z);
              });
}

// ----------------------------------------------------------------------------------------------------------- backward
// sums over the CTA's voxels of dt and dt * xhat per channel
template <bool XF, bool ZF> struct Both { Raw<XF> x; Raw<ZF> z; };

// The calls for channels whose rstd is far from 1
template <bool XF, bool ZF, int ACT> __device__ __noinline__ void sums_far(const GnParams &P, uint32_t far, double *sa, double *sb)
{
    const Place q = place(P, false);
    const int64_t line = q.sample * P.v + q.v0;
    far_sums<XF, ZF, ACT>(far_of(P, q.sample), Run{line * P.px + q.ch, P.apart * P.px, line * P.pdz + q.ch, P.apart * P.pdz, 0, 0, q.count},
                          far, q.ch, sa, sb);
}
template <bool XF, bool ZF, int ACT> __device__ __noinline__ void apply_far(const GnParams &P, const float2 *means, int g0)
{
    const Place q = place(P, true);
    const int64_t line = q.sample * P.v + q.v0;
    far_apply<XF, ZF, ACT>(far_of(P, q.sample), Run{line * P.px + q.ch, P.apart * P.px, line * P.pdz + q.ch, P.apart * P.pdz, line * P.po + q.ch, P.apart * P.po, q.count},
                           q.ch, means, g0);
}

template <bool XF, bool ZF, int ACT>
__global__ void __launch_bounds__(GT, resident(XF, true))
gn_bwd_sums_kernel(const __grid_constant__ GnParams P)
{
    extern __shared__ __align__(16) double sm[];                // the rings, then the sums over the lines
    constexpr int D = depth(XF, true);
    pdl_launch_dependents();
    pdl_wait();
    const Place q = place(P, false);
    const int mine = q.count;
    const int64_t line = q.sample * P.v + q.v0, xs = P.apart * P.px, x0 = line * P.px + q.ch, zs = P.apart * P.pdz, z0 = line * P.pdz + q.ch;
    const Ring<XF, D> rx(sm);
    const Ring<ZF, D> rz((char *)sm + Ring<XF, D>::BYTES);
    const auto start = [&](int i, int slot) { rx.load(slot, P.x, x0 + i * xs); rz.load(slot, P.dz, z0 + i * zs); };
    begin<D>(mine, start);
    double a[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = b[j] = 0.0;
    uint32_t far = 0;                                           // channels whose sums left fp32
    if (mine > 0) {
        const Affine f = affine(P, q.ch, stats_of(P, q));
        f32x2 s1[4], s2[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) s1[j] = s2[j] = 0;
        stream<D>(mine, start, [&](int slot) { return Both<XF, ZF>{rx.get(slot), rz.get(slot)}; },
                  [&](int, const Both<XF, ZF> &r) {
                      f32x2 d[4], dt[4];
                      slopes<XF, ZF, ACT>(P, f, r.x, r.z, d, dt);
#pragma unroll
                      for (int j = 0; j < 4; ++j) { s1[j] = add2(s1[j], dt[j]); s2[j] = fma2(dt[j], d[j], s2[j]); }
                  });
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float f1[2], f2[2];
            unpack2(s1[j], f1[0], f1[1]);
            unpack2(s2[j], f2[0], f2[1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float rstd = P.mean_rstd[q.sample * P.groups + group_of(P, q.ch + 2 * j + i)].y;
                a[2 * j + i] = f1[i];
                b[2 * j + i] = (double)f2[i] * rstd;
                far |= sum_is_far(rstd, f2[i]) ? 1u << (2 * j + i) : 0u;
            }
        }
    }
    landed<0>();
    __syncthreads();                                            // the rings make room
    const Totals tot = sum_lines(P.ty, P.uc, q.ty, q.unit, a, b, sm, [&](double *sa, double *sb) {
        if (far) sums_far<XF, ZF, ACT>(P, far, sa, sb);
    });
    const int cc = P.uc * 8, c0 = blockIdx.y * cc;
    double2 *out = P.part + (q.sample * P.parts + q.part) * P.c + c0;
    for (int i = threadIdx.x; i < cc && c0 + i < P.c; i += GT) out[i] = make_double2(tot.a(i), tot.b(i));
}

// chan[n][c] = sum over the parts, 8 channels per CTA
__global__ void __launch_bounds__(1024)
gn_bwd_parts_kernel(const GnParams P)
{
    __shared__ double2 red[128][9];
    pdl_launch_dependents();
    pdl_wait();
    const int per = P.c / 8;
    const int64_t sample = blockIdx.x / per;
    const int c0 = (int)(blockIdx.x - sample * per) * 8;
    const int col = threadIdx.x & 7, line = threadIdx.x >> 3;
    double s = 0.0, t = 0.0;
    const double2 *p = P.part + sample * P.parts * P.c + c0 + col;
#pragma unroll 4
    for (int i = line; i < P.parts; i += 128) { const double2 v = p[(int64_t)i * P.c]; s += v.x; t += v.y; }
    red[line][col] = make_double2(s, t);
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp >= 8) return;
    s = t = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) { s += red[i * 32 + lane][warp].x; t += red[i * 32 + lane][warp].y; }
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        t += __shfl_xor_sync(0xffffffffu, t, o);
    }
    if (lane == 0) P.chan[sample * P.c + c0 + warp] = make_double2(s, t);
}

// dx, and dw and db from the sums of all samples
template <bool XF, bool ZF, int ACT>
__global__ void __launch_bounds__(GT, resident(XF, true))
gn_bwd_apply_kernel(const __grid_constant__ GnParams P)
{
    extern __shared__ __align__(16) double sm[];                // the rings, then of this chunk's groups (mean(w dt), mean(w dt xhat))
    constexpr int D = depth(XF, true);
    pdl_launch_dependents();
    pdl_wait();
    const Place q = place(P, true);
    const int mine = q.count;
    const int64_t line = q.sample * P.v + q.v0 + (mine - 1) * P.apart;             // backwards from the last voxel
    const int64_t xs = P.apart * P.px, x0 = line * P.px + q.ch, zs = P.apart * P.pdz, z0 = line * P.pdz + q.ch, os = P.apart * P.po, o0 = line * P.po + q.ch;
    const Ring<XF, D> rx(sm);
    const Ring<ZF, D> rz((char *)sm + Ring<XF, D>::BYTES);
    float2 *means = (float2 *)((char *)sm + Ring<XF, D>::BYTES + Ring<ZF, D>::BYTES);
    const auto start = [&](int i, int slot) { rx.load(slot, P.x, x0 - i * xs); rz.load(slot, P.dz, z0 - i * zs); };
    begin<D>(mine, start);
    const int cc = P.uc * 8, c0 = blockIdx.y * cc, c1 = min(P.c, c0 + cc), g0 = c0 / P.cg, g1 = (c1 - 1) / P.cg;
    const double inv = P.inv_count;
    sum_groups(g0, g1, P.cg,
               [&](int g, int l, int lanes, double &s, double &t) {
                   for (int ch = g * P.cg + l; ch < (g + 1) * P.cg; ch += lanes) {
                       const double2 v = P.chan[q.sample * P.c + ch];
                       const double w = P.w ? P.w[ch] : 1.f;
                       s += w * v.x;
                       t += w * v.y;
                   }
               },
               [&](int g, double s, double t) { means[g - g0] = make_float2((float)(s * inv), (float)(t * inv)); });
    __syncthreads();
    if (blockIdx.y == 0 && (P.dw || P.db)) {                    // a few lanes per channel, four samples each where that is enough
        int lanes = 1;
        while (lanes < 32 && lanes * 4 < P.n) lanes *= 2;
        const int l = threadIdx.x % lanes, per = GT / lanes;
        for (int64_t c0 = (int64_t)blockIdx.x * per; c0 < P.c; c0 += (int64_t)gridDim.x * per) {      // the same turns for every thread
            const int64_t ch = c0 + threadIdx.x / lanes;
            double s = 0.0, t = 0.0;
            if (ch < P.c) {
#pragma unroll 4
                for (int i = l; i < P.n; i += lanes) { const double2 v = P.chan[(int64_t)i * P.c + ch]; s += v.x; t += v.y; }
            }
            for (int o = lanes / 2; o > 0; o >>= 1) {
                s += __shfl_xor_sync(0xffffffffu, s, o);
                t += __shfl_xor_sync(0xffffffffu, t, o);
            }
            if (ch < P.c && l == 0 && P.db) P.db[ch] = (float)s;
            if (ch < P.c && l == 0 && P.dw) P.dw[ch] = (float)t;
        }
    }
    if (mine == 0) return;
    const auto means_of = [&](int g) { return means[g - g0]; };
    const Affine f = affine(P, q.ch, stats_of(P, q));
    const Back k = back_terms(P, q.ch, stats_of(P, q), means_of);
    if (terms_are_far(P, q.ch, k, stats_of(P, q), means_of)) {
        landed<0>();
        apply_far<XF, ZF, ACT>(P, means, g0);
        return;
    }
    stream<D>(mine, start, [&](int slot) { return Both<XF, ZF>{rx.get(slot), rz.get(slot)}; },
              [&](int i, const Both<XF, ZF> &r) {
                  float o[8];
                  back_apply<XF, ZF, ACT>(P, f, k, r.x, r.z, o);
                  store8_whole<XF>(P.out, o0 - i * os, o);
              });
}

// ----------------------------------------------------------------------------------------------------------- host
// Units, lines and parts for a sample of v voxels: about `per_sm` CTAs per SM, none with fewer than 4 voxels per thread where that leaves it without
// work, none with more than RUN.
void split(GnParams &P, int per_sm)
{
    const int units = P.c / 8;
    P.chunks = (units + GT - 1) / GT;
    P.uc = (units + P.chunks - 1) / P.chunks;
    P.ty = GT / P.uc;
    const int64_t room = (int64_t)sm_count() * per_sm / ((int64_t)P.n * P.chunks), least = (P.v + (int64_t)P.ty * RUN - 1) / ((int64_t)P.ty * RUN);
    const int64_t need = (P.v + (int64_t)P.ty * 4 - 1) / ((int64_t)P.ty * 4);
    int64_t parts = need < room ? need : room;
    if (parts < least) parts = least;
    P.parts = (int32_t)parts;
    P.lead = P.ty;
    P.apart = (int64_t)P.ty * parts;
    P.span = P.v;
}

// The passes that apply have nothing to hand over at their end, so large tensors are cut into short runs, one after the other through the CTAs that
// the GPU holds: CTAs at different points of their work use the memory better than CTAs in step (128^3 x 64 bf16 forward: 153 -> 146 us).  Up
// to LONG_RUN units per thread of a resident grid the constants at the start of a CTA cost more than that (10^6 x 64: 72 -> 76).
constexpr int LONG_RUN = 64, SHORT_RUN = 16;
void short_runs(GnParams &P)
{
    if ((P.v + P.apart - 1) / P.apart <= LONG_RUN) return;
    P.lead = P.span = (int64_t)P.ty * SHORT_RUN;
    P.apart = P.ty;
    P.parts = (int32_t)((P.v + P.lead - 1) / P.lead);
}

// Whether the CTAs of the forward pass that apply also finish the sums, each those of its own groups: the launch of the kernel that does it otherwise costs
// 3 us, what a CTA reads for it less while that is little and one run per CTA (2 x 32,768 x 64 bf16: 18.2 -> 15.1 us, some of it from the sums' bank conflicts).
constexpr int FUSE_GROUPS = GT, FUSE_SUMS = 4096;
bool fuse(const GnParams &P)
{
    if ((P.v + P.apart - 1) / P.apart > LONG_RUN) return false;
    const int cc = P.uc * 8, groups = std::min(P.groups, (cc - 1) / P.cg + 2);        // of a chunk, at most
    const int64_t sums = P.stats ? P.cg : (int64_t)P.parts * std::min(P.chunks, (P.cg - 1) / cc + 2);
    return groups <= FUSE_GROUPS && groups * sums <= FUSE_SUMS;
}

size_t workspace(int64_t v, int n, int c, int groups)
{
    // the larger of the forward pass' [n][groups][parts][chunks] and the backward pass' [n][parts + 1][c]
    GnParams P = {};
    P.v = v; P.n = n; P.c = c;
    split(P, resident(false, false));                          // bf16 has the more parts
    const size_t fwd = (size_t)n * groups * P.parts * P.chunks + ((size_t)n * groups + 1) / 2;        // and the groups' first values
    split(P, resident(false, true));
    const size_t bwd = (size_t)n * c * (P.parts + 1);
    return (fwd > bwd ? fwd : bwd) * sizeof(double2);
}

lamp_status_t check_params(const lamp_group_norm_t *p, const lamp_tensor_t *x)
{
    if (!p || p->groups < 1 || x->c % p->groups) return LAMP_ERR_INVALID_ARG;
    if (x->c > 65536 || (int64_t)x->n * x->c > 2147483647ll) return LAMP_ERR_UNSUPPORTED;
    if (p->act < LAMP_ACT_NONE || p->act > LAMP_ACT_GELU) return LAMP_ERR_INVALID_ARG;
    if (!(p->eps >= 0.f) || !(p->slope - p->slope == 0.f)) return LAMP_ERR_INVALID_ARG;
    if (((uintptr_t)p->w | (uintptr_t)p->b) & 3) return LAMP_ERR_INVALID_ARG;
    return LAMP_OK;
}

lamp_status_t check_same(const lamp_tensor_t *t, const lamp_tensor_t *x)
{
    lamp_status_t s;
    if ((s = check_view(t, false)) != LAMP_OK) return s;
    if ((t->c & 7) || (t->c_pitch & 7) || (t->c_offset & 7)) return LAMP_ERR_UNSUPPORTED;
    if (t->n != x->n || t->d != x->d || t->h != x->h || t->w != x->w || t->c != x->c) return LAMP_ERR_INVALID_ARG;
    return LAMP_OK;
}

GnParams params(const lamp_group_norm_t *p, const lamp_tensor_t *x, const float *mean_rstd, void *ws)
{
    GnParams P = {};
    const TView v = make_view(x);
    P.x = v.p; P.px = v.pitch;
    P.n = x->n; P.v = (int64_t)x->d * x->h * x->w; P.c = x->c; P.groups = p->groups; P.cg = x->c / p->groups;
    P.inv_cg = ((1ull << 32) + P.cg - 1) / P.cg;
    if (P.v > 0) P.inv_count = 1.0 / ((double)P.v * P.cg);
    P.act = p->act; P.slope = p->slope; P.eps = p->eps; P.w = p->w; P.b = p->b;
    P.mean_rstd = (float2 *)mean_rstd;
    P.part = (double2 *)ws;
    return P;
}

bool short_launch(const GnParams &P) { return (int64_t)P.n * P.v * P.c <= 32 * 1024 * 1024; }

size_t larger(size_t a, size_t b) { return a > b ? a : b; }

template <bool XF, bool ZF, int ACT>
lamp_status_t forward(GnParams &P, cudaStream_t st)
{
    lamp_status_t s;
    const bool early = short_launch(P);
    const size_t rings = Ring<XF, depth(XF, false)>::BYTES;
    split(P, resident(XF, false));
    const dim3 grid((unsigned)(P.n * P.parts), (unsigned)P.chunks);
    P.ref = (double *)(P.part + (int64_t)P.n * P.groups * P.parts * P.chunks);
    if (!P.stats && (s = launch_pdl(early, gn_sums_kernel<XF>, grid, dim3(GT), larger(rings, lines_bytes(P.ty, P.uc)), st, P)) != LAMP_OK) return s;
    P.fused = fuse(P);
    if (!P.fused) {
        const int64_t all = (int64_t)P.n * P.groups;
        const bool many = P.stats ? P.cg > 256 : P.parts > 128;
        if ((s = launch_pdl(early, many ? gn_finish_kernel<GT / 32> : gn_finish_kernel<1>, dim3((unsigned)(many ? all : (all + GT / 32 - 1) / (GT / 32))), dim3(GT), 0, st, P)) !=
            LAMP_OK) return s;
        short_runs(P);
    }
    return launch_pdl(early, gn_apply_kernel<XF, ZF, ACT>, dim3((unsigned)(P.n * P.parts), (unsigned)P.chunks), dim3(GT), rings + FUSE_GROUPS * sizeof(float2), st, P);
}

template <bool XF, bool ZF, int ACT>
lamp_status_t backward(GnParams &P, cudaStream_t st)
{
    lamp_status_t s;
    const bool early = short_launch(P);
    constexpr int D = depth(XF, true);
    const size_t rings = Ring<XF, D>::BYTES + Ring<ZF, D>::BYTES;
    split(P, resident(XF, true));
    const dim3 grid((unsigned)(P.n * P.parts), (unsigned)P.chunks);
    P.chan = P.parts > 1 ? P.part + (int64_t)P.n * P.parts * P.c : P.part;
    static SmemAttrOnce sums, applies;
    if ((s = sums.ensure(gn_bwd_sums_kernel<XF, ZF, ACT>, (int)larger(rings, lines_bytes(GT, 1)))) != LAMP_OK) return s;
    if ((s = applies.ensure(gn_bwd_apply_kernel<XF, ZF, ACT>, (int)(rings + (size_t)GT * 8 * sizeof(float2)))) != LAMP_OK) return s;
    if ((s = launch_pdl(early, gn_bwd_sums_kernel<XF, ZF, ACT>, grid, dim3(GT), larger(rings, lines_bytes(P.ty, P.uc)), st, P)) != LAMP_OK) return s;
    if (P.parts > 1 && (s = launch_pdl(early, gn_bwd_parts_kernel, dim3((unsigned)(P.c / 8 * P.n)), dim3(1024), 0, st, P)) != LAMP_OK) return s;
    short_runs(P);
    return launch_pdl(early, gn_bwd_apply_kernel<XF, ZF, ACT>, dim3((unsigned)(P.n * P.parts), (unsigned)P.chunks), dim3(GT), rings + (size_t)P.uc * 8 * sizeof(float2), st, P);
}

template <bool XF, bool ZF>
lamp_status_t by_act(GnParams &P, bool back, cudaStream_t st)
{
    switch (P.act) {
    case LAMP_ACT_NONE: return back ? backward<XF, ZF, LAMP_ACT_NONE>(P, st) : forward<XF, ZF, LAMP_ACT_NONE>(P, st);
    case LAMP_ACT_LEAKY_RELU: return back ? backward<XF, ZF, LAMP_ACT_LEAKY_RELU>(P, st) : forward<XF, ZF, LAMP_ACT_LEAKY_RELU>(P, st);
    case LAMP_ACT_SILU: return back ? backward<XF, ZF, LAMP_ACT_SILU>(P, st) : forward<XF, ZF, LAMP_ACT_SILU>(P, st);
    default: return back ? backward<XF, ZF, LAMP_ACT_GELU>(P, st) : forward<XF, ZF, LAMP_ACT_GELU>(P, st);
    }
}

lamp_status_t by_type(GnParams &P, bool xf, bool zf, bool back, cudaStream_t st)
{
    if (!P.stats) {
        const lamp_status_t s = gn_small(P, xf, zf, back, st);
        if (s != LAMP_ERR_UNSUPPORTED) return s;
    }
    if (!xf) return by_act<false, false>(P, back, st);
    return zf ? by_act<true, true>(P, back, st) : by_act<true, false>(P, back, st);
}

lamp_status_t check_scratch(const GnParams &P, const void *ws, size_t ws_bytes)
{
    return !ws || ((uintptr_t)ws & 15) || ws_bytes < workspace(P.v, P.n, P.c, P.groups) ? LAMP_ERR_WORKSPACE : LAMP_OK;
}

}  // namespace

}  // namespace lamp

using namespace lamp;

extern "C" size_t lamp_group_norm_workspace_bytes(const lamp_group_norm_t *p, const lamp_tensor_t *x)
{
    if (!x || check_same(x, x) != LAMP_OK || check_params(p, x) != LAMP_OK) return 0;
    return voxels(x) == 0 ? 0 : workspace((int64_t)x->d * x->h * x->w, x->n, x->c, p->groups);
}

extern "C" lamp_status_t lamp_group_norm_act_fwd(const lamp_group_norm_t *p, const lamp_tensor_t *x, const double *stats, lamp_tensor_t *z,
                                                 float *mean_rstd, void *ws, size_t ws_bytes, void *cuda_stream)
{
    lamp_status_t s;
    if (!x || !z || (!mean_rstd && voxels(x) != 0)) return LAMP_ERR_INVALID_ARG;
    if ((s = check_same(x, x)) != LAMP_OK || (s = check_params(p, x)) != LAMP_OK || (s = check_same(z, x)) != LAMP_OK) return s;
    if (x->dtype == LAMP_BF16 && z->dtype == LAMP_F32) return LAMP_ERR_UNSUPPORTED;
    if (((uintptr_t)mean_rstd & 7) || ((uintptr_t)stats & 15)) return LAMP_ERR_INVALID_ARG;
    if (voxels(x) == 0) return LAMP_OK;
    GnParams P = params(p, x, mean_rstd, ws);
    P.stats = stats;
    if (!stats && (s = check_scratch(P, ws, ws_bytes)) != LAMP_OK) return s;
    const TView v = make_view(z);
    P.out = v.p; P.po = v.pitch;
    return by_type(P, x->dtype == LAMP_F32, z->dtype == LAMP_F32, false, (cudaStream_t)cuda_stream);
}

extern "C" lamp_status_t lamp_group_norm_act_bwd(const lamp_group_norm_t *p, const lamp_tensor_t *dz, const lamp_tensor_t *x, const float *mean_rstd,
                                                 lamp_tensor_t *dx, float *dw, float *db, void *ws, size_t ws_bytes, void *cuda_stream)
{
    lamp_status_t s;
    if (!x || !dz || !dx || (!mean_rstd && voxels(x) != 0)) return LAMP_ERR_INVALID_ARG;
    if ((s = check_same(x, x)) != LAMP_OK || (s = check_params(p, x)) != LAMP_OK || (s = check_same(dz, x)) != LAMP_OK || (s = check_same(dx, x)) != LAMP_OK) return s;
    if (dx->dtype != x->dtype || (x->dtype == LAMP_BF16 && dz->dtype == LAMP_F32)) return LAMP_ERR_UNSUPPORTED;
    if (((uintptr_t)mean_rstd & 7) || (((uintptr_t)dw | (uintptr_t)db) & 3)) return LAMP_ERR_INVALID_ARG;
    GnParams P = params(p, x, mean_rstd, ws);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (voxels(x) == 0) {                                       // sums over nothing
        if (dw) LAMP_CUDA_OK(cudaMemsetAsync(dw, 0, (size_t)x->c * 4, st));
        if (db) LAMP_CUDA_OK(cudaMemsetAsync(db, 0, (size_t)x->c * 4, st));
        return LAMP_OK;
    }
    if ((s = check_scratch(P, ws, ws_bytes)) != LAMP_OK) return s;
    const TView vz = make_view(dz), vd = make_view(dx);
    P.dz = vz.p; P.pdz = vz.pitch; P.out = vd.p; P.po = vd.pitch; P.dw = dw; P.db = db;
    return by_type(P, x->dtype == LAMP_F32, dz->dtype == LAMP_F32, true, st);
}
