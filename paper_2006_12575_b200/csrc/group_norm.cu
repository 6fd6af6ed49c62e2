// Group norm with an activation, channels last:  t = (x - mean_g) rstd_g w[c] + b[c],  z = act(t),  and its backward pass.
//
// The statistics of a group need all of its values before the first output: a pass that sums, a kernel that finishes the few
// sums, a pass that applies.  Forward both passes read x, backward both read x and dz; the second runs against the direction of the
// first, so that it starts with what the first left in L2 (126 MB).  Bound by memory.
// A voxel's channels are taken in units of 8 (16 bytes of bf16, 32 of fp32), a thread keeps its unit for all of its voxels, so
// everything per channel stays in registers; a CTA holds TY voxels side by side and a run of voxels of one sample.
// Sums: a thread adds d = x - k and d^2 of at most RUN voxels in fp32, k the mean of the first values it loads - without it the squares of
// data far from 0 lose the variance.  Between threads, CTAs and channels of a group the sums are fp64, taken about r, the group's first
// value, and added in a fixed order.
#include "block_norm.cuh"

namespace lamp {

namespace {

using namespace bn;
using ptx::f32x2; using ptx::fma2; using ptx::add2; using ptx::mul2; using ptx::twice; using ptx::pack2; using ptx::unpack2;

constexpr int GT = 256;                       // threads
// CTAs per SM that the streaming kernels are compiled and sized for
constexpr int resident(bool xf, bool back) { return (xf ? 3 : 4) - (back ? 1 : 0); }
constexpr int RUN = 256;                      // voxels that a thread sums at most

struct GnParams {
    const void *x, *dz;
    void *out;                                // z, or dx
    int64_t px, pdz, po;
    int64_t v;                                // voxels of one sample
    int32_t n, c, groups, cg;                 // cg = channels per group
    int32_t parts;                            // CTAs per sample (and chunk of channels)
    int64_t run;                              // voxels per CTA
    int32_t chunks, uc, ty;                   // chunks of channels, units of a chunk, voxels side by side
    int32_t act;
    float slope, eps;
    const float *w, *b;
    const double *stats;
    double2 *part;                            // forward [n][groups][parts][chunks], backward [n][parts][c]
    double2 *chan;                            // backward [n][c]
    float2 *mean_rstd;
    float *dw, *db;
};


// ----------------------------------------------------------------------------------------------------------- activations
// Two values at a time: the packed fp32 instructions halve what is issued, which with a SiLU or GELU bounds these kernels as much as memory does.
// FINE: fp32 outputs of the forward pass, with expf and erfcf.  Elsewhere e^x without the correction for the rounding of x log2(e) (2^-24 |x| of e^x),
// and the normal distribution by Abramowitz & Stegun 7.1.26: q(u) = (a1 s + .. + a5 s^5) e^(-u^2), s = 1 / (1 + p u), for erfc(u), u >= 0, off by at
// most 1.5e-7.  A derivative is a factor of size one, so both are within a few units of 2^-24 of it.
__device__ __forceinline__ float ex2(float x)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
    return e;
}
__device__ __forceinline__ f32x2 pair(float a, float b) { return pack2(__float_as_uint(a), __float_as_uint(b)); }
__device__ __forceinline__ f32x2 ex2_2(f32x2 v) { float a, b; unpack2(v, a, b); return pair(ex2(a), ex2(b)); }
__device__ __forceinline__ f32x2 rcp_2(f32x2 v) { float a, b; unpack2(v, a, b); return pair(reciprocal(a), reciprocal(b)); }
__device__ __forceinline__ f32x2 sigmoid_2(f32x2 t) { return rcp_2(add2(ex2_2(mul2(t, twice(-1.4426950408889634f))), twice(1.f))); }

// below = P(X <= t) of the normal distribution, density = e^(-t^2 / 2)
__device__ __forceinline__ void normal_2(f32x2 t, f32x2 &below, f32x2 &density)
{
    density = ex2_2(mul2(t, mul2(t, twice(-0.72134752044448170f))));
    float a, b;
    unpack2(t, a, b);
    const f32x2 s = rcp_2(fma2(pair(fabsf(a), fabsf(b)), twice(0.3275911f * 0.70710678118654752f), twice(1.f)));
    f32x2 q = fma2(s, twice(0.5f * 1.061405429f), twice(0.5f * -1.453152027f));
    q = fma2(s, q, twice(0.5f * 1.421413741f));
    q = fma2(s, q, twice(0.5f * -0.284496736f));
    q = fma2(s, q, twice(0.5f * 0.254829592f));
    q = mul2(mul2(q, s), density);
    float q0, q1, u0, u1;
    unpack2(q, q0, q1);
    unpack2(fma2(q, twice(-1.f), twice(1.f)), u0, u1);
    below = pair(a > 0.f ? u0 : q0, b > 0.f ? u1 : q1);
}
template <int ACT, bool FINE> __device__ __forceinline__ f32x2 activate(f32x2 t, float slope)
{
    if constexpr (ACT == LAMP_ACT_NONE) return t;
    float a, b;
    unpack2(t, a, b);
    if constexpr (ACT == LAMP_ACT_LEAKY_RELU) return pair(a > 0.f ? a : slope * a, b > 0.f ? b : slope * b);
    if constexpr (ACT == LAMP_ACT_SILU) {
        if (FINE) return pair(a * sigmoid<true>(a), b * sigmoid<true>(b));
        return mul2(t, sigmoid_2(t));
    }
    if (FINE) return pair(a * (0.5f * erfcf(a * -0.70710678118654752f)), b * (0.5f * erfcf(b * -0.70710678118654752f)));
    f32x2 below, density;
    normal_2(t, below, density);
    return mul2(t, below);
}
// v * act'(t)
template <int ACT> __device__ __forceinline__ f32x2 times_derivative(f32x2 v, f32x2 t, float slope)
{
    if constexpr (ACT == LAMP_ACT_NONE) return v;
    if constexpr (ACT == LAMP_ACT_LEAKY_RELU) {
        float a, b, x, y;
        unpack2(t, a, b);
        unpack2(v, x, y);
        return pair(a > 0.f ? x : a <= 0.f ? slope * x : a, b > 0.f ? y : b <= 0.f ? slope * y : b);       // NaN stays
    }
    if constexpr (ACT == LAMP_ACT_SILU) {
        // s (1 + t (1 - s)) = s + y - y s with y = t s
        const f32x2 s = sigmoid_2(t), y = mul2(t, s);
        return mul2(v, add2(fma2(mul2(y, twice(-1.f)), s, y), s));
    }
    f32x2 below, density;
    normal_2(t, below, density);
    return mul2(v, fma2(mul2(t, twice(0.3989422804014327f)), density, below));
}

// ----------------------------------------------------------------------------------------------------------- places
struct Place {
    int64_t sample, v0, v1;                   // voxels of this CTA
    int part, ch, unit, ty;                   // this thread's first channel, its unit in the chunk, its voxel line
    bool active;
};
__device__ __forceinline__ Place place(const GnParams &P)
{
    Place q;
    const int64_t at = blockIdx.x;
    q.sample = at / P.parts;
    q.part = (int)(at - q.sample * P.parts);
    q.ty = threadIdx.x / P.uc;
    q.unit = threadIdx.x - q.ty * P.uc;
    const int u = blockIdx.y * P.uc + q.unit;
    q.ch = u * 8;
    q.active = q.ty < P.ty && q.ch < P.c;
    q.v0 = q.part * P.run;
    q.v1 = min(P.v, q.v0 + P.run);
    return q;
}

// first voxel of this thread's last batch of U (below v0 where it has none)
template <int U> __device__ __forceinline__ int64_t last_batch(const GnParams &P, const Place &q)
{
    const int64_t first = q.v0 + q.ty;
    return first < q.v1 ? first + (q.v1 - first - 1) / (U * P.ty) * (U * P.ty) : q.v0 - 1;
}

// Sum over the CTA's voxel lines of 8 pairs of fp64 per thread; on return tot[2 * channel + {0, 1}] (channels of the chunk) is in shared memory.
__device__ __forceinline__ void sum_lines(const GnParams &P, const Place &q, const double (&a)[8], const double (&b)[8], double *sm)
{
    // [line][channel of the chunk], first all a, then all b; the totals replace line 0
    const int cc = P.uc * 8;
    double *sa = sm, *sb = sm + P.ty * cc;
    if (q.ty < P.ty) {
#pragma unroll
        for (int j = 0; j < 8; ++j) { sa[q.ty * cc + q.unit * 8 + j] = a[j]; sb[q.ty * cc + q.unit * 8 + j] = b[j]; }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * cc; i += GT) {
        double *s = i < cc ? sa + i : sb + (i - cc);
        double t = s[0];
        for (int l = 1; l < P.ty; ++l) t += s[l * cc];
        s[0] = t;
    }
    __syncthreads();
}

// ----------------------------------------------------------------------------------------------------------- forward
template <bool XF, int U>
__global__ void __launch_bounds__(GT, resident(XF, false))
gn_sums_kernel(const GnParams P)
{
    extern __shared__ __align__(16) double sm[];
    pdl_launch_dependents();
    pdl_wait();
    const Place q = place(P);
    const int64_t base = q.sample * P.v;
    f32x2 k[4], s1[4], s2[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = s1[j] = s2[j] = 0;
    int mine = 0;
    if (q.active) {
        mine = q.v1 > q.v0 + q.ty ? ((int)(q.v1 - q.v0) - q.ty + P.ty - 1) / P.ty : 0;
        const int64_t step = P.ty * P.px;
        int64_t at = (base + q.v0 + q.ty) * P.px + q.ch;
        Raw<XF> r[U];
        for (int left = mine; left > 0; left -= U, at += U * step) {
#pragma unroll
            for (int u = 0; u < U; ++u) if (u < left) r[u] = load_raw<XF>(P.x, at + u * step);
            if (left == mine) {
                f32x2 t[4], s[4] = {0, 0, 0, 0};
#pragma unroll
                for (int u = 0; u < U; ++u) if (u < left) {
                    to_pairs<XF>(r[u], t);
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[j] = add2(s[j], t[j]);
                }
                const float inv = -1.f / (float)(left < U ? left : U);
#pragma unroll
                for (int j = 0; j < 4; ++j) k[j] = mul2(s[j], twice(inv));      // -k
            }
#pragma unroll
            for (int u = 0; u < U; ++u) if (u < left) {
                f32x2 t[4];
                to_pairs<XF>(r[u], t);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x2 d = add2(t[j], k[j]);
                    s1[j] = add2(s1[j], d);
                    s2[j] = fma2(d, d, s2[j]);
                }
            }
        }
    }
    double a[8], b[8];
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
            const int64_t first = base * P.px + (q.ch + j) / P.cg * P.cg;
            const double r = XF ? ((const float *)P.x)[first] : bf2f(((const bf16 *)P.x)[first]);
            const double e = -(double)nk[j] - r, m = (double)mine;
            a[j] = (double)f1[j] + m * e;
            b[j] = (double)f2[j] + e * (2.0 * f1[j] + m * e);
        }
    }
    sum_lines(P, q, a, b, sm);
    // channels of a group
    const int cc = P.uc * 8, c0 = blockIdx.y * cc, c1 = min(P.c, c0 + cc);
    const int g0 = c0 / P.cg, g1 = (c1 - 1) / P.cg;
    int lanes = 1;
    while (lanes < 32 && lanes * 2 <= P.cg) lanes *= 2;
    const int l = threadIdx.x % lanes, per = GT / lanes;
    for (int g = g0; g <= g1; g += per) {                        // the same number of turns for every thread
        const int mg = g + threadIdx.x / lanes;
        double s = 0.0, t = 0.0;
        if (mg <= g1) {
            for (int ch = max(c0, mg * P.cg) + l; ch < min(c1, (mg + 1) * P.cg); ch += lanes) { s += sm[ch - c0]; t += sm[P.ty * cc + ch - c0]; }
        }
        for (int o = lanes / 2; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            t += __shfl_xor_sync(0xffffffffu, t, o);
        }
        if (mg <= g1 && l == 0) P.part[((q.sample * P.groups + mg) * P.parts + q.part) * P.chunks + blockIdx.y] = make_double2(s, t);
    }
}

// mean and rstd of a group from its partial sums, or from sums per channel; W warps per group: one where the sums are few (a CTA has 8 groups),
// all where they are many
template <bool XF, int W>
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
    const int g = (int)(at - sample * P.groups);
    double s = 0.0, t = 0.0, r = 0.0;
    if (P.stats) {
        const double2 *st = reinterpret_cast<const double2 *>(P.stats) + sample * P.c + g * P.cg;
#pragma unroll 4
        for (int i = first; i < P.cg; i += 32 * W) { const double2 v = st[i]; s += v.x; t += v.y; }
    } else {
        const int cc = P.uc * 8, k0 = g * P.cg / cc, k1 = ((g + 1) * P.cg - 1) / cc, ks = k1 - k0 + 1;
        const double2 *p = P.part + at * P.parts * P.chunks;
        const int64_t x0 = sample * P.v * P.px + g * P.cg;
        r = XF ? ((const float *)P.x)[x0] : bf2f(((const bf16 *)P.x)[x0]);
#pragma unroll 4
        for (int i = first; i < P.parts * ks; i += 32 * W) { const double2 v = p[i / ks * P.chunks + k0 + i % ks]; s += v.x; t += v.y; }
    }
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
    if (first == 0) {
        const double m = (double)P.v * P.cg, mu = s / m, var = t / m - mu * mu;
        P.mean_rstd[at] = make_float2((float)(r + mu), (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + (double)P.eps)));
    }
}

// -mean, rstd * w and b of this thread's channels
struct Affine { f32x2 nm[4], a[4], b[4]; };
__device__ __forceinline__ Affine affine(const GnParams &P, const Place &q)
{
    float nm[8], a[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 mr = P.mean_rstd[q.sample * P.groups + (q.ch + j) / P.cg];
        nm[j] = -mr.x;
        a[j] = mr.y * (P.w ? P.w[q.ch + j] : 1.f);
        b[j] = P.b ? P.b[q.ch + j] : 0.f;
    }
    Affine f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f.nm[j] = pack2(__float_as_uint(nm[2 * j]), __float_as_uint(nm[2 * j + 1]));
        f.a[j] = pack2(__float_as_uint(a[2 * j]), __float_as_uint(a[2 * j + 1]));
        f.b[j] = pack2(__float_as_uint(b[2 * j]), __float_as_uint(b[2 * j + 1]));
    }
    return f;
}

template <bool XF, bool ZF, int ACT, int U>
__global__ void __launch_bounds__(GT, resident(XF, false))
gn_apply_kernel(const GnParams P)
{
    pdl_launch_dependents();
    pdl_wait();
    const Place q = place(P);
    if (!q.active) return;
    const int64_t base = q.sample * P.v;
    const Affine f = affine(P, q);
    for (int64_t v = last_batch<U>(P, q); v >= q.v0; v -= (int64_t)U * P.ty) {
        Raw<XF> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = v + (int64_t)u * P.ty;
            if (at < q.v1) r[u] = load_raw<XF>(P.x, (base + at) * P.px + q.ch);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = v + (int64_t)u * P.ty;
            if (at >= q.v1) continue;
            f32x2 t[4];
            to_pairs<XF>(r[u], t);
            float z[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) unpack2(activate<ACT, ZF>(fma2(add2(t[j], f.nm[j]), f.a[j], f.b[j]), P.slope), z[2 * j], z[2 * j + 1]);
            store8_last<ZF>(P.out, (base + at) * P.po + q.ch, z);
        }
    }
}

// ----------------------------------------------------------------------------------------------------------- backward
// dt and (x - mean) of 8 channels
template <bool XF, bool ZF, int ACT>
__device__ __forceinline__ void slopes(const GnParams &P, const Affine &f, const Raw<XF> &rx, const Raw<ZF> &rz, f32x2 (&d)[4], f32x2 (&dt)[4])
{
    to_pairs<XF>(rx, d);
    to_pairs<ZF>(rz, dt);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        d[j] = add2(d[j], f.nm[j]);
        dt[j] = times_derivative<ACT>(dt[j], fma2(d[j], f.a[j], f.b[j]), P.slope);
    }
}

// sums over the CTA's voxels of dt and dt * xhat per channel
template <bool XF, bool ZF, int ACT, int U>
__global__ void __launch_bounds__(GT, resident(XF, true))
gn_bwd_sums_kernel(const GnParams P)
{
    extern __shared__ __align__(16) double sm[];
    pdl_launch_dependents();
    pdl_wait();
    const Place q = place(P);
    const int64_t base = q.sample * P.v;
    double a[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = b[j] = 0.0;
    if (q.active) {
        const Affine f = affine(P, q);
        f32x2 s1[4], s2[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) s1[j] = s2[j] = 0;
        for (int64_t v = q.v0 + q.ty; v < q.v1; v += (int64_t)U * P.ty) {
            Raw<XF> rx[U];
            Raw<ZF> rz[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t at = v + (int64_t)u * P.ty;
                if (at < q.v1) {
                    rx[u] = load_raw<XF>(P.x, (base + at) * P.px + q.ch);
                    rz[u] = load_raw<ZF>(P.dz, (base + at) * P.pdz + q.ch);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + (int64_t)u * P.ty >= q.v1) continue;
                f32x2 d[4], dt[4];
                slopes<XF, ZF, ACT>(P, f, rx[u], rz[u], d, dt);
#pragma unroll
                for (int j = 0; j < 4; ++j) { s1[j] = add2(s1[j], dt[j]); s2[j] = fma2(dt[j], d[j], s2[j]); }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float f1[2], f2[2];
            unpack2(s1[j], f1[0], f1[1]);
            unpack2(s2[j], f2[0], f2[1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float rstd = P.mean_rstd[q.sample * P.groups + (q.ch + 2 * j + i) / P.cg].y;
                a[2 * j + i] = f1[i];
                b[2 * j + i] = (double)f2[i] * rstd;
            }
        }
    }
    sum_lines(P, q, a, b, sm);
    const int cc = P.uc * 8, c0 = blockIdx.y * cc;
    double2 *out = P.part + (q.sample * P.parts + q.part) * P.c + c0;
    for (int i = threadIdx.x; i < cc && c0 + i < P.c; i += GT) out[i] = make_double2(sm[i], sm[P.ty * cc + i]);
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
template <bool XF, bool ZF, int ACT, int U>
__global__ void __launch_bounds__(GT, resident(XF, true))
gn_bwd_apply_kernel(const GnParams P)
{
    extern __shared__ __align__(16) float2 means[];             // of this chunk's groups: (mean(w dt), mean(w dt xhat))
    pdl_launch_dependents();
    pdl_wait();
    const Place q = place(P);
    const int64_t base = q.sample * P.v;
    const int cc = P.uc * 8, c0 = blockIdx.y * cc, c1 = min(P.c, c0 + cc), g0 = c0 / P.cg, g1 = (c1 - 1) / P.cg;
    {
        int lanes = 1;
        while (lanes < 32 && lanes * 2 <= P.cg) lanes *= 2;
        const int l = threadIdx.x % lanes, per = GT / lanes;
        const double inv = 1.0 / ((double)P.v * P.cg);
        for (int g = g0; g <= g1; g += per) {
            const int mg = g + threadIdx.x / lanes;
            double s = 0.0, t = 0.0;
            if (mg <= g1) {
                for (int i = l; i < P.cg; i += lanes) {
                    const int ch = mg * P.cg + i;
                    const double2 v = P.chan[q.sample * P.c + ch];
                    const double w = P.w ? P.w[ch] : 1.f;
                    s += w * v.x;
                    t += w * v.y;
                }
            }
            for (int o = lanes / 2; o > 0; o >>= 1) {
                s += __shfl_xor_sync(0xffffffffu, s, o);
                t += __shfl_xor_sync(0xffffffffu, t, o);
            }
            if (mg <= g1 && l == 0) means[mg - g0] = make_float2((float)(s * inv), (float)(t * inv));
        }
    }
    __syncthreads();
    if (blockIdx.y == 0 && (P.dw || P.db)) {                    // a warp per channel, the lanes over the samples
        const int lane = threadIdx.x & 31;
        for (int64_t ch = (int64_t)blockIdx.x * (GT / 32) + (threadIdx.x >> 5); ch < P.c; ch += (int64_t)gridDim.x * (GT / 32)) {
            double s = 0.0, t = 0.0;
            for (int i = lane; i < P.n; i += 32) { const double2 v = P.chan[(int64_t)i * P.c + ch]; s += v.x; t += v.y; }
            for (int o = 16; o > 0; o >>= 1) {
                s += __shfl_xor_sync(0xffffffffu, s, o);
                t += __shfl_xor_sync(0xffffffffu, t, o);
            }
            if (lane == 0 && P.db) P.db[ch] = (float)s;
            if (lane == 0 && P.dw) P.dw[ch] = (float)t;
        }
    }
    if (!q.active) return;
    const Affine f = affine(P, q);
    // dx = dt a + (x - mean) e + h,  e = -rstd^2 mean(w dt xhat), h = -rstd mean(w dt)
    f32x2 e[4], h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float ev[2], hv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int g = (q.ch + 2 * j + i) / P.cg;
            const float rstd = P.mean_rstd[q.sample * P.groups + g].y;
            const float2 m = means[g - g0];
            ev[i] = -rstd * (rstd * m.y);
            hv[i] = -rstd * m.x;
        }
        e[j] = pack2(__float_as_uint(ev[0]), __float_as_uint(ev[1]));
        h[j] = pack2(__float_as_uint(hv[0]), __float_as_uint(hv[1]));
    }
    for (int64_t v = last_batch<U>(P, q); v >= q.v0; v -= (int64_t)U * P.ty) {
        Raw<XF> rx[U];
        Raw<ZF> rz[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = v + (int64_t)u * P.ty;
            if (at < q.v1) {
                rx[u] = load_raw<XF>(P.x, (base + at) * P.px + q.ch);
                rz[u] = load_raw<ZF>(P.dz, (base + at) * P.pdz + q.ch);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = v + (int64_t)u * P.ty;
            if (at >= q.v1) continue;
            f32x2 d[4], dt[4];
            slopes<XF, ZF, ACT>(P, f, rx[u], rz[u], d, dt);
#pragma unroll
            for (int j = 0; j < 4; ++j) d[j] = fma2(dt[j], f.a[j], fma2(d[j], e[j], h[j]));
            float o[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) unpack2(d[j], o[2 * j], o[2 * j + 1]);
            store8_last<XF>(P.out, (base + at) * P.po + q.ch, o);
        }
    }
}

// ----------------------------------------------------------------------------------------------------------- host
// Units, lines and runs for a sample of v voxels: about `per_sm` CTAs per SM, none with less than a batch of u voxels per thread or more than
// RUN of them.
void split(GnParams &P, int u, int per_sm)
{
    const int units = P.c / 8;
    P.chunks = (units + GT - 1) / GT;
    P.uc = (units + P.chunks - 1) / P.chunks;
    P.ty = GT / P.uc;
    const int64_t room = (int64_t)sm_count() * per_sm / ((int64_t)P.n * P.chunks), least = (P.v + (int64_t)P.ty * RUN - 1) / ((int64_t)P.ty * RUN);
    const int64_t need = (P.v + (int64_t)P.ty * u - 1) / ((int64_t)P.ty * u);
    int64_t parts = need < room ? need : room;
    if (parts < least) parts = least;
    P.run = (P.v + parts - 1) / parts;
    P.run = (P.run + P.ty - 1) / P.ty * P.ty;
    P.parts = (int32_t)((P.v + P.run - 1) / P.run);
}

constexpr int SUM_U = 4, BWD_U = 2;           // voxels in flight per thread

size_t workspace(int64_t v, int n, int c)
{
    // the larger of the forward pass' [n][groups][parts][chunks] and the backward pass' [n][parts + 1][c], groups = c at most
    GnParams P = {};
    P.v = v; P.n = n; P.c = c;
    split(P, SUM_U, resident(false, false));
    const size_t fwd = (size_t)n * c * P.parts * P.chunks;
    split(P, BWD_U, resident(false, true));
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
    P.act = p->act; P.slope = p->slope; P.eps = p->eps; P.w = p->w; P.b = p->b;
    P.mean_rstd = (float2 *)mean_rstd;
    P.part = (double2 *)ws;
    return P;
}

bool short_launch(const GnParams &P) { return (int64_t)P.n * P.v * P.c <= 32 * 1024 * 1024; }

template <bool XF, bool ZF, int ACT>
lamp_status_t forward(GnParams &P, cudaStream_t st)
{
    lamp_status_t s;
    const bool early = short_launch(P);
    split(P, SUM_U, resident(XF, false));
    const dim3 grid((unsigned)(P.n * P.parts), (unsigned)P.chunks);
    if (!P.stats) {
        const size_t smem = (size_t)P.ty * P.uc * 8 * 2 * sizeof(double);
        if ((s = launch_pdl(early, gn_sums_kernel<XF, SUM_U>, grid, dim3(GT), smem, st, P)) != LAMP_OK) return s;
    }
    const int64_t all = (int64_t)P.n * P.groups;
    const bool many = P.stats ? P.cg > 256 : P.parts > 128;
    if ((s = launch_pdl(early, many ? gn_finish_kernel<XF, GT / 32> : gn_finish_kernel<XF, 1>, dim3((unsigned)(many ? all : (all + GT / 32 - 1) / (GT / 32))), dim3(GT), 0, st,
                        P)) != LAMP_OK) return s;
    return launch_pdl(early, gn_apply_kernel<XF, ZF, ACT, SUM_U>, grid, dim3(GT), 0, st, P);
}

template <bool XF, bool ZF, int ACT>
lamp_status_t backward(GnParams &P, cudaStream_t st)
{
    lamp_status_t s;
    const bool early = short_launch(P);
    split(P, BWD_U, resident(XF, true));
    const dim3 grid((unsigned)(P.n * P.parts), (unsigned)P.chunks);
    const size_t smem = (size_t)P.ty * P.uc * 8 * 2 * sizeof(double);
    P.chan = P.parts > 1 ? P.part + (int64_t)P.n * P.parts * P.c : P.part;
    if ((s = launch_pdl(early, gn_bwd_sums_kernel<XF, ZF, ACT, BWD_U>, grid, dim3(GT), smem, st, P)) != LAMP_OK) return s;
    if (P.parts > 1 && (s = launch_pdl(early, gn_bwd_parts_kernel, dim3((unsigned)(P.c / 8 * P.n)), dim3(1024), 0, st, P)) != LAMP_OK) return s;
    return launch_pdl(early, gn_bwd_apply_kernel<XF, ZF, ACT, BWD_U>, grid, dim3(GT), (size_t)P.uc * 8 * sizeof(float2), st, P);
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
    if (!xf) return by_act<false, false>(P, back, st);
    return zf ? by_act<true, true>(P, back, st) : by_act<true, false>(P, back, st);
}

lamp_status_t check_scratch(const GnParams &P, const void *ws, size_t ws_bytes)
{
    return !ws || ((uintptr_t)ws & 15) || ws_bytes < workspace(P.v, P.n, P.c) ? LAMP_ERR_WORKSPACE : LAMP_OK;
}

}  // namespace

}  // namespace lamp

using namespace lamp;

extern "C" size_t lamp_group_norm_workspace_bytes(const lamp_group_norm_t *p, const lamp_tensor_t *x)
{
    if (!x || check_same(x, x) != LAMP_OK || check_params(p, x) != LAMP_OK) return 0;
    return voxels(x) == 0 ? 0 : workspace((int64_t)x->d * x->h * x->w, x->n, x->c);
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
