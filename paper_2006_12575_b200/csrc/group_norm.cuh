// What the two forms of the group norm share (group_norm.cu: tensors that stream through, group_norm_small.cu: samples that a cluster holds).
// A voxel's channels are taken in units of 8 (16 bytes of bf16, 32 of fp32); a thread keeps its unit for all of its voxels, so everything per
// channel stays in registers.
#pragma once
#include "block_norm.cuh"

namespace lamp {
namespace gn {

using namespace bn;
using ptx::f32x2; using ptx::fma2; using ptx::add2; using ptx::mul2; using ptx::twice; using ptx::pack2; using ptx::unpack2;

constexpr int GT = 256;                       // threads

struct GnParams {
    const void *x, *dz;
    void *out;                                // z, or dx
    int64_t px, pdz, po;
    int64_t v;                                // voxels of one sample
    double inv_count;                         // 1 / values of a group
    int32_t n, c, groups, cg;                 // cg = channels per group
    uint64_t inv_cg;                          // 2^32 / cg, rounded up
    int32_t parts;                            // CTAs per sample (and chunk of channels)
    int64_t apart, lead, span;                // voxels between two of a thread, between the first ones of two CTAs, from a CTA's first one to its end
    int32_t chunks, uc, ty;                   // chunks of channels, units of a chunk, voxels side by side
    int32_t act;
    float slope, eps;
    const float *w, *b;
    const double *stats;
    double2 *part;                            // forward [n][groups][parts][chunks], backward [n][parts][c]
    double2 *chan;                            // backward [n][c]
    double *ref;                              // forward [n][groups], the first values
    float2 *mean_rstd;
    float *dw, *db;
    bool fused;                               // the apply pass finishes the sums itself
};

// ch / cg: inv_cg cg is less than cg above 2^32 and ch < 2^16, so what it adds stays below 1 / cg
__device__ __forceinline__ int group_of(const GnParams &P, int ch) { return (int)(((uint64_t)(uint32_t)ch * P.inv_cg) >> 32); }

// ----------------------------------------------------------------------------------------------------------- activations
// Two values at a time: the packed fp32 instructions halve what is issued, which with a SiLU or GELU bounds these kernels as much as memory does.
// FINE: fp32 outputs; forward with expf and erfcf, backward with the two functions below whose names say so.  Elsewhere e^x without the correction for the rounding
// of x log2(e) (2^-24 |x| of e^x), and the normal distribution by Abramowitz & Stegun 7.1.26: q(u) = (a1 s + .. + a5 s^5) e^(-u^2), s = 1 / (1 + p u), for
// erfc(u), u >= 0, off by at most 1.5e-7 of one: both less than half a step of a bf16 gradient of ordinary size.
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
// The sigmoid to a few units of 2^-24 of its own size.  The exponent is formed with its rounding error (by fma, which gives a product's remainder exactly,
// and the rest of the constant); that error, a small number, goes into 2^x as the factor 1 + ln(2) error.
__device__ __forceinline__ f32x2 sigmoid_fine_2(f32x2 t)
{
    float a, b;
    unpack2(t, a, b);
    const f32x2 u = pair(fminf(a, 127.f), fminf(b, 127.f));      // beyond, e^-t is 0 and the error would not stay small
    const f32x2 hi = mul2(u, twice(-1.4426950216293335f));
    const f32x2 over = fma2(u, twice(1.9259629911266175e-08f), fma2(u, twice(1.4426950216293335f), hi));         // hi - (-u log2 e)
    return rcp_2(fma2(ex2_2(hi), fma2(over, twice(-0.69314718f), twice(1.f)), twice(1.f)));
}
// GELU' = P(X <= t) + t p(t) = h(t) for t <= 0, 1 - h(-t) for t > 0, with h(-u) = e^(-u^2 / 2) (R(u) - u / sqrt(2 pi)), R(u) = e^(u^2 / 2) P(X <= -u).  R as a
// polynomial in s = 1 / (1 + p u): degree and p chosen, coefficients fitted for the least relative error, over u <= 14 (3.7e-8; 3.4e-7 in fp32).  The
// exponential is off by 2^-24 t^2 of itself, at most 2^-24 of one: carrying its exponent's rounding as above took 91 us on 81,840 x 320 fp32 backward, so
// it takes 89, by normal_2 87.
__device__ __forceinline__ f32x2 gelu_slope_fine_2(f32x2 t)
{
    float a, b;
    unpack2(t, a, b);
    const f32x2 u = pair(fabsf(a), fabsf(b)), density = ex2_2(mul2(t, mul2(t, twice(-0.72134752044448170f))));
    const f32x2 s = rcp_2(fma2(u, twice(0.295f), twice(1.f)));
    f32x2 q = fma2(s, twice(0.0394211486f), twice(-0.183406189f));
    q = fma2(s, q, twice(0.271016657f));
    q = fma2(s, q, twice(-0.117071159f));
    q = fma2(s, q, twice(0.166289002f));
    q = fma2(s, q, twice(0.0847447962f));
    q = fma2(s, q, twice(0.121699385f));
    q = fma2(s, q, twice(0.117289335f));
    q = fma2(s, q, twice(1.70069379e-05f));
    const f32x2 h = mul2(fma2(u, twice(-0.3989422804014327f), q), density);
    float h0, h1, r0, r1;
    unpack2(h, h0, h1);
    unpack2(fma2(h, twice(-1.f), twice(1.f)), r0, r1);
    return pair(a > 0.f ? r0 : a <= 0.f ? h0 : a, b > 0.f ? r1 : b <= 0.f ? h1 : b);                   // NaN stays
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
// v * act'(t); FINE: fp32 gradients
template <int ACT, bool FINE> __device__ __forceinline__ f32x2 times_derivative(f32x2 v, f32x2 t, float slope)
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
        const f32x2 s = FINE ? sigmoid_fine_2(t) : sigmoid_2(t), y = mul2(t, s);
        return mul2(v, add2(fma2(mul2(y, twice(-1.f)), s, y), s));
    }
    if (FINE) return mul2(v, gelu_slope_fine_2(t));
    f32x2 below, density;
    normal_2(t, below, density);
    return mul2(v, fma2(mul2(t, twice(0.3989422804014327f)), density, below));
}

// -mean, rstd * w and b of this thread's channels
struct Affine { f32x2 nm[4], a[4], b[4]; };
// mr(g): (mean, rstd) of group g
template <typename F> __device__ __forceinline__ Affine affine(const GnParams &P, int ch, F mr)
{
    float nm[8], a[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 s = mr(group_of(P, ch + j));
        nm[j] = -s.x;
        a[j] = s.y * (P.w ? P.w[ch + j] : 1.f);
        b[j] = P.b ? P.b[ch + j] : 0.f;
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

// dt and (x - mean) of 8 channels
template <bool XF, bool ZF, int ACT>
__device__ __forceinline__ void slopes(const GnParams &P, const Affine &f, const Raw<XF> &rx, const Raw<ZF> &rz, f32x2 (&d)[4], f32x2 (&dt)[4])
{
    to_pairs<XF>(rx, d);
    to_pairs<ZF>(rz, dt);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        d[j] = add2(d[j], f.nm[j]);
        dt[j] = times_derivative<ACT, XF>(dt[j], fma2(d[j], f.a[j], f.b[j]), P.slope);
    }
}

// z of 8 channels
template <bool XF, bool ZF, int ACT>
__device__ __forceinline__ void apply(const GnParams &P, const Affine &f, const Raw<XF> &r, float (&z)[8])
{
    f32x2 t[4];
    to_pairs<XF>(r, t);
#pragma unroll
    for (int j = 0; j < 4; ++j) unpack2(activate<ACT, ZF>(fma2(add2(t[j], f.nm[j]), f.a[j], f.b[j]), P.slope), z[2 * j], z[2 * j + 1]);
}

// dx = dt a + (x - mean) e + h,  e = -rstd^2 mean(w dt xhat), h = -rstd mean(w dt);  m: the two means
struct Back { f32x2 e[4], h[4]; };
template <typename F, typename G> __device__ __forceinline__ Back back_terms(const GnParams &P, int ch, F mr, G means)
{
    Back k;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float ev[2], hv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int g = group_of(P, ch + 2 * j + i);
            const float rstd = mr(g).y;
            const float2 m = means(g);
            ev[i] = -rstd * (rstd * m.y);
            hv[i] = -rstd * m.x;
        }
        k.e[j] = pair(ev[0], ev[1]);
        k.h[j] = pair(hv[0], hv[1]);
    }
    return k;
}
template <bool XF, bool ZF, int ACT>
__device__ __forceinline__ void back_apply(const GnParams &P, const Affine &f, const Back &k, const Raw<XF> &rx, const Raw<ZF> &rz, float (&o)[8])
{
    f32x2 d[4], dt[4];
    slopes<XF, ZF, ACT>(P, f, rx, rz, d, dt);
#pragma unroll
    for (int j = 0; j < 4; ++j) unpack2(fma2(dt[j], f.a[j], fma2(d[j], k.e[j], k.h[j])), o[2 * j], o[2 * j + 1]);
}


template <bool XF> __device__ __forceinline__ float value_at(const void *p, int64_t i) { return XF ? ((const float *)p)[i] : bf2f(((const bf16 *)p)[i]); }

// Deviations far from 1 (outside of 2^-24 .. 2^24): where dt (x - mean), or rstd^2 times the mean of w dt xhat, leaves fp32's range while dw and dx do not, the
// values go through the two functions below, which divide by the deviation first, in fp64.  The kernels reach them by calls that find their own places, so
// that they cost the usual values next to no registers.  (128^3 x 32 bf16 with a deviation of 1e25: 355 us for 114.)
__device__ __forceinline__ bool sum_is_far(float rstd, float s2)
{
    return rstd > 16777216.f || (rstd < 5.9604645e-8f && !(fabsf(s2) <= 3.4028235e38f));         // squares or products of small values vanish; of large ones overflow
}
// k: the terms as they came out.  Ordinary ones take a look at the smallest and the largest.
template <typename F, typename G> __device__ __forceinline__ bool terms_are_far(const GnParams &P, int ch, const Back &k, F mr, G means)
{
    float low = 3.4028235e38f, high = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float a, b;
        unpack2(k.e[j], a, b);
        low = fminf(low, fminf(fabsf(a), fabsf(b)));
        high = fmaxf(high, fmaxf(fabsf(a), fabsf(b)));
    }
    if (low >= 1.1754944e-38f && high <= 3.4028235e38f) return false;
    bool far = false;
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
        const int g = group_of(P, ch + j);
        const float rstd = mr(g).y, m = means(g).y, e = fabsf(rstd * (rstd * m));
        far |= (rstd > 16777216.f && e > 3.4028235e38f) || (rstd < 5.9604645e-8f && e < 1.1754944e-38f && m != 0.f);
    }
    return far;
}
// where a thread's values lie: the first of x, of dz and of dx, elements between two, how many
struct Run { int64_t x, xs, z, zs, o, os; int count; };
// what the functions need of the layer: mean and rstd of the sample's groups, channels of a group
struct Far { const void *x, *dz; void *out; const float *w, *b; const float2 *mr; int cg; float slope; };
__device__ __forceinline__ Far far_of(const GnParams &P, int64_t sample) { return Far{P.x, P.dz, P.out, P.w, P.b, P.mean_rstd + sample * P.groups, P.cg, P.slope}; }
// dt, and x in deviations from the mean; t as the forward pass forms it
template <bool XF, bool ZF, int ACT> __device__ __forceinline__ float far_slope(const Far &f, float2 mr, float w, float b, int64_t x, int64_t z, double &xhat)
{
    const float v = value_at<XF>(f.x, x), dz = value_at<ZF>(f.dz, z), t = fmaf(v - mr.x, mr.y * w, b);
    xhat = ((double)v - mr.x) * mr.y;
    float dt, same;
    unpack2(times_derivative<ACT, XF>(twice(dz), twice(t), f.slope), dt, same);
    return dt;
}
// Sums of dt and dt * xhat of the channels of `mask`, to where the thread's sums lie in shared memory.
template <bool XF, bool ZF, int ACT> __device__ __forceinline__ void far_sums(const Far &f, const Run &r, uint32_t mask, int ch, double *sa, double *sb)
{
    for (; mask; mask &= mask - 1) {
        const int j = __ffs(mask) - 1;
        const float2 mr = f.mr[(ch + j) / f.cg];
        const float w = f.w ? f.w[ch + j] : 1.f, b = f.b ? f.b[ch + j] : 0.f;
        double s = 0.0, t = 0.0;
#pragma unroll 1
        for (int i = 0; i < r.count; ++i) {
            double xhat;
            const double dt = far_slope<XF, ZF, ACT>(f, mr, w, b, r.x + i * r.xs + j, r.z + i * r.zs + j, xhat);
            s += dt;
            t = fma(dt, xhat, t);
        }
        sa[j] = s; sb[j] = t;
    }
}
// dx of all 8 channels; means: (mean(w dt), mean(w dt xhat)) of the groups from g0 on.  An element is read before it is written: dx may be x or dz.
template <bool XF, bool ZF, int ACT> __device__ __forceinline__ void far_apply(const Far &f, const Run &r, int ch, const float2 *means, int g0)
{
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
        const int g = (ch + j) / f.cg;
        const float2 mr = f.mr[g], m = means[g - g0];
        const float w = f.w ? f.w[ch + j] : 1.f, b = f.b ? f.b[ch + j] : 0.f;
#pragma unroll 1
        for (int i = 0; i < r.count; ++i) {
            double xhat;
            const double dt = far_slope<XF, ZF, ACT>(f, mr, w, b, r.x + i * r.xs + j, r.z + i * r.zs + j, xhat);
            const float o = (float)(mr.y * (w * dt - m.x - xhat * m.y));
            if (XF) ((float *)f.out)[r.o + i * r.os + j] = o; else ((bf16 *)f.out)[r.o + i * r.os + j] = f2bf(o);
        }
    }
}

// A thread's sums of d and d^2 about k (nk = -k) as fp64 sums about r
__device__ __forceinline__ void about(float nk, float s1, float s2, int n, double r, double &a, double &b)
{
    const double e = -(double)nk - r, m = (double)n;
    a = (double)s1 + m * e;
    b = (double)s2 + e * (2.0 * s1 + m * e);
}
// Whether the fp32 sum of a thread's squares may stand: finite, so that no square or shift left fp32's range; and, where eps does not hide it, well above the
// 256 halves of fp32's smallest step that squares may have lost.
__device__ __forceinline__ bool squares_hold(float s2, float eps) { return s2 <= 3.4028235e38f && (s2 >= 7.8886091e-31f || eps >= 7.8886091e-31f); }      // 2^-100
// The same sums about the group's first value, in fp64 from the values themselves, for the channels of `mask` where they may not: `count` voxels, `step`
// elements apart, the first at `at`; first: the sample's first voxel.  To where the thread's sums lie in shared memory.  The kernels reach it by calls
// that find their own places, as those for deviations far from 1 above.
template <bool XF> __device__ __forceinline__ void sums_again(const GnParams &P, uint32_t mask, int64_t at, int64_t step, int count, int64_t first, int ch, double *sa, double *sb)
{
    for (; mask; mask &= mask - 1) {
        const int j = __ffs(mask) - 1;
        const double r = value_at<XF>(P.x, first + group_of(P, ch + j) * P.cg);
        double s = 0.0, t = 0.0;
#pragma unroll 1
        for (int i = 0; i < count; ++i) {
            const double d = (double)value_at<XF>(P.x, at + i * step + j) - r;
            s += d;
            t = fma(d, d, t);
        }
        sa[j] = s; sb[j] = t;
    }
}
// 1 / sqrt(v): a step of Newton's method in fp64 from the fp32 value (2^-22 off before, 2^-43 after), the division and the root themselves - a microsecond
// together - only where fp32 has no such value
__device__ __forceinline__ double inverse_root(double v)
{
    if (!(v >= 1e-30 && v <= 1e30)) return 1.0 / sqrt(v);
    const double r = (double)rsqrtf((float)v);
    return r * (1.5 - 0.5 * v * r * r);
}
// from the sums about r of `1 / inv` values
__device__ __forceinline__ float2 mean_rstd_of(double s, double t, double r, double inv, float eps)
{
    const double mu = s * inv, var = t * inv - mu * mu;
    return make_float2((float)(r + mu), (float)inverse_root((var < 0.0 ? 0.0 : var) + (double)eps));
}

// Channel i of a line in shared memory: an empty place behind every two units, so that lanes with neighbouring units write to different banks.
__host__ __device__ constexpr int padded(int i) { return i + (i >> 4); }
// fp64 values of a line, and bytes of `ty` of them twice
__host__ __device__ constexpr int line_of(int uc) { return uc * 8 + (uc + 1) / 2; }
__host__ __device__ constexpr size_t lines_bytes(int ty, int uc) { return (size_t)ty * line_of(uc) * 2 * sizeof(double); }

// Sum over `ty` lines of uc units of 8 pairs of fp64 per thread, over the chunk's channels.  mend(sa, sb): a thread's last word on its own.
struct Totals {
    const double *sa, *sb;
    __device__ __forceinline__ double a(int i) const { return sa[padded(i)]; }
    __device__ __forceinline__ double b(int i) const { return sb[padded(i)]; }
};
template <typename M> __device__ __forceinline__ Totals sum_lines(int ty, int uc, int my_line, int my_unit, const double (&a)[8], const double (&b)[8], double *sm, M mend)
{
    const int cc = uc * 8, row = line_of(uc);
    double *sa = sm, *sb = sm + ty * row;
    if (my_line < ty) {
        const int at = my_line * row + padded(my_unit * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) { sa[at + j] = a[j]; sb[at + j] = b[j]; }
        mend(sa + at, sb + at);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * cc; i += GT) {
        double *s = i < cc ? sa + padded(i) : sb + padded(i - cc);
        double t = s[0];
#pragma unroll 8
        for (int l = 1; l < ty; ++l) t += s[l * row];
        s[0] = t;
    }
    __syncthreads();
    return Totals{sa, sb};
}

// For the groups g0 .. g1 in turn, several at a time: load(group, lane, lanes) -> sums of its values `lane`, lane + lanes, .. of `count`, their sum to
// done(group, s, t) in one lane.  Few groups of many values take several warps each.  Every thread takes part.
template <typename L, typename D> __device__ __forceinline__ void sum_groups(int g0, int g1, int count, L load, D done)
{
    __shared__ double2 red[GT / 32];
    int lanes = 1;
    while (lanes * 2 <= count && (lanes < 32 || (lanes * 2 <= GT && lanes * 2 * (g1 - g0 + 1) <= GT))) lanes *= 2;
    const int l = threadIdx.x % lanes, per = GT / lanes, wide = lanes < 32 ? lanes : 32;
    for (int g = g0; g <= g1; g += per) {                        // the same number of turns for every thread; one where lanes > 32
        const int mg = g + threadIdx.x / lanes;
        double s = 0.0, t = 0.0;
        if (mg <= g1) load(mg, l, lanes, s, t);
        for (int o = wide / 2; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            t += __shfl_xor_sync(0xffffffffu, t, o);
        }
        if (lanes > 32) {
            if (l % 32 == 0) red[threadIdx.x / 32] = make_double2(s, t);
            __syncthreads();
            if (l == 0)
                for (int w = 1; w < lanes / 32; ++w) { s += red[threadIdx.x / 32 + w].x; t += red[threadIdx.x / 32 + w].y; }
        }
        if (mg <= g1 && l == 0) done(mg, s, t);
    }
}

}  // namespace gn

// group_norm_small.cu.  The pass in the form in which a cluster holds what a group needs (forward, or backward with dz set; P.part takes [n][c] pairs of
// fp64 where dw or db is asked for); LAMP_ERR_UNSUPPORTED, and nothing launched, where it cannot hold it.
lamp_status_t gn_small(const gn::GnParams &P, bool xf, bool zf, bool back, cudaStream_t st);

}  // namespace lamp
