// Backward pass of the norms around a residual block (block_norm.cuh has the layout).  Per row, with th, yh the normalised
// t and y, and all means over the channels (mean(a), mean(b) only for LayerNorm):
//     a  = dh w_pre,        dt = dout + rstd_t (a - mean(a) - th mean(a th)),          dx = dt
//     b  = dt r g w_post,   dy = rstd_y (b - mean(b) - yh mean(b yh)),                 dlogit = dt r (yh w_post + b_post) g (1 - g)
// Means and deviations are computed again from the rows, which are read anyway.  Bound by memory: t, y, dout, dh read once, dx
// and dy written once (133 us with the finish kernel on 81,840 x 320, fp32 stream, gate per element, at a floor of 88).
// Parameter gradients are sums over voxels of four products per channel, P = dt g' yh, Q = dt g' (g' = the gate where it has
// a value per element, else 1), dh th and dh: each thread adds them up for its own channels over the rows it works on, a CTA
// joins its threads in a fixed order and leaves one row of 4 c partial sums in the workspace; block_norm_finish_kernel adds
// those in a fixed order (fp64) and forms  dw_post = r g P, db_post = r g Q, dr = g (w P + b Q), dg = r (w P + b Q).
#include "block_norm.cuh"

namespace lamp {

namespace {

using namespace bn;

struct BwdParams {
    const void *y, *t, *dout, *dh, *logits;
    void *dx, *dy, *dl;
    int64_t py, pt, pdo, pdh, pl, pdx, pdy, pdl;
    int64_t rows;
    int32_t parts, c, rms;
    float eps;
    const float *post_w, *post_b, *pre_w, *gate, *res;
    float *part;                     // [samples * parts][4][c] or NULL
};

// The running sums of a row group sit in shared memory, [sum][half][slot] float4 with slot = group * units + unit: 64 or
// more accumulators per thread would leave 8 warps per SM (measured on 81,840 x 320, fp32 stream, gate per element, this
// kernel alone: 265 us; in shared memory, with packed fp32 arithmetic, 129).
template <bool SF, bool BF, int TPR, int U, int MAXT, int MINB, bool LOGITS>
__global__ void __launch_bounds__(MAXT, MINB)
block_norm_bwd_kernel(const BwdParams P)
{
    using ptx::f32x2; using ptx::fma2; using ptx::add2; using ptx::mul2; using ptx::twice; using ptx::pack2; using ptx::unpack2;
    extern __shared__ __align__(16) float par[];
    __shared__ float red[2][32];
    const int threads = TPR ? TPR : blockDim.x;
    const int groups = TPR ? blockDim.x / TPR : 1, group = TPR ? threadIdx.x / TPR : 0, tt = TPR ? threadIdx.x % TPR : threadIdx.x;
    const int units = P.c / 8;
    const bool post = P.y != nullptr, pre = P.dh != nullptr, want = P.part != nullptr;
    const int64_t sample = blockIdx.x / P.parts, part = blockIdx.x - sample * P.parts;
    const int64_t base = sample * P.rows;
    pdl_launch_dependents();
    pdl_wait();
    for (int ch = threadIdx.x; ch < P.c; ch += blockDim.x) {
        const float rg = (P.res ? P.res[ch] : 1.f) * (P.gate ? P.gate[sample * P.c + ch] : 1.f);
        store_par(par, 0, units, ch, rg * (P.post_w ? P.post_w[ch] : 1.f));
        store_par(par, 1, units, ch, P.pre_w ? P.pre_w[ch] : 1.f);
        if (LOGITS) store_par(par, 2, units, ch, P.post_b ? rg * P.post_b[ch] : 0.f);
    }
    const float4 *par4 = reinterpret_cast<const float4 *>(par);
    float4 *sums = reinterpret_cast<float4 *>(par) + (LOGITS ? 6 : 4) * units;
    const int slots = groups * units;
    if (want)
        for (int i = threadIdx.x; i < 8 * slots; i += blockDim.x) sums[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    __syncthreads();
    // sums k and k + 1 of a unit: a += f1 f2, b += f1
    auto gather = [&](int k, int unit, const f32x2 (&f1)[4], const f32x2 (&f2)[4]) {
        ulonglong2 *p = reinterpret_cast<ulonglong2 *>(sums + k * 2 * slots + group * units + unit);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            ulonglong2 a = p[h * slots], b = p[(2 + h) * slots];
            a.x = fma2(f1[2 * h], f2[2 * h], a.x); a.y = fma2(f1[2 * h + 1], f2[2 * h + 1], a.y);
            b.x = add2(b.x, f1[2 * h]); b.y = add2(b.y, f1[2 * h + 1]);
            p[h * slots] = a; p[(2 + h) * slots] = b;
        }
    };
    const float inv_c = 1.f / (float)P.c;
    int turn = 0;
    const int64_t step = (int64_t)P.parts * groups;
    for (int64_t r0 = part * groups; r0 < P.rows; r0 += step) {
        const int64_t row = r0 + group, r = base + row;
        const bool active = row < P.rows;
        Raw<SF> rt[U], rdo[U];
        Raw<BF> ry[U], rdh[U], rl[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int ch = (u * threads + tt) * 8;
            const bool in = active && ch < P.c;
            rt[u] = in && pre ? load_raw<SF>(P.t, r * P.pt + ch) : zero_raw<SF>();
            ry[u] = in && post ? load_raw<BF>(P.y, r * P.py + ch) : zero_raw<BF>();
            rdh[u] = in && pre ? load_raw<BF>(P.dh, r * P.pdh + ch) : zero_raw<BF>();
            rdo[u] = in && P.dout ? load_raw<SF>(P.dout, r * P.pdo + ch) : zero_raw<SF>();
            if (LOGITS) rl[u] = in ? load_raw<BF>(P.logits, r * P.pl + ch) : zero_raw<BF>();
        }
        f32x2 th[U][4], yh[U][4], dt[U][4];
        float mt = 0.f, my = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) { to_pairs<SF>(rt[u], th[u]); to_pairs<BF>(ry[u], yh[u]); }
        if (!P.rms) {
            f32x2 st = 0, sy = 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) { st = add2(st, th[u][j]); sy = add2(sy, yh[u][j]); }
            mt = both(st); my = both(sy);
            row_sum2<TPR>(mt, my, red, turn);
            mt *= inv_c; my *= inv_c;
        }
        f32x2 qt2 = 0, qy2 = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if ((u * threads + tt) * 8 >= P.c) continue;               // stays zero
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!P.rms) { th[u][j] = add2(th[u][j], twice(-mt)); yh[u][j] = add2(yh[u][j], twice(-my)); }
                qt2 = fma2(th[u][j], th[u][j], qt2);
                qy2 = fma2(yh[u][j], yh[u][j], qy2);
            }
        }
        float qt = both(qt2), qy = both(qy2);
        row_sum2<TPR>(qt, qy, red, turn);
        // a row past the end takes part with zeros only, whatever eps is
        const float rst = active ? rsqrtf(qt * inv_c + P.eps) : 0.f, rsy = active ? rsqrtf(qy * inv_c + P.eps) : 0.f;
        if (pre) {
            f32x2 s1 = 0, s2 = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int unit = u * threads + tt;
                f32x2 w[4] = {0, 0, 0, 0}, d[4];
                to_pairs<BF>(rdh[u], d);
                if (unit < units) load_par(par4, 1, units, unit, w);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    th[u][j] = mul2(th[u][j], twice(rst));
                    dt[u][j] = mul2(d[j], w[j]);
                    s1 = add2(s1, dt[u][j]);
                    s2 = fma2(dt[u][j], th[u][j], s2);
                }
                if (want && active && unit < units) gather(2, unit, d, th[u]);
            }
            float m1 = both(s1), m2 = both(s2);
            row_sum2<TPR>(m1, m2, red, turn);
            m1 = P.rms ? 0.f : m1 * inv_c; m2 *= inv_c;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                f32x2 d[4];
                to_pairs<SF>(rdo[u], d);
#pragma unroll
                for (int j = 0; j < 4; ++j) dt[u][j] = fma2(twice(rst), fma2(th[u][j], twice(-m2), add2(dt[u][j], twice(-m1))), d[j]);
            }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) to_pairs<SF>(rdo[u], dt[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = u * threads + tt;
            if (active && unit < units) store_pairs<SF>(P.dx, r * P.pdx + unit * 8, dt[u]);
        }
        if (post) {
            f32x2 s1 = 0, s2 = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int unit = u * threads + tt;
                const bool in = active && unit < units;
                f32x2 w[4] = {0, 0, 0, 0};
                if (in) load_par(par4, 0, units, unit, w);
#pragma unroll
                for (int j = 0; j < 4; ++j) yh[u][j] = mul2(yh[u][j], twice(rsy));
                if (LOGITS) {
                    f32x2 g[4], wb[4] = {0, 0, 0, 0};
                    to_pairs<BF>(rl[u], g);
                    if (in) load_par(par4, 2, units, unit, wb);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float a, b, ga, gb, sa, sb;
                        unpack2(g[j], a, b);
                        sigmoid_slope<BF>(a, ga, sa);
                        sigmoid_slope<BF>(b, gb, sb);
                        g[j] = pack2(__float_as_uint(ga), __float_as_uint(gb));
                        // dlogit = dt r N(y) g (1 - g)
                        wb[j] = mul2(mul2(dt[u][j], fma2(yh[u][j], w[j], wb[j])), pack2(__float_as_uint(sa), __float_as_uint(sb)));
                        dt[u][j] = mul2(dt[u][j], g[j]);
                    }
                    if (in) store_pairs<BF>(P.dl, r * P.pdl + unit * 8, wb);
                }
                if (want && in) gather(0, unit, dt[u], yh[u]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    dt[u][j] = mul2(dt[u][j], w[j]);
                    s1 = add2(s1, dt[u][j]);
                    s2 = fma2(dt[u][j], yh[u][j], s2);
                }
            }
            float m1 = both(s1), m2 = both(s2);
            row_sum2<TPR>(m1, m2, red, turn);
            m1 = P.rms ? 0.f : m1 * inv_c; m2 *= inv_c;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int unit = u * threads + tt;
#pragma unroll
                for (int j = 0; j < 4; ++j) dt[u][j] = mul2(twice(rsy), fma2(yh[u][j], twice(-m2), add2(dt[u][j], twice(-m1))));
                if (active && unit < units) store_pairs<BF>(P.dy, r * P.pdy + unit * 8, dt[u]);
            }
        }
    }
    if (!want) return;
    __syncthreads();
    // the groups' sums, added in group order
    float4 *dst = reinterpret_cast<float4 *>(P.part + (int64_t)blockIdx.x * 4 * P.c);
    for (int i = threadIdx.x; i < 8 * units; i += blockDim.x) {
        const int kh = i / units, unit = i - kh * units;
        float4 s = sums[kh * slots + unit];
        for (int g = 1; g < groups; ++g) {
            const float4 v = sums[kh * slots + g * units + unit];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        dst[(kh >> 1) * (P.c / 4) + unit * 2 + (kh & 1)] = s;
    }
}

// 32 channels per CTA (one per lane); its warps share the partial rows of a sample, or, with as many samples as warps or more,
// take whole samples.
struct FinishParams {
    const float *part;
    int32_t parts, c;
    int64_t samples;
    const float *post_w, *post_b, *gate, *res;
    float *dpost_w, *dpost_b, *dpre_w, *dpre_b, *dgate, *dres;
};

constexpr int FIN_WARPS = 32;
__global__ void __launch_bounds__(FIN_WARPS * 32)
block_norm_finish_kernel(const FinishParams P)
{
    __shared__ double sm[FIN_WARPS][4][32];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ch = blockIdx.x * 32 + lane;
    const bool in = ch < P.c;
    const double w = in && P.post_w ? P.post_w[ch] : 1.0, b = in && P.post_b ? P.post_b[ch] : 0.0, r = in && P.res ? P.res[ch] : 1.0;
    const bool whole = P.samples >= FIN_WARPS;                      // a warp takes whole samples
    double tot[5] = {0, 0, 0, 0, 0};                                // dw_post, db_post, dw_pre, db_pre, dr
    for (int64_t s = whole ? warp : 0; s < P.samples; s += whole ? FIN_WARPS : 1) {
        double v[4] = {0, 0, 0, 0};
        if (in) {
            const int step = whole ? 1 : FIN_WARPS;
#pragma unroll 4
            for (int p = whole ? 0 : warp; p < P.parts; p += step) {
                const float *src = P.part + (s * P.parts + p) * 4 * P.c + ch;
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] += (double)src[(int64_t)k * P.c];
            }
        }
        const double g = in && P.gate ? P.gate[s * P.c + ch] : 1.0;
        if (!whole && P.gate) {                                     // the sample's sums over all warps, in warp order
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 4; ++k) sm[warp][k][lane] = v[k];
            __syncthreads();
            if (warp < 4) {                                         // one warp per sum
                double a = 0;
                for (int i = 0; i < FIN_WARPS; ++i) a += sm[i][warp][lane];
                sm[0][warp][lane] = a;
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = warp == 0 ? sm[0][k][lane] : 0.0;
        }
        if (P.dgate && in && (whole || warp == 0)) P.dgate[s * P.c + ch] = (float)(r * (w * v[0] + b * v[1]));
        tot[0] += r * g * v[0]; tot[1] += r * g * v[1]; tot[2] += v[2]; tot[3] += v[3]; tot[4] += g * (w * v[0] + b * v[1]);
    }
    float *outs[5] = {P.dpost_w, P.dpost_b, P.dpre_w, P.dpre_b, P.dres};
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) sm[warp][k][lane] = tot[k];
    __syncthreads();
    if (warp < 4 && in && outs[warp]) {
        double v = 0;
        for (int i = 0; i < FIN_WARPS; ++i) v += sm[i][warp][lane];
        outs[warp][ch] = (float)v;
    }
    __syncthreads();
    sm[warp][0][lane] = tot[4];
    __syncthreads();
    if (warp == 0 && in && P.dres) {
        double v = 0;
        for (int i = 0; i < FIN_WARPS; ++i) v += sm[i][0][lane];
        P.dres[ch] = (float)v;
    }
}

int64_t parts_of(const lamp_tensor_t *t, const lamp_block_norm_t *p, int64_t *samples)
{
    const Shape sh = shape_of(t->c);
    *samples = p->gate ? t->n : 1;
    const int64_t rows = voxels(t) / (*samples > 0 ? *samples : 1), need = (rows + sh.rows_per_cta - 1) / sh.rows_per_cta;
    // as many CTAs as are resident at once: 80 registers with one unit per thread (three CTAs of 256 threads: 99 us against 110
    // with two on 120,000 x 256 bf16), 128 with two
    int64_t room = (int64_t)sm_count() * (sh.threads <= 256 ? (sh.u == 1 ? 768 : 512) / sh.threads : 1) / (*samples > 0 ? *samples : 1);
    if (room < 1) room = 1;
    return need < room ? need : room;
}

template <bool SF, bool BF, int TPR, int U, int MAXT, int MINB>
lamp_status_t launch(const BwdParams &P, int64_t samples, const Shape &sh, cudaStream_t st)
{
    const int groups = TPR ? sh.threads / TPR : 1;
    const int smem = P.c * (P.logits ? 12 : 8) + (P.part ? groups * P.c * 16 : 0);
    auto kernel = P.logits ? block_norm_bwd_kernel<SF, BF, TPR, U, MAXT, MINB, true> : block_norm_bwd_kernel<SF, BF, TPR, U, MAXT, MINB, false>;
    if (smem > 32 * 1024) {                                  // static shared memory counts too: well below the 48 KB default
        static SmemAttrOnce attr[2];
        const lamp_status_t s = attr[P.logits ? 1 : 0].ensure(kernel, MAX_C * 28);
        if (s != LAMP_OK) return s;
    }
    return launch_pdl(samples * P.parts <= 8 * (int64_t)sm_count(), kernel, dim3((unsigned)(samples * P.parts)), dim3(sh.threads), (size_t)smem, st, P);
}

template <bool SF, bool BF>
lamp_status_t dispatch(const BwdParams &P, int64_t samples, const Shape &sh, cudaStream_t st)
{
    if (sh.tpr == 4) return launch<SF, BF, 4, 1, 256, 3>(P, samples, sh, st);
    if (sh.tpr == 8) return launch<SF, BF, 8, 1, 256, 3>(P, samples, sh, st);
    if (sh.tpr == 16) return launch<SF, BF, 16, 1, 256, 3>(P, samples, sh, st);
    if (sh.tpr == 32 && sh.u == 1) return launch<SF, BF, 32, 1, 256, 3>(P, samples, sh, st);
    if (sh.tpr == 32) return launch<SF, BF, 32, 2, 256, 2>(P, samples, sh, st);
    return launch<SF, BF, 0, 2, 512, 1>(P, samples, sh, st);
}

}  // namespace

}  // namespace lamp

using namespace lamp;

extern "C" size_t lamp_block_norm_bwd_workspace_bytes(const lamp_tensor_t *t, const lamp_block_norm_t *p)
{
    if (!t || check_norm_tensor(t, t) != LAMP_OK || check_norm_params(p, t) != LAMP_OK) return 0;
    int64_t samples;
    const int64_t parts = parts_of(t, p, &samples);
    return (size_t)(samples * parts) * 4 * t->c * sizeof(float);
}

extern "C" lamp_status_t lamp_block_norm_bwd(const lamp_block_norm_t *p, const lamp_tensor_t *y, const lamp_tensor_t *t, const lamp_tensor_t *dout,
                                             const lamp_tensor_t *dh, lamp_tensor_t *dx, lamp_tensor_t *dy, lamp_tensor_t *dgate_logits,
                                             const lamp_block_norm_grads_t *grads, void *ws, size_t ws_bytes, void *cuda_stream)
{
    lamp_status_t s;
    if (!t || (s = check_norm_tensor(t, t)) != LAMP_OK) return t ? s : LAMP_ERR_INVALID_ARG;
    if ((s = check_norm_params(p, t)) != LAMP_OK) return s;
    if ((!dout && !dh) || !dx || (y == nullptr) != (dy == nullptr)) return LAMP_ERR_INVALID_ARG;
    if ((p->gate_logits == nullptr) != (dgate_logits == nullptr) || (!y && (p->gate_logits || p->gate || p->res_scale))) return LAMP_ERR_INVALID_ARG;
    const lamp_tensor_t *stream[2] = {dout, dx}, *branch[5] = {y, dh, dy, p->gate_logits, dgate_logits};
    for (const lamp_tensor_t *v : stream) {
        if (!v) continue;
        if ((s = check_norm_tensor(v, t)) != LAMP_OK) return s;
        if (v->dtype != t->dtype) return LAMP_ERR_UNSUPPORTED;
    }
    int bf = -1;
    for (const lamp_tensor_t *v : branch) {
        if (!v) continue;
        if ((s = check_norm_tensor(v, t)) != LAMP_OK) return s;
        if (bf >= 0 && v->dtype != bf) return LAMP_ERR_UNSUPPORTED;
        bf = v->dtype;
    }
    if (bf < 0) return LAMP_ERR_INVALID_ARG;                           // neither a post-norm nor a pre-norm
    if (t->dtype == LAMP_BF16 && bf == LAMP_F32) return LAMP_ERR_UNSUPPORTED;
    const lamp_block_norm_grads_t none = {}, *g = grads ? grads : &none;
    const bool want = g->post_w || g->post_b || g->pre_w || g->pre_b || g->gate || g->res_scale;
    if (((uintptr_t)g->post_w | (uintptr_t)g->post_b | (uintptr_t)g->pre_w | (uintptr_t)g->pre_b | (uintptr_t)g->gate | (uintptr_t)g->res_scale) & 3)
        return LAMP_ERR_INVALID_ARG;
    if (g->gate && !p->gate) return LAMP_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    int64_t samples;
    const int64_t parts = parts_of(t, p, &samples);
    if (voxels(t) == 0) {                                              // empty sums
        float *z[5] = {g->post_w, g->post_b, g->pre_w, g->pre_b, g->res_scale};
        for (float *q : z) if (q) LAMP_CUDA_OK(cudaMemsetAsync(q, 0, (size_t)t->c * 4, st));
        if (g->gate && t->n) LAMP_CUDA_OK(cudaMemsetAsync(g->gate, 0, (size_t)t->n * t->c * 4, st));
        return LAMP_OK;
    }
    if (samples * parts > 2147483647ll) return LAMP_ERR_UNSUPPORTED;
    if (want && (!ws || ((uintptr_t)ws & 15) || ws_bytes < (size_t)(samples * parts) * 4 * t->c * sizeof(float))) return LAMP_ERR_WORKSPACE;
    BwdParams P = {};
    auto put = [](const lamp_tensor_t *v, auto &ptr, int64_t &pitch) { if (v) { const TView w = make_view(v); ptr = w.p; pitch = w.pitch; } };
    put(y, P.y, P.py); put(t, P.t, P.pt); put(dout, P.dout, P.pdo); put(dh, P.dh, P.pdh); put(p->gate_logits, P.logits, P.pl);
    put(dx, P.dx, P.pdx); put(dy, P.dy, P.pdy); put(dgate_logits, P.dl, P.pdl);
    P.rows = voxels(t) / samples; P.parts = (int32_t)parts; P.c = t->c; P.rms = p->rms; P.eps = p->eps;
    P.post_w = p->post_w; P.post_b = p->post_b; P.pre_w = p->pre_w; P.gate = p->gate; P.res = p->res_scale;
    P.part = want ? (float *)ws : nullptr;
    const Shape sh = shape_of(P.c);
    if (t->dtype == LAMP_BF16) s = dispatch<false, false>(P, samples, sh, st);
    else s = bf == LAMP_F32 ? dispatch<true, true>(P, samples, sh, st) : dispatch<true, false>(P, samples, sh, st);
    if (s != LAMP_OK || !want) return s;
    FinishParams F = {(const float *)ws, (int32_t)parts, P.c, samples, P.post_w, P.post_b, P.gate, P.res, g->post_w, g->post_b, g->pre_w, g->pre_b, g->gate, g->res_scale};
    return launch_pdl(true, block_norm_finish_kernel, dim3((unsigned)((P.c + 31) / 32)), dim3(FIN_WARPS * 32), 0, st, F);
}
