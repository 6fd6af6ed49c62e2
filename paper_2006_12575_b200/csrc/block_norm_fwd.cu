// Forward pass of the norms around a residual block:  t = x + r g N_post(y),  h = N_pre(t)  (block_norm.cuh has the layout).
// Bound by memory: y and x are read once, t and h (bf16, fp32 or e4m3 with its scales) written once; everything between
// stays in registers.  The factors r g w and r g b of the post-norm (g per sample) and w, b of the pre-norm are combined once per
// CTA and kept in shared memory; a CTA stays within one sample.
#include "block_norm.cuh"
#include "fp8.cuh"

namespace lamp {

namespace {

using namespace bn;

struct FwdParams {
    const void *y, *x, *logits;
    void *out, *h;
    int64_t py, px, pl, po, ph;
    int64_t rows;                    // rows of one sample (all rows where the gate does not depend on the sample)
    int32_t parts;                   // CTAs per sample
    int32_t c, rms;
    float eps;
    const float *post_w, *post_b, *pre_w, *pre_b, *gate, *res;
    uint8_t *hq;
    int64_t hq_pitch;
    float *hs;
    int64_t hs_pitch;
};

template <bool SF, bool BF, int TPR, int U, int MAXT, int MINB, bool LOGITS>
__global__ void __launch_bounds__(MAXT, MINB)
block_norm_fwd_kernel(const FwdParams P)
{
    using ptx::f32x2; using ptx::fma2; using ptx::add2; using ptx::mul2; using ptx::twice; using ptx::pack2; using ptx::unpack2;
    extern __shared__ __align__(16) float par[];
    __shared__ float red[2][32];
    const int threads = TPR ? TPR : blockDim.x;                    // per row
    const int groups = TPR ? blockDim.x / TPR : 1, group = TPR ? threadIdx.x / TPR : 0, tt = TPR ? threadIdx.x % TPR : threadIdx.x;
    const int units = P.c / 8;
    const bool post = P.y != nullptr, pre = P.h != nullptr || P.hq != nullptr;
    const int64_t sample = blockIdx.x / P.parts, part = blockIdx.x - sample * P.parts;
    const int64_t base = sample * P.rows;
    pdl_launch_dependents();
    pdl_wait();
    for (int ch = threadIdx.x; ch < P.c; ch += blockDim.x) {
        const float rg = (P.res ? P.res[ch] : 1.f) * (P.gate ? P.gate[sample * P.c + ch] : 1.f);
        store_par(par, 0, units, ch, post ? rg * (P.post_w ? P.post_w[ch] : 1.f) : 0.f);
        store_par(par, 1, units, ch, post && P.post_b ? rg * P.post_b[ch] : 0.f);
        store_par(par, 2, units, ch, P.pre_w ? P.pre_w[ch] : 1.f);
        store_par(par, 3, units, ch, P.pre_b ? P.pre_b[ch] : 0.f);
    }
    __syncthreads();
    const float4 *par4 = reinterpret_cast<const float4 *>(par);
    const float inv_c = 1.f / (float)P.c;
    int turn = 0;

    Raw<BF> ry[U], rl[U];
    Raw<SF> rx[U];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int ch = (u * threads + tt) * 8;
            const bool in = row < P.rows && ch < P.c;
            rx[u] = in ? load_raw<SF>(P.x, (base + row) * P.px + ch) : zero_raw<SF>();
            if (post) ry[u] = in ? load_raw<BF>(P.y, (base + row) * P.py + ch) : zero_raw<BF>();
            if (LOGITS) rl[u] = in ? load_raw<BF>(P.logits, (base + row) * P.pl + ch) : zero_raw<BF>();
        }
    };
    // centres v (not for rms) and returns 1 / deviation; channels behind c stay zero
    auto centre = [&](f32x2 (&v)[U][4]) {
        float mean = 0.f;
        if (!P.rms) {
            f32x2 s = 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) s = add2(s, v[u][j]);
            mean = row_sum<TPR>(both(s), red, turn) * inv_c;
        }
        f32x2 q = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if ((u * threads + tt) * 8 >= P.c) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!P.rms) v[u][j] = add2(v[u][j], twice(-mean));
                q = fma2(v[u][j], v[u][j], q);
            }
        }
        return rsqrtf(row_sum<TPR>(both(q), red, turn) * inv_c + P.eps);
    };
    const int64_t step = (int64_t)P.parts * groups;
    int64_t r0 = part * groups;
    if (r0 < P.rows) fetch(r0 + group);
    for (; r0 < P.rows; r0 += step) {                              // the same number of turns for every thread of the CTA
        const int64_t row = r0 + group;
        const bool active = row < P.rows;
        f32x2 t[U][4], v[U][4], lg[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            to_pairs<SF>(rx[u], t[u]);
            if (post) to_pairs<BF>(ry[u], v[u]);
            if (LOGITS) to_pairs<BF>(rl[u], lg[u]);
        }
        if (r0 + step < P.rows) fetch(row + step);                 // in flight while this row is worked on
        if (post) {
            const float rstd = centre(v);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int unit = u * threads + tt;
                if (unit >= units) continue;
                f32x2 w[4], b[4];
                uint32_t stored[4];
                load_par(par4, 0, units, unit, w);
                load_par(par4, 1, units, unit, b);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    f32x2 branch = fma2(mul2(v[u][j], twice(rstd)), w[j], b[j]);
                    if (LOGITS) {
                        float p, q;
                        unpack2(lg[u][j], p, q);
                        branch = mul2(branch, pack2(__float_as_uint(sigmoid<BF>(p)), __float_as_uint(sigmoid<BF>(q))));
                    }
                    t[u][j] = add2(t[u][j], branch);
                    if constexpr (!SF) {                           // t as stored
                        float p, q;
                        unpack2(t[u][j], p, q);
                        const __nv_bfloat162 h = __floats2bfloat162_rn(p, q);
                        const uint32_t bits = *reinterpret_cast<const uint32_t *>(&h);
                        stored[j] = bits;
                        t[u][j] = pack2(bits << 16, bits & 0xFFFF0000u);
                    }
                }
                if (!active) continue;
                if constexpr (SF) store_pairs<SF>(P.out, (base + row) * P.po + unit * 8, t[u]);
                else *reinterpret_cast<uint4 *>((bf16 *)P.out + (base + row) * P.po + unit * 8) = make_uint4(stored[0], stored[1], stored[2], stored[3]);
            }
        }
        if (pre) {
            const float rstd = centre(t);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int unit = u * threads + tt;
                const bool in = unit < units;
                if (in) {
                    f32x2 w[4], b[4];
                    load_par(par4, 2, units, unit, w);
                    load_par(par4, 3, units, unit, b);
#pragma unroll
                    for (int j = 0; j < 4; ++j) t[u][j] = fma2(mul2(t[u][j], twice(rstd)), w[j], b[j]);
                    if (P.h && active) store_pairs<BF>(P.h, (base + row) * P.ph + unit * 8, t[u]);
                }
                if (P.hq) {                                        // 16 threads hold one block of 128 channels
                    float f[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) unpack2(t[u][j], f[2 * j], f[2 * j + 1]);
                    if (!in) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] = 0.f;
                    }
                    float m;
                    const uint2 codes = encode_block<(TPR == 0 || TPR > 16 ? 16 : TPR)>(f, m);
                    if (in && active) {
                        *reinterpret_cast<uint2 *>(P.hq + (base + row) * P.hq_pitch + unit * 8) = codes;
                        if ((unit & 15) == 0) P.hs[(unit >> 4) * P.hs_pitch + base + row] = __fmul_rn(m, 1.0f / 448.0f);
                    }
                }
            }
        }
    }
}

// CTAs of 256 threads per SM that a kernel is compiled for: the grid is that many per SM, so that all are resident at once (four
// per SM where three fit cost a second, mostly empty wave: 120 us against 114 on 131,072 x 512).  Three mean 80 registers;
// with two units per thread and fp32 or gate rows in flight as well they would spill.
__host__ __device__ constexpr int fwd_ctas(bool wide_rows, int u) { return wide_rows && u == 2 ? 2 : 3; }

template <bool SF, bool BF, int TPR, int U, int MAXT>
lamp_status_t launch(const FwdParams &P, int64_t samples, const Shape &sh, cudaStream_t st)
{
    const int smem = P.c * 16;
    auto kernel = P.logits ? block_norm_fwd_kernel<SF, BF, TPR, U, MAXT, MAXT == 256 ? fwd_ctas(true, U) : 1, true>
                           : block_norm_fwd_kernel<SF, BF, TPR, U, MAXT, MAXT == 256 ? fwd_ctas(SF, U) : 1, false>;
    if (smem > 32 * 1024) {                                  // static shared memory counts too: well below the 48 KB default
        static SmemAttrOnce attr[2];
        const lamp_status_t s = attr[P.logits ? 1 : 0].ensure(kernel, MAX_C * 16);
        if (s != LAMP_OK) return s;
    }
    return launch_pdl(samples * P.parts <= 8 * (int64_t)sm_count(), kernel, dim3((unsigned)(samples * P.parts)), dim3(sh.threads), (size_t)smem, st, P);
}

template <bool SF, bool BF>
lamp_status_t dispatch(const FwdParams &P, int64_t samples, const Shape &sh, cudaStream_t st)
{
    if (sh.tpr == 4) return launch<SF, BF, 4, 1, 256>(P, samples, sh, st);
    if (sh.tpr == 8) return launch<SF, BF, 8, 1, 256>(P, samples, sh, st);
    if (sh.tpr == 16) return launch<SF, BF, 16, 1, 256>(P, samples, sh, st);
    if (sh.tpr == 32 && sh.u == 1) return launch<SF, BF, 32, 1, 256>(P, samples, sh, st);
    if (sh.tpr == 32) return launch<SF, BF, 32, 2, 256>(P, samples, sh, st);
    return sh.threads <= 256 ? launch<SF, BF, 0, 2, 256>(P, samples, sh, st) : launch<SF, BF, 0, 2, 512>(P, samples, sh, st);
}

}  // namespace

lamp_status_t check_norm_tensor(const lamp_tensor_t *t, const lamp_tensor_t *like)
{
    lamp_status_t s = check_view(t, false);
    if (s != LAMP_OK) return s;
    if ((t->c & 7) || (t->c_pitch & 7) || (t->c_offset & 7) || t->c > bn::MAX_C) return LAMP_ERR_UNSUPPORTED;
    if (t->n != like->n || t->d != like->d || t->h != like->h || t->w != like->w || t->c != like->c) return LAMP_ERR_INVALID_ARG;
    return LAMP_OK;
}

lamp_status_t check_norm_params(const lamp_block_norm_t *p, const lamp_tensor_t *like)
{
    if (!p || (p->rms != 0 && p->rms != 1) || !(p->eps >= 0.f) || (p->gate && p->gate_logits)) return LAMP_ERR_INVALID_ARG;
    if (((uintptr_t)p->post_w | (uintptr_t)p->post_b | (uintptr_t)p->pre_w | (uintptr_t)p->pre_b | (uintptr_t)p->gate | (uintptr_t)p->res_scale) & 3)
        return LAMP_ERR_INVALID_ARG;
    return p->gate_logits ? check_norm_tensor(p->gate_logits, like) : LAMP_OK;
}

}  // namespace lamp

using namespace lamp;

extern "C" lamp_status_t lamp_block_norm_fwd(const lamp_block_norm_t *p, const lamp_tensor_t *y, const lamp_tensor_t *x, lamp_tensor_t *out,
                                             lamp_tensor_t *h, const lamp_fp8_operand_t *h_fp8, void *cuda_stream)
{
    lamp_status_t s;
    if (!x || (s = check_norm_tensor(x, x)) != LAMP_OK) return x ? s : LAMP_ERR_INVALID_ARG;
    if ((s = check_norm_params(p, x)) != LAMP_OK) return s;
    if ((y == nullptr) != (out == nullptr) || (!y && !h && !h_fp8)) return LAMP_ERR_INVALID_ARG;
    if (!y && (p->gate_logits || p->gate || p->res_scale)) return LAMP_ERR_INVALID_ARG;
    const lamp_tensor_t *branch[3] = {y, h, p->gate_logits};
    int bf = -1;                                                       // type of the branch tensors: one for all
    for (const lamp_tensor_t *t : branch) {
        if (!t) continue;
        if ((s = check_norm_tensor(t, x)) != LAMP_OK) return s;
        if (bf >= 0 && t->dtype != bf) return LAMP_ERR_UNSUPPORTED;
        bf = t->dtype;
    }
    if (bf < 0) bf = x->dtype;
    if (out && (s = check_norm_tensor(out, x)) != LAMP_OK) return s;
    if (out && out->dtype != x->dtype) return LAMP_ERR_UNSUPPORTED;
    if (x->dtype == LAMP_BF16 && bf == LAMP_F32) return LAMP_ERR_UNSUPPORTED;
    const int64_t rows = voxels(x);
    if (h_fp8) {
        if ((s = check_fp8_operand(h_fp8)) != LAMP_OK) return s;
        if (h_fp8->rows != rows || h_fp8->k != x->c || h_fp8->tile_scale) return LAMP_ERR_INVALID_ARG;
    }
    if (rows == 0) return LAMP_OK;
    FwdParams P = {};
    const TView vx = make_view(x);
    P.x = vx.p; P.px = vx.pitch;
    if (y) {
        const TView vy = make_view(y), vo = make_view(out);
        P.y = vy.p; P.py = vy.pitch; P.out = vo.p; P.po = vo.pitch;
    }
    if (p->gate_logits) { const TView v = make_view(p->gate_logits); P.logits = v.p; P.pl = v.pitch; }
    if (h) { const TView v = make_view(h); P.h = v.p; P.ph = v.pitch; }
    if (h_fp8) { P.hq = (uint8_t *)h_fp8->q; P.hq_pitch = h_fp8->q_pitch; P.hs = h_fp8->scale; P.hs_pitch = h_fp8->scale_pitch; }
    P.c = x->c; P.rms = p->rms; P.eps = p->eps;
    P.post_w = p->post_w; P.post_b = p->post_b; P.pre_w = p->pre_w; P.pre_b = p->pre_b; P.gate = p->gate; P.res = p->res_scale;
    const int64_t samples = p->gate ? x->n : 1;
    P.rows = rows / samples;
    const Shape sh = shape_of(P.c);
    const int64_t need = (P.rows + sh.rows_per_cta - 1) / sh.rows_per_cta;
    const int ctas = fwd_ctas(p->gate_logits || x->dtype == LAMP_F32, sh.u);
    int64_t room = (int64_t)sm_count() * (sh.threads <= 256 ? ctas * 256 / sh.threads : 1) / samples;
    if (room < 1) room = 1;
    P.parts = (int32_t)(need < room ? need : room);
    if (samples * P.parts > 2147483647ll) return LAMP_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (x->dtype == LAMP_BF16) return dispatch<false, false>(P, samples, sh, st);
    return bf == LAMP_F32 ? dispatch<true, true>(P, samples, sh, st) : dispatch<true, false>(P, samples, sh, st);
}
