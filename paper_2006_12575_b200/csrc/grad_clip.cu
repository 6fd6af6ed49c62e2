// Global norm of the gradients of many tensors, and clipping by it.
//
// Bound by memory: the norm reads every gradient once, the scaling reads and writes it.  The tensors' table travels in the
// kernel's parameters (a captured graph keeps it), so no copy to the device precedes a call.  The elements are cut into pieces of
// 32 KB, laid from a 128-byte boundary of their tensor; the CTAs take them in turn, the scaling backwards, so that it
// starts with what the norm left in L2.
// Sums: 8 squares in fp32 where that stays well inside its range, otherwise the 8 again in fp64; fp64 beyond, per thread, then over the
// CTA in a fixed order, one partial sum per CTA.  Every CTA of the scaling adds all of them in the same order: no counter, no atomic, nothing
// that has to be zero beforehand.
#include "block_norm.cuh"

namespace lamp {

namespace {

using namespace bn;

constexpr int CT = 256, UNITS = 8;              // threads, 16-byte units of a piece per thread: neighbouring lanes take neighbouring units
// Elements of a piece that T threads take: a CTA's 32 KB, or a warp's 4 KB where all of the gradients are few
template <int T> __host__ __device__ constexpr int piece_of(bool f32) { return T * UNITS * (f32 ? 4 : 8); }
constexpr int CTAS = 4;                       // per SM, all of them resident

struct Entry {
    const void *g;
    void *out;
    int64_t n;
    int64_t f32;
};
// Every line of the parameters that a kernel touches is a miss at first, 0.5 us each in turn: the search runs over an array of its own, and where
// the pieces are few a piece has its tensor written beside it.
template <int N> struct Table {
    int32_t count, pieces;
    int32_t first[N];                         // pieces of the tensors in front of it
    Entry e[N];
};
constexpr int SMALL = 110, LARGE = 900;       // parameters of 4 KB and of just under 32 KB
constexpr int CLUSTER = 8, FEW = 2 * CLUSTER * (CT / 32);          // pieces of a warp each: two per warp of a cluster
struct FewTable {
    int32_t pieces;
    uint8_t owner[FEW], index[FEW];           // of each piece: its tensor, its number there
    Entry e[SMALL];
};
static_assert(sizeof(Table<LARGE>) + 64 <= 32764 && sizeof(Table<SMALL>) <= 4040 && sizeof(FewTable) <= 4040 && FEW <= 255, "kernel parameters");

// elements in front of the first 128-byte boundary: a warp's 512 bytes are then whole lines
__host__ __device__ __forceinline__ int64_t head_of(const void *p, int64_t n, bool f32)
{
    const int64_t h = (int64_t)((128 - ((uintptr_t)p & 127)) & 127) / (f32 ? 4 : 2);
    return h < n ? h : n;
}
template <int T> __host__ __forceinline__ int64_t pieces_of(const lamp_grad_t &t)
{
    if (t.n == 0) return 0;
    const bool f32 = t.dtype == LAMP_F32;
    const int64_t body = t.n - head_of(t.g, t.n, f32), piece = piece_of<T>(f32);
    return body == 0 ? 1 : (body + piece - 1) / piece;
}

// Piece `index` of W threads of a tensor: f(entry, first element of its body, its end, elements of the head)
template <int W, typename F> __device__ __forceinline__ void piece(const Entry &e, int index, F f)
{
    const int64_t h = head_of(e.g, e.n, e.f32), b0 = h + (int64_t)index * piece_of<W>(e.f32), b1 = b0 + piece_of<W>(e.f32);
    f(e, b0, b1 < e.n ? b1 : e.n, index == 0 ? h : 0);
}

// Where each tensor's pieces begin, in shared memory: all of it in one access per thread.  (A search in the parameters themselves misses at every
// step: 366 tensors of 15,000 took 37 us.)  Needs nothing of the launch before, so it comes ahead of the wait for that.
template <int N> __device__ __forceinline__ void stage_first(const Table<N> &T, int *first)
{
    const int *p = T.first;
    asm volatile("" : "+l"(p));                  // as memory, which lanes read side by side, not as constants, which they read one by one
    for (int i = threadIdx.x; i < T.count; i += CT) first[i] = p[i];
    __syncthreads();
}
// The pieces `me`, me + step, .. of the tensors, forwards or BACK
template <int W, bool BACK, int N, typename F>
__device__ __forceinline__ void for_pieces(const Table<N> &T, const int *first, int me, int step, F f)
{
    if (me >= T.pieces) return;
    const int turns = (T.pieces - me + step - 1) / step;
    int p = me + (BACK ? turns - 1 : 0) * step;
    int lo = 0, hi = T.count - 1;
    for (int t = 0; t < turns; ++t, p += BACK ? -step : step) {
        while (lo < hi) {                     // the entry of piece p: the last that begins at it or before it
            const int mid = (lo + hi + 1) / 2;
            if (first[mid] <= p) lo = mid; else hi = mid - 1;
        }
        piece<W>(T.e[lo], p - first[lo], f);
        if (BACK) lo = p - step >= first[lo] ? lo : 0;          // in the same tensor, or the ones in front of it
        else hi = lo + 1 < T.count && first[lo + 1] <= p + step ? T.count - 1 : lo;
    }
}

__device__ __forceinline__ float element(const void *p, int64_t i, int f32) { return f32 ? ((const float *)p)[i] : bf2f(((const bf16 *)p)[i]); }

// 16 bytes as pairs of fp32, and their squares added to `s`
template <bool F32> __device__ __forceinline__ void unit_pairs(const uint4 &u, ptx::f32x2 (&v)[F32 ? 2 : 4])
{
    if constexpr (F32) {
        v[0] = ptx::pack2(u.x, u.y); v[1] = ptx::pack2(u.z, u.w);
    } else {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = ptx::pack2(w[i] << 16, w[i] & 0xFFFF0000u);
    }
}
template <int N> __device__ __forceinline__ bool nonzero(const uint4 (&r)[N])
{
    uint32_t any = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) any |= r[n].x | r[n].y | r[n].z | r[n].w;
    return any != 0;
}
// N units = 8 values
template <bool F32, int N> __device__ __forceinline__ void add_squares(const uint4 (&r)[N], double &acc)
{
    constexpr int PAIRS = F32 ? 2 : 4;
    static_assert(N * PAIRS == 4, "");
    ptx::f32x2 v[N][PAIRS], sum = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        unit_pairs<F32>(r[n], v[n]);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) sum = ptx::fma2(v[n][i], v[n][i], sum);
    }
    const float s = both(sum);
    if (s >= 8.6736174e-19f && s <= 1.3292279957849159e36f) {        // 2^-60 .. 2^120: what underflowed is nothing beside s
        acc += (double)s;
    } else if (nonzero<N>(r)) {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                float a, b;
                ptx::unpack2(v[n][i], a, b);
                acc = fma((double)a, (double)a, acc);
                acc = fma((double)b, (double)b, acc);
            }
    }
}

// The units of a piece: all of them loaded, the ones that the tensor's end cuts left zero.  f(first element) for the elements of a cut unit.
template <int W, bool F32, typename Tail>
__device__ __forceinline__ void load_piece(const void *g, int64_t b0, int64_t b1, uint4 (&r)[UNITS], Tail tail)
{
    constexpr int E = F32 ? 4 : 8;
    const uint4 *p = (const uint4 *)((const char *)g + b0 * (F32 ? 4 : 2)) + threadIdx.x % W;
    if (b1 - b0 == piece_of<W>(F32)) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) r[u] = p[u * W];
        return;
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int64_t at = b0 + (int64_t)(u * W + threadIdx.x % W) * E;
        r[u] = make_uint4(0, 0, 0, 0);
        if (at + E <= b1) r[u] = p[u * W];
        else for (int64_t i = at; i < b1; ++i) tail(i);
    }
}

template <int W, bool F32> __device__ __forceinline__ void piece_squares(const void *g, int64_t b0, int64_t b1, double &acc)
{
    constexpr int N = F32 ? 2 : 1;
    uint4 r[UNITS];
    load_piece<W, F32>(g, b0, b1, r, [&](int64_t i) { const double v = element(g, i, F32); acc = fma(v, v, acc); });
#pragma unroll
    for (int u = 0; u < UNITS; u += N) {
        uint4 e[N];
#pragma unroll
        for (int n = 0; n < N; ++n) e[n] = r[u + n];
        add_squares<F32, N>(e, acc);
    }
}

// the head of a tensor and a piece of it
template <int W> __device__ __forceinline__ void add_piece(const Entry &e, int64_t b0, int64_t b1, int64_t h, double &acc)
{
    for (int64_t i = threadIdx.x % W; i < h; i += W) { const double v = element(e.g, i, e.f32); acc = fma(v, v, acc); }
    if (e.f32) piece_squares<W, true>(e.g, b0, b1, acc);
    else piece_squares<W, false>(e.g, b0, b1, acc);
}
// Sum over the CTA, in every thread; fixed order.
__device__ __forceinline__ double block_sum(double v, double *red)
{
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = red[0];
    for (int i = 1; i < CT / 32; ++i) t += red[i];
    return t;
}

template <int N>
__global__ void __launch_bounds__(CT, CTAS)
grad_norm_parts_kernel(const __grid_constant__ Table<N> T, double *__restrict__ part)
{
    __shared__ double red[CT / 32];
    __shared__ int first[N];
    pdl_launch_dependents();
    stage_first(T, first);
    pdl_wait();
    double acc = 0.0;
    for_pieces<CT, false>(T, first, blockIdx.x, gridDim.x, [&](const Entry &e, int64_t b0, int64_t b1, int64_t h) { add_piece<CT>(e, b0, b1, h, acc); });
    acc = block_sum(acc, red);
    if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

// norm and factor of all partial sums, the same in every CTA
__device__ __forceinline__ float clip_factor(const double *part, int parts, float max_norm, float &norm, double *red)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += CT) s += part[i];
    norm = (float)sqrt(block_sum(s, red));
    return norm <= max_norm ? 1.f : max_norm / norm;
}

__global__ void __launch_bounds__(CT)
grad_norm_finish_kernel(const double *part, int parts, float max_norm, float *norm, float *factor)
{
    __shared__ double red[CT / 32];
    pdl_launch_dependents();
    pdl_wait();
    float v;
    const float f = clip_factor(part, parts, max_norm, v, red);
    if (threadIdx.x == 0) {
        *norm = v;
        if (factor) *factor = f;
    }
}

template <bool F32> __device__ __forceinline__ void scale_element(const Entry &e, int64_t i, float f)
{
    if (F32) ((float *)e.out)[i] = ((const float *)e.g)[i] * f;
    else ((bf16 *)e.out)[i] = f2bf(bf2f(((const bf16 *)e.g)[i]) * f);
}

template <int W, bool F32> __device__ __forceinline__ void piece_scale(const Entry &e, int64_t b0, int64_t b1, float f)
{
    if (((uintptr_t)e.out ^ (uintptr_t)e.g) & 15) {                   // the two cannot both be on 16-byte boundaries: an element per lane
        for (int64_t i = b0 + threadIdx.x % W; i < b1; i += W) scale_element<F32>(e, i, f);
        return;
    }
    constexpr int E = F32 ? 4 : 8, PAIRS = F32 ? 2 : 4;
    uint4 r[UNITS];
    load_piece<W, F32>(e.g, b0, b1, r, [&](int64_t i) { scale_element<F32>(e, i, f); });
    uint4 *o = (uint4 *)((char *)e.out + b0 * (F32 ? 4 : 2)) + threadIdx.x % W;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        ptx::f32x2 v[PAIRS];
        float x[8];
        unit_pairs<F32>(r[u], v);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) ptx::unpack2(ptx::mul2(v[i], ptx::twice(f)), x[2 * i], x[2 * i + 1]);
        uint4 w;
        if constexpr (F32) w = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
        else w = pack8(x);
        if (b1 - b0 == piece_of<W>(F32) || b0 + (int64_t)(u * W + threadIdx.x % W + 1) * E <= b1) __stcs(o + u * W, w);
    }
}

template <int W> __device__ __forceinline__ void scale_piece(const Entry &e, int64_t b0, int64_t b1, int64_t h, float f)
{
    if (f == 1.f && e.out == e.g) return;
    for (int64_t i = threadIdx.x % W; i < h; i += W) {
        if (e.f32) scale_element<true>(e, i, f);
        else scale_element<false>(e, i, f);
    }
    if (e.f32) piece_scale<W, true>(e, b0, b1, f);
    else piece_scale<W, false>(e, b0, b1, f);
}

template <int N>
__global__ void __launch_bounds__(CT, CTAS)
grad_scale_kernel(const __grid_constant__ Table<N> T, const double *part, int parts, float max_norm, float *norm, float *factor)
{
    __shared__ double red[CT / 32];
    __shared__ int first[N];
    pdl_launch_dependents();
    stage_first(T, first);
    pdl_wait();
    float v;
    const float f = clip_factor(part, parts, max_norm, v, red);
    if (blockIdx.x == 0 && threadIdx.x == 0) {                        // every launch of a call writes the same values
        *norm = v;
        *factor = f;
    }
    for_pieces<CT, true>(T, first, gridDim.x - 1 - blockIdx.x, gridDim.x, [&](const Entry &e, int64_t b0, int64_t b1, int64_t h) { scale_piece<CT>(e, b0, b1, h, f); });
}

// All of it in one launch where the gradients are few: a cluster, a piece per warp, the CTAs' sums over distributed shared memory in rank order.
// (62 vectors of 512: two launches took 6.9 us and 9.4 a call, this 6.7 and 6.8.)
__global__ void __launch_bounds__(CT)
grad_clip_small_kernel(const __grid_constant__ FewTable T, float max_norm, float *norm, float *factor, int scale)
{
    __shared__ double red[CT / 32], mine;
    pdl_launch_dependents();
    pdl_wait();
    uint32_t rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int me = rank * (CT / 32) + (threadIdx.x >> 5), all = CLUSTER * (CT / 32);
    double acc = 0.0;
    for (int p = me; p < T.pieces; p += all)
        piece<32>(T.e[T.owner[p]], T.index[p], [&](const Entry &e, int64_t b0, int64_t b1, int64_t h) { add_piece<32>(e, b0, b1, h, acc); });
    acc = block_sum(acc, red);
    if (threadIdx.x == 0) mine = acc;
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
    double sum = 0.0;
    for (uint32_t i = 0; i < CLUSTER; ++i) {
        uint32_t a;
        double v;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(ptx::smem_u32(&mine)), "r"(i));
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(a) : "memory");
        sum += v;
    }
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");    // this CTA has read its peers' sums; waited for at the end
    const float v = (float)sqrt(sum), f = v <= max_norm ? 1.f : max_norm / v;
    if (rank == 0 && threadIdx.x == 0) {
        *norm = v;
        if (factor) *factor = f;
    }
    if (scale)
        for (int p = me; p < T.pieces; p += all)
            piece<32>(T.e[T.owner[p]], T.index[p], [&](const Entry &e, int64_t b0, int64_t b1, int64_t h) { scale_piece<32>(e, b0, b1, h, f); });
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

// ----------------------------------------------------------------------------------------------------------- host
constexpr int SHORT = 4096;                   // pieces up to which the next launch is scheduled early
int max_ctas() { return sm_count() * CTAS; }

lamp_status_t check_grads(const lamp_grad_t *grads, int32_t count, bool outs)
{
    if (count < 0 || (count > 0 && !grads)) return LAMP_ERR_INVALID_ARG;
    if (count > (1 << 20)) return LAMP_ERR_UNSUPPORTED;
    int64_t total = 0;
    for (int32_t i = 0; i < count; ++i) {
        const lamp_grad_t &t = grads[i];
        if (t.dtype != LAMP_BF16 && t.dtype != LAMP_F32) return LAMP_ERR_UNSUPPORTED;
        if (t.n < 0) return LAMP_ERR_INVALID_ARG;
        if (t.n > (1ll << 40)) return LAMP_ERR_UNSUPPORTED;
        if ((total += t.n) > (1ll << 42)) return LAMP_ERR_UNSUPPORTED;  // 2^29 pieces
        if (t.n == 0) continue;
        const uintptr_t mask = t.dtype == LAMP_F32 ? 3 : 1;
        if (!t.g || ((uintptr_t)t.g & mask) || (outs && (!t.out || ((uintptr_t)t.out & mask)))) return LAMP_ERR_INVALID_ARG;
    }
    return LAMP_OK;
}

// Fills a table from entry i on; returns the entry behind it.
template <int N>
int32_t fill(Table<N> &T, const lamp_grad_t *grads, int32_t count, int32_t i)
{
    T.count = T.pieces = 0;
    for (; i < count && T.count < N; ++i) {
        const int64_t p = pieces_of<CT>(grads[i]);
        if (p == 0) continue;
        T.first[T.count] = T.pieces;
        T.e[T.count++] = Entry{grads[i].g, grads[i].out, grads[i].n, grads[i].dtype == LAMP_F32};
        T.pieces += (int32_t)p;
    }
    return i;
}

template <int N> int ctas(const Table<N> &T) { return T.pieces < max_ctas() ? T.pieces : max_ctas(); }

// Many pieces: four to a CTA, one CTA after the other.  CTAs at different points of their work use the memory better than resident ones in step, which
// pays for the sum over the parts at the start of each (211 M mixed gradients: 324 us resident, 303 so, 310 with two or eight).
template <int N> int scale_ctas(const Table<N> &T) { return T.pieces <= 8 * max_ctas() ? ctas(T) : (T.pieces + 3) / 4; }

template <int N>
lamp_status_t run(const lamp_grad_t *grads, int32_t count, float max_norm, float *norm, float *factor, bool scale, double *part, cudaStream_t st)
{
    lamp_status_t s;
    Table<N> T;
    int parts = 0, tables = 0;
    for (int32_t i = 0; i < count;) {
        i = fill(T, grads, count, i);
        const int g = ctas(T);
        if (g == 0) break;                                            // nothing but empty tensors left
        if ((s = launch_pdl(T.pieces <= SHORT, grad_norm_parts_kernel<N>, dim3((unsigned)g), dim3(CT), 0, st, T, part + parts)) != LAMP_OK) return s;
        parts += g;
        ++tables;
    }
    if (!scale || parts == 0) return launch_pdl(true, grad_norm_finish_kernel, dim3(1), dim3(CT), 0, st, (const double *)part, parts, max_norm, norm, factor);
    int32_t i = 0;
    for (int t = 0; t < tables; ++t) {
        i = fill(T, grads, count, i);
        if ((s = launch_pdl(T.pieces <= SHORT, grad_scale_kernel<N>, dim3((unsigned)scale_ctas(T)), dim3(CT), 0, st, T, (const double *)part, parts, max_norm, norm,
                            factor)) != LAMP_OK) return s;
    }
    return LAMP_OK;
}

// Whether all of the gradients are FEW pieces of a warp (512 KB) at most, and the table of them.
bool fill_few(FewTable &T, const lamp_grad_t *grads, int32_t count)
{
    if (count > SMALL) return false;
    T.pieces = 0;
    for (int32_t i = 0; i < count; ++i) {
        const int64_t p = pieces_of<32>(grads[i]);
        if (T.pieces + p > FEW) return false;
        for (int64_t k = 0; k < p; ++k) { T.owner[T.pieces] = (uint8_t)i; T.index[T.pieces++] = (uint8_t)k; }
        T.e[i] = Entry{grads[i].g, grads[i].out, grads[i].n, grads[i].dtype == LAMP_F32};
    }
    return T.pieces > 0;
}
lamp_status_t run_few(const FewTable &T, float max_norm, float *norm, float *factor, bool scale, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CLUSTER);
    cfg.blockDim = dim3(CT);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = CLUSTER;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, grad_clip_small_kernel, T, max_norm, norm, factor, scale ? 1 : 0) == cudaSuccess ? LAMP_OK : LAMP_ERR_CUDA;
}

size_t workspace(int32_t count)
{
    const size_t tables = count <= SMALL ? 1 : (size_t)(count + LARGE - 1) / LARGE;
    return tables * max_ctas() * sizeof(double);
}

lamp_status_t clip(const lamp_grad_t *grads, int32_t count, float max_norm, float *norm, float *factor, bool scale, void *ws, size_t ws_bytes, void *stream)
{
    lamp_status_t s;
    if ((s = check_grads(grads, count, scale)) != LAMP_OK) return s;
    if (!norm || ((uintptr_t)norm & 3) || (scale && !factor) || ((uintptr_t)factor & 3) || !(max_norm >= 0.f)) return LAMP_ERR_INVALID_ARG;
    if (!ws || ((uintptr_t)ws & 15) || ws_bytes < lamp_grad_norm_workspace_bytes(grads, count)) return LAMP_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    FewTable T;
    if (fill_few(T, grads, count)) return run_few(T, max_norm, norm, factor, scale, st);
    return count <= SMALL ? run<SMALL>(grads, count, max_norm, norm, factor, scale, (double *)ws, st)
                          : run<LARGE>(grads, count, max_norm, norm, factor, scale, (double *)ws, st);
}

}  // namespace

}  // namespace lamp

using namespace lamp;

extern "C" size_t lamp_grad_norm_workspace_bytes(const lamp_grad_t *grads, int32_t count)
{
    return check_grads(grads, count, false) == LAMP_OK ? workspace(count) : 0;
}
extern "C" lamp_status_t lamp_grad_norm(const lamp_grad_t *grads, int32_t count, float max_norm, float *norm, float *factor, void *ws, size_t ws_bytes,
                                        void *cuda_stream)
{
    return clip(grads, count, max_norm, norm, factor, false, ws, ws_bytes, cuda_stream);
}
extern "C" lamp_status_t lamp_grad_clip(const lamp_grad_t *grads, int32_t count, float max_norm, float *norm, float *factor, void *ws, size_t ws_bytes,
                                        void *cuda_stream)
{
    return clip(grads, count, max_norm, norm, factor, true, ws, ws_bytes, cuda_stream);
}
