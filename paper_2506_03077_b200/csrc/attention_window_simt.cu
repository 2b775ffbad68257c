// Attention with a sliding window and sink keys on CUDA cores (fp32 arithmetic): the fp32 precision mode, and what the
// tensor-core kernels are checked against.  Tiles of 32 queries and 32 keys; a query tile visits the key tiles its window
// reaches and those that hold sinks.  Online softmax with warp-shuffle row maxima and sums.  The backward is deterministic:
// one kernel owns a key tile (dK, dV), another a query tile (dQ); a sink tile's query tiles are cut into segments that are
// joined in order (window_join_kernel below, which the tensor-core backward uses as well).
#include "common.cuh"
#include "window.cuh"

namespace sbp {
namespace {

constexpr int TILE = 32;

// dst[r][c] = src[(row0 + r) * stride + c], 32 rows of DH values, zeros from `rows` on and in rows `skip`
template <typename T, int DH, typename Skip>
__device__ __forceinline__ void load_rows(float *dst, const T *src, int row0, int rows, int64_t stride, Skip skip) {
    constexpr int LD = DH + 4, N = Vec<T>::N;
    for (int i = threadIdx.x; i < 32 * (DH / N); i += 256) {
        const int r = i / (DH / N), c = (i % (DH / N)) * N;
        Vec<T> v;
#pragma unroll
        for (int e = 0; e < N; e++) v.v[e] = 0.f;
        if (row0 + r < rows && !skip(row0 + r)) v.load(src + (int64_t)(row0 + r) * stride + c);
#pragma unroll
        for (int e = 0; e < N; e++) dst[r * LD + c + e] = v.v[e];
    }
}
template <typename T, int DH>
__device__ __forceinline__ void load_rows(float *dst, const T *src, int row0, int rows, int64_t stride) {
    load_rows<T, DH>(dst, src, row0, rows, stride, [](int) { return false; });
}
// of K or V: rows that no query sees may hold anything
template <typename T, int DH>
__device__ __forceinline__ void load_keys(float *dst, const T *src, int row0, const WindowShape &w) {
    load_rows<T, DH>(dst, src, row0, w.q0 + w.n, (int64_t)w.Hkv * DH, [&](int r) { return w.unseen(r); });
}
// s[i] = <A[4 warp + i], B[lane]>
template <int DH>
__device__ __forceinline__ void dots(const float *A, const float *B, int w, int lane, float s[4]) {
    constexpr int LD = DH + 4;
    s[0] = s[1] = s[2] = s[3] = 0.f;
#pragma unroll 8
    for (int x = 0; x < DH; x += 4) {
        const float4 b = *reinterpret_cast<const float4 *>(B + lane * LD + x);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float4 a = *reinterpret_cast<const float4 *>(A + (w * 4 + i) * LD + x);
            s[i] = fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, s[i]))));
        }
    }
}
__device__ __forceinline__ bool visible(const WindowShape &w, int q, int k) {
    return k <= q && q < w.q0 + w.n && (q - k < w.window || k < w.sinks);
}

// grid (query tiles, Hq); warp w owns query rows 4w .. 4w + 3, a lane a key
template <typename T, int DH>
__global__ void __launch_bounds__(256)
    window_fwd_kernel(const T *q, const T *k, const T *v, const WindowShape w, T *o, float *lse) {
    pdl_enter();
    constexpr int LD = DH + 4, D = DH / 32;
    extern __shared__ __align__(16) float smem[];
    float *Qs = smem, *Ks = Qs + 32 * LD, *Vs = Ks + 32 * LD;
    const int h = blockIdx.y, g = h / (w.Hq / w.Hkv), qt0 = blockIdx.x * TILE;
    const int wp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int kv = w.q0 + w.n;
    const float scale = rsqrtf((float)DH);
    load_rows<T, DH>(Qs, q + (int64_t)h * DH, qt0, w.n, (int64_t)w.Hq * DH);
    float m[4], l[4], acc[4][D];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int e = 0; e < D; e++) acc[i][e] = 0.f;
    }
    const int q_last = w.q0 + (qt0 + TILE < w.n ? qt0 + TILE : w.n) - 1;
    const KeySpan span = key_span<TILE>(w, w.q0 + qt0, q_last);
    for (int j = 0; j < span.count(); j++) {
        const int k0 = span.tile(j) * TILE;
        __syncthreads();
        load_keys<T, DH>(Ks, k + (int64_t)g * DH, k0, w);
        load_keys<T, DH>(Vs, v + (int64_t)g * DH, k0, w);
        __syncthreads();
        float s[4];
        dots<DH>(Qs, Ks, wp, lane, s);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const bool ok = visible(w, w.q0 + qt0 + wp * 4 + i, k0 + lane);
            const float x = ok ? s[i] * scale : -INFINITY;
            const float top = fmaxf(m[i], warp_max(x));
            const float ref = top == -INFINITY ? 0.f : top;       // a row that has seen no key yet
            const float pr = ok ? __expf(x - ref) : 0.f, keep = __expf(m[i] - ref);
            l[i] = l[i] * keep + warp_sum(pr);
            m[i] = top;
#pragma unroll
            for (int e = 0; e < D; e++) acc[i][e] *= keep;
            for (int c = 0; c < 32; c++) {
                const float pc = __shfl_sync(0xffffffffu, pr, c);
#pragma unroll
                for (int e = 0; e < D; e++) acc[i][e] = fmaf(pc, Vs[c * LD + e * 32 + lane], acc[i][e]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int r = qt0 + wp * 4 + i;
        if (r >= w.n) continue;
        const float inv = 1.f / l[i];
#pragma unroll
        for (int e = 0; e < D; e++) o[((int64_t)r * w.Hq + h) * DH + e * 32 + lane] = from_f32<T>(acc[i][e] * inv);
        if (lane == 0) lse[(int64_t)h * w.n + r] = m[i] + logf(l[i]);
    }
}

// Rows of dk and dv that no query of the chunk sees have no owner among the key tiles: their gradients are zero (`count`
// 16-byte pieces of each; sink rows among them are written later in the stream).
__device__ __forceinline__ void clear_unseen(void *dk, void *dv, int64_t count) {
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < count; i += (int64_t)gridDim.x * blockDim.x) {
        static_cast<uint4 *>(dk)[i] = make_uint4(0u, 0u, 0u, 0u);
        static_cast<uint4 *>(dv)[i] = make_uint4(0u, 0u, 0u, 0u);
    }
}
template <typename T>
__global__ void __launch_bounds__(256) window_delta_any_kernel(const T *o, const T *dout, int n, int Hq, int dh, float *delta, WsHeader *hdr,
                                                               void *dk, void *dv, int64_t unseen16) {
    pdl_enter();
    if (blockIdx.x == 0 && threadIdx.x == 0) clear_status(hdr);
    clear_unseen(dk, dv, unseen16);
    const int64_t r = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    if (r >= (int64_t)n * Hq) return;
    float s = 0.f;
    for (int j = lane; j < dh; j += 32) s = fmaf(to_f32(o[r * dh + j]), to_f32(dout[r * dh + j]), s);
    s = warp_sum(s);
    if (lane == 0) delta[(r % Hq) * n + r / Hq] = s;
}

// P and dS of the warp's four query rows against key `lane`
template <int DH>
__device__ __forceinline__ void p_ds(const float *Qs, const float *Ds, const float *Ks, const float *Vs, const float *lse,
                                     const float *delta, int wp, int lane, const WindowShape &w, int q0, int k0, float scale,
                                     float p[4], float ds[4]) {
    float s[4], dp[4];
    dots<DH>(Qs, Ks, wp, lane, s);
    dots<DH>(Ds, Vs, wp, lane, dp);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        p[i] = visible(w, q0 + wp * 4 + i, k0 + lane) ? __expf(s[i] * scale - lse[wp * 4 + i]) : 0.f;
        ds[i] = p[i] * (dp[i] - delta[wp * 4 + i]) * scale;
    }
}
__device__ __forceinline__ void put4(void *dst, int64_t at, const float (&a)[4], int mode) {
    if (mode == GRAD_BF16_SET) {
        const __nv_bfloat162 x = __floats2bfloat162_rn(a[0], a[1]), y = __floats2bfloat162_rn(a[2], a[3]);
        *reinterpret_cast<uint2 *>(static_cast<bf16 *>(dst) + at) =
            make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y));
        return;
    }
    float4 *d = reinterpret_cast<float4 *>(static_cast<float *>(dst) + at);
    float4 v = make_float4(a[0], a[1], a[2], a[3]);
    if (mode == GRAD_F32_ADD) {
        const float4 b = *d;
        v.x += b.x; v.y += b.y; v.z += b.z; v.w += b.w;
    }
    *d = v;
}

// grid (items, Hkv); thread (row tid / 8, dims (tid % 8) * 4 + 32 e ..)
template <typename T, int DH>
__global__ void __launch_bounds__(256)
    window_dkdv_kernel(const T *q, const T *k, const T *v, const T *dout, const float *lse, const float *delta,
                       const WindowShape w, const KeyWork<TILE> work, void *dk, void *dv, int mode, float *part, int part_rows) {
    pdl_enter();
    constexpr int LD = DH + 4, NE = DH / 32;
    extern __shared__ __align__(16) float smem[];
    float *Ks = smem, *Vs = Ks + 32 * LD, *Qs = Vs + 32 * LD, *Ds = Qs + 32 * LD;
    float *Ps = Ds + 32 * LD, *Ss = Ps + 32 * 33, *lse_s = Ss + 32 * 33, *delta_s = lse_s + 32;
    const int g = blockIdx.y, G = w.Hq / w.Hkv, kv = w.q0 + w.n, item = blockIdx.x;
    const int wp = threadIdx.x >> 5, lane = threadIdx.x & 31, kr = threadIdx.x >> 3, sub = threadIdx.x & 7;
    const float scale = rsqrtf((float)DH);
    int kt, begin, end, seg;
    work.item(w, item, kt, begin, end, seg);
    const int k0 = kt * TILE;
    load_keys<T, DH>(Ks, k + (int64_t)g * DH, k0, w);
    load_keys<T, DH>(Vs, v + (int64_t)g * DH, k0, w);
    float ak[NE][4], av[NE][4];
#pragma unroll
    for (int e = 0; e < NE; e++)
#pragma unroll
        for (int c = 0; c < 4; c++) ak[e][c] = av[e][c] = 0.f;
    for (int h = g * G; h < (g + 1) * G; h++) {
        for (int qt = begin; qt < end; qt++) {
            const int r0 = qt * TILE;
            __syncthreads();
            load_rows<T, DH>(Qs, q + (int64_t)h * DH, r0, w.n, (int64_t)w.Hq * DH);
            load_rows<T, DH>(Ds, dout + (int64_t)h * DH, r0, w.n, (int64_t)w.Hq * DH);
            if (threadIdx.x < 32) {
                const int r = r0 + threadIdx.x;
                lse_s[threadIdx.x] = r < w.n ? lse[(int64_t)h * w.n + r] : 0.f;
                delta_s[threadIdx.x] = r < w.n ? delta[(int64_t)h * w.n + r] : 0.f;
            }
            __syncthreads();
            float p[4], ds[4];
            p_ds<DH>(Qs, Ds, Ks, Vs, lse_s, delta_s, wp, lane, w, w.q0 + r0, k0, scale, p, ds);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                Ps[(wp * 4 + i) * 33 + lane] = p[i];
                Ss[(wp * 4 + i) * 33 + lane] = ds[i];
            }
            __syncthreads();
            for (int r = 0; r < TILE; r++) {
                const float pv = Ps[r * 33 + kr], sv = Ss[r * 33 + kr];
#pragma unroll
                for (int e = 0; e < NE; e++) {
                    const float4 d = *reinterpret_cast<const float4 *>(Ds + r * LD + e * 32 + sub * 4);
                    const float4 x = *reinterpret_cast<const float4 *>(Qs + r * LD + e * 32 + sub * 4);
                    av[e][0] = fmaf(pv, d.x, av[e][0]); av[e][1] = fmaf(pv, d.y, av[e][1]);
                    av[e][2] = fmaf(pv, d.z, av[e][2]); av[e][3] = fmaf(pv, d.w, av[e][3]);
                    ak[e][0] = fmaf(sv, x.x, ak[e][0]); ak[e][1] = fmaf(sv, x.y, ak[e][1]);
                    ak[e][2] = fmaf(sv, x.z, ak[e][2]); ak[e][3] = fmaf(sv, x.w, ak[e][3]);
                }
            }
        }
    }
    const bool joined = seg >= 0 && kr < work.joined_rows(w, kt);
#pragma unroll
    for (int e = 0; e < NE; e++) {
        if (joined) {
            float *out = part + (((int64_t)item * w.Hkv + g) * 2 * part_rows + kr) * DH + e * 32 + sub * 4;
            put4(out, 0, ak[e], GRAD_F32_SET);
            put4(out, (int64_t)part_rows * DH, av[e], GRAD_F32_SET);
        } else if (seg <= 0 && k0 + kr < kv) {
            const int64_t at = ((int64_t)(k0 + kr) * w.Hkv + g) * DH + e * 32 + sub * 4;
            put4(dk, at, ak[e], mode);
            put4(dv, at, av[e], mode);
        }
    }
}

// grid (query tiles, Hq)
template <typename T, int DH>
__global__ void __launch_bounds__(256)
    window_dq_kernel(const T *q, const T *k, const T *v, const T *dout, const float *lse, const float *delta,
                     const WindowShape w, void *dq, int mode) {
    pdl_enter();
    constexpr int LD = DH + 4, NE = DH / 32;
    extern __shared__ __align__(16) float smem[];
    float *Ks = smem, *Vs = Ks + 32 * LD, *Qs = Vs + 32 * LD, *Ds = Qs + 32 * LD;
    float *Ss = Ds + 32 * LD, *lse_s = Ss + 32 * 33, *delta_s = lse_s + 32;
    const int h = blockIdx.y, g = h / (w.Hq / w.Hkv), r0 = blockIdx.x * TILE, kv = w.q0 + w.n;
    const int wp = threadIdx.x >> 5, lane = threadIdx.x & 31, qr = threadIdx.x >> 3, sub = threadIdx.x & 7;
    const float scale = rsqrtf((float)DH);
    load_rows<T, DH>(Qs, q + (int64_t)h * DH, r0, w.n, (int64_t)w.Hq * DH);
    load_rows<T, DH>(Ds, dout + (int64_t)h * DH, r0, w.n, (int64_t)w.Hq * DH);
    if (threadIdx.x < 32) {
        const int r = r0 + threadIdx.x;
        lse_s[threadIdx.x] = r < w.n ? lse[(int64_t)h * w.n + r] : 0.f;
        delta_s[threadIdx.x] = r < w.n ? delta[(int64_t)h * w.n + r] : 0.f;
    }
    float aq[NE][4];
#pragma unroll
    for (int e = 0; e < NE; e++)
#pragma unroll
        for (int c = 0; c < 4; c++) aq[e][c] = 0.f;
    const int q_last = w.q0 + (r0 + TILE < w.n ? r0 + TILE : w.n) - 1;
    const KeySpan span = key_span<TILE>(w, w.q0 + r0, q_last);
    for (int j = 0; j < span.count(); j++) {
        const int k0 = span.tile(j) * TILE;
        __syncthreads();
        load_keys<T, DH>(Ks, k + (int64_t)g * DH, k0, w);
        load_keys<T, DH>(Vs, v + (int64_t)g * DH, k0, w);
        __syncthreads();
        float p[4], ds[4];
        p_ds<DH>(Qs, Ds, Ks, Vs, lse_s, delta_s, wp, lane, w, w.q0 + r0, k0, scale, p, ds);
#pragma unroll
        for (int i = 0; i < 4; i++) Ss[(wp * 4 + i) * 33 + lane] = ds[i];
        __syncthreads();
        for (int c = 0; c < TILE; c++) {
            const float sv = Ss[qr * 33 + c];
#pragma unroll
            for (int e = 0; e < NE; e++) {
                const float4 x = *reinterpret_cast<const float4 *>(Ks + c * LD + e * 32 + sub * 4);
                aq[e][0] = fmaf(sv, x.x, aq[e][0]); aq[e][1] = fmaf(sv, x.y, aq[e][1]);
                aq[e][2] = fmaf(sv, x.z, aq[e][2]); aq[e][3] = fmaf(sv, x.w, aq[e][3]);
            }
        }
    }
    if (r0 + qr < w.n)
#pragma unroll
        for (int e = 0; e < NE; e++)
            put4(dq, ((int64_t)(r0 + qr) * w.Hq + h) * DH + e * 32 + sub * 4, aq[e], mode == GRAD_BF16_SET ? mode : GRAD_F32_SET);
}

// A thread per four values of (key, KV head, dK or dV); the keys are those of the first st tiles, `lead` of them, then those of
// the tiles from wt0 on.
__global__ void __launch_bounds__(256)
    window_join_kernel(const float *part, int tile, int st, int segs, int wt0, int wsegs, int lead, int rows, int Hkv, int dh, int64_t count,
                       void *dk, void *dv, int mode) {
    pdl_enter();
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= count) return;
    const int per = dh / 4, d = (int)(t % per) * 4, which = (int)(t / per) & 1;
    const int64_t unit = t / (2 * per);
    const int i = (int)(unit / Hkv), g = (int)(unit % Hkv);
    const bool head = i < lead;
    const int key = head ? i : wt0 * tile + i - lead, kt = key / tile, row = key - kt * tile;
    const int n = head ? segs : wsegs, item0 = head ? kt * segs : st * segs + (kt - wt0) * wsegs;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    const float *p = part + ((((int64_t)item0 * Hkv + g) * 2 + which) * rows + row) * dh + d;
    const int64_t step = (int64_t)Hkv * 2 * rows * dh;
#pragma unroll 4
    for (int k = 0; k < n; k++) {
        const float4 a = *reinterpret_cast<const float4 *>(p + k * step);
        s[0] += a.x; s[1] += a.y; s[2] += a.z; s[3] += a.w;
    }
    put4(which ? dv : dk, ((int64_t)key * Hkv + g) * dh + d, s, mode);
}

template <typename K>
bool set_smem(K kernel, size_t bytes) {
    return cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
}

template <typename T, int DH>
int fwd(const T *q, const T *k, const T *v, const WindowShape &w, T *o, float *lse, cudaStream_t st) {
    const size_t smem = (size_t)3 * 32 * (DH + 4) * sizeof(float);
    static PerDevice configured;
    if (!configured.get([&] { return set_smem(window_fwd_kernel<T, DH>, smem) ? 1 : 0; })) return STREAMBP_E_CUDA;
    SBP_LAUNCH((window_fwd_kernel<T, DH>), dim3((w.n + TILE - 1) / TILE, w.Hq), 256, smem, st, q, k, v, w, o, lse);
    return STREAMBP_OK;
}
template <typename T, int DH>
int bwd(const T *q, const T *k, const T *v, const T *o, const T *dout, const float *lse, const WindowShape &w, int mode,
        void *dq, void *dk, void *dv, float *delta, float *part, WsHeader *hdr, cudaStream_t st) {
    const size_t smem = ((size_t)4 * 32 * (DH + 4) + 2 * 32 * 33 + 64) * sizeof(float);
    static PerDevice configured;
    if (!configured.get([&] { return set_smem(window_dkdv_kernel<T, DH>, smem) && set_smem(window_dq_kernel<T, DH>, smem) ? 1 : 0; }))
        return STREAMBP_E_CUDA;
    const int64_t rows = (int64_t)w.n * w.Hq;
    const KeyWork<TILE> work = key_work<TILE>(w, TILE, 1, 0);
    const int64_t unseen16 = mode == GRAD_F32_ADD ? 0 : (int64_t)work.lo * TILE * w.Hkv * DH * (mode == GRAD_BF16_SET ? 2 : 4) / 16;
    SBP_LAUNCH(window_delta_any_kernel<T>, (unsigned)((rows * 32 + 255) / 256), 256, 0, st, o, dout, w.n, w.Hq, DH, delta, hdr, dk, dv,
               unseen16);
    const int part_rows = work.slot_rows(w);
    SBP_LAUNCH((window_dkdv_kernel<T, DH>), dim3(work.items(), w.Hkv), 256, smem, st, q, k, v, dout, lse, (const float *)delta, w,
               work, dk, dv, mode, part, part_rows);
    SBP_LAUNCH((window_dq_kernel<T, DH>), dim3((w.n + TILE - 1) / TILE, w.Hq), 256, smem, st, q, k, v, dout, lse,
               (const float *)delta, w, dq, mode);
    return attention_window_join(part, work, w, DH, mode, dk, dv, st);
}

}  // namespace

template <int TK>
int attention_window_join(const float *part, const KeyWork<TK> &work, const WindowShape &w, int dh, int mode, void *dk, void *dv,
                          cudaStream_t stream) {
    const int64_t lead = work.join_lead(w), count = (lead + work.join_behind(w)) * w.Hkv * (dh / 2), blocks = (count + 255) / 256;
    if (blocks > 0x7fffffff) return STREAMBP_E_SHAPE;
    if (count == 0) return STREAMBP_OK;
    SBP_LAUNCH(window_join_kernel, (unsigned)blocks, 256, 0, stream, part, TK, work.st, work.segs, work.wt0, work.wsegs, (int)lead,
               work.slot_rows(w), w.Hkv, dh, count, dk, dv, mode);
    return STREAMBP_OK;
}
template int attention_window_join<128>(const float *, const KeyWork<128> &, const WindowShape &, int, int, void *, void *, cudaStream_t);

template <typename T>
int attention_window_fwd_simt(const T *q, const T *k, const T *v, const WindowShape &w, int dh, T *o, float *lse, cudaStream_t st) {
    return dh == 64 ? fwd<T, 64>(q, k, v, w, o, lse, st) : fwd<T, 128>(q, k, v, w, o, lse, st);
}
template <typename T>
int attention_window_bwd_simt(const T *q, const T *k, const T *v, const T *o, const T *dout, const float *lse, const WindowShape &w,
                              int dh, int mode, void *dq, void *dk, void *dv, float *delta, float *part, WsHeader *hdr,
                              cudaStream_t st) {
    return dh == 64 ? bwd<T, 64>(q, k, v, o, dout, lse, w, mode, dq, dk, dv, delta, part, hdr, st)
                    : bwd<T, 128>(q, k, v, o, dout, lse, w, mode, dq, dk, dv, delta, part, hdr, st);
}
template int attention_window_fwd_simt<float>(const float *, const float *, const float *, const WindowShape &, int, float *, float *, cudaStream_t);
template int attention_window_fwd_simt<bf16>(const bf16 *, const bf16 *, const bf16 *, const WindowShape &, int, bf16 *, float *, cudaStream_t);
template int attention_window_bwd_simt<float>(const float *, const float *, const float *, const float *, const float *, const float *,
                                              const WindowShape &, int, int, void *, void *, void *, float *, float *, WsHeader *, cudaStream_t);
template int attention_window_bwd_simt<bf16>(const bf16 *, const bf16 *, const bf16 *, const bf16 *, const bf16 *, const float *,
                                             const WindowShape &, int, int, void *, void *, void *, float *, float *, WsHeader *, cudaStream_t);

}  // namespace sbp
