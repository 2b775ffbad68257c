// Distillation from a teacher's top logits: the loss of a row and the gradient of its logits.
//
// A row has k entries (id c_i, value t_i) and a weight w.  p = softmax(z / tau) over the whole vocabulary.
//   list only:  q = softmax(t / tau) over the entries,   L = sum q_i (log q_i - log p_ci),  Q = 1, q_r = 0
//   with tail:  q_i = exp t_i,  q_r = 1 - sum q_i,  L as above + q_r log(q_r / p_r),  p_r the mass of unlisted tokens,  Q = sum q_i + q_r
//   dL/dz_j = (Q p_j - sum_{c_i = j} q_i) / tau for listed j,  (Q p_j - q_r p_j / p_r) / tau for the others
#include <algorithm>

#include "vocab_rows.cuh"

namespace sbp {

namespace {
constexpr int kThreads = 512, kWarps = kThreads / 32, kMaxTop = STREAMBP_TOP_MAX, kMaxCluster = 8;

struct DistillArgs {
    const int64_t *ids;
    const float *values, *weight;       // weight is optional
    float *row_loss;                    // optional
    int64_t rows, ld, ldd;
    int vocab, k, tail;
    Heat heat;
    WsHeader *hdr;                      // optional: the first row with an id outside the vocabulary goes there
    const int *gate;
};

__device__ __forceinline__ void st_remote_f64(uint32_t a, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(a), "d"(v) : "memory");
}

// What a block knows of its segment of a row, for the others: the maximum m, the sums of exp((z - m) / tau) over its unlisted
// and its listed tokens, sum q (log q - (z - m) / tau) over its entries and the sum of their q.
struct Segment {
    double m, rest, listed, loss, q;
};

// A row's logits stay in the shared memory of `cluster` blocks (three blocks an SM, so that one loads while others compute
// and store): they are read from HBM once and their gradient is written once, which is what bounds the kernel.  Listed
// tokens are taken out of the row (their logits become -inf) before the sums, so that the mass of the others is a sum of
// its own and not a difference; their gradients are written over the zeros of the streaming pass.
template <typename T, typename TO>
__global__ void __launch_bounds__(kThreads) distill_kernel(const T *logits, TO *d_logits, DistillArgs a, int cluster) {
    pdl_enter();
    if (gated_off(a.gate)) return;
    constexpr int N = RowGroups<T>::N;
    extern __shared__ __align__(16) unsigned char s_raw[];
    T *s_row = reinterpret_cast<T *>(s_raw);            // groups g0 .. g1 - 1 of the row
    __shared__ float s_max[kWarps], s_sum[kWarps];
    __shared__ Segment s_seg[kMaxCluster];
    __shared__ int s_id[kMaxTop];
    __shared__ double s_q[kMaxTop], s_logq[kMaxTop], s_part[2];
    __shared__ float s_z[kMaxTop], s_e[kMaxTop];
    const int64_t r = blockIdx.x / cluster;
    const int rank = (int)(blockIdx.x % cluster), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (blockIdx.x == 0 && a.hdr)
        report_first(a.ids, a.rows * a.k, a.k, a.hdr, [&](int64_t id, int64_t i) {
            return (id < -1 || id >= a.vocab) && (!a.weight || a.weight[i / a.k] != 0.f);
        });
    const RowGroups<T> row(logits + r * a.ld, a.vocab);
    TO *d = d_logits ? d_logits + r * a.ldd : nullptr;
    const int per = (row.groups + cluster - 1) / cluster;
    const int g0 = min(rank * per, row.groups), g1 = min(g0 + per, row.groups);
    const int e0 = max(0, row.first(g0)), e1 = g1 > g0 ? min(a.vocab, row.first(g1)) : e0;      // elements of the segment
    const float w = a.weight ? a.weight[r] : 1.f;
    // entries of the row: the first warp finds q
    if (w != 0.f && warp == 0) {
        const int64_t at = r * a.k;
        float t[kMaxTop / 32];
        int id[kMaxTop / 32], any = 0;
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < kMaxTop / 32; j++) {
            const int i = lane + 32 * j;
            id[j] = -1;
            t[j] = -INFINITY;
            if (i < a.k) {
                const int64_t x = a.ids[at + i];
                if (x >= 0 && x < a.vocab) {
                    id[j] = (int)x;
                    t[j] = a.values[at + i];
                    any = 1;
                }
            }
            top = fmaxf(top, t[j]);
        }
        top = warp_max(top);
        any = __any_sync(0xffffffffu, any);
        // (in 64 bits: what is left of 1 for the tail is a difference)
        const double inv = (double)a.heat.hi + (double)a.heat.lo, t0 = top == -INFINITY ? 0.0 : (double)top;
        double q[kMaxTop / 32], sum = 0.0;
#pragma unroll
        for (int j = 0; j < kMaxTop / 32; j++) {
            q[j] = id[j] < 0 ? 0.0 : a.tail ? exp((double)t[j]) : exp(((double)t[j] - t0) * inv);
            sum += q[j];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const double logsum = log(sum);
#pragma unroll
        for (int j = 0; j < kMaxTop / 32; j++) {
            const int i = lane + 32 * j;
            if (i >= a.k) continue;
            s_id[i] = id[j];
            s_q[i] = a.tail || sum == 0.0 ? q[j] : q[j] / sum;
            s_logq[i] = a.tail ? (double)t[j] : ((double)t[j] - t0) * inv - logsum;
        }
        if (lane == 0) {
            s_part[0] = a.tail ? sum : sum == 0.0 ? 0.0 : 1.0;                  // the sum of q
            s_part[1] = a.tail && any ? fmax(0.0, 1.0 - sum) : 0.0;
        }
    }
    if (w != 0.f)
        for (int v = g0 + tid; v < g1; v += kThreads) {
            if (row.whole(v)) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(s_row + (size_t)(v - g0) * N)),
                             "l"(row.base + (int64_t)v * N)
                             : "memory");
            } else {
#pragma unroll
                for (int i = 0; i < N; i++) {
                    const int e = row.first(v) + i;
                    s_row[(v - g0) * N + i] = e >= 0 && e < a.vocab ? row.base[(int64_t)v * N + i] : from_f32<T>(-INFINITY);
                }
            }
        }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    const double mass = w != 0.f ? s_part[0] : 0.0;
    double rest_q = w != 0.f ? s_part[1] : 0.0;
    if (mass == 0.0 && rest_q == 0.0) {         // no weight or no entries: the row takes no part
        if (d)
            for (int e = e0 + tid; e < e1; e += kThreads) d[e] = from_f32<TO>(0.f);
        if (rank == 0 && tid == 0 && a.row_loss) a.row_loss[r] = 0.f;
        return;
    }
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // (waited for before the others' memory is written)
    // maximum; the segment's listed logits
    float m = -INFINITY;
    for (int v = tid; v < g1 - g0; v += kThreads) {
        Vec<T> x;
        x.load(s_row + (size_t)v * N);
#pragma unroll
        for (int i = 0; i < N; i++) m = fmaxf(m, x.v[i]);
    }
    m = warp_max(m);
    if (lane == 0) s_max[warp] = m;
    const int mine = tid < a.k && s_id[tid] >= e0 && s_id[tid] < e1 ? s_id[tid] - row.first(g0) : -1;   // place in s_row of entry tid
    if (mine >= 0) s_z[tid] = to_f32(s_row[mine]);
    __syncthreads();
    if (mine >= 0) s_row[mine] = from_f32<T>(-INFINITY);
    m = s_max[0];
#pragma unroll
    for (int i = 1; i < kWarps; i++) m = fmaxf(m, s_max[i]);
    const float mf = finite_or_zero(m), c = a.heat.hi * kLog2e;
    __syncthreads();
    // the sum over unlisted tokens
    float sum = 0.f;
    for (int v = tid; v < g1 - g0; v += kThreads) {
        Vec<T> x;
        x.load(s_row + (size_t)v * N);
#pragma unroll
        for (int i = 0; i < N; i++) sum += exp2_approx((x.v[i] - mf) * c);
    }
    sum = warp_sum(sum);
    if (lane == 0) s_sum[warp] = sum;
    if (tid < kMaxTop) s_e[tid] = mine >= 0 ? exp2_approx((s_z[tid] - mf) * c) : 0.f;
    __syncthreads();
    if (warp == 0) {
        const double inv = (double)a.heat.hi + (double)a.heat.lo;
        Segment s{(double)m, lane < kWarps ? (double)s_sum[lane] : 0.0, 0.0, 0.0, 0.0};
        for (int i = lane; i < a.k; i += 32) {
            if (s_id[i] < e0 || s_id[i] >= e1) continue;
            bool again = false;
            for (int j = 0; j < i; j++) again |= s_id[j] == s_id[i];
            if (!again) s.listed += (double)s_e[i];
            const double q = s_q[i];
            if (q != 0.0) s.loss += q * (s_logq[i] - ((double)s_z[i] - (double)mf) * inv);
            s.q += q;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s.rest += __shfl_xor_sync(0xffffffffu, s.rest, o);
            s.listed += __shfl_xor_sync(0xffffffffu, s.listed, o);
            s.loss += __shfl_xor_sync(0xffffffffu, s.loss, o);
            s.q += __shfl_xor_sync(0xffffffffu, s.q, o);
        }
        if (cluster > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        if (lane < cluster) {
            const uint32_t to = map_to_cta(smem_u32(&s_seg[rank]), lane);
            st_remote_f64(to, s.m);
            st_remote_f64(to + 8, s.rest);
            st_remote_f64(to + 16, s.listed);
            st_remote_f64(to + 24, s.loss);
            st_remote_f64(to + 32, s.q);
        }
    } else if (cluster > 1) {
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
    if (cluster > 1) cluster_sync_all();
    else __syncthreads();
    double M = s_seg[0].m;
    for (int i = 1; i < cluster; i++) M = fmax(M, s_seg[i].m);
    const double Mf = M == -INFINITY ? 0.0 : M;
    double S = 0.0, rest = 0.0, loss = 0.0;
    const double inv = (double)a.heat.hi + (double)a.heat.lo;
    for (int i = 0; i < cluster; i++) {
        const Segment &s = s_seg[i];
        const double f = s.m == -INFINITY ? 0.0 : (double)exp2f((float)((s.m - Mf) * inv * 1.4426950408889634));
        rest += s.rest * f;
        S += (s.rest + s.listed) * f;
    }
    if (rest == 0.0) rest_q = 0.0;              // there is no token for the tail
    const double Q = mass + rest_q;
    if (rank == 0 && tid == 0 && a.row_loss) {
        const double logS = S == 0.0 ? 0.0 : log(S);
        for (int i = 0; i < cluster; i++) {
            const Segment &s = s_seg[i];
            loss += s.loss;
            if (s.q != 0.0) loss += s.q * (((s.m == -INFINITY ? Mf : Mf - s.m)) * inv + logS);
        }
        if (rest_q != 0.0) loss += rest_q * (log(rest_q) - (log(rest) - logS));
        a.row_loss[r] = (float)loss;
    }
    if (!d) return;
    // gradient: unlisted tokens by one factor
    const double scale = (double)w * inv, own = m == -INFINITY ? 0.0 : (double)exp2f((float)(((double)m - Mf) * inv * 1.4426950408889634));
    const double of_p = S == 0.0 ? 0.0 : Q / S;
    const float factor = (float)(scale * own * (of_p - (rest_q != 0.0 ? rest_q / rest : 0.0)));
    constexpr int NO = Vec<TO>::N;
    const RowGroups<TO> out(d + e0, e1 - e0);
    const T *seg = s_row + (e0 - row.first(g0));
    for (int v = tid; v < out.groups; v += kThreads) {
        const int f = out.first(v);
        Vec<TO> o;
#pragma unroll
        for (int i = 0; i < NO; i++) {
            const int e = f + i;
            o.v[i] = e >= 0 && e < e1 - e0 ? factor * exp2_approx((to_f32(seg[e]) - mf) * c) : 0.f;
        }
        if (out.whole(v)) {
            o.store(d + e0 + f);
        } else {
#pragma unroll
            for (int i = 0; i < NO; i++)
                if (f + i >= 0 && f + i < e1 - e0) d[e0 + f + i] = from_f32<TO>(o.v[i]);
        }
    }
    __syncthreads();
    if (mine >= 0) {        // listed tokens; a token listed again has the sum of its entries
        double q = 0.0;
        bool again = false;
        for (int j = 0; j < a.k; j++) {
            if (s_id[j] != s_id[tid]) continue;
            again |= j < tid;
            q += s_q[j];
        }
        if (!again) d[s_id[tid]] = from_f32<TO>((float)(scale * (of_p * own * (double)s_e[tid] - q)));
    }
}

// Blocks to a row: at most kSegment bytes of it in each (three blocks an SM); more where rows are few, none with less than
// two groups a thread.
constexpr int64_t kSegment = 72 << 10;
template <typename T>
int row_cluster(int64_t rows, int64_t vocab) {
    int c = 1;
    while (c < kMaxCluster && (vocab * (int64_t)sizeof(T) > c * kSegment ||
                               (rows * c < 2 * 148 && vocab / (2 * c) >= 2 * kThreads * Vec<T>::N)))
        c *= 2;
    return c;
}

template <typename T, typename TO>
int launch(const T *logits, TO *d_logits, const DistillArgs &a, cudaStream_t st) {
    const int c = row_cluster<T>(a.rows, a.vocab);
    const int64_t groups = (a.vocab + Vec<T>::N - 1) / Vec<T>::N + 1;
    const int smem = (int)((groups + c - 1) / c * 16);
    static PerDevice ready;
    auto kernel = distill_kernel<T, TO>;
    if (!ready.get([&] { return cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 208 << 10)) ? 1 : 0; }))
        return STREAMBP_E_CUDA;
    return launch_clusters(kernel, dim3((unsigned)(a.rows * c)), kThreads, smem, c, 1, st, logits, d_logits, a, c);
}
}  // namespace

template <typename T, typename TO>
int distill_topk(const T *logits, int64_t ld, int64_t rows, int64_t vocab, const DistillRows &ds, TO *d_logits, int64_t ldd,
                 WsHeader *hdr, cudaStream_t st) {
    if (rows <= 0) return STREAMBP_OK;
    const DistillArgs a{ds.ids, ds.values, ds.weight, ds.row_loss, rows, ld, ldd, (int)vocab, ds.k, ds.tail ? 1 : 0,
                        make_heat(ds.temperature), hdr, call_state().gate};
    return launch<T, TO>(logits, d_logits, a, st);
}
template int distill_topk<float, float>(const float *, int64_t, int64_t, int64_t, const DistillRows &, float *, int64_t, WsHeader *,
                                        cudaStream_t);
template int distill_topk<bf16, bf16>(const bf16 *, int64_t, int64_t, int64_t, const DistillRows &, bf16 *, int64_t, WsHeader *,
                                      cudaStream_t);
template int distill_topk<float, bf16>(const float *, int64_t, int64_t, int64_t, const DistillRows &, bf16 *, int64_t, WsHeader *,
                                       cudaStream_t);

__global__ void __launch_bounds__(256) distill_marks_kernel(DistillRows ds, int64_t T_, int64_t vocab, int64_t *__restrict__ marks,
                                                            WsHeader *hdr) {
    pdl_enter();
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < T_ * ds.k; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t t = i / ds.k;
        const bool part = ds.weight[t] != 0.f;
        if (i == t * ds.k) marks[t] = part ? 0 : 1;
        if (part && (ds.ids[i] < -1 || ds.ids[i] >= vocab)) set_status(hdr, STREAMBP_E_BAD_LABEL, (int)t);
    }
}
int distill_marks(const DistillRows &ds, int64_t T_, int64_t vocab, int64_t *marks, WsHeader *hdr, cudaStream_t st) {
    const int64_t blocks = std::min<int64_t>((T_ * ds.k + 255) / 256, 148 * 8);
    SBP_LAUNCH(distill_marks_kernel, (unsigned)blocks, 256, 0, st, ds, T_, vocab, marks, hdr);
    return STREAMBP_OK;
}

__global__ void __launch_bounds__(1024) loss_weighted_kernel(const float *__restrict__ row_loss, const float *__restrict__ weight,
                                                             int64_t rows, WsHeader *hdr, const int *gate) {
    pdl_enter();
    __shared__ double red[32];
    if (gated_off(gate)) return;
    double acc = 0.0;
    for (int64_t r = threadIdx.x; r < rows; r += blockDim.x)
        if (weight[r] != 0.f) acc += (double)weight[r] * (double)row_loss[r];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 32; w++) acc += red[w];
        hdr->loss_sum += acc;
    }
}
int loss_accumulate_weighted(const float *row_loss, const float *weight, int64_t rows, WsHeader *hdr, cudaStream_t st) {
    SBP_LAUNCH(loss_weighted_kernel, 1, 1024, 0, st, row_loss, weight, rows, hdr, call_state().gate);
    return STREAMBP_OK;
}

}  // namespace sbp
