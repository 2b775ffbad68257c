// Log-probabilities of given tokens, entropy and the top alternatives of rows of logits, and their gradient.
//
// Per row, with p = softmax(z / tau):  lse = log sum exp(z / tau),  logp = z_y / tau - lse,
// H = - sum p log p = log S - W / (tau S) of the statistics S, W of vocab_rows.cuh, and the k largest logits.
#include <algorithm>

#include "vocab_rows.cuh"

namespace sbp {

namespace {
constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxTop = STREAMBP_TOP_MAX, kCandidates = 1024, kMaxCluster = 8;

__device__ __forceinline__ void st_remote_f32(uint32_t a, float v) { st_remote_u32(a, __float_as_uint(v)); }

// The list of a row's segment: its k largest elements in order.
//
// A thread's elements are a stripe of the segment, and each thread knows the first of its largest (`best`, 0: none).  The
// k-th largest of these is not above the k-th largest element, and at most k stripes reach it: only those are read again,
// and what reaches it there (mostly little more than k elements) is ranked by counting.
template <typename T>
struct TopOfSegment {
    unsigned long long cand[kCandidates];
    int stripe[kThreads];
    int n_cand, n_stripes;

    // elements of the stripes in the list that reach `bound`; kept in cand where `keep`
    __device__ __forceinline__ void scan(const RowGroups<T> &row, int g0, int g1, unsigned long long bound, int n_str, bool keep) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        int mine = 0;
        for (int s = warp; s < n_str; s += kWarps)
            for (int v = g0 + stripe[s] + lane * kThreads; v < g1; v += 32 * kThreads) {
                float x[RowGroups<T>::N];
                row.load(v, x, 0.f);
#pragma unroll
                for (int i = 0; i < RowGroups<T>::N; i++) {
                    const int e = row.first(v) + i;
                    if (e < 0 || e >= row.n) continue;
                    const unsigned long long o = order_of(x[i], e);
                    if (o < bound) continue;
                    if (keep) {
                        const int at = atomicAdd(&n_cand, 1);
                        if (at < kCandidates) cand[at] = o;
                    } else {
                        mine++;
                    }
                }
            }
        if (!keep && mine) atomicAdd(&n_cand, mine);
    }

    __device__ __forceinline__ void list(const RowGroups<T> &row, int g0, int g1, unsigned long long best, int k,
                                         unsigned long long *out) {
        unsigned long long bound = 0;
        if (__syncthreads_count(best != 0) > k)
            for (int bit = 63; bit >= 0; bit--) {
                const unsigned long long trial = bound | 1ull << bit;
                const int reach = __syncthreads_count(best >= trial);
                if (reach >= k) bound = trial;
                if (reach == k) break;
            }
        if (threadIdx.x == 0) n_cand = n_stripes = 0;
        for (int i = threadIdx.x; i < k; i += kThreads) out[i] = 0;
        __syncthreads();
        if (best != 0 && best >= bound) stripe[atomicAdd(&n_stripes, 1)] = threadIdx.x;
        __syncthreads();
        const int n_str = n_stripes;
        scan(row, g0, g1, bound, n_str, true);
        __syncthreads();
        if (n_cand > kCandidates) {
            // rows whose large elements crowd into few stripes: a higher bound, bit by bit, until few enough reach it
            unsigned long long b = 0;
            for (int bit = 63; bit >= 0; bit--) {
                __syncthreads();
                if (threadIdx.x == 0) n_cand = 0;
                __syncthreads();
                scan(row, g0, g1, b | 1ull << bit, n_str, false);
                __syncthreads();
                const int reach = n_cand;
                if (reach >= k) b |= 1ull << bit;
                if (reach >= k && reach <= kCandidates) break;
            }
            __syncthreads();
            if (threadIdx.x == 0) n_cand = 0;
            __syncthreads();
            scan(row, g0, g1, b, n_str, true);
            __syncthreads();
        }
        const int n = n_cand;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const unsigned long long o = cand[i];
            int rank = 0;
            for (int j = 0; j < n; j++) rank += cand[j] > o;
            if (rank < k) out[rank] = o;
        }
        __syncthreads();
    }
};

struct ScoreArgs {
    const int64_t *tokens;      // optional
    int64_t ignore, rows, ld;
    int vocab, k;
    Heat heat;
    float *logp, *lse, *entropy, *top_logp;     // all optional
    int64_t *top_ids;
    WsHeader *hdr;              // optional: the first token outside the vocabulary goes there
    const int *gate;
};

// One pass over the row with the running maximum and sums in every thread, `cluster` blocks to a row where there are few
// rows.  Bound by HBM: a row of logits is read once; what the list reads again (k stripes) is a few kilobytes in L2.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) token_logprobs_kernel(const T *__restrict__ logits, ScoreArgs a, int cluster) {
    pdl_enter();
    constexpr int N = RowGroups<T>::N, U = 16 / N;
    if (gated_off(a.gate)) return;
    __shared__ RowStats s_warp[kWarps], s_cta[kMaxCluster];
    __shared__ TopOfSegment<T> top;
    __shared__ unsigned long long s_list[TOP ? kMaxTop : 1], s_lists[TOP ? kMaxCluster * kMaxTop : 1];
    const int64_t r = blockIdx.x / cluster;
    const int rank = (int)(blockIdx.x % cluster), tid = threadIdx.x;
    if (blockIdx.x == 0 && a.hdr)
        report_first(a.tokens, a.tokens ? a.rows : 0, 1, a.hdr,
                     [&](int64_t y, int64_t) { return y != a.ignore && (y < 0 || y >= a.vocab); });
    const int64_t y = a.tokens ? a.tokens[r] : 0;
    if (a.tokens && (y == a.ignore || y < 0 || y >= a.vocab)) {
        if (rank == 0) {
            if (tid == 0) {
                if (a.logp) a.logp[r] = 0.f;
                if (a.lse) a.lse[r] = 0.f;
                if (a.entropy) a.entropy[r] = 0.f;
            }
            if (TOP)
                for (int i = tid; i < a.k; i += kThreads) {
                    if (a.top_logp) a.top_logp[r * a.k + i] = -INFINITY;
                    if (a.top_ids) a.top_ids[r * a.k + i] = -1;
                }
        }
        return;
    }
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // (waited for before the others' memory is written)
    const RowGroups<T> row(logits + r * a.ld, a.vocab);
    const int per = (row.groups + cluster - 1) / cluster;
    const int g0 = min(rank * per, row.groups), g1 = min(g0 + per, row.groups);
    const float c = a.heat.hi * kLog2e;
    RowStats st{-INFINITY, 0.f, 0.f};
    int first = g0 + tid < g1 ? max(0, row.first(g0 + tid)) : -1;      // where the largest so far came first
    for (int v0 = g0 + tid; v0 < g1; v0 += U * kThreads) {
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int v = v0 + u * kThreads;
            if (v < g1) {
                row.load(v, x[u], -INFINITY);
            } else {
#pragma unroll
                for (int i = 0; i < N; i++) x[u][i] = -INFINITY;
            }
        }
        float mx = x[0][0];
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < N; i++) mx = fmaxf(mx, x[u][i]);
        if (mx > st.m) {
            if (st.m > -INFINITY) {
                const float dm = fmaxf(st.m - mx, kDeep), f = exp2_approx(dm * c);
                st.W = f * fmaf(dm, st.S, st.W);
                st.S *= f;
            }
            st.m = mx;
            if (TOP) {
#pragma unroll
                for (int u = U - 1; u >= 0; u--)
#pragma unroll
                    for (int i = N - 1; i >= 0; i--)
                        if (x[u][i] == mx) first = row.first(v0 + u * kThreads) + i;
            }
        }
        const float m = finite_or_zero(st.m);
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float d = x[u][i] - m, e = exp2_approx(d * c);
                st.S += e;
                st.W = fmaf(e, fmaxf(d, kDeep), st.W);
            }
    }
    const unsigned long long best = TOP && first >= 0 ? order_of(st.m, first) : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        RowStats b;
        b.m = __shfl_xor_sync(0xffffffffu, st.m, o);
        b.S = __shfl_xor_sync(0xffffffffu, st.S, o);
        b.W = __shfl_xor_sync(0xffffffffu, st.W, o);
        st = join(st, b, c);
    }
    if ((tid & 31) == 0) s_warp[tid >> 5] = st;
    __syncthreads();
    st = s_warp[0];
    for (int w = 1; w < kWarps; w++) st = join(st, s_warp[w], c);
    if (cluster > 1) {
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (tid < cluster) {
            const uint32_t to = map_to_cta(smem_u32(&s_cta[rank]), tid);
            st_remote_f32(to, st.m);
            st_remote_f32(to + 4, st.S);
            st_remote_f32(to + 8, st.W);
        }
        cluster_sync_all();
        st = s_cta[0];
        for (int w = 1; w < cluster; w++) st = join(st, s_cta[w], c);
    }
    const float m = finite_or_zero(st.m), logS = logf(st.S);
    const bool none = st.S == 0.f, broken = !(st.S < INFINITY);
    auto logp_of = [&](float z) {
        const float d = z - m;
        return none ? -INFINITY : broken ? NAN : d > -INFINITY ? fmaf(d, a.heat.hi, fmaf(d, a.heat.lo, -logS)) : -INFINITY;
    };
    if (rank == 0 && tid == 0) {
        if (a.logp) a.logp[r] = logp_of(to_f32(logits[r * a.ld + y]));
        if (a.lse) a.lse[r] = broken ? NAN : fmaf(m, a.heat.hi, fmaf(m, a.heat.lo, logS));
        if (a.entropy) a.entropy[r] = none ? 0.f : broken ? NAN : logS - (st.W / st.S) * a.heat.hi;
    }
    if constexpr (TOP) {
        if (broken) {       // (the same in every block of the row)
            if (rank == 0)
                for (int i = tid; i < a.k; i += kThreads) {
                    if (a.top_logp) a.top_logp[r * a.k + i] = NAN;
                    if (a.top_ids) a.top_ids[r * a.k + i] = -1;
                }
            return;
        }
        top.list(row, g0, g1, best, a.k, s_list);
        if (cluster > 1) {
            const uint32_t to = map_to_cta(smem_u32(s_lists + rank * kMaxTop), 0);
            for (int i = tid; i < a.k; i += kThreads) {
                st_remote_u32(to + 8 * i, (uint32_t)s_list[i]);
                st_remote_u32(to + 8 * i + 4, (uint32_t)(s_list[i] >> 32));
            }
            cluster_sync_all();
            if (rank != 0) return;
            // an element's place is the number of larger ones: its own list's and, by bisection, the others'
            for (int i = tid; i < cluster * a.k; i += kThreads) {
                const int l = i / a.k;
                const unsigned long long o = s_lists[l * kMaxTop + i % a.k];
                int place = i % a.k;
                for (int q = 0; q < cluster && o; q++) {
                    if (q == l) continue;
                    int lo = 0, hi = a.k;
                    while (lo < hi) {
                        const int mid = (lo + hi) / 2;
                        if (s_lists[q * kMaxTop + mid] > o) lo = mid + 1;
                        else hi = mid;
                    }
                    place += lo;
                }
                if (o && place < a.k) s_list[place] = o;
            }
            __syncthreads();
        }
        for (int i = tid; i < a.k; i += kThreads) {
            if (a.top_logp) a.top_logp[r * a.k + i] = logp_of(value_of(s_list[i]));
            if (a.top_ids) a.top_ids[r * a.k + i] = index_of(s_list[i]);
        }
    }
}

// dz = (dlogp (1[y] - p) + dlse p - dH p (log p + H)) / tau; each thread a few groups of one row, a row cut over blocks.
struct ScoreGradArgs {
    const int64_t *tokens;      // optional
    int64_t ignore, ld, ldd;
    int vocab;
    Heat heat;
    const float *lse, *entropy, *d_logp, *d_lse, *d_entropy;    // entropy with d_entropy; the three gradients are optional
};
constexpr int kGradGroups = 4;
template <typename T>
__global__ void __launch_bounds__(kThreads) token_logprobs_bwd_kernel(const T *logits, T *d_logits, ScoreGradArgs a) {
    pdl_enter();
    constexpr int N = RowGroups<T>::N;
    const int64_t r = blockIdx.x;
    T *d = d_logits + r * a.ldd;
    const RowGroups<T> out(d, a.vocab);
    const int64_t y = a.tokens ? a.tokens[r] : -1;
    const bool part = !a.tokens || (y != a.ignore && y >= 0 && y < a.vocab);
    const RowGroups<T> in(logits + r * a.ld, a.vocab);
    const bool same = in.off == out.off;
    const float lse = part ? a.lse[r] : 0.f, gp = part && a.d_logp && a.tokens ? a.d_logp[r] : 0.f, gl = part && a.d_lse ? a.d_lse[r] : 0.f;
    const float gh = part && a.d_entropy ? a.d_entropy[r] : 0.f, H = part && a.d_entropy ? a.entropy[r] : 0.f;
    const float c0 = gl - gp - gh * H;
    const bool none = lse == -INFINITY;      // every logit is -inf: p is 0
    auto grad = [&](float z, int e) {
        const float lp = fmaf(z, a.heat.hi, fmaf(z, a.heat.lo, -lse));
        float p = exp2_approx(lp * kLog2e);
        if (z == -INFINITY) p = 0.f;
        float g = p * (p > 0.f || p != p ? fmaf(-gh, lp, c0) : 0.f);
        if (none) g = 0.f;
        if (e == y) g += gp;
        return fmaf(g, a.heat.hi, g * a.heat.lo);
    };
    const int v0 = (blockIdx.y * kGradGroups) * kThreads + threadIdx.x;
    float x[kGradGroups][N];
#pragma unroll
    for (int u = 0; u < kGradGroups; u++) {
        const int v = v0 + u * kThreads;
        if (!part || v >= out.groups) continue;
        if (same) {
            in.load(v, x[u], 0.f);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) {
                const int e = out.first(v) + i;
                x[u][i] = e >= 0 && e < a.vocab ? to_f32(logits[r * a.ld + e]) : 0.f;
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kGradGroups; u++) {
        const int v = v0 + u * kThreads;
        if (v >= out.groups) continue;
        const int e0 = out.first(v);
        Vec<T> o;
#pragma unroll
        for (int i = 0; i < N; i++) o.v[i] = part ? grad(x[u][i], e0 + i) : 0.f;
        if (out.whole(v)) {
            o.store(d + e0);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++)
                if (e0 + i >= 0 && e0 + i < a.vocab) d[e0 + i] = from_f32<T>(o.v[i]);
        }
    }
}

// Blocks to a row: enough for two blocks an SM where rows are few, none with less than two groups a thread.
template <typename T>
int row_cluster(int64_t rows, int64_t vocab) {
    int c = 1;
    while (c < kMaxCluster && rows * c < 2 * 148 && vocab / (2 * c) >= 2 * kThreads * Vec<T>::N) c *= 2;
    return c;
}
}  // namespace

template <typename T>
int token_logprobs(const T *logits, int64_t ld, int64_t rows, int64_t vocab, const int64_t *tokens, int64_t ignore,
                   float temperature, int k, float *logp, float *lse, float *entropy, float *top_logp, int64_t *top_ids,
                   WsHeader *hdr, cudaStream_t st) {
    const ScoreArgs a{tokens, ignore, rows, ld, (int)vocab, k, make_heat(temperature), logp, lse, entropy, top_logp, top_ids, hdr,
                      call_state().gate};
    const int c = row_cluster<T>(rows, vocab);
    auto kernel = k ? token_logprobs_kernel<T, true> : token_logprobs_kernel<T, false>;
    return launch_clusters(kernel, dim3((unsigned)(rows * c)), kThreads, 0, c, 1, st, logits, a, c);
}
template <typename T>
int token_logprobs_bwd(const T *logits, int64_t ld, int64_t rows, int64_t vocab, const int64_t *tokens, int64_t ignore,
                       float temperature, const float *lse, const float *entropy, const float *d_logp, const float *d_lse,
                       const float *d_entropy, T *d_logits, int64_t ldd, cudaStream_t st) {
    const ScoreGradArgs a{tokens, ignore, ld, ldd, (int)vocab, make_heat(temperature), lse, entropy, d_logp, d_lse, d_entropy};
    const int64_t groups = (vocab + Vec<T>::N - 1) / Vec<T>::N + 1, per = kThreads * kGradGroups;
    SBP_LAUNCH(token_logprobs_bwd_kernel<T>, dim3((unsigned)rows, (unsigned)((groups + per - 1) / per)), kThreads, 0, st, logits,
               d_logits, a);
    return STREAMBP_OK;
}

template int token_logprobs<float>(const float *, int64_t, int64_t, int64_t, const int64_t *, int64_t, float, int, float *, float *,
                                   float *, float *, int64_t *, WsHeader *, cudaStream_t);
template int token_logprobs<bf16>(const bf16 *, int64_t, int64_t, int64_t, const int64_t *, int64_t, float, int, float *, float *,
                                  float *, float *, int64_t *, WsHeader *, cudaStream_t);
template int token_logprobs_bwd<float>(const float *, int64_t, int64_t, int64_t, const int64_t *, int64_t, float, const float *,
                                       const float *, const float *, const float *, const float *, float *, int64_t, cudaStream_t);
template int token_logprobs_bwd<bf16>(const bf16 *, int64_t, int64_t, int64_t, const int64_t *, int64_t, float, const float *,
                                      const float *, const float *, const float *, const float *, bf16 *, int64_t, cudaStream_t);

}  // namespace sbp
