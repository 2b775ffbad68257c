// Log-probabilities of given tokens, entropy and the top alternatives of rows of logits, and their gradient.
//
// Per row, with p = softmax(z / tau):  lse = log sum exp(z / tau),  logp = z_y / tau - lse,
// H = - sum p log p = log S - W / (tau S) of the statistics S, W of vocab_rows.cuh, and the k largest logits.
//
// Bound by HBM where rows are many.  Measured: 1024 x 152064 fp32 without a list in 97 us (6.4 TB/s, a copy's rate), with 16
// alternatives 104 (6.0); 2048 x 152064 bf16 in 103 and 123 us (6.0 and 5.1 TB/s: twice the exponentials a byte).  3 rows of 152064
// in 11 us, half of which is the list: its bound, what reaches it, the ranks and the cluster's join come one after another.
// Gradient: 2048 x 32003 bf16 in 42 us (5.6 TB/s with what skipped rows save), 2048 x 152064 fp32 in 379 (6.6).
#include <algorithm>

#include "vocab_rows.cuh"

namespace sbp {

namespace {
constexpr int kMaxTop = STREAMBP_TOP_MAX, kCandidates = 1056, kMaxCluster = 8;
constexpr int kManyThreads = 256, kFewThreads = 1024;      // of a block where rows are many, and few

__device__ __forceinline__ void st_remote_f32(uint32_t a, float v) { st_remote_u32(a, __float_as_uint(v)); }
__device__ __forceinline__ float value_of_key(uint32_t key) { return value_of((unsigned long long)key << 32); }
__device__ __forceinline__ uint32_t key_of(float v) { return (uint32_t)(order_of(v, 0) >> 32); }

// The list of a row's segment: its k largest elements in order.
//
// A thread's elements (every THREADS-th whole group) are cut into kParts parts (fewer where it has few), and the pass over the
// row leaves each part's largest value in `part`.  Of m >= k disjoint sets of elements, the k-th largest of the sets' largest
// values is not above the k-th largest element; the sets are 32 groups of threads where k is well below 32 (one warp finds
// the bound), else the threads.  Only parts that reach the bound hold what is on the list: mostly little more than k parts, each
// a few groups, are read again, and what reaches the bound there (mostly little more than k elements) is ranked by counting.
template <typename T, int THREADS>
struct TopOfSegment {
    static constexpr int kParts = THREADS > 256 ? 2 : 8, kOf32 = 24;
    unsigned long long cand[kCandidates];
    float part[kParts][THREADS];
    unsigned short item[kParts * THREADS];       // parts that reach the bound: part * THREADS + thread
    uint32_t set[32], s_bound;
    int n_cand, n_items, n_warp[THREADS / 32];

    __device__ __forceinline__ void offer(float x, int e, uint32_t bound, bool keep, int &mine) {
        if (key_of(x) < bound) return;
        if (keep) {
            const int at = atomicAdd(&n_cand, 1);
            if (at < kCandidates) cand[at] = order_of(x, e);
        } else {
            mine++;
        }
    }
    // elements of the listed parts and of the segment's ragged ends with key >= bound, kept in cand where there is room
    __device__ __forceinline__ void gather(const RowGroups<T> &row, int g0, int g1, int w0, int w1, int per_part, uint32_t bound, bool keep) {
        constexpr int N = RowGroups<T>::N;
        const int n = n_items * per_part;
        int mine = 0;
        for (int q = threadIdx.x; q < n; q += THREADS) {
            const int it = item[q / per_part], v = w0 + it % THREADS + (it / THREADS * per_part + q % per_part) * THREADS;
            if (v >= w1) continue;
            float x[N];
            row.load(v, x, 0.f);
#pragma unroll
            for (int i = 0; i < N; i++) offer(x[i], row.first(v) + i, bound, keep, mine);
        }
        if (threadIdx.x < 2 * N) {
            // (one group at each end, which may be the same one)
            const int v = threadIdx.x < N ? g0 : g1 - 1, e = row.first(v) + threadIdx.x % N;
            if (g0 < g1 && (v < w0 || v >= w1) && !(threadIdx.x >= N && v == g0) && e >= 0 && e < row.n)
                offer(to_f32(row.base[(int64_t)v * N + threadIdx.x % N]), e, bound, keep, mine);
        }
        if (!keep && mine) atomicAdd(&n_cand, mine);
    }
    __device__ __forceinline__ void restart() {
        __syncthreads();
        if (threadIdx.x == 0) n_cand = 0;
        __syncthreads();
    }

    // best: the largest value of this thread's elements, if it has any
    __device__ __forceinline__ void list(const RowGroups<T> &row, int g0, int g1, int w0, int w1, int per_part, bool has, float best, int k,
                                         unsigned long long *out) {
        constexpr int N = RowGroups<T>::N;
        const int tid = threadIdx.x, lane = tid & 31;
        uint32_t bound = 0;
        const uint32_t key = has ? key_of(best) : 0;
        if (tid == 0) n_cand = n_items = 0;
        for (int i = tid; i < k; i += THREADS) out[i] = 0;
        if (k <= kOf32 && w1 - w0 >= THREADS) {
            uint32_t top = key;
#pragma unroll
            for (int o = THREADS / 64; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (tid % (THREADS / 32) == 0) set[tid / (THREADS / 32)] = top;
            __syncthreads();
            if (tid < 32) {
                const uint32_t mine = set[lane];
                int above = 0;
#pragma unroll
                for (int j = 0; j < 32; j++) {
                    const uint32_t other = __shfl_sync(0xffffffffu, mine, j);
                    above += other > mine || (other == mine && j < lane);
                }
                if (above == k - 1) s_bound = mine;         // (0 where fewer than k sets have elements)
            }
            __syncthreads();
            bound = s_bound;
        } else if (__syncthreads_count(has) > k) {
            for (int bit = 31; bit >= 0; bit--) {
                const uint32_t trial = bound | 1u << bit;
                const int reach = __syncthreads_count(key >= trial);
                if (reach >= k) bound = trial;
                if (reach == k) break;
            }
        }
        __syncthreads();
        if (has && key >= bound)
            for (int p = 0; p < kParts; p++)
                if (w0 + tid + p * per_part * THREADS < w1 && key_of(part[p][tid]) >= bound)
                    item[atomicAdd(&n_items, 1)] = (unsigned short)(p * THREADS + tid);
        __syncthreads();
        gather(row, g0, g1, w0, w1, per_part, bound, true);
        __syncthreads();
        bool ties = false;
        if (n_cand > kCandidates) {
            // many equal values at the bound, or large values crowded into few parts: the k-th largest value itself, bit by
            // bit where more than the list's length lie above the bound
            restart();
            gather(row, g0, g1, w0, w1, per_part, bound + 1, true);
            __syncthreads();
            if (n_cand > kCandidates) {
                uint32_t b = 0;
                for (int bit = 31; bit >= 0; bit--) {
                    restart();
                    gather(row, g0, g1, w0, w1, per_part, b | 1u << bit, false);
                    __syncthreads();
                    if (n_cand >= k) b |= 1u << bit;
                }
                bound = b;
                restart();
                gather(row, g0, g1, w0, w1, per_part, bound + 1, true);
                __syncthreads();
            }
            ties = n_cand < k;
        }
        const int n = min(n_cand, kCandidates);
        for (int i = tid; i < n; i += THREADS) {
            const unsigned long long o = cand[i];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < n; j++) rank += cand[j] > o;
            if (rank < k) out[rank] = o;
        }
        if (ties) {
            // behind them the first elements of the bound's value, looked for in the row's order
            int have = n;
            for (int v0 = g0; v0 < g1 && have < k; v0 += THREADS) {
                const int v = v0 + tid;
                float x[N];
                uint32_t equal = 0;
                if (v < g1) {
                    row.load(v, x, 0.f);
#pragma unroll
                    for (int i = 0; i < N; i++) {
                        const int e = row.first(v) + i;
                        if (e >= 0 && e < row.n && key_of(x[i]) == bound) equal |= 1u << i;
                    }
                }
                int before = __popc(equal);
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int t = __shfl_up_sync(0xffffffffu, before, o);
                    if (lane >= o) before += t;
                }
                if (lane == 31) n_warp[tid >> 5] = before;
                __syncthreads();
                int at = have + before - __popc(equal);
                for (int w = 0; w < THREADS / 32; w++) {
                    if (w < (tid >> 5)) at += n_warp[w];
                    have += n_warp[w];
                }
                for (; equal && at < k; equal &= equal - 1, at++) out[at] = order_of(value_of_key(bound), row.first(v) + __ffs(equal) - 1);
                __syncthreads();
            }
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
    WsHeader *hdr;              // optional: a token outside the vocabulary goes there
    bool scan;                  // found by one block, else by each row's
    const int *gate;
};

// One pass over the row with the running maximum and sums in every thread.  Bound by HBM: a row of logits is read once; what
// the list reads again is a few kilobytes.  Blocks of 256 threads, one to a row, where there are rows to fill the GPU; else
// blocks of 1024 and up to eight to a row, so that a thread has all of its loads in flight at once.
template <typename T, bool TOP, bool ENT, int THREADS>
__device__ __forceinline__ void score_row(const T *__restrict__ logits, const ScoreArgs &a, int cluster) {
    // (loads of a thread in flight: 1024 x 152064 fp32 with 16 alternatives 104 us with eight and 116 with four, without 103 and 97)
    constexpr int U = TOP && THREADS == kManyThreads && sizeof(T) == 4 ? 8 : 4, kWarps = THREADS / 32, kParts = TopOfSegment<T, THREADS>::kParts;
    __shared__ RowStats s_warp[kWarps], s_row, s_cta[kMaxCluster];
    __shared__ TopOfSegment<T, TOP ? THREADS : 32> top;
    __shared__ unsigned long long s_list[TOP ? kMaxTop : 1], s_lists[TOP && THREADS == kFewThreads ? kMaxCluster * kMaxTop : 1];
    const int64_t r = blockIdx.x / cluster;
    const int rank = (int)(blockIdx.x % cluster), tid = threadIdx.x, lane = tid & 31;
    const int64_t y = a.tokens ? a.tokens[r] : 0;
    if (a.tokens && (y == a.ignore || y < 0 || y >= a.vocab)) {
        if (rank == 0) {
            if (tid == 0) {
                if (y != a.ignore && a.hdr && !a.scan) set_status(a.hdr, STREAMBP_E_BAD_LABEL, (int)r);
                if (a.logp) a.logp[r] = 0.f;
                if (a.lse) a.lse[r] = 0.f;
                if (a.entropy) a.entropy[r] = 0.f;
            }
            if (TOP)
                for (int i = tid; i < a.k; i += THREADS) {
                    if (a.top_logp) a.top_logp[r * a.k + i] = -INFINITY;
                    if (a.top_ids) a.top_ids[r * a.k + i] = -1;
                }
        }
        return;
    }
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // (waited for before the others' memory is written)
    const RowGroups<T> row(logits + r * a.ld, a.vocab);
    const int per = (row.groups + cluster - 1) / cluster;
    const int g0 = min(rank * per, row.groups), g1 = min(g0 + per, row.groups);         // the segment's groups
    const int w0 = max(g0, row.whole_begin()), w1 = max(w0, min(g1, row.whole_end()));  // the whole ones among them
    // groups of a thread in one part: whole batches
    const int rounds = (w1 - w0 + THREADS - 1) / THREADS, per_part = max(1, ((rounds + kParts - 1) / kParts + U - 1) / U) * U;
    const float c = a.heat.hi * kLog2e;
    const float zy = rank == 0 && tid == 0 && a.logp ? to_f32(logits[r * a.ld + y]) : 0.f;
    Running<T, ENT> run;
    for (int p = 0; p < (TOP ? kParts : 1); p++) {
        run.largest = -INFINITY;
        const int end = TOP ? min(w1, w0 + (p + 1) * per_part * THREADS) : w1;
        int v0 = w0 + p * per_part * THREADS + tid;
        Raw<T> x[U];
        for (; v0 + (U - 1) * THREADS < end; v0 += U * THREADS) {
#pragma unroll
            for (int u = 0; u < U; u++) row.load_whole(v0 + u * THREADS, x[u]);
            run.add(x, c);
        }
        if (v0 < end) {
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (v0 + u * THREADS < end) row.load_whole(v0 + u * THREADS, x[u]);
                else x[u].fill(-INFINITY);
            }
            run.add(x, c);
        }
        if (TOP) top.part[p][tid] = run.largest;
    }
    bool has = w0 + tid < w1;
    if (tid == 0 && g0 < g1 && (w0 != g0 || w1 != g1)) {        // the ragged ends
        Raw<T> x[U];
#pragma unroll
        for (int u = 0; u < U; u++) x[u].fill(-INFINITY);
        if (w0 != g0) row.load(g0, x[0]);
        if (w1 != g1 && g1 - 1 >= w0) row.load(g1 - 1, x[1]);
        run.add(x, c);
        has = true;
    }
    RowStats st;
    {
        float lo, hi;
        run.S.get(lo, hi);
        st.S = lo + hi;
        run.W.get(lo, hi);
        st.W = lo + hi;
        st.m = run.m;
    }
    auto joined = [&](int first) {          // over the lanes of a warp
#pragma unroll
        for (int o = first; o > 0; o >>= 1) {
            RowStats b;
            b.m = __shfl_xor_sync(0xffffffffu, st.m, o);
            b.S = __shfl_xor_sync(0xffffffffu, st.S, o);
            b.W = __shfl_xor_sync(0xffffffffu, st.W, o);
            st = join(st, b, c);
        }
    };
    joined(16);
    if (lane == 0) s_warp[tid >> 5] = st;
    __syncthreads();
    if (tid < 32) {
        st = lane < kWarps ? s_warp[lane] : RowStats{-INFINITY, 0.f, 0.f};
        joined(kWarps / 2);
        if (lane == 0) s_row = st;
        if (cluster > 1) {
            st.m = __shfl_sync(0xffffffffu, st.m, 0);
            st.S = __shfl_sync(0xffffffffu, st.S, 0);
            st.W = __shfl_sync(0xffffffffu, st.W, 0);
            asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
            if (lane < cluster) {
                const uint32_t to = map_to_cta(smem_u32(&s_cta[rank]), lane);
                st_remote_f32(to, st.m);
                st_remote_f32(to + 4, st.S);
                st_remote_f32(to + 8, st.W);
            }
            __syncwarp();
        }
    } else if (cluster > 1) {
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");      // (waited for where the whole row's sums are needed)
    __syncthreads();
    if constexpr (TOP)
        if (s_row.S < INFINITY) top.list(row, g0, g1, w0, w1, per_part, has, run.m, a.k, s_list);     // (else the row is broken, and has no list)
    if (cluster > 1) {
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        if (tid < 32) {
            st = lane < cluster ? s_cta[lane] : RowStats{-INFINITY, 0.f, 0.f};
            joined(kMaxCluster / 2);
            if (lane == 0) s_row = st;
        }
        __syncthreads();
    }
    st = s_row;
    const float top_m = finite_or_zero(st.m), logS = logf(st.S);
    const bool none = st.S == 0.f, broken = !(st.S < INFINITY);
    auto logp_of = [&](float z) {
        const float d = z - top_m;
        return none ? -INFINITY : broken ? NAN : d > -INFINITY ? fmaf(d, a.heat.hi, fmaf(d, a.heat.lo, -logS)) : -INFINITY;
    };
    if (rank == 0 && tid == 0) {
        if (a.logp) a.logp[r] = logp_of(zy);
        if (a.lse) a.lse[r] = broken ? NAN : fmaf(top_m, a.heat.hi, fmaf(top_m, a.heat.lo, logS));
        if (ENT) a.entropy[r] = none ? 0.f : broken ? NAN : logS - (st.W / st.S) * a.heat.hi;
    }
    if constexpr (TOP) {
        if (broken) {       // (the same in every block of the row)
            if (rank == 0)
                for (int i = tid; i < a.k; i += THREADS) {
                    if (a.top_logp) a.top_logp[r * a.k + i] = NAN;
                    if (a.top_ids) a.top_ids[r * a.k + i] = -1;
                }
            return;
        }
        if (THREADS == kFewThreads && cluster > 1) {
            const uint32_t to = map_to_cta(smem_u32(s_lists + rank * kMaxTop), 0);
            for (int i = tid; i < a.k; i += THREADS) {
                st_remote_u32(to + 8 * i, (uint32_t)s_list[i]);
                st_remote_u32(to + 8 * i + 4, (uint32_t)(s_list[i] >> 32));
            }
            asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
            if (rank != 0) return;
            // an element's place is the number of larger ones, by bisection of all lists at once
            for (int i = tid; i < cluster * a.k; i += THREADS) {
                const unsigned long long o = s_lists[i / a.k * kMaxTop + i % a.k];
                int larger[kMaxCluster] = {}, place = 0;
                for (int step = kMaxTop; step > 0; step >>= 1) {
                    if (step > a.k) continue;
#pragma unroll
                    for (int q = 0; q < kMaxCluster; q++)
                        if (q < cluster && larger[q] + step <= a.k && s_lists[q * kMaxTop + larger[q] + step - 1] > o) larger[q] += step;
                }
#pragma unroll
                for (int q = 0; q < kMaxCluster; q++) place += larger[q];
                if (o && place < a.k) s_list[place] = o;
            }
            __syncthreads();
        }
        for (int i = tid; i < a.k; i += THREADS) {
            if (a.top_logp) a.top_logp[r * a.k + i] = logp_of(value_of(s_list[i]));
            if (a.top_ids) a.top_ids[r * a.k + i] = index_of(s_list[i]);
        }
    }
}

template <typename T, bool TOP, bool ENT, int THREADS>
__global__ void __launch_bounds__(THREADS) token_logprobs_kernel(const T *__restrict__ logits, ScoreArgs a, int cluster) {
    pdl_enter();
    if (gated_off(a.gate)) return;
    score_row<T, TOP, ENT, THREADS>(logits, a, cluster);
    // (the last block of the first row: where a row has several, another one writes the results)
    if ((int)blockIdx.x == cluster - 1 && a.hdr && a.scan)
        report_first(a.tokens, a.tokens ? a.rows : 0, 1, a.hdr,
                     [&](int64_t y, int64_t) { return y != a.ignore && (y < 0 || y >= a.vocab); });
}

// dz = (dlogp (1[y] - p) + dlse p - dH p (log p + H)) / tau.  Reads and writes the row once; about ten operations an
// element, so that two bytes in and two out still leave HBM the bound.
struct ScoreGradArgs {
    const int64_t *tokens;      // optional
    int64_t ignore, ld, ldd;
    int vocab;
    Heat heat;
    const float *lse, *entropy, *d_logp, *d_lse, *d_entropy;    // entropy with d_entropy; the three gradients are optional
};
constexpr int kGradThreads = 256, kGradGroups = 4, kGradRounds = 4;
template <typename T, bool LO>
__global__ void __launch_bounds__(kGradThreads) token_logprobs_bwd_kernel(const T *logits, T *d_logits, ScoreGradArgs a) {
    pdl_enter();
    constexpr int N = RowGroups<T>::N, H = N / 2;
    const int64_t r = blockIdx.x;
    T *d = d_logits + r * a.ldd;
    const RowGroups<T> out(d, a.vocab), in(logits + r * a.ld, a.vocab);
    const int64_t y = a.tokens ? a.tokens[r] : -1;
    const bool none = a.lse[r] == -INFINITY;       // every logit is -inf: p is 0
    const float lse = none ? 0.f : a.lse[r];
    const float gp = a.d_logp ? a.d_logp[r] : 0.f, gl = a.d_lse ? a.d_lse[r] : 0.f, gh = a.d_entropy ? a.d_entropy[r] : 0.f;
    const float ent = a.d_entropy ? a.entropy[r] : 0.f, tau = a.heat.hi;
    const bool part = !a.tokens || (y != a.ignore && y >= 0 && y < a.vocab), same = in.off == out.off;
    const float c0 = (gl - gp - gh * ent) * tau, c1 = -gh * tau;
    // log p below this (-inf among them) counts as this: p is 0, and so is its product with log p.  (log p and not the logit, whose
    // bound lse - 1e4 would be lse itself where lse is large: p of a masked token 1.)
    constexpr float kLeast = -1e4f, kLowest = -3.402823466e38f;
    const int per_block = kGradRounds * kGradGroups * kGradThreads;
    const int g0 = blockIdx.y * per_block, g1 = min(out.groups, g0 + per_block);
    const float inv_hi = a.heat.hi, inv_lo = a.heat.lo;
    auto grad = [&](Pair z) {
        float l[2], q[2];
        Pair lp = fma2(z, Pair(inv_hi, inv_hi), Pair(-lse, -lse));
        if (LO) {
            z.get(l[0], l[1]);          // (-inf times the second part of 1 / tau may be +inf)
            lp = fma2(Pair(max_nan(l[0], kLowest), max_nan(l[1], kLowest)), Pair(inv_lo, inv_lo), lp);
        }
        lp.get(l[0], l[1]);
        lp = Pair(max_nan(l[0], kLeast), max_nan(l[1], kLeast));
        (lp * Pair(kLog2e, kLog2e)).get(q[0], q[1]);
        return Pair(exp2_approx(q[0]), exp2_approx(q[1])) * fma2(lp, Pair(c1, c1), Pair(c0, c0));
    };
    if (part && same) {
        const int w0 = max(g0, out.whole_begin()), w1 = min(g1, out.whole_end());
        const int at = part && a.d_logp ? (int)((y + out.off) / N) : -1, in_at = (int)((y + out.off) % N);     // the token's group
        auto one = [&](int v, const Raw<T> &x) {
            Pair p[H];
            x.pairs(p);
            Vec<T> o;
#pragma unroll
            for (int i = 0; i < H; i++) grad(p[i]).get(o.v[2 * i], o.v[2 * i + 1]);
            if (v == at) {
#pragma unroll
                for (int i = 0; i < N; i++)
                    if (i == in_at) o.v[i] = fmaf(gp, tau, o.v[i]);
            }
            o.store(d + out.first(v));
        };
        Raw<T> x[kGradGroups];
        int v0 = w0 + threadIdx.x;
        for (; v0 + (kGradGroups - 1) * kGradThreads < w1; v0 += kGradGroups * kGradThreads) {
#pragma unroll
            for (int u = 0; u < kGradGroups; u++) in.load_whole(v0 + u * kGradThreads, x[u]);
#pragma unroll
            for (int u = 0; u < kGradGroups; u++) one(v0 + u * kGradThreads, x[u]);
        }
#pragma unroll
        for (int u = 0; u < kGradGroups; u++)
            if (v0 + u * kGradThreads < w1) in.load_whole(v0 + u * kGradThreads, x[u]);
#pragma unroll
        for (int u = 0; u < kGradGroups; u++)
            if (v0 + u * kGradThreads < w1) one(v0 + u * kGradThreads, x[u]);
    }
    // element by element: the ragged ends, rows that start elsewhere than their gradient, zeros
    auto slow = [&](int v) {
        const int e0 = out.first(v);
        Vec<T> o;
#pragma unroll
        for (int i = 0; i < H; i++) {
            const int e = e0 + 2 * i;
            Pair g(0.f, 0.f);
            if (part)
                g = grad(Pair(e >= 0 && e < a.vocab ? to_f32(logits[r * a.ld + e]) : 0.f,
                              e + 1 >= 0 && e + 1 < a.vocab ? to_f32(logits[r * a.ld + e + 1]) : 0.f));
            g.get(o.v[2 * i], o.v[2 * i + 1]);
#pragma unroll
            for (int j = 0; j < 2; j++)
                if (part && e + j == y) o.v[2 * i + j] = fmaf(gp, tau, o.v[2 * i + j]);
        }
        if (out.whole(v)) {
            o.store(d + e0);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++)
                if (e0 + i >= 0 && e0 + i < a.vocab) d[e0 + i] = from_f32<T>(o.v[i]);
        }
    };
    if (!part || !same) {
        for (int v = g0 + threadIdx.x; v < g1; v += kGradThreads) slow(v);
    } else if (threadIdx.x < 2 && g0 < g1) {
        const int v = threadIdx.x ? g1 - 1 : g0;
        if (!out.whole(v) && !(threadIdx.x && v == g0)) slow(v);
    }
}

// Where rows fill the GPU several times, blocks of 256 threads take one each; fewer rows are cut over as many blocks of 1024
// as fit at once (one an SM), none with less than a batch of loads a thread.
constexpr int64_t kFewRows = 148;
template <typename T>
int row_cluster(int64_t rows, int64_t vocab) {
    int c = 1;
    while (c < kMaxCluster && rows * 2 * c <= 148 && vocab / (2 * c) >= kFewThreads * Vec<T>::N) c *= 2;
    return c;
}
template <typename T, bool TOP, bool ENT>
int launch_score(const T *logits, const ScoreArgs &a, cudaStream_t st) {
    if (a.rows > kFewRows || a.vocab <= kManyThreads * 4 * Vec<T>::N)
        return launch_clusters(token_logprobs_kernel<T, TOP, ENT, kManyThreads>, dim3((unsigned)a.rows), kManyThreads, 0, 1, 1, st, logits, a, 1);
    const int c = row_cluster<T>(a.rows, a.vocab);
    return launch_clusters(token_logprobs_kernel<T, TOP, ENT, kFewThreads>, dim3((unsigned)(a.rows * c)), kFewThreads, 0, c, 1, st, logits, a, c);
}
}  // namespace

template <typename T>
int token_logprobs(const T *logits, int64_t ld, int64_t rows, int64_t vocab, const int64_t *tokens, int64_t ignore,
                   float temperature, int k, float *logp, float *lse, float *entropy, float *top_logp, int64_t *top_ids,
                   WsHeader *hdr, cudaStream_t st) {
    const bool scan = rows <= kScanMost || vocab * (int64_t)sizeof(T) >= kScanRow;
    if (hdr && !scan) SBP_TRY(clear_status_launch(hdr, st));
    const ScoreArgs a{tokens, ignore, rows, ld, (int)vocab, k, make_heat(temperature), logp, lse, entropy, top_logp, top_ids, hdr, scan,
                      call_state().gate};
    if (k) return entropy ? launch_score<T, true, true>(logits, a, st) : launch_score<T, true, false>(logits, a, st);
    return entropy ? launch_score<T, false, true>(logits, a, st) : launch_score<T, false, false>(logits, a, st);
}
template <typename T>
int token_logprobs_bwd(const T *logits, int64_t ld, int64_t rows, int64_t vocab, const int64_t *tokens, int64_t ignore,
                       float temperature, const float *lse, const float *entropy, const float *d_logp, const float *d_lse,
                       const float *d_entropy, T *d_logits, int64_t ldd, cudaStream_t st) {
    const ScoreGradArgs a{tokens, ignore, ld, ldd, (int)vocab, make_heat(temperature), lse, entropy, d_logp, d_lse, d_entropy};
    const int64_t groups = (vocab + Vec<T>::N - 1) / Vec<T>::N + 1, per = kGradThreads * kGradGroups * kGradRounds;
    auto kernel = a.heat.lo != 0.f ? token_logprobs_bwd_kernel<T, true> : token_logprobs_bwd_kernel<T, false>;
    SBP_LAUNCH(kernel, dim3((unsigned)rows, (unsigned)((groups + per - 1) / per)), kGradThreads, 0, st, logits,
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
