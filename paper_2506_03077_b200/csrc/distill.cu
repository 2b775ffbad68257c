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
constexpr int kThreads = 512, kCompute = kThreads - 32, kComputeWarps = kCompute / 32, kMaxTop = STREAMBP_TOP_MAX, kMaxCluster = 8;

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

// What a block knows of its segment of a row, for the others: the maximum m, the sums of exp((z - m) / tau) over its tokens
// (with a tail: over the unlisted and over the listed ones), and sum q (log q - z / tau) over the entries that lie in it.
struct Segment {
    float m, S, rest, pad;
    double loss;
};
struct Entries {
    int id[kMaxTop], place[kMaxTop], first[kMaxTop];    // the token (-1: none), where its logit lies in this block's shared memory (-1: elsewhere), the entry that lists it first
    float z[kMaxTop], q[kMaxTop], q_all[kMaxTop];       // of the first entry of a token; q_all: the q of all its entries
    double logq[kMaxTop];
    double mass, rest;                                  // sum of the q, and what is left for the tail
    float mass_f, rest_f;
};

// The row's entries, by one warp.  With a tail what is left of 1 is a difference, so those exponentials are taken in 64 bits.
__device__ __forceinline__ void read_entries(const DistillArgs &a, int64_t r, Entries &s) {
    constexpr int J = kMaxTop / 32;
    const int lane = threadIdx.x & 31;
    float t[J], top = -INFINITY;
    int id[J];
    bool any = false;
#pragma unroll
    for (int j = 0; j < J; j++) {
        const int i = lane + 32 * j;
        id[j] = -1;
        t[j] = -INFINITY;
        if (i < a.k) {
            const int64_t x = a.ids[r * a.k + i];
            const float v = a.values[r * a.k + i];
            if (x >= 0 && x < a.vocab) {
                id[j] = (int)x;
                t[j] = v;
                any = true;
            }
            s.id[i] = id[j];
        }
        top = fmaxf(top, t[j]);
    }
    if (a.tail) {
        double q[J], sum = 0.0;
#pragma unroll
        for (int j = 0; j < J; j++) {
            q[j] = 0.0;
            if (32 * j < a.k && id[j] >= 0) q[j] = exp((double)t[j]);
            sum += q[j];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
#pragma unroll
        for (int j = 0; j < J; j++)
            if (lane + 32 * j < a.k) {
                s.q[lane + 32 * j] = (float)q[j];
                s.logq[lane + 32 * j] = (double)t[j];
            }
        any = __any_sync(0xffffffffu, any);
        if (lane == 0) s.rest = any ? fmax(0.0, 1.0 - sum) : 0.0;
    } else {
        top = warp_max(top);
        const float t0 = finite_or_zero(top);
        float q[J], sum = 0.f;
#pragma unroll
        for (int j = 0; j < J; j++) {
            q[j] = id[j] < 0 ? 0.f : expf(fmaf(t[j] - t0, a.heat.hi, (t[j] - t0) * a.heat.lo));
            if (t[j] == -INFINITY) q[j] = 0.f;
            sum += q[j];
        }
        sum = warp_sum(sum);
        const double inv = (double)a.heat.hi + (double)a.heat.lo, logsum = (double)logf(sum);
        const float over = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int j = 0; j < J; j++)
            if (lane + 32 * j < a.k) {
                s.q[lane + 32 * j] = q[j] * over;
                s.logq[lane + 32 * j] = ((double)t[j] - (double)t0) * inv - logsum;
            }
        if (lane == 0) s.rest = 0.0;
    }
    // (of the q as they are held, so that their roundings weigh log q - log p and not each of the two)
    __syncwarp();
    double mass = 0.0;
#pragma unroll
    for (int j = 0; j < J; j++)
        if (lane + 32 * j < a.k) mass += (double)s.q[lane + 32 * j];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, o);
    if (lane == 0) {
        s.mass = mass;
        s.mass_f = (float)mass;
        s.rest_f = (float)s.rest;
    }
}

// Which entries lie in elements e0 .. e1 - 1 (at s_row + id - first), and which list the same token; by the same warp.  A hash
// table (kHash ints) tells whether any token is listed twice; only then every pair is looked at.
constexpr int kHash = 512;
__device__ __forceinline__ void place_entries(const DistillArgs &a, int e0, int e1, int first_element, Entries &s, int *table) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < kHash / 128; i++) reinterpret_cast<int4 *>(table)[lane + 32 * i] = make_int4(-1, -1, -1, -1);
    __syncwarp();
    bool twice = false;
    for (int i = lane; i < a.k; i += 32) {
        const int id = s.id[i];
        if (id < 0) continue;
        for (uint32_t at = (uint32_t)id * 2654435761u >> 23;; at = (at + 1) & (kHash - 1)) {       // (at most kMaxTop of the places are taken)
            const int was = atomicCAS(table + at, -1, id);
            twice |= was == id;
            if (was == -1 || was == id) break;
        }
    }
    twice = __any_sync(0xffffffffu, twice);
    for (int i = lane; i < a.k; i += 32) {
        const int id = s.id[i];
        int first = i;
        float q = s.q[i];
        if (twice && id >= 0) {
            q = 0.f;
            for (int j = a.k - 1; j >= 0; j--)
                if (s.id[j] == id) {
                    first = j;
                    q += s.q[j];
                }
        }
        s.first[i] = first;
        s.q_all[i] = q;
        s.place[i] = id >= e0 && id < e1 ? id - first_element : -1;
    }
}

__device__ __forceinline__ void compute_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kCompute) : "memory"); }

// The part of a row that one block of a cluster holds.
template <typename T, typename TO>
struct RowSegment {
    int n, groups, g0, w0, w1, e0, e1, first;     // groups in all and from where; the whole ones among them (counted from g0); elements, and the one at the start of the block's buffer
    __device__ __forceinline__ RowSegment(const T *p, int vocab, int rank, int log_cluster) {
        const RowGroups<T> row(p, vocab);
        n = vocab;
        const int per = (row.groups + (1 << log_cluster) - 1) >> log_cluster;
        g0 = min(rank * per, row.groups);
        const int g1 = min(g0 + per, row.groups);
        groups = g1 - g0;
        w0 = max(g0, row.whole_begin()) - g0;
        w1 = max(w0, min(g1, row.whole_end()) - g0);
        first = row.first(g0);
        e0 = max(0, first);
        e1 = g1 > g0 ? min(vocab, row.first(g1)) : e0;
    }
    // by one warp: the whole groups by the copy engine, the ragged ends element by element; all of it reports to `bar`
    __device__ __forceinline__ void copy(const T *p, T *s_row, uint32_t bar) const {
        constexpr int N = RowGroups<T>::N;
        const int lane = threadIdx.x & 31, end = lane / N, v = end ? groups - 1 : 0;
        if (end < 2 && groups > 0 && (v < w0 || v >= w1)) {
            const int e = first + v * N + lane % N;
            s_row[v * N + lane % N] = e >= 0 && e < n ? p[e] : from_f32<T>(-INFINITY);
        }
        __syncwarp();
        if (lane == 0) {
            const uint32_t bytes = (uint32_t)(w1 - w0) * 16;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // (what was read and written here before comes first)
            mbar_expect_tx(bar, bytes);
            if (bytes)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                                 smem_u32(s_row + w0 * N)), "l"(p + (first + w0 * N)), "r"(bytes), "r"(bar)
                             : "memory");
        }
        __syncwarp();
    }
    __device__ __forceinline__ void zeros(TO *d) const {
        constexpr int NO = Vec<TO>::N;
        const RowGroups<TO> out(d + e0, e1 - e0);
        Vec<TO> zero;
#pragma unroll
        for (int i = 0; i < NO; i++) zero.v[i] = 0.f;
        for (int v = threadIdx.x; v < out.groups; v += kCompute) {
            const int f = out.first(v);
            if (out.whole(v)) {
                zero.store(d + e0 + f);
            } else {
#pragma unroll
                for (int i = 0; i < NO; i++)
                    if (f + i >= 0 && f + i < e1 - e0) d[e0 + f + i] = from_f32<TO>(0.f);
            }
        }
    }
};

// Persistent clusters of up to eight blocks, two blocks an SM (so that one's loads, barriers and stores are the other's time to
// compute), take rows in turn.  A row's logits stay in the blocks' shared memory from the sums to the gradient, so they are
// read from HBM once and the gradient is written once, which is what bounds the kernel.  The last warp reads and places
// the next row's entries, writes the listed tokens' gradients of the row before over those of the streaming pass, and its
// loss.  With a tail the listed tokens are taken out of the row first (their logits become -inf), so that the mass of the others is a
// sum of its own and not a difference.
template <typename T, typename TO>
__global__ void __launch_bounds__(kThreads, 2) distill_kernel(const T *logits, TO *d_logits, DistillArgs a, int log_cluster) {
    pdl_enter();
    if (gated_off(a.gate)) return;
    constexpr int N = RowGroups<T>::N, U = 4, NO = Vec<TO>::N;
    extern __shared__ __align__(128) unsigned char s_raw[];
    __shared__ __align__(16) int s_hash[kHash];
    __shared__ __align__(8) unsigned long long s_bar;       // the row is there
    __shared__ int s_abort;
    __shared__ RowStats s_warp[kComputeWarps];
    // (a block may post a row's statistics while another's last warp finishes the row two before: four places)
    __shared__ Segment s_seg[4][kMaxCluster];
    __shared__ Entries s_entries[2];
    __shared__ float s_at[2], s_of_p[2], s_rest[2], s_total[2];
    const int cluster = 1 << log_cluster, rank = (int)(blockIdx.x & (cluster - 1)), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t step = gridDim.x >> log_cluster;
    const float c = a.heat.hi * kLog2e;
    const bool reader = warp == kComputeWarps;
    auto weight = [&](int64_t r) { return r < a.rows ? (a.weight ? a.weight[r] : 1.f) : 0.f; };
    // (rows that start alike in their 16 bytes are cut alike)
    const bool alike = (a.ld * sizeof(T)) % 16 == 0;
    RowSegment<T, TO> sg(logits, a.vocab, rank, log_cluster);
    auto segment = [&](int64_t r) { return alike ? sg : RowSegment<T, TO>(logits + r * a.ld, a.vocab, rank, log_cluster); };
    // the last warp's part for a row that is done but for its listed tokens
    auto finish = [&](int64_t r, float w, int slot, int at_seg) {
        const Entries &s = s_entries[slot];
        const float at = s_at[slot], total = s_total[slot], rest = s_rest[slot];
        const double rest_q = rest == 0.f ? 0.0 : s.rest;
        const bool none = s.mass_f == 0.f && s.rest_f == 0.f;
        const float scale = fmaf(w, a.heat.hi, w * a.heat.lo), of_p = s_of_p[slot];
        if (d_logits && !none)
            for (int i = lane; i < a.k; i += 32)
                if (s.place[i] >= 0 && s.first[i] == i)
                    d_logits[r * a.ldd + s.id[i]] = from_f32<TO>(scale * fmaf(of_p, exp2_approx((s.z[i] - at) * c), -s.q_all[i]));
        if (rank == 0 && a.row_loss) {
            double loss = lane < cluster ? s_seg[at_seg][lane].loss : 0.0;
#pragma unroll
            for (int o = kMaxCluster / 2; o > 0; o >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, o);
            const double inv = (double)a.heat.hi + (double)a.heat.lo, logS = total == 0.f ? 0.0 : (double)logf(total);
            if (s.mass != 0.0) loss += s.mass * ((double)at * inv + logS);
            if (rest_q != 0.0) loss += rest_q * (double)(logf((float)rest_q) - logf(rest / total));
            if (lane == 0) a.row_loss[r] = none ? 0.f : (float)loss;
        }
    };
    int64_t r = blockIdx.x >> log_cluster;
    float w = weight(r), w_next = weight(r + step), w_before = 0.f;
    const uint32_t bar = smem_u32(&s_bar);
    T *s_row = reinterpret_cast<T *>(s_raw);
    uint32_t parity = 0;
    if (tid == 0) {
        s_abort = 0;
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (reader) {
        if (w != 0.f) {
            const RowSegment<T, TO> seg = segment(r);
            read_entries(a, r, s_entries[0]);
            place_entries(a, seg.e0, seg.e1, seg.first, s_entries[0], s_hash);
        }
    }
    if (cluster > 1) cluster_sync_all();        // (all blocks are there before one writes into another's memory)
    __syncthreads();
    int slot = 0, turn = 0;
    for (; r < a.rows; r += step, slot ^= 1, turn = (turn + 1) & 3) {
        const float w_later = weight(r + 2 * step);
        if (reader) {
            // (after a wait that ran out nothing more is copied)
            if (w != 0.f && *(volatile int *)&s_abort == 0) segment(r).copy(logits + r * a.ld, s_row, bar);
            if (w != 0.f && cluster > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
            if (w_before != 0.f) finish(r - step, w_before, slot ^ 1, (turn + 3) & 3);
            __syncwarp();
            if (w_next != 0.f) {
                const RowSegment<T, TO> seg = segment(r + step);
                read_entries(a, r + step, s_entries[slot ^ 1]);
                place_entries(a, seg.e0, seg.e1, seg.first, s_entries[slot ^ 1], s_hash);
            }
            if (w == 0.f && rank == 0 && lane == 0 && a.row_loss) a.row_loss[r] = 0.f;
            if (w != 0.f && cluster > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        } else {
            if (!alike) sg = segment(r);
            TO *d = d_logits ? d_logits + r * a.ldd : nullptr;
            if (w == 0.f) {         // the row takes no part
                if (d) sg.zeros(d);
            } else {
                Entries &s = s_entries[slot];
                mbar_wait(bar, parity, &s_abort);
                parity ^= 1;
                if (a.tail) {
                    if (tid < a.k && s.place[tid] >= 0 && s.first[tid] == tid) {
                        s.z[tid] = to_f32(s_row[s.place[tid]]);
                        s_row[s.place[tid]] = from_f32<T>(-INFINITY);
                    }
                    compute_sync();
                }
                const int n = sg.groups;
                Running<T, false, U> run;
                auto at_group = [&](int v) { return *reinterpret_cast<const uint4 *>(s_row + v * N); };
                int v = tid;
                for (; v + (U - 1) * kCompute < n; v += U * kCompute) {
                    Raw<T> x[U];
#pragma unroll
                    for (int u = 0; u < U; u++) x[u].w = at_group(v + u * kCompute);
                    run.add(x, c);
                }
                if (v < n) {
                    Raw<T> x[U];
#pragma unroll
                    for (int u = 0; u < U; u++) {
                        if (v + u * kCompute < n) x[u].w = at_group(v + u * kCompute);
                        else x[u].fill(-INFINITY);
                    }
                    run.add(x, c);
                }
                float m = run.m, S;
                {
                    float lo, hi;
                    run.S.get(lo, hi);
                    S = lo + hi;
                }
                // over the lanes of a warp
                auto joined = [&] {
                    const float top = warp_max(m), at = finite_or_zero(top);
                    S = warp_sum(S * exp2_approx((m - at) * c));
                    m = top;
                };
                joined();
                if (lane == 0) s_warp[warp] = RowStats{m, S, 0.f};
                compute_sync();
                if (warp == 0) {
                    const RowStats st = lane < kComputeWarps ? s_warp[lane] : RowStats{-INFINITY, 0.f, 0.f};
                    m = st.m;
                    S = st.S;
                    joined();
                    float rest = S;
                    if (a.tail) {       // the listed tokens come back
                        float top = m;
                        for (int i = lane; i < a.k; i += 32)
                            if (s.place[i] >= 0 && s.first[i] == i) top = fmaxf(top, s.z[i]);
                        top = warp_max(top);
                        const float at = finite_or_zero(top);
                        rest = S * exp2_approx((m - at) * c);
                        float listed = 0.f;
                        for (int i = lane; i < a.k; i += 32)
                            if (s.place[i] >= 0 && s.first[i] == i) listed += exp2_approx((s.z[i] - at) * c);
                        S = rest + warp_sum(listed);
                        m = top;
                    }
                    if (lane < cluster) {
                        const uint32_t to = map_to_cta(smem_u32(&s_seg[turn][rank]), lane);
                        st_remote_u32(to, __float_as_uint(m));
                        st_remote_u32(to + 4, __float_as_uint(S));
                        st_remote_u32(to + 8, __float_as_uint(rest));
                    }
                } else if (warp == 1) {
                    const double inv = (double)a.heat.hi + (double)a.heat.lo;
                    double loss = 0.0;
                    for (int i = lane; i < a.k; i += 32) {
                        if (s.place[i] < 0) continue;
                        if (!a.tail) s.z[i] = to_f32(s_row[s.place[i]]);
                        const float q = s.q[i];
                        if (q != 0.f) loss += (double)q * (s.logq[i] - (double)(a.tail ? s.z[s.first[i]] : s.z[i]) * inv);
                    }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, o);
                    if (lane < cluster) st_remote_f64(map_to_cta(smem_u32(&s_seg[turn][rank].loss), lane), loss);
                }
                __syncwarp();
                if (cluster > 1) asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
                else compute_sync();
                // the row: every eight lanes join the segments for themselves
                Segment g{-INFINITY, 0.f, 0.f, 0.f, 0.0};
                if ((lane & (kMaxCluster - 1)) < cluster) g = s_seg[turn][lane & (kMaxCluster - 1)];
                float at = g.m;
#pragma unroll
                for (int o = kMaxCluster / 2; o > 0; o >>= 1) at = fmaxf(at, __shfl_xor_sync(0xffffffffu, at, o));
                at = finite_or_zero(at);
                const float f = exp2_approx((g.m - at) * c);
                float total = g.S * f, rest = g.rest * f;
#pragma unroll
                for (int o = kMaxCluster / 2; o > 0; o >>= 1) {
                    total += __shfl_xor_sync(0xffffffffu, total, o);
                    if (a.tail) rest += __shfl_xor_sync(0xffffffffu, rest, o);
                }
                const float mass = s.mass_f, rest_q = a.tail && rest != 0.f ? s.rest_f : 0.f;      // (or there is no token for the tail)
                const bool none = mass == 0.f && s.rest_f == 0.f;                                   // no entries: the row takes no part
                const float of_p = total == 0.f ? 0.f : (mass + rest_q) / total, scale = fmaf(w, a.heat.hi, w * a.heat.lo);
                const float factor = scale * (of_p - (rest_q != 0.f ? rest_q / rest : 0.f));
                if (tid == 0) {
                    s_at[slot] = at;
                    s_of_p[slot] = of_p;
                    s_rest[slot] = rest;
                    s_total[slot] = total;
                }
                if (d && none) {
                    sg.zeros(d);
                } else if (d) {
                    auto grad = [&](Pair z) {
                        float x[2];
                        ((z + Pair(-at, -at)) * Pair(c, c)).get(x[0], x[1]);
                        return Pair(exp2_approx(x[0]), exp2_approx(x[1])) * Pair(factor, factor);
                    };
                    TO *to = d + sg.e0;
                    const RowGroups<TO> out(to, sg.e1 - sg.e0);
                    const T *from = s_row + (sg.e0 - sg.first);
                    const int lead = sg.e0 - sg.first - out.off;         // element 0 of out's group 0 lies at s_row + lead
                    const int whole = out.whole_end();
                    if (lead % N == 0) {
                        // groups of the gradient are made of whole groups of the row
                        for (int v = tid + out.whole_begin(); v < whole; v += kCompute) {
                            Vec<TO> o;
#pragma unroll
                            for (int i = 0; i < NO; i += N) {
                                Raw<T> x;
                                x.w = *reinterpret_cast<const uint4 *>(s_row + lead + v * NO + i);
                                Pair p[N / 2];
                                x.pairs(p);
#pragma unroll
                                for (int j = 0; j < N / 2; j++) grad(p[j]).get(o.v[i + 2 * j], o.v[i + 2 * j + 1]);
                            }
                            o.store(to + out.first(v));
                        }
                    } else {
                        for (int v = tid + out.whole_begin(); v < whole; v += kCompute) {
                            Vec<TO> o;
                            const int f = out.first(v);
#pragma unroll
                            for (int i = 0; i < NO; i += 2) grad(Pair(to_f32(from[f + i]), to_f32(from[f + i + 1]))).get(o.v[i], o.v[i + 1]);
                            o.store(to + f);
                        }
                    }
                    if (tid < 2 * NO) {         // the ragged ends (one group at each, which may be the same one)
                        const int v = tid < NO ? 0 : out.groups - 1, f = out.first(v) + tid % NO;
                        if (out.groups > 0 && !out.whole(v) && !(tid >= NO && v == 0) && f >= 0 && f < out.n) {
                            float g, unused;
                            grad(Pair(to_f32(from[f]), 0.f)).get(g, unused);
                            to[f] = from_f32<TO>(g);
                        }
                    }
                }
            }
        }
        __syncthreads();
        w_before = w;
        w = w_next;
        w_next = w_later;
    }
    if (reader && w_before != 0.f) finish(r - step, w_before, slot ^ 1, (turn + 3) & 3);
    // (the last block of the first cluster looks through the ids)
    if ((int)blockIdx.x == cluster - 1 && a.hdr)
        report_first(a.ids, a.rows * a.k, a.k, a.hdr, [&](int64_t id, int64_t i) {
            return (id < -1 || id >= a.vocab) && (!a.weight || a.weight[i / a.k] != 0.f);
        });
}

// Blocks to a row: as few as hold it with two blocks an SM, and more where there are SMs for them and each thread keeps a
// group.  Rows that eight such blocks do not hold have one block an SM.
constexpr int kShared = 100 << 10, kSharedLong = 208 << 10;
template <typename T>
int row_cluster(int64_t rows, int64_t vocab) {
    int c = 1;
    while (c < kMaxCluster && (vocab * (int64_t)sizeof(T) + 32 * c > (int64_t)c * kShared ||
                               (rows * 2 * c <= 148 && vocab / (2 * c) >= kCompute * Vec<T>::N)))
        c *= 2;
    return c;
}

// Clusters of c blocks that the GPU holds at once.
template <typename F>
int resident_clusters(F kernel, int c, int smem) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)(296 / c * c));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cudaLaunchAttribute attr[1];
    memset(attr, 0, sizeof(attr));
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)c;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (!cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedLong)) ||
        !cuda_ok(cudaOccupancyMaxActiveClusters(&n, kernel, &cfg)))
        return 0;
    return n;
}

template <typename T, typename TO>
int launch(const T *logits, TO *d_logits, const DistillArgs &a, cudaStream_t st) {
    const int c = row_cluster<T>(a.rows, a.vocab);
    const int64_t groups = (a.vocab + Vec<T>::N - 1) / Vec<T>::N + 1;
    const int smem = (groups + c - 1) / c * 16 <= kShared ? kShared : kSharedLong;
    static PerDevice clusters[2][4];
    auto kernel = distill_kernel<T, TO>;
    int log_c = 0;
    while (1 << log_c < c) log_c++;
    const int most = clusters[smem == kSharedLong][log_c].get([&] { return resident_clusters(kernel, c, smem); });
    if (most < 1) return STREAMBP_E_CUDA;
    // (rows are dealt out evenly)
    const int64_t turns = (a.rows + most - 1) / most, n = (a.rows + turns - 1) / turns;
    return launch_clusters(kernel, dim3((unsigned)(n * c)), kThreads, smem, c, 1, st, logits, d_logits, a, log_c);
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
int distill_take_fault() { return take_fault_local(); }
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
