// Distillation from a teacher's top logits: the loss of a row and the gradient of its logits.
//
// A row has k entries (id c_i, value t_i) and a weight w.  p = softmax(z / tau) over the whole vocabulary.
//   list only:  q = softmax(t / tau) over the entries,   L = sum q_i (log q_i - log p_ci),  Q = 1, q_r = 0
//   with tail:  q_i = exp t_i,  q_r = 1 - sum q_i,  L as above + q_r log(q_r / p_r),  p_r the mass of unlisted tokens,  Q = sum q_i + q_r
//   dL/dz_j = (Q p_j - sum_{c_i = j} q_i) / tau for listed j,  (Q p_j - q_r p_j / p_r) / tau for the others
//
// Bound by HBM, one reading and one writing of a row, as far as the phases of a block (entries, sums, the others' sums, gradient)
// hide one another's.  Measured: 1024 x 152064 fp32 with 32 entries 220 us (5.7 TB/s), 2048 x 32000 with 64 and a tail 101 (5.2);
// bf16 has twice the exponentials a byte: 2048 x 152064 in 255 us (4.9), 1500 x 50001 with 100 entries and a tail 73 (3.7; two and
// a half rounds of rows on the GPU).  A maximum of its own for the unlisted tokens takes 1 us of the two with a tail.
#include <algorithm>

#include "vocab_rows.cuh"

namespace sbp {

namespace {
constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxTop = STREAMBP_TOP_MAX, kTopWarps = kMaxTop / 32, kMaxCluster = 8, kHash = 512;

struct DistillArgs {
    const int64_t *ids;
    const float *values, *weight;       // weight is optional
    float *row_loss;                    // optional
    int64_t rows, ld, ldd;
    int vocab, k;
    Heat heat;
    WsHeader *hdr;                      // optional: a row with an id outside the vocabulary goes there
    bool scan;                          // found by one block, else by each row's
    const int *gate;
};

__device__ __forceinline__ void st_remote_f64(uint32_t a, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(a), "d"(v) : "memory");
}

// What a block knows of its segment of a row, for the others: the maximum m and the sum S of exp((z - m) / tau) over its tokens
// (with a tail: over the listed ones, and the same of the unlisted ones by themselves), and sum q (log q - z / tau) over the
// entries that lie in it.
struct Segment {
    float m, S, m_rest, rest;
    double loss;
};

__device__ __forceinline__ double entry_sum(const double (*red)[2], int which) {
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kTopWarps; w++) s += red[w][which];
    return s;
}
// sums over the first kTopWarps warps (every thread of the block calls; one barrier), which stay in red for entry_sum
__device__ __forceinline__ void entry_sums(double &a, double &b, double (*red)[2]) {
    const int warp = threadIdx.x >> 5;
    if (warp < kTopWarps) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if ((threadIdx.x & 31) == 0) {
            red[warp][0] = a;
            red[warp][1] = b;
        }
    }
    __syncthreads();
    a = entry_sum(red, 0);
    b = entry_sum(red, 1);
}

// `cluster` blocks to a row, a segment each: the entries while the segment comes to L2, the sums while it streams in, the other
// blocks' sums, the gradient while it streams in again and out.  The second reading comes from L2 (row_cluster keeps what is under way well below its size), so
// HBM reads a row once and writes its gradient once, which is what bounds the kernel.  Thread i < k has entry i.
//
// With a tail the mass of the unlisted tokens has to be a sum of its own: a difference of two sums would lose it where the
// list has nearly all.  And it has a maximum of its own: relative to the row's it underflows where the student is sure of listed
// tokens (87 tau above the others), which is where the tail has most to say.  A bit for each group of 16 bytes tells the streaming
// sum to leave out groups with listed tokens, whose unlisted ones are added by the group's first entry.  Listed tokens' gradients
// are written over those of the streaming pass.
template <typename T, typename TO, bool TAIL>
__device__ __forceinline__ void distill_row(const T *logits, TO *d_logits, const DistillArgs &a, int cluster) {
    constexpr int N = RowGroups<T>::N, NO = Vec<TO>::N, U = 4;
    extern __shared__ uint32_t s_bits[];                // TAIL: a bit for each group of the segment
    __shared__ int s_hash[kHash], s_id[kMaxTop];
    __shared__ float s_q[kMaxTop], s_top[kTopWarps];
    __shared__ double s_red[kTopWarps][2], s_red2[kTopWarps][2];
    __shared__ float4 s_warp[kWarps];
    __shared__ Segment s_seg[kMaxCluster];
    const int64_t r = blockIdx.x / cluster;
    const int rank = (int)(blockIdx.x % cluster), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const float w = a.weight ? a.weight[r] : 1.f, c = a.heat.hi * kLog2e;
    const double inv = (double)a.heat.hi + (double)a.heat.lo;
    const T *z = logits + r * a.ld;
    const RowGroups<T> row(z, a.vocab);
    TO *d = d_logits ? d_logits + r * a.ldd : nullptr;
    const int per = (row.groups + cluster - 1) / cluster;
    const int g0 = min(rank * per, row.groups), g1 = min(g0 + per, row.groups);
    const int w0 = max(g0, row.whole_begin());
    int w1 = max(w0, min(g1, row.whole_end()));
    const int e0 = max(0, row.first(g0)), e1 = g1 > g0 ? min(a.vocab, row.first(g1)) : e0;      // elements of the segment
    auto zeros = [&] {
        if (!d) return;
        const RowGroups<TO> out(d + e0, e1 - e0);
        Vec<TO> zero;
#pragma unroll
        for (int i = 0; i < NO; i++) zero.v[i] = 0.f;
        for (int v = tid; v < out.groups; v += kThreads) {
            const int f = out.first(v);
            if (out.whole(v)) {
                zero.store(d + e0 + f);
            } else {
#pragma unroll
                for (int i = 0; i < NO; i++)
                    if (f + i >= 0 && f + i < e1 - e0) d[e0 + f + i] = from_f32<TO>(0.f);
            }
        }
    };
    // (asked for at once)
    int64_t id64 = -1;
    float t = -INFINITY;
    if (tid < a.k) {
        id64 = a.ids[r * a.k + tid];
        t = a.values[r * a.k + tid];
    }
    if (w == 0.f) {         // the row takes no part
        zeros();
        if (rank == 0 && tid == 0 && a.row_loss) a.row_loss[r] = 0.f;
        return;
    }
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // (waited for before the others' memory is written)
    // The segment is on its way to L2 while the entries are dealt with.  (Asked for only where the row has entries, that is once they
    // are there: 1024 x 152064 fp32 222 us for 219, 2048 x 32000 with a tail 102 for 101.)
    if (warp == kWarps - 1) {
        constexpr int kPiece = 1024;
        for (int v = w0 + lane * kPiece; v < w1; v += 32 * kPiece)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(row.base + (int64_t)v * N), "r"(16 * min(kPiece, w1 - v)) : "memory");
    }
    // entry tid
    int id = -1;
    if (id64 >= 0 && id64 < a.vocab) id = (int)id64;
    else if (id64 != -1 && a.hdr && !a.scan && rank == 0) set_status(a.hdr, STREAMBP_E_BAD_LABEL, (int)r);
    if (id < 0) t = -INFINITY;
    const bool here = id >= e0 && id < e1;
    const float zi = here ? to_f32(z[id]) : -INFINITY;
    // which token was listed before, which groups have listed tokens, the q
    if (tid < kMaxTop) {
        s_id[tid] = id;
        for (int i = tid; i < kHash; i += kMaxTop) s_hash[i] = -1;
        const float top = warp_max(t);
        if (lane == 0) s_top[warp] = top;
    }
    if (TAIL)
        for (int i = tid; i < (g1 - g0 + 31) / 32; i += kThreads) s_bits[i] = 0;
    __syncthreads();
    bool shared_group = false;          // any two of the segment's entries
    if (TAIL && here) {
        const int g = (id + row.off) / N - g0;
        shared_group = atomicOr(&s_bits[g >> 5], 1u << (g & 31)) >> (g & 31) & 1;
    }
    bool twice = false;
    if (id >= 0)
        for (uint32_t at = (uint32_t)id * 2654435761u >> 23;; at = (at + 1) & (kHash - 1)) {       // (at most kMaxTop of the places are taken)
            const int was = atomicCAS(&s_hash[at], -1, id);
            twice |= was == id;
            if (was == -1 || was == id) break;
        }
    const bool any_twice = __syncthreads_or(twice);
    if (TAIL) shared_group = __syncthreads_or(shared_group);
    float t0 = s_top[0];
#pragma unroll
    for (int i = 1; i < kTopWarps; i++) t0 = fmaxf(t0, s_top[i]);
    t0 = finite_or_zero(t0);
    // (with a tail what is left of 1 is a difference, so those exponentials are taken in 64 bits)
    double e = 0.0;
    if (id >= 0) e = TAIL ? exp((double)t) : t == -INFINITY ? 0.0 : (double)expf(fmaf(t - t0, a.heat.hi, (t - t0) * a.heat.lo));
    double sum = e, listed = id >= 0 ? 1.0 : 0.0;
    entry_sums(sum, listed, s_red);
    if (listed == 0.0) w1 = w0;         // no entries: none of the row's values is used (nor those of its ragged ends, below)
    const float q = TAIL ? (float)e : sum == 0.0 ? 0.f : (float)e / (float)sum;
    if (tid < kMaxTop) s_q[tid] = q;
    {
        double q_sum = (double)q, l = 0.0;      // (of the q as they are held, so that their roundings weigh log q - log p and not each of the two)
        if (here && q != 0.f) l = (double)q * ((TAIL ? (double)t : ((double)t - (double)t0) * inv - (double)logf((float)sum)) - (double)zi * inv);
        entry_sums(q_sum, l, s_red2);
    }
    // the entry that lists its token first has the q of all that do
    bool first = here;
    float q_all = q;
    if (any_twice && here) {
        q_all = 0.f;
        for (int j = a.k - 1; j >= 0; j--)
            if (s_id[j] == id) {
                first = j == tid;
                q_all += s_q[j];
            }
    }
    float m_own = -INFINITY, rest_own = 0.f;    // TAIL: of the unlisted tokens beside the entry's
    if (TAIL && here) {
        // the first entry of a group adds its unlisted tokens; each token's first entry the token
        const int g = (id + row.off) / N;
        bool of_group = true;
        uint32_t mask = 1u << ((id + row.off) % N);
        if (shared_group)
            for (int j = 0; j < a.k; j++) {
                const int other = s_id[j];
                if (other < e0 || other >= e1 || (other + row.off) / N != g) continue;
                if (j < tid) of_group = false;
                mask |= 1u << ((other + row.off) % N);
            }
        float x[N];
        row.load(g, x, -INFINITY);
#pragma unroll
        for (int i = 0; i < N; i++) {
            if (!of_group || (mask >> i & 1)) x[i] = -INFINITY;
            m_own = fmaxf(m_own, x[i]);
        }
        const float at = finite_or_zero(m_own);
#pragma unroll
        for (int i = 0; i < N; i++) rest_own += exp2_approx((x[i] - at) * c);
    }
    // the sums over the segment (TAIL: but for groups with listed tokens)
    Running<T, false> run;
    {
        auto skip = [&](int v, Raw<T> &x) {
            if (TAIL && (s_bits[(v - g0) >> 5] >> ((v - g0) & 31) & 1)) x.fill(-INFINITY);
        };
        Raw<T> x[U];
        int v = w0 + tid;
        for (; v + (U - 1) * kThreads < w1; v += U * kThreads) {
#pragma unroll
            for (int u = 0; u < U; u++) row.load_whole(v + u * kThreads, x[u]);
#pragma unroll
            for (int u = 0; u < U; u++) skip(v + u * kThreads, x[u]);
            run.add(x, c);
        }
        if (v < w1) {
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (v + u * kThreads < w1) row.load_whole(v + u * kThreads, x[u]);
                else x[u].fill(-INFINITY);
            }
#pragma unroll
            for (int u = 0; u < U; u++)
                if (v + u * kThreads < w1) skip(v + u * kThreads, x[u]);
            run.add(x, c);
        }
        if (tid >= kThreads - 2 && g0 < g1 && listed != 0.0) {      // the ragged ends (one group at each, which may be the same one)
            const int v = tid == kThreads - 2 ? g0 : g1 - 1;
            if ((v < w0 || v >= w1) && !(tid == kThreads - 1 && v == g0)) {
                Raw<T> y[1];
                row.load(v, y[0]);
                skip(v, y[0]);
                run.add(y, c);
            }
        }
    }
    const double mass = entry_sum(s_red2, 0), loss = entry_sum(s_red2, 1);
    const double rest_all = TAIL && entry_sum(s_red, 1) != 0.0 ? fmax(0.0, 1.0 - entry_sum(s_red, 0)) : 0.0;
    float m = run.m, S, m_rest = -INFINITY, rest = 0.f;
    {
        float lo, hi;
        run.S.get(lo, hi);
        S = lo + hi;
    }
    auto join = [&](float &m1, float &S1, float m2, float S2) {
        const float both = fmaxf(m1, m2), at = finite_or_zero(both);
        S1 = S1 * exp2_approx((m1 - at) * c) + S2 * exp2_approx((m2 - at) * c);
        m1 = both;
    };
    if (TAIL) {
        m_rest = m;
        rest = S;
        join(m_rest, rest, m_own, rest_own);
        m = fmaxf(-INFINITY, first ? zi : -INFINITY);           // (-inf for NaN, which S tells)
        S = first ? exp2_approx((zi - finite_or_zero(m)) * c) : 0.f;
    }
    auto joined = [&](int from) {          // over the lanes of a warp
#pragma unroll
        for (int o = from; o > 0; o >>= 1) {
            join(m, S, __shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, S, o));
            if (TAIL) join(m_rest, rest, __shfl_xor_sync(0xffffffffu, m_rest, o), __shfl_xor_sync(0xffffffffu, rest, o));
        }
    };
    joined(16);
    if (lane == 0) s_warp[warp] = make_float4(m, S, m_rest, rest);
    __syncthreads();
    if (warp == 0) {
        const float4 st = lane < kWarps ? s_warp[lane] : make_float4(-INFINITY, 0.f, -INFINITY, 0.f);
        m = st.x;
        S = st.y;
        m_rest = st.z;
        rest = st.w;
        joined(kWarps / 2);
        m = __shfl_sync(0xffffffffu, m, 0);
        S = __shfl_sync(0xffffffffu, S, 0);
        m_rest = __shfl_sync(0xffffffffu, m_rest, 0);
        rest = __shfl_sync(0xffffffffu, rest, 0);
        if (cluster > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        if (lane < cluster) {
            const uint32_t to = map_to_cta(smem_u32(&s_seg[rank]), lane);
            st_remote_u32(to, __float_as_uint(m));
            st_remote_u32(to + 4, __float_as_uint(S));
            if (TAIL) {
                st_remote_u32(to + 8, __float_as_uint(m_rest));
                st_remote_u32(to + 12, __float_as_uint(rest));
            }
            st_remote_f64(to + 16, loss);
        }
        __syncwarp();
    } else if (cluster > 1) {
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    else __syncthreads();
    // the row: every eight lanes join the segments for themselves
    Segment g{-INFINITY, 0.f, -INFINITY, 0.f, 0.0};
    if ((lane & (kMaxCluster - 1)) < cluster) g = s_seg[lane & (kMaxCluster - 1)];
    float at = g.m, at_rest = TAIL ? g.m_rest : -INFINITY;
#pragma unroll
    for (int o = kMaxCluster / 2; o > 0; o >>= 1) {
        at = fmaxf(at, __shfl_xor_sync(0xffffffffu, at, o));
        if (TAIL) at_rest = fmaxf(at_rest, __shfl_xor_sync(0xffffffffu, at_rest, o));
    }
    at = finite_or_zero(fmaxf(at, at_rest));
    float total = g.S * exp2_approx((g.m - at) * c);
    rest = TAIL ? g.rest * exp2_approx((g.m_rest - finite_or_zero(at_rest)) * c) : 0.f;
#pragma unroll
    for (int o = kMaxCluster / 2; o > 0; o >>= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, o);
        if (TAIL) rest += __shfl_xor_sync(0xffffffffu, rest, o);
    }
    const float lower = TAIL ? exp2_approx((at_rest - at) * c) : 0.f;      // turns sums relative to at_rest into sums relative to at
    if (TAIL) total = fmaf(rest, lower, total);
    // (rest is 0 where every unlisted logit is -inf, and at least 1 elsewhere: its largest term)
    const float rest_q = TAIL && rest != 0.f ? (float)rest_all : 0.f;
    const bool none = mass == 0.0 && rest_all == 0.0;                       // no entries, or all of q = 0: the row takes no part
    const float of_p = total == 0.f ? 0.f : ((float)mass + rest_q) / total, scale = fmaf(w, a.heat.hi, w * a.heat.lo);
    // An unlisted token's gradient is (Q p_j - q_r p_j / p_r) w / tau.  Both terms are multiples of exp((z_j - at_rest) / tau), which
    // does not underflow where p_j / p_r matters.  (A listed token's may overflow there: its gradient is written over it.)
    const float from_at = rest_q != 0.f ? at_rest : at;
    const float factor = scale * (rest_q != 0.f ? fmaf(of_p, lower, -rest_q / rest) : of_p);
    if (rank == 0 && warp == kWarps - 1 && a.row_loss) {
        double l = lane < kMaxCluster ? g.loss : 0.0;
#pragma unroll
        for (int o = kMaxCluster / 2; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        const double logS = total == 0.f ? 0.0 : (double)logf(total);
        if (mass != 0.0) l += mass * ((double)at * inv + logS);
        if (rest_q != 0.f) l += rest_all * ((double)logf(rest_q) - log((double)rest / (double)total) - ((double)at_rest - (double)at) * inv);
        if (lane == 0) a.row_loss[r] = none ? 0.f : (float)l;
    }
    if (none) {
        zeros();
        return;
    }
    if (!d) return;
    // the gradient; a segment's part of the row and of the gradient may start differently in their 16 bytes
    auto grad = [&](Pair x) {
        float y[2];
        ((x + Pair(-from_at, -from_at)) * Pair(c, c)).get(y[0], y[1]);
        return Pair(exp2_approx(y[0]), exp2_approx(y[1])) * Pair(factor, factor);
    };
    const RowGroups<TO> out(d, a.vocab);
    const int lead = row.off - out.off;         // element 0 of out's group 0 is element `lead` of the row's groups
    // groups of the gradient that begin in the segment
    auto from = [&](int group) { return group <= 0 ? 0 : group >= row.groups ? out.groups : (group * N - lead + NO - 1) / NO; };
    const int v0 = from(g0), v1 = from(g1), x0 = max(v0, out.whole_begin()), x1 = min(v1, out.whole_end());
    if (lead % N == 0) {
        // (they are made of whole groups of the row)
        constexpr int H = NO / N;
        const T *src = row.base + lead;
        for (int v = x0 + tid; v < x1; v += U * kThreads) {
            Raw<T> x[U][H];
#pragma unroll
            for (int u = 0; u < U; u++)
#pragma unroll
                for (int h = 0; h < H; h++)
                    if (v + u * kThreads < x1) x[u][h].w = *reinterpret_cast<const uint4 *>(src + (int64_t)(v + u * kThreads) * NO + h * N);
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (v + u * kThreads >= x1) continue;
                Vec<TO> o;
#pragma unroll
                for (int h = 0; h < H; h++) {
                    Pair p[N / 2];
                    x[u][h].pairs(p);
#pragma unroll
                    for (int i = 0; i < N / 2; i++) grad(p[i]).get(o.v[h * N + 2 * i], o.v[h * N + 2 * i + 1]);
                }
                o.store(d + out.first(v + u * kThreads));
            }
        }
    } else {
        for (int v = x0 + tid; v < x1; v += kThreads) {
            Vec<TO> o;
            const int first_element = out.first(v);
#pragma unroll
            for (int i = 0; i < NO; i += 2) grad(Pair(to_f32(z[first_element + i]), to_f32(z[first_element + i + 1]))).get(o.v[i], o.v[i + 1]);
            o.store(d + first_element);
        }
    }
    for (int i = tid; i < 2 * NO; i += kThreads) {      // the row's ragged ends (one group at each, which may be the same one)
        const int v = i < NO ? 0 : out.groups - 1, element = out.first(v) + i % NO;
        if (v < v0 || v >= v1 || out.whole(v) || (i >= NO && v == 0) || element < 0 || element >= a.vocab) continue;
        float y, unused;
        grad(Pair(to_f32(z[element]), 0.f)).get(y, unused);
        d[element] = from_f32<TO>(y);
    }
    // listed tokens: by the block that wrote the group they lie in
    const int mine = id >= 0 ? (id + out.off) / NO : -1;
    bool writes = mine >= v0 && mine < v1;
    if (lead % N == 0 && NO == N) writes = first;
    float z_mine = zi;
    if (!(lead % N == 0 && NO == N) && writes) {
        // (its logit and its other entries may belong to another block)
        z_mine = to_f32(z[id]);
        q_all = 0.f;
        for (int j = a.k - 1; j >= 0; j--)
            if (s_id[j] == id) {
                writes = j == tid;
                q_all += s_q[j];
            }
    }
    __syncthreads();
    if (writes) d[id] = from_f32<TO>(scale * fmaf(of_p, exp2_approx((z_mine - at) * c), -q_all));
}

template <typename T, typename TO, bool TAIL>
__global__ void __launch_bounds__(kThreads, 4) distill_kernel(const T *logits, TO *d_logits, DistillArgs a, int cluster) {
    pdl_enter();
    if (gated_off(a.gate)) return;
    distill_row<T, TO, TAIL>(logits, d_logits, a, cluster);
    // (the last block of the first row: where a row has several, another one writes the results)
    if ((int)blockIdx.x == cluster - 1 && a.hdr && a.scan)
        report_first(a.ids, a.rows * a.k, a.k, a.hdr, [&](int64_t id, int64_t i) {
            return (id < -1 || id >= a.vocab) && (!a.weight || a.weight[i / a.k] != 0.f);
        });
}

// Blocks to a row: so many that the rows under way (four blocks an SM) stay below kUnderWay bytes, which L2 has to hold until
// they are read again, beside their gradients; more where rows are few, none with less than two groups a thread.
constexpr int64_t kUnderWay = 64 << 20;
template <typename T>
int row_cluster(int64_t rows, int64_t vocab) {
    int c = 1;
    while (c < kMaxCluster && vocab / (2 * c) >= 2 * kThreads * Vec<T>::N &&
           (148 * 4 / c * vocab * (int64_t)sizeof(T) > kUnderWay || rows * c < 2 * 148))
        c *= 2;
    return c;
}

template <typename T, typename TO>
int launch(const T *logits, TO *d_logits, const DistillArgs &a, bool tail, cudaStream_t st) {
    const int c = row_cluster<T>(a.rows, a.vocab);
    const int64_t groups = (a.vocab + Vec<T>::N - 1) / Vec<T>::N + 1;
    const int smem = tail ? (int)(((groups + c - 1) / c + 31) / 32 * 4) : 0;
    auto kernel = tail ? distill_kernel<T, TO, true> : distill_kernel<T, TO, false>;
    return launch_clusters(kernel, dim3((unsigned)(a.rows * c)), kThreads, smem, c, 1, st, logits, d_logits, a, c);
}
}  // namespace

template <typename T, typename TO>
int distill_topk(const T *logits, int64_t ld, int64_t rows, int64_t vocab, const DistillRows &ds, TO *d_logits, int64_t ldd,
                 WsHeader *hdr, cudaStream_t st) {
    if (rows <= 0) return STREAMBP_OK;
    const bool scan = rows * ds.k <= kScanMost;
    if (hdr && !scan) SBP_TRY(clear_status_launch(hdr, st));
    const DistillArgs a{ds.ids, ds.values, ds.weight, ds.row_loss, rows, ld, ldd, (int)vocab, ds.k,
                        make_heat(ds.temperature), hdr, scan, call_state().gate};
    return launch<T, TO>(logits, d_logits, a, ds.tail, st);
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
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    unsigned weighted = 0;
    for (int64_t t = (int64_t)blockIdx.x * warps + (threadIdx.x >> 5); t < T_; t += (int64_t)gridDim.x * warps) {      // a warp to a row
        const bool on = ds.weight[t] != 0.f;
        bool entry = false, bad = false;
        for (int i = lane; on && i < ds.k; i += 32) {
            const int64_t id = ds.ids[t * ds.k + i];
            entry |= id >= 0 && id < vocab;
            bad |= id < -1 || id >= vocab;
        }
        entry = __any_sync(0xffffffffu, entry);
        bad = __any_sync(0xffffffffu, bad);
        if (lane) continue;
        marks[t] = entry ? 0 : 1;
        if (bad) set_status(hdr, STREAMBP_E_BAD_LABEL, (int)t);
        weighted += on;
    }
    if (weighted) atomicAdd(&hdr->n_valid, (unsigned long long)weighted);
}
int distill_marks(const DistillRows &ds, int64_t T_, int64_t vocab, int64_t *marks, WsHeader *hdr, cudaStream_t st) {
    const int64_t blocks = std::min<int64_t>((T_ + 7) / 8, 148 * 8);
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
