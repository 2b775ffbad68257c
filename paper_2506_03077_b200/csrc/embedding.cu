// Embedding lookup with a scale, and its gradient by sorted tokens.
//
//   out[t] = scale table[id_t],      d_table[v] (+)= scale sum over t with id_t = v of d_out[t]
// The gradient sorts the tokens by id (stable, by digits of 8 bits), so that equal ids lie side by side in token order, cuts the
// sorted list into chunks of equal length and sums the runs of a chunk in order.  A run that crosses chunks leaves one partial
// sum a chunk in the workspace; a second launch adds them in order.  So a token that fills half the batch costs no more than
// many that come once, and equal inputs give equal bits.
#include <algorithm>

#include "embedding.cuh"
#include "vocab_rows.cuh"

namespace sbp {

namespace {
constexpr int kThreads = 256, kWarps = kThreads / 32, kBins = 256;

// ---- lookup: a warp to a token's piece of kPiece bytes ------------------------------------------------------------------
template <typename T>
struct LookupArgs {
    const T *table;
    const int64_t *ids;
    T *out;
    int64_t n, vocab, ld, ldo, padding;
    int d;
    float scale;
    WsHeader *hdr;
};
constexpr int kLookupGroups = 4;
template <typename T, bool GROUPED>
__global__ void __launch_bounds__(kThreads) embedding_lookup_kernel(LookupArgs<T> a) {
    pdl_enter();
    constexpr int N = GROUPED ? Vec<T>::N : 1;
    if (blockIdx.x == 0 && blockIdx.y == 0)
        report_first(a.ids, a.n, 1, a.hdr, [&](int64_t id, int64_t) { return id != a.padding && (id < 0 || id >= a.vocab); });
    const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (t >= a.n) return;
    const int64_t id = a.ids[t];
    const bool zero = id == a.padding || id < 0 || id >= a.vocab;
    const T *from = a.table + (zero ? 0 : id) * a.ld;
    T *to = a.out + t * a.ldo;
    const int c0 = (blockIdx.y * kLookupGroups * 32 + (threadIdx.x & 31)) * N;
    if constexpr (GROUPED) {
        Vec<T> x[kLookupGroups];
#pragma unroll
        for (int u = 0; u < kLookupGroups; u++) {
            const int c = c0 + u * 32 * N;
            if (c < a.d && !zero) x[u].load(from + c);
        }
#pragma unroll
        for (int u = 0; u < kLookupGroups; u++) {
            const int c = c0 + u * 32 * N;
            if (c >= a.d) continue;
#pragma unroll
            for (int i = 0; i < N; i++) x[u].v[i] = zero ? 0.f : x[u].v[i] * a.scale;
            x[u].store(to + c);
        }
    } else {
#pragma unroll
        for (int u = 0; u < kLookupGroups; u++) {
            const int c = c0 + u * 32;
            if (c < a.d) to[c] = from_f32<T>(zero ? 0.f : to_f32(from[c]) * a.scale);
        }
    }
}

// ---- sort ---------------------------------------------------------------------------------------------------------------
// Tokens that take no part have the key `vocab`, which comes last.
__device__ __forceinline__ int key_of(int64_t id, int64_t vocab, int64_t padding) {
    return id == padding || id < 0 || id >= vocab ? (int)vocab : (int)id;
}
struct SortPass {
    const int64_t *ids;         // first pass: keys come from here, tokens are the positions
    const int *keys, *tokens;
    int *keys_out, *tokens_out, *counts;        // counts: [kBins][tiles]
    int64_t vocab, padding;
    int n, tile, shift;
    WsHeader *hdr;              // first pass: the status
};
__device__ __forceinline__ int sort_key(const SortPass &p, int i) {
    return p.ids ? key_of(p.ids[i], p.vocab, p.padding) : p.keys[i];
}
__global__ void __launch_bounds__(kThreads) sort_count_kernel(SortPass p) {
    pdl_enter();
    const int tiles = gridDim.x - (p.hdr ? 1 : 0), tile = blockIdx.x;
    if (tile == tiles) {
        report_first(p.ids, p.n, 1, p.hdr, [&](int64_t id, int64_t) { return id != p.padding && (id < 0 || id >= p.vocab); });
        return;
    }
    __shared__ int s_bins[kBins];
    s_bins[threadIdx.x] = 0;
    __syncthreads();
    const int i1 = min(p.n, (tile + 1) * p.tile);
    for (int i = tile * p.tile + threadIdx.x; i < i1; i += kThreads) atomicAdd(&s_bins[sort_key(p, i) >> p.shift & (kBins - 1)], 1);
    __syncthreads();
    p.counts[threadIdx.x * tiles + tile] = s_bins[threadIdx.x];
}
__global__ void __launch_bounds__(kThreads) sort_move_kernel(SortPass p) {
    pdl_enter();
    const int tiles = gridDim.x, tile = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ int s_next[kBins], s_warp[kWarps][kBins], s_sum[kWarps];
    // where this tile's elements of bin `tid` begin: behind all smaller bins and the bin's part in the tiles before
    int all = 0, before = 0;
    for (int t = 0; t < tiles; t++) {
        const int c = p.counts[tid * tiles + t];
        all += c;
        if (t < tile) before += c;
    }
    int up = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, up, o);
        if (lane >= o) up += x;
    }
    if (lane == 31) s_sum[warp] = up;
    __syncthreads();
    int base = up - all + before;
    for (int w = 0; w < warp; w++) base += s_sum[w];
    s_next[tid] = base;
    const int i1 = min(p.n, (tile + 1) * p.tile);
    for (int i0 = tile * p.tile; i0 < i1; i0 += kThreads) {
        for (int w = 0; w < kWarps; w++) s_warp[w][tid] = 0;
        __syncthreads();
        const int i = i0 + tid;
        int key = 0, bin = -1;
        if (i < i1) {
            key = sort_key(p, i);
            bin = key >> p.shift & (kBins - 1);
        }
        const unsigned same = __match_any_sync(0xffffffffu, bin);
        const int rank = __popc(same & ((1u << lane) - 1));
        if (bin >= 0 && rank == 0) s_warp[warp][bin] = __popc(same);
        __syncthreads();
        {   // bin `tid`: the warps' places, and where the next round begins
            int at = s_next[tid];
            for (int w = 0; w < kWarps; w++) {
                const int c = s_warp[w][tid];
                s_warp[w][tid] = at;
                at += c;
            }
            s_next[tid] = at;
        }
        __syncthreads();
        if (bin >= 0) {
            const int to = s_warp[warp][bin] + rank;
            p.keys_out[to] = key;
            p.tokens_out[to] = p.ids ? i : p.tokens[i];
        }
        __syncthreads();
    }
}

// ---- sums of runs -------------------------------------------------------------------------------------------------------
template <typename T>
struct RunArgs {
    const int *keys, *tokens;       // sorted
    const T *dy;
    float *d_table, *partials;      // partials: [chunks][2][d]; 0: of a run that began before, 1: of one that goes on (a chunk inside one run: 0)
    int64_t ldy;
    int n, chunk, d, vocab, accumulate;
    float scale;
};
constexpr int kMaxChunk = 128;
template <typename T, int N>
__global__ void __launch_bounds__(kThreads) embedding_runs_kernel(RunArgs<T> a) {
    pdl_enter();
    __shared__ int s_key[kMaxChunk + 2], s_tok[kMaxChunk];
    const int i0 = blockIdx.x * a.chunk, len = min(a.chunk, a.n - i0);
    for (int i = threadIdx.x; i < len + 2; i += kThreads) {
        const int at = i0 + i - 1;
        s_key[i] = at >= 0 && at < a.n ? a.keys[at] : -1;
    }
    for (int i = threadIdx.x; i < len; i += kThreads) s_tok[i] = a.tokens[i0 + i];
    __syncthreads();
    const int c = (blockIdx.y * kThreads + threadIdx.x) * N;
    if (c >= a.d) return;
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; e++) sum[e] = 0.f;
    bool begun = s_key[0] == s_key[1];          // the run began in an earlier chunk
    constexpr int U = 4;
    for (int i = 0; i < len; i += U) {
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (i + u >= len || s_key[i + u + 1] >= a.vocab) continue;
            const T *p = a.dy + (int64_t)s_tok[i + u] * a.ldy + c;
            if constexpr (N == 1) {
                x[u][0] = to_f32(*p);
            } else {
                Vec<T> v;
                v.load(p);
#pragma unroll
                for (int e = 0; e < N; e++) x[u][e] = v.v[e];
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (i + u >= len) continue;
            const int key = s_key[i + u + 1];
            if (key >= a.vocab) continue;
#pragma unroll
            for (int e = 0; e < N; e++) sum[e] += x[u][e];
            const bool last = i + u + 1 == len, goes_on = s_key[i + u + 2] == key;
            if (goes_on && !last) continue;
            float *to;
            if (begun || goes_on) {
                to = a.partials + ((int64_t)blockIdx.x * 2 + (begun ? 0 : 1)) * a.d + c;
#pragma unroll
                for (int e = 0; e < N; e++) to[e] = sum[e];
            } else {
                to = a.d_table + (int64_t)key * a.d + c;
#pragma unroll
                for (int e = 0; e < N; e++) to[e] = a.accumulate ? fmaf(sum[e], a.scale, to[e]) : sum[e] * a.scale;
            }
            begun = false;
#pragma unroll
            for (int e = 0; e < N; e++) sum[e] = 0.f;
        }
    }
}

// The partial sums of a run that crosses chunks, by the block of the chunk that it begins in: 32 columns, 8 sections of chunks.
struct JoinArgs {
    const int *keys;
    const float *partials;
    float *d_table;
    int n, chunk, d, vocab, accumulate;
    float scale;
};
__global__ void __launch_bounds__(kThreads) embedding_join_kernel(JoinArgs a) {
    pdl_enter();
    const int b = blockIdx.x, last = min((b + 1) * a.chunk, a.n) - 1;
    const int key = a.keys[last];
    if (last + 1 >= a.n || key >= a.vocab || a.keys[last + 1] != key) return;               // no run goes on
    if (a.keys[b * a.chunk] == key && b > 0 && a.keys[b * a.chunk - 1] == key) return;      // it began before
    // the run's last element: the last one with this key
    int lo = last + 1, hi = a.n - 1;
    while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (a.keys[mid] == key) lo = mid;
        else hi = mid - 1;
    }
    const int b1 = lo / a.chunk;                // chunks b (slot 1) and b + 1 .. b1 (slot 0)
    __shared__ float s_sum[8][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.y * 32 + x;
    const int per = (b1 - b + 7) / 8, q0 = b + 1 + y * per, q1 = min(q0 + per, b1 + 1);
    float s = 0.f;
    if (c < a.d) {
        if (y == 0) s = a.partials[((int64_t)b * 2 + 1) * a.d + c];
#pragma unroll 4
        for (int q = q0; q < q1; q++) s += a.partials[(int64_t)q * 2 * a.d + c];
    }
    s_sum[y][x] = s;
    __syncthreads();
    if (y || c >= a.d) return;
    for (int i = 1; i < 8; i++) s += s_sum[i][x];
    float *to = a.d_table + (int64_t)key * a.d + c;
    *to = a.accumulate ? fmaf(s, a.scale, *to) : s * a.scale;
}

}  // namespace

EmbeddingPlan embedding_plan(int64_t n, int64_t vocab, int64_t d) {
    EmbeddingPlan p;
    p.passes = 1;
    while (p.passes < 4 && (vocab >> (8 * p.passes)) != 0) p.passes++;          // (`vocab` itself is a key)
    // tiles of the sort: at most 64, whole rounds of a block
    const int64_t per = (n + 63) / 64;
    p.tile = (int)std::max<int64_t>(1024, (per + kThreads - 1) / kThreads * kThreads);
    p.tiles = (int)((n + p.tile - 1) / p.tile);
    // chunks of the sorted list: about sixteen blocks of 256 threads with 8 columns each an SM
    const int64_t strips = (d + 2047) / 2048;
    p.chunk = (int)std::min<int64_t>(kMaxChunk, std::max<int64_t>(8, n * strips / (148 * 16)));
    p.chunks = (int)((n + p.chunk - 1) / p.chunk);
    return p;
}

template <typename T>
int embedding_fwd(const T *table, int64_t ld, const int64_t *ids, int64_t n, int64_t vocab, int64_t d, float scale,
                  int64_t padding, T *out, int64_t ldo, WsHeader *hdr, cudaStream_t st) {
    const LookupArgs<T> a{table, ids, out, n, vocab, ld, ldo, padding, (int)d, scale, hdr};
    constexpr int N = Vec<T>::N;
    const bool grouped = d % N == 0 && ld % N == 0 && ldo % N == 0 && reinterpret_cast<uintptr_t>(table) % 16 == 0 &&
                         reinterpret_cast<uintptr_t>(out) % 16 == 0;
    const int64_t piece = 32 * kLookupGroups * (grouped ? N : 1);
    const dim3 grid((unsigned)((n + kWarps - 1) / kWarps), (unsigned)((d + piece - 1) / piece));
    if (grouped) SBP_LAUNCH((embedding_lookup_kernel<T, true>), grid, kThreads, 0, st, a);
    else SBP_LAUNCH((embedding_lookup_kernel<T, false>), grid, kThreads, 0, st, a);
    return STREAMBP_OK;
}

template <typename T>
int embedding_bwd(const T *dy, int64_t ldy, const int64_t *ids, int64_t n, int64_t vocab, int64_t d, float scale, int64_t padding,
                  float *d_table, bool accumulate, const EmbeddingPlan &p, int *const (&keys)[2], int *const (&tokens)[2],
                  int *counts, float *partials, WsHeader *hdr, cudaStream_t st) {
    if (!accumulate) SBP_TRY(fill_zero(d_table, sizeof(float) * (size_t)vocab * d, st));
    for (int i = 0; i < p.passes; i++) {
        SortPass s{i ? nullptr : ids, keys[(i + 1) & 1], tokens[(i + 1) & 1], keys[i & 1], tokens[i & 1], counts, vocab, padding,
                   (int)n, p.tile, 8 * i, i ? nullptr : hdr};
        SBP_LAUNCH(sort_count_kernel, (unsigned)(p.tiles + (i ? 0 : 1)), kThreads, 0, st, s);
        SBP_LAUNCH(sort_move_kernel, (unsigned)p.tiles, kThreads, 0, st, s);
    }
    const int done = (p.passes - 1) & 1;
    const RunArgs<T> r{keys[done], tokens[done], dy, d_table, partials, ldy, (int)n, p.chunk, (int)d, (int)vocab, accumulate ? 1 : 0, scale};
    constexpr int N = Vec<T>::N;
    if (d % N == 0 && ldy % N == 0 && reinterpret_cast<uintptr_t>(dy) % 16 == 0)
        SBP_LAUNCH((embedding_runs_kernel<T, N>), dim3((unsigned)p.chunks, (unsigned)((d / N + kThreads - 1) / kThreads)), kThreads, 0, st, r);
    else
        SBP_LAUNCH((embedding_runs_kernel<T, 1>), dim3((unsigned)p.chunks, (unsigned)((d + kThreads - 1) / kThreads)), kThreads, 0, st, r);
    const JoinArgs j{keys[done], partials, d_table, (int)n, p.chunk, (int)d, (int)vocab, accumulate ? 1 : 0, scale};
    if (p.chunks > 1) SBP_LAUNCH(embedding_join_kernel, dim3((unsigned)p.chunks, (unsigned)((d + 31) / 32)), kThreads, 0, st, j);
    return STREAMBP_OK;
}

template int embedding_fwd<float>(const float *, int64_t, const int64_t *, int64_t, int64_t, int64_t, float, int64_t, float *, int64_t,
                                  WsHeader *, cudaStream_t);
template int embedding_fwd<bf16>(const bf16 *, int64_t, const int64_t *, int64_t, int64_t, int64_t, float, int64_t, bf16 *, int64_t,
                                 WsHeader *, cudaStream_t);
template int embedding_bwd<float>(const float *, int64_t, const int64_t *, int64_t, int64_t, int64_t, float, int64_t, float *, bool,
                                  const EmbeddingPlan &, int *const (&)[2], int *const (&)[2], int *, float *, WsHeader *, cudaStream_t);
template int embedding_bwd<bf16>(const bf16 *, int64_t, const int64_t *, int64_t, int64_t, int64_t, float, int64_t, float *, bool,
                                 const EmbeddingPlan &, int *const (&)[2], int *const (&)[2], int *, float *, WsHeader *, cudaStream_t);

}  // namespace sbp
