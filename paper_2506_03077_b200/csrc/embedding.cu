// Embedding lookup with a scale, and its gradient by sorted tokens.
//
//   out[t] = scale table[id_t],      d_table[v] (+)= scale sum over t with id_t = v of d_out[t]
// The gradient sorts the tokens by id (stable, by digits of 9 bits), so that equal ids lie side by side in token order, cuts the
// sorted list into chunks of equal length and sums the runs of a chunk in order.  A run that crosses chunks leaves one partial
// sum a chunk in the workspace; a second launch adds them in order.  So a token that fills half the batch costs no more than
// many that come once, and equal inputs give equal bits.
//
// Bound by HBM: a looked-up row in and out, a gradient row in and a row of the table in and out.  Measured: lookup of 32768 rows of
// 3584 bf16 in 52 us (6.2 TB/s with rows that come again from L2); gradient of the same into 152064 rows 127 us: sort 15, sums 96
// (6.1 TB/s), joins 12, launches.
#include <algorithm>
#include <atomic>

#include "embedding.cuh"
#include "vocab_rows.cuh"

namespace sbp {

namespace {
constexpr int kThreads = 256, kWarps = kThreads / 32;

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
    bool scan;              // one block looks for ids outside the table, else each token's warp
};
constexpr int kLookupGroups = 4;
template <typename T, bool GROUPED>
__global__ void __launch_bounds__(kThreads) embedding_lookup_kernel(LookupArgs<T> a) {
    pdl_enter();
    constexpr int N = GROUPED ? Vec<T>::N : 1;
    if (blockIdx.x == 0 && blockIdx.y == 0 && a.scan)
        report_first(a.ids, a.n, 1, a.hdr, [&](int64_t id, int64_t) { return id != a.padding && (id < 0 || id >= a.vocab); });
    const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (t >= a.n) return;
    const int64_t id = a.ids[t];
    const bool zero = id == a.padding || id < 0 || id >= a.vocab;
    if (zero && !a.scan && id != a.padding && blockIdx.y == 0 && (threadIdx.x & 31) == 0) set_status(a.hdr, STREAMBP_E_BAD_LABEL, (int)t);
    const T *from = a.table + (zero ? 0 : id) * a.ld;
    T *to = a.out + t * a.ldo;
    const int c0 = (blockIdx.y * kLookupGroups * 32 + (threadIdx.x & 31)) * N;
    if constexpr (GROUPED) {
        Raw<T> x[kLookupGroups];                // (as they came until all are on the way)
#pragma unroll
        for (int u = 0; u < kLookupGroups; u++) {
            const int c = c0 + u * 32 * N;
            x[u].w = make_uint4(0, 0, 0, 0);
            if (c < a.d && !zero) x[u].w = *reinterpret_cast<const uint4 *>(from + c);
        }
#pragma unroll
        for (int u = 0; u < kLookupGroups; u++) {
            const int c = c0 + u * 32 * N;
            if (c >= a.d) continue;
            Vec<T> o;
            o.load(reinterpret_cast<const T *>(&x[u].w));
#pragma unroll
            for (int i = 0; i < N; i++) o.v[i] = zero ? 0.f : o.v[i] * a.scale;
            o.store(to + c);
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
// Keys are ids; tokens that take no part have the key `vocab`, which comes last.  A pass sorts by one digit of up to 9 bits
// and keeps the order of equal digits: rank within the warp by matching lanes, warps and blocks behind one another.
constexpr int kDigit = 9, kBins = 1 << kDigit, kNoneBad = 0x7fffffff;

__device__ __forceinline__ bool no_part(int64_t id, int64_t vocab, int64_t padding) { return id == padding || id < 0 || id >= vocab; }

// exclusive sums over kBins values, one in each of the first kBins threads of a block (s_sum: kBins / 32 ints)
__device__ __forceinline__ int bins_before(int count, int *s_sum) {
    const int tid = threadIdx.x, lane = tid & 31;
    int up = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, up, o);
        if (lane >= o) up += x;
    }
    if (lane == 31 && tid < kBins) s_sum[tid >> 5] = up;
    __syncthreads();
    int base = up - count;
    if (tid < kBins)
        for (int w = 0; w < (tid >> 5); w++) base += s_sum[w];
    return base;
}

struct SortArgs {
    const int64_t *ids;
    int *keys, *tokens;         // sorted
    int *owners;                // [0] is set to 0 here (embedding_runs_kernel)
    float *zero;                // optional: the table to clear, `zeros` floats
    int64_t zeros, vocab, padding;
    int n, passes;
    WsHeader *hdr;
};
// Up to 64 K tokens: one cluster of up to sixteen blocks (eight where the device has no room for more) sorts in one launch, keys and tokens in registers, handed over through
// shared memory; the other blocks of the launch clear a small table meanwhile.
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortPortable = 8, kSortBlocks = 16;
template <int ITEMS>
__global__ void __launch_bounds__(kSortThreads) sort_cluster_kernel(SortArgs a, int cluster) {
    pdl_enter();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if ((int)blockIdx.x >= cluster) {
        const int64_t step = (int64_t)(gridDim.x - cluster) * kSortThreads, at = (int64_t)(blockIdx.x - cluster) * kSortThreads + tid;
        float4 *z = reinterpret_cast<float4 *>(a.zero);
        for (int64_t i = at; i < a.zeros / 4; i += step) z[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at < a.zeros % 4) a.zero[a.zeros / 4 * 4 + at] = 0.f;
        return;
    }
    constexpr int kHold = ITEMS * kSortThreads;             // elements of a block
    extern __shared__ __align__(16) unsigned char s_raw[];
    int2 *s_hold = reinterpret_cast<int2 *>(s_raw);
    unsigned short *s_count = reinterpret_cast<unsigned short *>(s_raw + sizeof(int2) * kHold);     // [warps][kBins]
    __shared__ uint32_t s_total[kSortBlocks][kBins / 2];
    __shared__ int s_base[kBins], s_sum[kBins / 32], s_bad[kSortBlocks], s_worst;
    const int rank = blockIdx.x;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");       // (waited for before the others' memory is written)
    if (tid == 0) s_worst = kNoneBad;
    __syncthreads();
    int key[ITEMS], token[ITEMS], bad = kNoneBad;
#pragma unroll
    for (int j = 0; j < ITEMS; j++) {
        token[j] = rank * kHold + (warp * ITEMS + j) * 32 + lane;
        key[j] = (int)a.vocab;
        if (token[j] < a.n) {
            const int64_t id = a.ids[token[j]];
            if (!no_part(id, a.vocab, a.padding)) key[j] = (int)id;
            else if (id != a.padding) bad = min(bad, token[j]);
        }
    }
    if (bad != kNoneBad) atomicMin(&s_worst, bad);
    if (rank == 0 && tid == 0) a.owners[0] = 0;
    for (int pass = 0; pass < a.passes; pass++) {
        const int shift = pass * kDigit;
        for (int i = tid; i < kSortWarps * kBins / 8; i += kSortThreads) reinterpret_cast<uint4 *>(s_count)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        unsigned short place[ITEMS], *mine = s_count + warp * kBins;
#pragma unroll
        for (int j = 0; j < ITEMS; j++) {
            // (elements behind the last token are of no bin)
            const int bin = token[j] < a.n ? key[j] >> shift & (kBins - 1) : -1;
            const unsigned same = __match_any_sync(0xffffffffu, bin);
            const int lower = __popc(same & ((1u << lane) - 1));
            place[j] = bin >= 0 ? (unsigned short)(mine[bin] + lower) : 0;
            __syncwarp();
            if (bin >= 0 && lower == 0) mine[bin] = (unsigned short)(mine[bin] + __popc(same));
            __syncwarp();
        }
        __syncthreads();
        if (pass == 0) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        if (tid < kBins / 2) {          // two bins a thread, added as one word (a block's counts are below 2^14)
            uint32_t at = 0, *count = reinterpret_cast<uint32_t *>(s_count) + tid;
#pragma unroll 8
            for (int w = 0; w < kSortWarps; w++) {
                const uint32_t c = count[w * kBins / 2];
                count[w * kBins / 2] = at;
                at += c;
            }
            for (int q = 0; q < cluster; q++) st_remote_u32(map_to_cta(smem_u32(&s_total[rank][tid]), q), at);
        }
        if (pass == 0 && tid == kSortThreads - 1) st_remote_u32(map_to_cta(smem_u32(&s_bad[rank]), 0), (uint32_t)s_worst);
        __syncwarp();
        cluster_sync_all();
        int all = 0, before = 0;
        if (tid < kBins)
            for (int q = 0; q < cluster; q++) {
                const int c = reinterpret_cast<const unsigned short *>(s_total[q])[tid];
                all += c;
                if (q < rank) before += c;
            }
        const int base = bins_before(all, s_sum) + before;
        if (tid < kBins) s_base[tid] = base;
        __syncthreads();
        const bool last = pass == a.passes - 1;
#pragma unroll
        for (int j = 0; j < ITEMS; j++) {
            if (token[j] >= a.n) continue;
            const int bin = key[j] >> shift & (kBins - 1), to = s_base[bin] + s_count[warp * kBins + bin] + place[j];
            if (last) {
                a.keys[to] = key[j];
                a.tokens[to] = token[j];
            } else {
                const uint32_t at = map_to_cta(smem_u32(s_hold + to % kHold), to / kHold);
                asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(at), "r"(key[j]), "r"(token[j]) : "memory");
            }
        }
        if (last) break;
        __syncwarp();
        cluster_sync_all();
#pragma unroll
        for (int j = 0; j < ITEMS; j++) {
            const int at = (warp * ITEMS + j) * 32 + lane;
            token[j] = a.n;
            if (rank * kHold + at < a.n) {
                const int2 e = s_hold[at];
                key[j] = e.x;
                token[j] = e.y;
            }
        }
    }
    if (rank == 0 && tid == 0) {
        int worst = kNoneBad;
        for (int q = 0; q < cluster; q++) worst = min(worst, s_bad[q]);
        a.hdr->status = worst == kNoneBad ? STREAMBP_OK : STREAMBP_E_BAD_LABEL;
        a.hdr->detail = worst == kNoneBad ? 0 : worst;
    }
}

// More tokens: two launches a pass over up to 64 tiles of the list.
struct SortPass {
    const int64_t *ids;         // first pass: keys come from here, tokens are the positions
    const int *keys, *tokens;
    int *keys_out, *tokens_out, *counts;        // counts: [kBins][tiles], then [tiles] the first token outside the vocabulary
    int *owners;
    int64_t vocab, padding;
    int n, tile, shift;
    WsHeader *hdr;
};
__device__ __forceinline__ int sort_key(const SortPass &p, int i, int &bad) {
    if (!p.ids) return p.keys[i];
    const int64_t id = p.ids[i];
    if (!no_part(id, p.vocab, p.padding)) return (int)id;
    if (id != p.padding) bad = min(bad, i);
    return (int)p.vocab;
}
__global__ void __launch_bounds__(kBins) sort_count_kernel(SortPass p) {
    pdl_enter();
    const int tiles = gridDim.x, tile = blockIdx.x, tid = threadIdx.x;
    __shared__ int s_bins[kBins], s_bad;
    s_bins[tid] = 0;
    if (tid == 0) s_bad = kNoneBad;
    __syncthreads();
    const int64_t i1 = min((int64_t)p.n, (int64_t)(tile + 1) * p.tile);
    int bad = kNoneBad;
#pragma unroll 4
    for (int64_t i = (int64_t)tile * p.tile + tid; i < i1; i += kBins)
        atomicAdd(&s_bins[sort_key(p, (int)i, bad) >> p.shift & (kBins - 1)], 1);
    if (bad != kNoneBad) atomicMin(&s_bad, bad);
    __syncthreads();
    p.counts[tid * tiles + tile] = s_bins[tid];
    if (p.ids && tid == 0) p.counts[kBins * tiles + tile] = s_bad;
}
__global__ void __launch_bounds__(kBins) sort_move_kernel(SortPass p) {
    pdl_enter();
    constexpr int kWarps = kBins / 32;
    const int tiles = gridDim.x, tile = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ int s_next[kBins], s_warp[kWarps][kBins], s_sum[kWarps];
    if (p.ids && tile == 0 && tid == 0) {
        int worst = kNoneBad;
        for (int t = 0; t < tiles; t++) worst = min(worst, p.counts[kBins * tiles + t]);
        p.hdr->status = worst == kNoneBad ? STREAMBP_OK : STREAMBP_E_BAD_LABEL;
        p.hdr->detail = worst == kNoneBad ? 0 : worst;
        p.owners[0] = 0;
    }
    // where this tile's elements of bin `tid` begin: behind all smaller bins and the bin's part in the tiles before
    int all = 0, before = 0;
#pragma unroll 8
    for (int t = 0; t < tiles; t++) {
        const int c = p.counts[tid * tiles + t];
        all += c;
        if (t < tile) before += c;
    }
    s_next[tid] = bins_before(all, s_sum) + before;
    const int64_t i1 = min((int64_t)p.n, (int64_t)(tile + 1) * p.tile);
    int unused = kNoneBad;
    for (int64_t i0 = (int64_t)tile * p.tile; i0 < i1; i0 += kBins) {
#pragma unroll
        for (int w = 0; w < kWarps; w++) s_warp[w][tid] = 0;
        __syncthreads();
        const int64_t i = i0 + tid;
        int key = 0, bin = -1;
        if (i < i1) {
            key = sort_key(p, (int)i, unused);
            bin = key >> p.shift & (kBins - 1);
        }
        const unsigned same = __match_any_sync(0xffffffffu, bin);
        const int rank = __popc(same & ((1u << lane) - 1));
        if (bin >= 0 && rank == 0) s_warp[warp][bin] = __popc(same);
        __syncthreads();
        {   // bin `tid`: the warps' places, and where the next round begins
            int at = s_next[tid];
#pragma unroll
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
            p.tokens_out[to] = p.ids ? (int)i : p.tokens[i];
        }
        __syncthreads();
    }
}

// ---- sums of runs -------------------------------------------------------------------------------------------------------
// 16 bytes of a row where rows are made of them (N > 1), else one element, as they came; and their values.
template <typename T, int N> struct Piece {
    typedef uint4 In;
    static __device__ __forceinline__ void load(const T *p, In &x) { x = *reinterpret_cast<const uint4 *>(p); }
    static __device__ __forceinline__ void get(const In &x, float (&v)[Vec<T>::N]) {
        Vec<T> t;
        t.load(reinterpret_cast<const T *>(&x));
#pragma unroll
        for (int i = 0; i < Vec<T>::N; i++) v[i] = t.v[i];
    }
};
template <typename T> struct Piece<T, 1> {
    typedef T In;
    static __device__ __forceinline__ void load(const T *p, In &x) { x = *p; }
    template <int M> static __device__ __forceinline__ void get(const In &x, float (&v)[M]) { v[0] = to_f32(x); }
};
template <typename T>
struct RunArgs {
    const int *keys, *tokens;       // sorted
    const T *dy;
    float *d_table, *partials;      // partials: [chunks][2][dp]; 0: of a run that began before, 1: of one that goes on (a chunk inside one run: 0)
    int *owners;                    // [0] how many runs go on behind the chunk they begin in; from [4] on their chunk, last chunk and key, four ints each
    int64_t ldy;
    int n, chunk, chunks, d, dp, vocab, accumulate;
    float scale;
    int clears;                     // blocks that clear the table's other rows
};
// Rows r0 .. r1 - 1 of the table that have no token are cleared, a warp to a row; find(r) tells the block in s_has which of the
// rows from r on have one, as many as it has threads.
template <typename F>
__device__ __forceinline__ void clear_rows(float *d_table, int d, int64_t r0, int64_t r1, int *s_has, F find) {
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    for (int64_t r = r0; r < r1; r += blockDim.x) {
        find(r);
        __syncthreads();
        for (int i = threadIdx.x >> 5; i < (int)blockDim.x && r + i < r1; i += warps) {
            if (s_has[i]) continue;
            float *to = d_table + (r + i) * d;
            if (d % 4 == 0)
                for (int c = lane * 4; c < d; c += 128) *reinterpret_cast<float4 *>(to + c) = make_float4(0.f, 0.f, 0.f, 0.f);
            else
                for (int c = lane; c < d; c += 32) to[c] = 0.f;
        }
        __syncthreads();
    }
}
// The table's part `part` of `parts`; whether a row has a token its thread finds in the sorted keys, seven keys at a time.
static __device__ __noinline__ void clear_others(const int *__restrict__ keys, int n, float *d_table, int64_t vocab, int d, int part, int parts) {
    __shared__ int s_has[256];
    const int tid = threadIdx.x;
    clear_rows(d_table, d, vocab * part / parts, vocab * (part + 1) / parts, s_has, [&](int64_t r) {
        int lo = 0, left = n;               // the first key that is not below the row lies in lo .. lo + left
        while (left > 0) {
            const int step = left / 8 + 1;
            int below = 0;
#pragma unroll
            for (int i = 1; i < 8; i++) {
                const int at = i * step - 1;
                if (at < left) below += keys[lo + at] < r + tid;
            }
            lo += below * step;
            left = min(left - below * step, step - 1);
        }
        s_has[tid] = lo < n && keys[lo] == r + tid;
    });
}
constexpr int kMaxChunk = 128, kRunThreads = 256;
constexpr int64_t kSmallTable = 16 << 20;       // elements
// Each thread owns the columns of one 16-byte group of d_out and walks the chunk, four rows of d_out (and, added to, of the
// table) in flight.  What bounds it is HBM: d_out once, the table's rows once in each direction.
template <typename T, int N>
__global__ void __launch_bounds__(kRunThreads) embedding_runs_kernel(RunArgs<T> a) {
    pdl_enter();
    __shared__ int s_key[kMaxChunk + 2], s_tok[kMaxChunk];
    if ((int)blockIdx.x >= a.chunks) {
        const int part = (blockIdx.x - a.chunks) * gridDim.y + blockIdx.y;
        if (part < a.clears) clear_others(a.keys, a.n, a.d_table, a.vocab, a.d, part, a.clears);
        return;
    }
    const int64_t i0 = (int64_t)blockIdx.x * a.chunk;
    const int len = (int)min((int64_t)a.chunk, a.n - i0);
    for (int i = threadIdx.x; i < len + 2; i += blockDim.x) {
        const int64_t at = i0 + i - 1;
        s_key[i] = at >= 0 && at < a.n ? a.keys[at] : -1;
    }
    for (int i = threadIdx.x; i < len; i += blockDim.x) s_tok[i] = a.tokens[i0 + i];
    __syncthreads();
    const int c = (blockIdx.y * blockDim.x + threadIdx.x) * N;
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; e++) sum[e] = 0.f;
    bool begun = s_key[0] == s_key[1];          // the run began in an earlier chunk
    constexpr int U = 4;
    for (int i = 0; i < len && s_key[i + 1] < a.vocab && c < a.d; i += U) {
        // (values stay as they came until all are on the way)
        typename Piece<T, N>::In x[U];
        typename Piece<float, N>::In old[U][sizeof(float) / sizeof(T)];
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (i + u >= len || s_key[i + u + 1] >= a.vocab) continue;
            Piece<T, N>::load(a.dy + (int64_t)s_tok[i + u] * a.ldy + c, x[u]);
            // the table's row of a run that ends here (a crossing run's is read for nothing, at most twice a chunk)
            if (a.accumulate && s_key[i + u + 2] != s_key[i + u + 1]) {
                const float *t = a.d_table + (int64_t)s_key[i + u + 1] * a.d + c;
#pragma unroll
                for (int e = 0; e < N; e += 4) Piece<float, N>::load(t + e, old[u][e / 4]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (i + u >= len) continue;
            const int key = s_key[i + u + 1];
            if (key >= a.vocab) continue;
            float v[N];
            Piece<T, N>::get(x[u], v);
#pragma unroll
            for (int e = 0; e < N; e++) sum[e] += v[e];
            const bool last = i + u + 1 == len, goes_on = s_key[i + u + 2] == key;
            if (goes_on && !last) continue;
            float *to;
            if (begun || goes_on) {
                to = a.partials + ((int64_t)blockIdx.x * 2 + (begun ? 0 : 1)) * a.dp + c;
            } else {
                to = a.d_table + (int64_t)key * a.d + c;
                if (a.accumulate) {
#pragma unroll
                    for (int e = 0; e < N; e += 4) {
                        float o[4];
                        Piece<float, N>::get(old[u][e / 4], o);
#pragma unroll
                        for (int f = 0; f < 4 && e + f < N; f++) sum[e + f] = fmaf(sum[e + f], a.scale, o[f]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < N; e++) sum[e] *= a.scale;
                }
            }
            if constexpr (N == 1) {
                *to = sum[0];
            } else {
#pragma unroll
                for (int e = 0; e < N; e += 4) *reinterpret_cast<float4 *>(to + e) = make_float4(sum[e], sum[e + 1], sum[e + 2], sum[e + 3]);
            }
            begun = false;
#pragma unroll
            for (int e = 0; e < N; e++) sum[e] = 0.f;
        }
    }
    __syncwarp();
    if (blockIdx.y == 0 && threadIdx.x < 32) {
        const int key = s_key[len], lane = threadIdx.x;
        // a run that goes on, and did not begin in an earlier chunk
        if (s_key[len + 1] == key && key < a.vocab && !(s_key[1] == key && s_key[0] == key)) {
            // the last chunk that begins with this key: 32 guesses at a time, the next 32 chunks first
            auto same = [&](int64_t q) { return q < a.chunks && a.keys[q * a.chunk] == key; };
            int last = blockIdx.x + 1;          // begins with it
            unsigned yes = __ballot_sync(0xffffffffu, same(last + 1 + lane));
            last += yes == 0xffffffffu ? 32 : __ffs(~yes) - 1;
            if (yes == 0xffffffffu) {
                int64_t step = 1;
                while (step * 32 < a.chunks) step *= 32;
                for (; step >= 1; step /= 32) {
                    yes = __ballot_sync(0xffffffffu, same(last + (lane + 1) * step));
                    last += (int)((yes == 0xffffffffu ? 32 : __ffs(~yes) - 1) * step);
                }
            }
            // (their order does not matter)
            if (lane == 0) reinterpret_cast<int4 *>(a.owners)[1 + atomicAdd(a.owners, 1)] = make_int4(blockIdx.x, last, key, 0);
        }
    }
}

// Up to kFewTokens tokens, in one launch without a sort: the block of a token that is the first with its id adds all of them, in
// their order, eight rows in flight.  Bound by latency: 50 tokens of 256 columns with the rest of 4096 rows cleared in 4.5 us (by
// sort, sums and joins 10), 128 tokens of two ids in 9.0 (10.6; 512 of them would take 57 against 14, though 512 of many ids 11).
constexpr int kFewTokens = 128;
template <typename T>
struct FewArgs {
    const int64_t *ids;
    const T *dy;
    float *d_table;
    int64_t ldy, vocab, padding;
    int n, d, accumulate, clears;
    float scale;
    WsHeader *hdr;
};
template <typename T, int N>
__global__ void __launch_bounds__(kRunThreads) embedding_few_kernel(FewArgs<T> a) {
    pdl_enter();
    constexpr int U = 8;
    __shared__ int s_id[kFewTokens], s_bad, s_has[kRunThreads];
    const int tid = threadIdx.x, lane = tid & 31, t = blockIdx.x;
    if (tid == 0) s_bad = kNoneBad;
    __syncthreads();
    for (int i = tid; i < kFewTokens; i += blockDim.x) {
        const int64_t id = i < a.n ? a.ids[i] : a.padding;
        const bool none = i >= a.n || no_part(id, a.vocab, a.padding);
        s_id[i] = none ? -1 : (int)id;
        if (none && id != a.padding) atomicMin(&s_bad, i);
    }
    __syncthreads();
    if (t == 0 && blockIdx.y == 0 && tid == 0) {
        a.hdr->status = s_bad == kNoneBad ? STREAMBP_OK : STREAMBP_E_BAD_LABEL;
        a.hdr->detail = s_bad == kNoneBad ? 0 : s_bad;
    }
    if (t >= a.n) {
        const int part = (t - a.n) * gridDim.y + blockIdx.y;
        if (part < a.clears)
            clear_rows(a.d_table, a.d, a.vocab * part / a.clears, a.vocab * (part + 1) / a.clears, s_has, [&](int64_t r) {
                s_has[tid] = 0;
                __syncthreads();
                for (int i = tid; i < a.n; i += blockDim.x)
                    if (s_id[i] >= r && s_id[i] < r + blockDim.x) s_has[s_id[i] - r] = 1;
            });
        return;
    }
    const int id = s_id[t], c = (blockIdx.y * blockDim.x + tid) * N;
    if (id < 0) return;
    uint32_t same[kFewTokens / 32];             // the tokens with this id
#pragma unroll
    for (int w = 0; w < kFewTokens / 32; w++) same[w] = __ballot_sync(0xffffffffu, s_id[w * 32 + lane] == id);
    bool first = true;
#pragma unroll
    for (int w = 0; w < kFewTokens / 32; w++) first = first && (w * 32 > t || (same[w] & (t - w * 32 >= 32 ? ~0u : (1u << (t - w * 32)) - 1)) == 0);
    if (!first || c >= a.d) return;
    float *to = a.d_table + (int64_t)id * a.d + c;
    typename Piece<float, N>::In old[sizeof(float) / sizeof(T)];
    if (a.accumulate) {
#pragma unroll
        for (int e = 0; e < N; e += 4) Piece<float, N>::load(to + e, old[e / 4]);
    }
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; e++) sum[e] = 0.f;
#pragma unroll
    for (int w = 0; w < kFewTokens / 32; w++)
        for (uint32_t left = same[w]; left;) {
            typename Piece<T, N>::In x[U];
            int have = 0;
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (!left) continue;
                Piece<T, N>::load(a.dy + (int64_t)(w * 32 + __ffs(left) - 1) * a.ldy + c, x[u]);
                left &= left - 1;
                have = u + 1;
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (u >= have) continue;
                float v[N];
                Piece<T, N>::get(x[u], v);
#pragma unroll
                for (int e = 0; e < N; e++) sum[e] += v[e];
            }
        }
#pragma unroll
    for (int e = 0; e < N; e += 4) {
        float o[4] = {0.f, 0.f, 0.f, 0.f};
        if (a.accumulate) Piece<float, N>::get(old[e / 4], o);
#pragma unroll
        for (int f = 0; f < 4 && e + f < N; f++) sum[e + f] = fmaf(sum[e + f], a.scale, o[f]);
    }
    if constexpr (N == 1) {
        *to = sum[0];
    } else {
#pragma unroll
        for (int e = 0; e < N; e += 4) *reinterpret_cast<float4 *>(to + e) = make_float4(sum[e], sum[e + 1], sum[e + 2], sum[e + 3]);
    }
}

// The partial sums of a run that crosses chunks, 128 columns at a time (an item): a warp adds those of a run of up to kShort
// chunks, a block's warps a section each of a longer one's, and the sections are added in order.
struct JoinArgs {
    const int *owners;
    const float *partials;
    float *d_table;
    int d, dp, accumulate;
    float scale;
};
constexpr int kShort = 128;
__global__ void __launch_bounds__(256) embedding_join_kernel(JoinArgs a) {
    pdl_enter();
    __shared__ float4 s_sum[8][32];
    __shared__ int s_first[8], s_last[8], s_key[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int strips = (a.d + 127) / 128;
    const int64_t items = (int64_t)a.owners[0] * strips;
    // eight items a block, one where the blocks suffice for that (long runs are then spread best)
    const int each = items > gridDim.x ? 8 : 1;
    for (int64_t it0 = (int64_t)blockIdx.x * each; it0 < items; it0 += (int64_t)gridDim.x * each) {
        const int64_t it = it0 + warp;
        const bool own = warp < each && it < items;
        int b = 0, last = 0, key = 0;
        const int c = (int)(it % strips) * 128 + lane * 4;
        float old[4] = {0.f, 0.f, 0.f, 0.f};
        auto before = [&](int k, int col) {
            const float *t = a.d_table + (int64_t)k * a.d + col;
            if (a.accumulate)
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (col + e < a.d) old[e] = t[e];
        };
        if (own) {
            const int4 o = reinterpret_cast<const int4 *>(a.owners)[1 + it / strips];
            b = o.x;
            last = o.y;
            key = o.z;
            if (last - b <= kShort) before(key, c);
        }
        // chunk from's sum of its last run and the first runs of chunks q0 .. q1 - 1
        auto add = [&](int col, int from, bool with_from, int q0, int q1) {
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
            if (col >= a.dp) return s;
            if (with_from) s = *reinterpret_cast<const float4 *>(a.partials + ((int64_t)from * 2 + 1) * a.dp + col);
#pragma unroll 8
            for (int q = q0; q < q1; q++) {
                const float4 t = *reinterpret_cast<const float4 *>(a.partials + (int64_t)q * 2 * a.dp + col);
                s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
            }
            return s;
        };
        auto put = [&](float4 s, int k, int col) {
            const float v[4] = {s.x, s.y, s.z, s.w};
            float *to = a.d_table + (int64_t)k * a.d + col;
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (col + e < a.d) to[e] = fmaf(v[e], a.scale, old[e]);
        };
        if (own && last - b <= kShort) put(add(c, b, true, b + 1, last + 1), key, c);
        const bool is_long = own && last - b > kShort;
        if (!__syncthreads_or(is_long)) continue;
        if (lane == 0) {
            s_first[warp] = is_long ? b : -1;
            s_last[warp] = last;
            s_key[warp] = key;
        }
        __syncthreads();
        for (int w = 0; w < each; w++) {
            const int first = s_first[w];
            if (first < 0) continue;
            const int per = (s_last[w] - first + 7) / 8, q0 = first + 1 + warp * per, col = (int)((it0 + w) % strips) * 128 + lane * 4;
            if (warp == 0) before(s_key[w], col);
            s_sum[warp][lane] = add(col, first, warp == 0, q0, min(q0 + per, s_last[w] + 1));
            __syncthreads();
            if (warp == 0) {
                float4 s = s_sum[0][lane];
                for (int i = 1; i < 8; i++) {
                    const float4 t = s_sum[i][lane];
                    s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
                }
                put(s, s_key[w], col);
            }
            __syncthreads();
        }
    }
}

}  // namespace

EmbeddingPlan embedding_plan(int64_t n, int64_t vocab, int64_t d) {
    EmbeddingPlan p;
    p.passes = 1;
    while (p.passes < 4 && (vocab >> (kDigit * p.passes)) != 0) p.passes++;     // (`vocab` itself is a key)
    p.one_launch = n <= (int64_t)kSortPortable * kSortThreads * 8;
    // tiles of the sort's launches: at most 64, whole rounds of a block
    const int64_t per = (n + 63) / 64;
    p.tile = (int)((per + kBins - 1) / kBins * kBins);
    p.tiles = (int)((n + p.tile - 1) / p.tile);
    // chunks of the sorted list: about eight blocks of 256 threads with 8 columns each an SM
    const int64_t strips = (d + 2047) / 2048;
    p.chunk = (int)std::min<int64_t>(kMaxChunk, std::max<int64_t>(8, n * strips / (148 * 8)));
    p.chunks = (int)((n + p.chunk - 1) / p.chunk);
    p.partial_width = (int)((d + 3) / 4 * 4);
    return p;
}
int embedding_counts(const EmbeddingPlan &p) { return p.one_launch ? 0 : (kBins + 1) * p.tiles; }

namespace {
std::atomic<int> g_sort_cap{kSortBlocks};
template <int ITEMS> constexpr int kSortSmem = ITEMS * kSortThreads * 8 + kSortWarps * kBins * 2;
// The largest cluster of the sort that the device can hold, 0 for an error (of which a call with less than kSortPortable is refused:
// the plan counts on that many).
template <int ITEMS>
int sort_cluster_limit() {
    static PerDevice cache;
    return cache.get([] {
        auto kernel = sort_cluster_kernel<ITEMS>;
        if (!cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortSmem<ITEMS>))) return 0;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) {
            cudaLaunchConfig_t cfg;
            memset(&cfg, 0, sizeof(cfg));
            cfg.gridDim = dim3(kSortBlocks, 1, 1);
            cfg.blockDim = dim3(kSortThreads, 1, 1);
            cfg.dynamicSmemBytes = kSortSmem<ITEMS>;
            cudaLaunchAttribute attr;
            memset(&attr, 0, sizeof(attr));
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = kSortBlocks;
            attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            int clusters = 0;
            if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters >= 1) return kSortBlocks;
        }
        cudaGetLastError();
        return kSortPortable;
    });
}
template <int ITEMS>
int launch_sort(const SortArgs &a, int cluster, cudaStream_t st) {
    const int64_t zero_blocks = std::min<int64_t>(148, (a.zeros + 4 * kSortThreads - 1) / (4 * kSortThreads));
    const int64_t blocks = cluster + (zero_blocks + cluster - 1) / cluster * cluster;
    return launch_clusters(sort_cluster_kernel<ITEMS>, dim3((unsigned)blocks), kSortThreads, kSortSmem<ITEMS>, cluster, 1, st, a, cluster);
}
}  // namespace

int embedding_cap_sort(int blocks) { return g_sort_cap.exchange(blocks); }

template <typename T>
int embedding_fwd(const T *table, int64_t ld, const int64_t *ids, int64_t n, int64_t vocab, int64_t d, float scale,
                  int64_t padding, T *out, int64_t ldo, WsHeader *hdr, cudaStream_t st) {
    const bool scan = n <= kScanMost || d * (int64_t)sizeof(T) >= kScanRow;
    if (!scan) SBP_TRY(clear_status_launch(hdr, st));
    const LookupArgs<T> a{table, ids, out, n, vocab, ld, ldo, padding, (int)d, scale, hdr, scan};
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
                  int *counts, int *owners, float *partials, WsHeader *hdr, cudaStream_t st) {
    constexpr int N = Vec<T>::N;
    const bool grouped = d % N == 0 && ldy % N == 0 && reinterpret_cast<uintptr_t>(dy) % 16 == 0;
    const int64_t groups = grouped ? d / N : d, strips = (groups + kRunThreads - 1) / kRunThreads;
    int threads = (int)(((groups + strips - 1) / strips + 31) / 32 * 32);
    if (n <= kFewTokens && !accumulate) threads = std::max(threads, 128);       // (for the rows that are cleared)
    // Blocks that clear rows: 64 KB each, less where its threads are fewer than those rows, more where the GPU is full of them.
    const int64_t clears =
        accumulate ? 0 : std::min<int64_t>({148 * 2048 / threads, vocab, std::max(vocab * d / 16384 + 1, (vocab + threads - 1) / threads)});
    if (n <= kFewTokens) {
        const FewArgs<T> f{ids, dy, d_table, ldy, vocab, padding, (int)n, (int)d, accumulate ? 1 : 0, (int)clears, scale, hdr};
        const dim3 grid((unsigned)(n + (clears + strips - 1) / strips), (unsigned)strips);
        if (grouped) SBP_LAUNCH((embedding_few_kernel<T, N>), grid, threads, 0, st, f);
        else SBP_LAUNCH((embedding_few_kernel<T, 1>), grid, threads, 0, st, f);
        return STREAMBP_OK;
    }
    int done = 0;
    // A small table is cleared beside the sort (3000 tokens, 50001 x 64: 17.7 us, with its rows without tokens cleared beside the
    // sums 20.5); a large one beside the sums, where tokens' rows need not be cleared (16384 tokens, 152064 x 3584: 373 us against 566).
    const bool clear_first = !accumulate && p.one_launch && vocab * d <= kSmallTable;
    if (p.one_launch) {
        const SortArgs s{ids, keys[0], tokens[0], owners, clear_first ? d_table : nullptr, clear_first ? vocab * d : 0, vocab, padding, (int)n,
                         p.passes, hdr};
        // (sixteen blocks: 65536 tokens 94 us against 104, 32768 127 against 132)
        const int most = std::min({sort_cluster_limit<1>(), sort_cluster_limit<2>(), sort_cluster_limit<4>(), sort_cluster_limit<8>(),
                                   g_sort_cap.load()});
        if (most < kSortPortable) return STREAMBP_E_CUDA;       // (fewer blocks would leave tokens out)
        int cluster = 1;
        while (2 * cluster <= most && n > (int64_t)cluster * kSortThreads) cluster *= 2;
        const int64_t each = (n + (int64_t)cluster * kSortThreads - 1) / ((int64_t)cluster * kSortThreads);
        if (each <= 1) SBP_TRY(launch_sort<1>(s, cluster, st));
        else if (each <= 2) SBP_TRY(launch_sort<2>(s, cluster, st));
        else if (each <= 4) SBP_TRY(launch_sort<4>(s, cluster, st));
        else SBP_TRY(launch_sort<8>(s, cluster, st));
    } else {
        for (int i = 0; i < p.passes; i++) {
            const SortPass s{i ? nullptr : ids, keys[(i + 1) & 1], tokens[(i + 1) & 1], keys[i & 1], tokens[i & 1], counts, owners, vocab,
                             padding, (int)n, p.tile, kDigit * i, hdr};
            SBP_LAUNCH(sort_count_kernel, (unsigned)p.tiles, kBins, 0, st, s);
            SBP_LAUNCH(sort_move_kernel, (unsigned)p.tiles, kBins, 0, st, s);
        }
        done = (p.passes - 1) & 1;
    }
    const RunArgs<T> r{keys[done], tokens[done], dy, d_table, partials, owners, ldy, (int)n, p.chunk, p.chunks, (int)d, p.partial_width, (int)vocab,
                       accumulate ? 1 : 0, scale, clear_first ? 0 : (int)clears};
    const dim3 grid((unsigned)(p.chunks + (r.clears + strips - 1) / strips), (unsigned)strips);
    if (grouped) SBP_LAUNCH((embedding_runs_kernel<T, N>), grid, threads, 0, st, r);
    else SBP_LAUNCH((embedding_runs_kernel<T, 1>), grid, threads, 0, st, r);
    const JoinArgs j{owners, partials, d_table, (int)d, p.partial_width, accumulate ? 1 : 0, scale};
    const int64_t most = (int64_t)p.chunks * ((d + 127) / 128);
    SBP_LAUNCH(embedding_join_kernel, (unsigned)std::min<int64_t>(most, 148 * 8), 256, 0, st, j);
    return STREAMBP_OK;
}

template int embedding_fwd<float>(const float *, int64_t, const int64_t *, int64_t, int64_t, int64_t, float, int64_t, float *, int64_t,
                                  WsHeader *, cudaStream_t);
template int embedding_fwd<bf16>(const bf16 *, int64_t, const int64_t *, int64_t, int64_t, int64_t, float, int64_t, bf16 *, int64_t,
                                 WsHeader *, cudaStream_t);
template int embedding_bwd<float>(const float *, int64_t, const int64_t *, int64_t, int64_t, int64_t, float, int64_t, float *, bool,
                                  const EmbeddingPlan &, int *const (&)[2], int *const (&)[2], int *, int *, float *, WsHeader *, cudaStream_t);
template int embedding_bwd<bf16>(const bf16 *, int64_t, const int64_t *, int64_t, int64_t, int64_t, float, int64_t, float *, bool,
                                 const EmbeddingPlan &, int *const (&)[2], int *const (&)[2], int *, int *, float *, WsHeader *, cudaStream_t);

}  // namespace sbp
