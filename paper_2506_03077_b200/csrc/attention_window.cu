// Attention with a sliding window and sink keys on tcgen05 tensor cores (bf16 operands, head_dim 64 or 128): the queries
// of one chunk against the key tiles their window reaches and the tiles that hold sinks; nothing else is loaded.
//
// Forward (attn_window_fwd_kernel): two persistent CTAs per SM, each walking items: 128 rows of queries, which are the rows
// of as many heads of one group as divide up, against the key tiles they see.  Few items: a cluster to each, which shares
// its key tiles and joins the sums.
//   warp 0      : TMA producer -- query tiles, K and V tiles of 64 keys through rings; runs ahead into the next item
//   warp 1      : MMA issuer (warp-uniform issue) -- S = Q K^T into tensor memory two or three tiles ahead, O += P V with P
//                 read from tensor memory (packed over the columns of its S: the product that reads P is queued before the
//                 one that overwrites S, one thread's MMAs run in order)
//   warps 2..5  : softmax -- a thread owns a query row: its scores in registers, row maximum and sum private; the running
//                 output is rescaled only when a row's maximum grows by more than 2^8 (exact: the final division uses the
//                 same reference)
// What two CTAs of one chain each buy: one's latencies (tensor-memory loads, hand-offs) fall into the other's exponentials,
// and short windows -- a handful of key tiles between fetching queries and storing outputs -- pay neither launch nor set-up
// nor first loads per tile.  Key tiles of 64 rather than 128 waste less at the two ends of a window and leave tensor memory
// for scores ahead (16384 rows, window 128, heads of 64: 125 -> 107 us; window 1024, heads of 128: 350 -> 305 us).
// A row may see nothing of the first tiles of its list: its maximum stays -infinity and it adds exact zeros until it sees
// a key.  Every query sees its own key, so no row ends empty.  Groups of 32 columns that no row of a warp sees are skipped,
// and the sink tile that the window does not reach is cut to its sinks (16 columns for up to 16 of them).  32 rows of four
// heads span 96 keys fewer than 128 rows of one (16384 rows, window 128, heads of 64: 96 -> 86 us).
// What bounds it: the exponentials and the conversions around them, ~770 of the ~1600 cycles of a CTA's step of 128 x 64
// scores, and the latencies that two chains do not hide.  2048 rows behind 14336, window 4096, 32:8 heads of 128: 160 us,
// 860 TFLOP/s among calls on other inputs (146 us, 940 TFLOP/s in a short run of the same); 16384 rows, window 4096: 870 us.
//
// Backward (attn_window_bwd_kernel): two CTA roles in one grid, both deterministic (no floating-point atomics).
//   dK/dV: one CTA per (key tile, KV head) loops over the query heads of the group and the query tiles that see the tile;
//          a sink tile, which every later query sees, and all tiles where there are few, are cut into segments of query
//          tiles whose fp32 sums meet in the workspace and are joined in order by window_join_kernel
//   dQ   : one CTA per (query tile, head) loops over the key tiles of its span; few of them: a cluster to each, which shares
//          the key tiles and adds the sums in order
// A tile's rows are those of one head, or of several of a group where that saves tile pairs (bwd_heads; PACKED kernels).
// Softmax work is split in time (P for dV first, then dS), packed operands stay in tensor memory, every product is a full
// tile; gradients leave through blocks of shared memory and TMA stores or adds, fp32 sums rounded once.
// What bounds it: one iteration's chain of products and exponentials, ~2900 (dK/dV) and ~2500 cycles (dQ) for 128 x 128
// scores at heads of 128, of which the tensor pipe is busy 2048 and 1536.  Heads of 64 run two CTAs with inner tiles of 64 per
// SM.  1024 rows behind 7168, window 2048, 28:4 heads of 128: 128 us (590 TFLOP/s counting five products a pair); 8191
// rows, window 512, 32:8 heads of 64: 242 us.
//
// All mbarrier waits are bounded (sm100.cuh).
#include <cstring>

#include "sm100.cuh"
#include "window.cuh"

namespace sbp {
namespace {

constexpr int TILE = 128;                 // queries to a tile; keys to a tile of the backward
constexpr int SUB_BYTES = TILE * 64 * 2;  // one [128 rows][64 columns] swizzled sub-tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Descriptor steps of a [128 rows][DH] tile stored as 64-column sub-tiles: K-major (contraction along the columns, 16 a
// step) and MN-major (contraction along the rows, 16 a step).
__device__ __forceinline__ uint32_t klo(uint32_t tile) { return desc_lo(tile, 16); }
__host__ __device__ constexpr uint32_t kstep(int kk) { return (uint32_t)((kk >> 2) * (SUB_BYTES >> 4) + (kk & 3) * 2); }
__host__ __device__ constexpr uint32_t mnstep(int kk) { return (uint32_t)(kk * 128); }

template <int DH, int SUB = SUB_BYTES>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, uint32_t bar, int head, int row) {
#pragma unroll
    for (int c = 0; c < DH / 64; c++) tma_load_2d(dst + c * SUB, map, bar, head * DH + c * 64, row);
}

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&h);
}
// Two fp32 values in one 64-bit register: sm_100 multiplies and adds them with one instruction.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split(f32x2 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// P of 32 scores of a row: 2^(s * scale + shift), shift of each pair from `shift(e)`.  HIDDEN: pairs that are not seen get 0.
// (Every fourth to every second pair through a polynomial on the fma units instead of ex2 changed no time by more than the
// noise, here and in the forward: the kernels are not bound by the special-function unit.)
template <bool HIDDEN, typename F>
__device__ __forceinline__ void exponentials(const uint32_t (&rs)[32], float scale, uint32_t see, F shift, f32x2 (&pv)[16]) {
    const f32x2 sc = pair(scale, scale);
#pragma unroll
    for (int e = 0; e < 16; e++) {
        const f32x2 x = fma2(pair(__uint_as_float(rs[2 * e]), __uint_as_float(rs[2 * e + 1])), sc, shift(e));
        float a, b;
        split(x, a, b);
        if (HIDDEN) {
            if (!(see >> (2 * e) & 1u)) a = -INFINITY;
            if (!(see >> (2 * e + 1) & 1u)) b = -INFINITY;
        }
        pv[e] = pair(fast_exp2(a), fast_exp2(b));
    }
}
__device__ __forceinline__ uint32_t pack_pair(f32x2 v) {
    float a, b;
    split(v, a, b);
    return pack_bf16(a, b);
}

// Rows of K and V that no query of the chunk sees may hold anything, and 0 times that need not be 0.  They are the zeros that a
// copy puts where its tensor ends: sinks are read from a tensor that ends with them (edge tile), the first tile of the windows
// from one that begins with their first row (Gap).  Where one tile holds both the last sinks and the first row of the windows
// (CLEAR kernels), the warp that issues its products overwrites the rows between them.
struct Gap {
    int tile, from;       // the first tile of the windows where no query sees its first rows (-1: none); the windows' first row
};
template <int T>
Gap gap_of(const WindowShape &w, bool &clear) {
    Gap g = {-1, w.seen_from()};
    clear = false;
    if (g.from <= w.sinks || g.from % T == 0) return g;          // nothing between the sinks and the windows; a whole tile
    if (w.sinks > g.from / T * T) clear = true;
    else g.tile = g.from / T;
    return g;
}
template <int DH, int ROWS, int SUB>
__device__ __forceinline__ void clear_unseen(const WindowShape &w, uint32_t tile, int k0, int lane) {
    if (k0 >= w.seen_from() || k0 + ROWS <= w.sinks) return;
    for (int r = lane; r < ROWS; r += 32)
        if (w.unseen(k0 + r))
            for (int e = 0; e < DH / 8; e++)
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + (e >> 3) * SUB + r * 128 + (e & 7) * 16), "r"(0) : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}
// bits [0, n) of 32, n clamped
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : (n >= 32 ? 0xffffffffu : (1u << n) - 1u); }
// Which of the keys k0 + base .. + 31 the query row sees, as bits.
__device__ __forceinline__ uint32_t visible_keys(const WindowShape &w, int row, int k0, int base) {
    const int at = k0 + base;
    return below(row + 1 - at) & (~below(row - w.window + 1 - at) | below(w.sinks - at));
}
// Which of a tile's columns base .. + 31 see the key, as bits: columns are query rows q0 .. of `heads` heads each, the heads
// of a row side by side; `cols` are used.
__device__ __forceinline__ uint32_t visible_columns(const WindowShape &w, int key, int q0, int heads, int cols, int base) {
    auto before = [&](int row) { return below(min(max(row - q0, 0), 128) * heads - base); };     // the columns of rows q0 .. row - 1
    const uint32_t behind = below(cols - base) & ~before(key);
    return key < w.sinks ? behind : behind & before(key + w.window);
}
// Whether a (query tile, key tile) pair holds hidden pairs: the diagonal or the window's far edge crosses it.
__device__ __forceinline__ bool mixed(const WindowShape &w, int q0, int rows, int k0, int keys) {
    return k0 + keys - 1 > q0 || (q0 + rows - 1 - k0 >= w.window && k0 + keys > w.sinks);
}

__device__ __forceinline__ void leave(volatile int *abort_flag) {
    if (*abort_flag) {   // give copies that are still in flight time to land before shared memory is released
        const unsigned long long t0 = global_timer();
        while (global_timer() - t0 < 200000ull) { }
    }
}

// ---------------------------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------------------------
constexpr int KT = 64;                    // keys per tile of the forward: two S tiles fit beside O in half of tensor memory
struct FwdParams {
    WindowShape w;
    float *lse;         // [Hq, n]
    float scale_log2;   // log2(e) / sqrt(head_dim)
    int heads, tokens;  // rows of a tile: `tokens` query rows of `heads` heads of one group, the heads of a row side by side
    int q_tiles, items; // items = q_tiles * Hq / heads, the last query tiles (longest spans) first, heads side by side
    int split;          // CTAs that share an item's key tiles, a cluster (SPLIT kernel)
    bf16 *o;            // SPLIT kernel
    int edge, edge_keys;// the sink tile that holds sinks in its first rows only (-1: none), and those rows rounded up to 16
    Gap gap;
};

template <int DH> struct Fwd {
    static constexpr int kQ = TILE * DH * 2, kKV = KT * DH * 2;
    static constexpr int kQRing = DH == 64 ? 2 : 1, kRing = DH == 64 ? 3 : 2;      // what leaves room for two CTAs
    static constexpr int kS = (256 - DH) / KT;             // S tiles in tensor memory: 3 or 2
    static constexpr int kThreads = 64 + 128;
    static constexpr int kStaging = 4 * 2 * 2048;          // two 32 x 32 blocks of O per softmax warp
    static constexpr int kSlack = 768;                     // what two CTAs leave for aligning the tiles to 1024 bytes
    static constexpr int kSmem = kQRing * kQ + 2 * kRing * kKV + kStaging + kSlack + 256;
    static_assert(2 * (kSmem + 1024) <= 233472, "two CTAs share an SM");
    static_assert((2 * kQRing + 4 * kRing + 3 * kS) * 8 <= 232, "barriers");
};
constexpr int KSUB = KT * 64 * 2;         // one [64 keys][64 columns] swizzled sub-tile
__host__ __device__ constexpr uint32_t kvstep(int kk) { return (uint32_t)((kk >> 2) * (KSUB >> 4) + (kk & 3) * 2); }

struct RingAt {                                            // stage and phase of the next use of a ring of N stages
    uint32_t st = 0, ph = 0;
    template <int N> __device__ __forceinline__ void next() {
        if (++st == N) { st = 0; ph ^= 1u; }
    }
};

// The running maximum of a row takes in the maximum `mt` of a tile; O and l are rescaled where it grew by more than 2^8
// (the product with the previous P has to have completed: `rest` waits for it).
template <int DH, typename F>
__device__ __forceinline__ bool take_maximum(float mt, uint32_t tO, bool later, float &m_used, float &l, F rest) {
    float factor = 1.f;
    bool rescale = false;
    if (mt > m_used + 8.f) {                              // also true on the first tile with a visible key:
        rescale = m_used != -INFINITY;                    // nothing to rescale then, the row's O is zero or not yet written
        if (rescale) factor = fast_exp2(m_used - mt);
        m_used = mt;
        l *= factor;
    }
    if (later && __any_sync(0xffffffffu, rescale)) {
        if (!rest()) return false;
        tc_fence_after();
#pragma unroll 1
        for (int c = 0; c < DH / 32; c++) {
            uint32_t o[32];
            tmem_ld32(tO + c * 32, o);
#pragma unroll
            for (int e = 0; e < 32; e++) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
            tmem_st32(tO + c * 32, o);
        }
    }
    return true;
}

// One key tile of a query row: scores from tensor memory, P packed over the first 32 of their 64 columns.  HIDDEN: the tile
// holds keys the row does not see (see[]: the ones it does).
template <bool HIDDEN, int DH, typename F>
__device__ __forceinline__ bool softmax_tile(float scale_log2, uint32_t tS, uint32_t tO, const uint32_t (&see)[2], bool later,
                                             float &m_used, float &l, F rest) {
    uint32_t r[KT];
    tmem_ld32_async(tS, r);
    tmem_ld32_async(tS + 32, r + 32);
    // of each group of 32 columns: whether some row of the warp sees one (else its P is zero without an exponential), and
    // whether every row sees all (else the hidden scores are struck out)
    bool some[2] = {true, true};
    if (HIDDEN) {
        some[0] = __any_sync(0xffffffffu, see[0] != 0u);
        some[1] = __any_sync(0xffffffffu, see[1] != 0u);
    }
    tmem_wait_ld();
    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int c = 0; c < 2; c++) {
        if (HIDDEN && !__all_sync(0xffffffffu, see[c] == 0xffffffffu)) {
            if (!some[c]) continue;
#pragma unroll
            for (int e = 0; e < 32; e++)
                if (!(see[c] >> e & 1u)) r[c * 32 + e] = 0xff800000u;              // -inf
        }
#pragma unroll
        for (int e = 0; e < 32; e++) m4[e & 3] = fmaxf(m4[e & 3], __uint_as_float(r[c * 32 + e]));
    }
    if (!take_maximum<DH>(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * scale_log2, tO, later, m_used, l, rest)) return false;
    const float neg_m = HIDDEN && m_used == -INFINITY ? 0.f : -m_used;        // nothing seen so far: exact zeros
    float l4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 2; c++) {
        uint32_t pk[16];
        if (!HIDDEN || some[c]) {
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                const float p0 = fast_exp2(fmaf(__uint_as_float(r[c * 32 + e]), scale_log2, neg_m));
                const float p1 = fast_exp2(fmaf(__uint_as_float(r[c * 32 + e + 1]), scale_log2, neg_m));
                l4[(e >> 1) & 3] += p0 + p1;
                pk[e >> 1] = pack_bf16(p0, p1);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; e++) pk[e] = 0u;
        }
        tmem_st16(tS + c * 16, pk);
    }
    l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
    return true;
}

template <int N>
__device__ __forceinline__ void ld_cluster(uint32_t addr, float (&v)[N]) {
    static_assert(N == 2 || N == 4, "8 or 16 bytes");
    if (N == 4) asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[N - 2]), "=f"(v[N - 1]) : "r"(addr));
    else asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(addr));
}

// SPLIT: one item to a cluster, its key tiles dealt to the CTAs in order; each leaves O, the reference of its exponentials
// and their sum in its shared memory, and the rows are joined from there, dealt to the warps of all.
template <int DH, bool SPLIT, bool CLEAR>
__global__ void __launch_bounds__(Fwd<DH>::kThreads, 2)
    attn_window_fwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                           const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_ke,
                           const __grid_constant__ CUtensorMap map_ve, const __grid_constant__ CUtensorMap map_kg,
                           const __grid_constant__ CUtensorMap map_vg, const __grid_constant__ CUtensorMap map_o, const FwdParams p) {
    pdl_enter();
    typedef Fwd<DH> F;
    constexpr int N = F::kRing, NQ = F::kQRing, NS = F::kS;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    const uint32_t sQ = base, sK = sQ + NQ * F::kQ, sV = sK + N * F::kKV, sO = sV + N * F::kKV;
    uint8_t *aux = smem_raw + (base - raw) + NQ * F::kQ + 2 * N * F::kKV + F::kStaging;
    const uint32_t bars = smem_u32(aux);
    const uint32_t q_full = bars, q_empty = q_full + 8 * NQ, k_full = q_empty + 8 * NQ, k_empty = k_full + 8 * N,
                   v_full = k_empty + 8 * N, v_empty = v_full + 8 * N, s_full = v_empty + 8 * N, p_full = s_full + 8 * NS,
                   pv_done = p_full + 8 * NS;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(aux + 232);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(aux + 240);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = SPLIT ? (int)cluster_cta_rank() : 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < NQ; s++) {
            mbar_init(q_full + 8 * s, 1);
            mbar_init(q_empty + 8 * s, 1);
        }
        for (int s = 0; s < N; s++) {
            mbar_init(k_full + 8 * s, 1);
            mbar_init(k_empty + 8 * s, 1);
            mbar_init(v_full + 8 * s, 1);
            mbar_init(v_empty + 8 * s, 1);
        }
        for (int s = 0; s < NS; s++) {
            mbar_init(s_full + 8 * s, 1);
            mbar_init(p_full + 8 * s, 4);
            mbar_init(pv_done + 8 * s, 1);
        }
        // a base that needs more alignment than the carve-out leaves cannot be used
        *abort_flag = (int)(base - raw) > F::kSlack ? 1 : 0;
        if (*abort_flag) atomicExch(&g_tc_fault, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(tmem_slot), 256);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;      // O (DH columns), then the S tiles (64 columns each)
    const bool usable = *abort_flag == 0;

    // an item: the query tile's rows of some heads of a group against key tiles begin .. end - 1 of its span
    struct Item { int h0, t0, first, begin, end; KeySpan span; };
    const int groups = p.w.Hq / p.heads;
    auto item_at = [&](int i) {
        Item t;
        t.h0 = i % groups * p.heads;
        t.t0 = (p.q_tiles - 1 - i / groups) * p.tokens;
        const int rows = p.w.n - t.t0 < p.tokens ? p.w.n - t.t0 : p.tokens;
        t.first = p.w.q0 + t.t0;
        t.span = key_span<KT>(p.w, t.first, t.first + rows - 1);
        const int count = t.span.count();
        t.begin = SPLIT ? (int)((long long)count * rank / p.split) : 0;
        t.end = SPLIT ? (int)((long long)count * (rank + 1) / p.split) : count;
        return t;
    };
    // the items of this CTA: SPLIT, the cluster's one, or none where there are fewer key tiles than CTAs
    const Item mine = item_at(SPLIT ? (int)blockIdx.x / p.split : 0);
    auto first_item = [&] { return SPLIT ? (int)blockIdx.x / p.split : (int)blockIdx.x; };
    auto next_item = [&](int i) { return SPLIT ? p.items : i + (int)gridDim.x; };
    auto is_item = [&](int i) { return i < p.items && (!SPLIT || mine.begin < mine.end); };
    // keys of a tile that take part: all, or the sinks at the head of the edge tile where the window does not reach it
    auto keys_of = [&](const Item &t, int j) { return j < t.span.ns && j == p.edge ? p.edge_keys : KT; };

    if (!usable) {
        // nothing was issued: fall through to the common exit
    } else if (warp == 0) {
        if (lane == 0) {
            RingAt q, kv;
            bool alive = true;
            for (int i = first_item(); is_item(i) && alive; i = next_item(i)) {
                const Item t = item_at(i);
                const int g = t.h0 / (p.w.Hq / p.w.Hkv);
                if (!mbar_wait(q_empty + 8 * q.st, q.ph ^ 1u, abort_flag)) break;
                mbar_expect_tx(q_full + 8 * q.st, (uint32_t)(p.heads * p.tokens * DH * 2));
#pragma unroll
                for (int c = 0; c < DH / 64; c++)
                    tma_load_3d(sQ + q.st * F::kQ + c * SUB_BYTES, &map_q, q_full + 8 * q.st, c * 64, t.h0, t.t0);
                q.next<NQ>();
                for (int j = t.begin; j < t.end; j++) {
                    const int tile = t.span.tile(j), keys = keys_of(t, j);
                    const bool part = j < t.span.ns && j == p.edge, gap = tile == p.gap.tile;
                    const int row = tile * KT - (gap ? p.gap.from : 0);
                    const uint32_t bytes = (uint32_t)keys * DH * 2u;
                    if (!mbar_wait(k_empty + 8 * kv.st, kv.ph ^ 1u, abort_flag)) { alive = false; break; }
                    mbar_expect_tx(k_full + 8 * kv.st, bytes);
#pragma unroll
                    for (int c = 0; c < DH / 64; c++)
                        tma_load_2d(sK + kv.st * F::kKV + c * KSUB, part ? &map_ke : gap ? &map_kg : &map_k, k_full + 8 * kv.st, g * DH + c * 64, row);
                    if (!mbar_wait(v_empty + 8 * kv.st, kv.ph ^ 1u, abort_flag)) { alive = false; break; }
                    mbar_expect_tx(v_full + 8 * kv.st, bytes);
#pragma unroll
                    for (int c = 0; c < DH / 64; c++)
                        tma_load_2d(sV + kv.st * F::kKV + c * KSUB, part ? &map_ve : gap ? &map_vg : &map_v, v_full + 8 * kv.st, g * DH + c * 64, row);
                    kv.next<N>();
                }
            }
        }
    } else if (warp == 1) {
        constexpr uint32_t idesc_pv = make_idesc(TILE, DH, false, true);
        // two cursors over the same sequence of (item, tile): S runs up to NS tiles ahead of P V
        RingAt q, k, v, bs, bp;                         // rings: Q and K (by S), V (by P V), S tiles (by S and by P V)
        int is = first_item(), js = 0, ip = is, jp = 0;
        Item ts, tp;
        if (is_item(is)) {
            ts = tp = item_at(is);
            js = jp = ts.begin;
        }
        bool alive = true;
        auto issue_s = [&]() -> bool {                  // S = Q K^T of the next tile; the last of an item hands Q back
            if (!is_item(is)) return true;
            if (js == ts.begin && !mbar_wait_warp(q_full + 8 * q.st, q.ph, abort_flag)) return false;
            if (!mbar_wait_warp(k_full + 8 * k.st, k.ph, abort_flag)) return false;
            tc_fence_after();
            const uint32_t q_lo = klo(sQ + q.st * F::kQ), k_lo = klo(sK + k.st * F::kKV);
            const uint32_t idesc_s = make_idesc(TILE, keys_of(ts, js), false, false), d = tmem + DH + bs.st * KT;
#pragma unroll
            for (int kk = 0; kk < DH / 16; kk++) umma_ss_w(d, q_lo + kstep(kk), k_lo + kvstep(kk), idesc_s, kk != 0);
            umma_commit_w(s_full + 8 * bs.st);
            umma_commit_w(k_empty + 8 * k.st);
            k.next<N>();
            bs.next<NS>();
            if (++js == ts.end) {
                umma_commit_w(q_empty + 8 * q.st);
                q.next<NQ>();
                is = next_item(is);
                if (is_item(is)) {
                    ts = item_at(is);
                    js = ts.begin;
                }
            }
            return true;
        };
        for (int s = 0; s < NS && alive; s++) alive = issue_s();
        while (alive && is_item(ip)) {
            // O += P V once P is stored; the S tile that P lay in then takes the scores NS tiles further on
            if (!mbar_wait_warp(v_full + 8 * v.st, v.ph, abort_flag)) break;
            if (CLEAR) clear_unseen<DH, KT, KSUB>(p.w, sV + v.st * F::kKV, tp.span.tile(jp) * KT, lane);
            if (!mbar_wait_warp(p_full + 8 * bp.st, bp.ph, abort_flag)) break;
            tc_fence_after();
            const uint32_t v_lo = desc_lo(sV + v.st * F::kKV, KSUB), a = tmem + DH + bp.st * KT;
            const int slices = keys_of(tp, jp) / 16;
#pragma unroll
            for (int kk = 0; kk < KT / 16; kk++)
                if (kk < slices) umma_ts_w(tmem, a + kk * 8, v_lo + mnstep(kk), idesc_pv, jp != tp.begin || kk != 0);
            umma_commit_w(v_empty + 8 * v.st);
            umma_commit_w(pv_done + 8 * bp.st);
            v.next<N>();
            bp.next<NS>();
            alive = issue_s();
            if (++jp == tp.end) {
                ip = next_item(ip);
                if (is_item(ip)) {
                    tp = item_at(ip);
                    jp = tp.begin;
                }
            }
        }
    } else {
        const int quarter = warp & 3;
        const int row = quarter * 32 + lane, token = row / p.heads, head = row % p.heads;
        const int seen_as = token < p.tokens ? token : p.tokens - 1;       // rows that are none of the tile's see as its last
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tO = tmem + lane_base;
        const uint32_t stage0 = sO + quarter * 4096u;
        RingAt b, before;                                // S tile of this step and of the one before
        bool alive = true;
        // P V of the step before has completed.  One barrier per S tile: a warp may be a tile or two ahead of the others,
        // and S of a tile, which it has seen, was issued behind the last use of that tile's barrier -- a single barrier
        // could still be two phases back and pass for done.
        auto rest = [&]() -> bool { return mbar_wait(pv_done + 8 * before.st, before.ph, abort_flag); };
        for (int i = first_item(); is_item(i) && alive; i = next_item(i)) {
            const Item t = item_at(i);
            const int q_abs = t.first + seen_as;
            float m_used = -INFINITY, l = 0.f;
            for (int j = t.begin; j < t.end; j++) {
                const int k0 = t.span.tile(j) * KT;
                const uint32_t tS = tmem + DH + b.st * KT + lane_base;
                const bool hidden = mixed(p.w, t.first, p.tokens, k0, KT);
                uint32_t see[2];
                if (hidden) {
                    see[0] = visible_keys(p.w, q_abs, k0, 0);
                    see[1] = visible_keys(p.w, q_abs, k0, 32);
                }
                if (!mbar_wait(s_full + 8 * b.st, b.ph, abort_flag)) { alive = false; break; }
                tc_fence_after();
                alive = hidden ? softmax_tile<true, DH>(p.scale_log2, tS, tO, see, j > t.begin, m_used, l, rest)
                               : softmax_tile<false, DH>(p.scale_log2, tS, tO, see, j > t.begin, m_used, l, rest);
                if (!alive) break;
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * b.st);
                before = b;
                b.next<NS>();
            }
            if (!alive || !rest()) { alive = false; break; }
            tc_fence_after();
            if (SPLIT) {       // the rings of K and V are done with: O there, 16-byte groups of eight rows on different banks
                if (quarter * 32 < p.heads * p.tokens) {
#pragma unroll 1
                    for (int c = 0; c < DH / 32; c++) {
                        uint32_t o[32];
                        tmem_ld32(tO + c * 32, o);
#pragma unroll
                        for (int e = 0; e < 8; e++)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                                         ::"r"(sK + (uint32_t)(row * DH * 4 + (((c * 8 + e) ^ (row & 7)) << 4))), "r"(o[4 * e]),
                                         "r"(o[4 * e + 1]), "r"(o[4 * e + 2]), "r"(o[4 * e + 3]) : "memory");
                    }
                    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(sO + row * 8u), "f"(m_used), "f"(l) : "memory");
                }
                continue;
            }
            // O / l through 32 x 32 blocks in shared memory (rows of 64 bytes, 64-byte swizzle) and TMA stores, which clip
            // the rows behind the last query; the warp's next P is handed over only after its O has been read
            const float inv = 1.f / l;
#pragma unroll 1
            for (int c = 0; c < DH / 32; c++) {
                uint32_t o[32];
                tmem_ld32(tO + c * 32, o);
                const uint32_t stage = stage0 + (c & 1) * 2048u;
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");    // the block before last
                __syncwarp();
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    uint32_t wd[4];
#pragma unroll
                    for (int u = 0; u < 4; u++)
                        wd[u] = pack_bf16(__uint_as_float(o[e + 2 * u]) * inv, __uint_as_float(o[e + 2 * u + 1]) * inv);
                    const uint32_t at = stage + (uint32_t)lane * 64u + ((uint32_t)((e >> 3) ^ ((lane >> 1) & 3)) << 4);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(wd[0]), "r"(wd[1]), "r"(wd[2]), "r"(wd[3]) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    tma_store_3d(&map_o, stage, c * 32, t.h0, t.t0 + quarter * (32 / p.heads));
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
            }
            if (t.t0 + token < p.w.n) p.lse[(long long)(t.h0 + head) * p.w.n + t.t0 + token] = (m_used + log2f(l)) * kLn2;
        }
        if (SPLIT && mine.begin == mine.end) asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(sO + row * 8u), "f"(-INFINITY), "f"(0.f) : "memory");
        if (!SPLIT && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }

    __syncwarp();
    if (SPLIT) {
        cluster_sync_all();
        // out = sum_c 2^(m_c - m) O_c / sum_c 2^(m_c - m) l_c over the CTAs c; four rows to a warp at a time, a lane has DH / 32
        // columns of each
        if (!*abort_flag) {
            constexpr int NC = DH / 32;
            const Item &t = mine;
            const int rows = (p.w.n - t.t0 < p.tokens ? p.w.n - t.t0 : p.tokens) * p.heads, warps = p.split * (F::kThreads / 32);
            for (int r0 = rank * (F::kThreads / 32) + warp; r0 < rows; r0 += 4 * warps) {
                // lane (row i, CTA c): their reference, sum and weight
                const int c_l = lane & 7, r_l = r0 + (lane >> 3) * warps;
                float m = -INFINITY, l = 0.f;
                if (c_l < p.split && r_l < rows) {
                    const uint32_t at = map_to_cta(sO, (uint32_t)c_l) + r_l * 8u;
                    m = ld_cluster_f32(at);
                    l = ld_cluster_f32(at + 4u);
                }
                float top = m;
#pragma unroll
                for (int x = 1; x < 8; x *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                const float f = m == -INFINITY ? 0.f : fast_exp2(m - top);
                float sum = l * f;
#pragma unroll
                for (int x = 1; x < 8; x *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, x);
                const float weight = f / sum;
                float acc[4][NC];
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int e = 0; e < NC; e++) acc[i][e] = 0.f;
#pragma unroll 2
                for (int c = 0; c < p.split; c++) {
                    const uint32_t from = map_to_cta(sK, (uint32_t)c);
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int r = r0 + i * warps;
                        const float wt = __shfl_sync(0xffffffffu, weight, i * 8 + c);
                        float o[NC];
                        if (r >= rows) continue;
                        ld_cluster<NC>(from + (uint32_t)(r * DH * 4 + (((lane * NC >> 2) ^ (r & 7)) << 4) + (lane * NC & 3) * 4), o);
#pragma unroll
                        for (int e = 0; e < NC; e++)
                            if (wt != 0.f) acc[i][e] = fmaf(o[e], wt, acc[i][e]);      // nothing seen there: O may never have been written
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int r = r0 + i * warps;
                    if (r >= rows) break;
                    const int h = t.h0 + r % p.heads, at = t.t0 + r / p.heads;
                    bf16 *out = p.o + ((long long)at * p.w.Hq + h) * DH + lane * NC;
#pragma unroll
                    for (int e = 0; e < NC; e += 2) *reinterpret_cast<uint32_t *>(out + e) = pack_bf16(acc[i][e], acc[i][e + 1]);
                }
                if (c_l == 0 && r_l < rows)
                    p.lse[(long long)(t.h0 + r_l % p.heads) * p.w.n + t.t0 + r_l / p.heads] = (top + log2f(sum)) * kLn2;
            }
        }
        __syncwarp();
    }
    leave(abort_flag);
    tc_fence_before();
    __syncthreads();
    if (SPLIT) cluster_sync_all();          // no CTA leaves while another may read its sums
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 256);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------------------------
// What the two head sizes need of an SM decides their shape.  Heads of 128: inner tiles of 128 (every product a full one),
// all of tensor memory, one CTA of sixteen softmax warps per SM.  Heads of 64: the products are short and what bounds an
// iteration is its chain of loads, exponentials and hand-offs, so inner tiles of 64 and half of tensor memory let two
// independent CTAs of eight softmax warps share an SM, each in the other's latencies.
template <int DH> struct Bwd {
    static constexpr int IT = DH == 64 ? kBwdRows64 : kBwdRows128;   // query rows (dK/dV role) or keys (dQ role) of an inner tile
    static constexpr int kGroups = IT / 32;                          // softmax warpgroups, 32 columns of a row each
    static constexpr int kThreads = 64 + 128 * kGroups;
    static constexpr int kBlocks = DH == 64 ? 2 : 1;
    static constexpr uint32_t kCols = DH == 64 ? 256 : 512;
    static constexpr int kOut = TILE * DH * 2, kIn = IT * DH * 2;    // bytes of a resident and of an inner tile
    static constexpr int kInSub = IT * 64 * 2;
    static constexpr int kQStages = 3, kKStages = 3;
    static constexpr int kSlack = 768;                               // what is left for aligning the tiles to 1024 bytes
    static constexpr int kTiles = 2 * kOut + 5 * kIn;
    static constexpr int kSmem = kTiles + 4 * IT * 4 /* lse, delta x 2 stages */ + 256 + kSlack;
    static_assert(kBlocks * (kSmem + 1024) <= 233472 && 4 * kGroups * 8192 <= kTiles, "backward roles exceed the shared memory of an SM");
    typedef KeyWork<TILE> Work;
    __host__ __device__ static constexpr uint32_t step(int kk) { return (uint32_t)((kk >> 2) * (kInSub >> 4) + (kk & 3) * 2); }
};
template <int DH>
struct BwdParams {
    WindowShape w;
    typename Bwd<DH>::Work work;
    const float *lse;     // [Hq, n]
    const float *delta;   // [Hq, n]
    void *dq, *dk, *dv;   // [n, Hq, DH], [q0 + n, Hkv, DH]
    float *part;          // sums of segments: [item][Hkv][dK, dV][part_rows][DH]
    int part_rows;
    int mode;             // GradMode of dk, dv (dq: fp32 or bf16, always overwritten)
    Gap gap;              // dQ role: the first tile of the windows where no query sees its first rows
    int edge, edge_keys;  // dQ role: the sink tile that holds sinks in its first rows only (-1: none), those rows rounded up to 32
    int split;                      // PACKED: CTAs that share a dQ item's key tiles, a cluster (1: none)
    int n_dkdv, n_dq_first;         // dK/dV CTAs; dQ CTAs that are dispatched before them (all or none)
    float scale, scale_log2;
    // PACKED: several heads of a group share a tile.  Heads of a query row, query rows of an inner tile (dK/dV role), the rows
    // that these make, query rows of a resident tile (dQ role).
    template <bool PACKED> __host__ __device__ int heads() const { return PACKED ? work.heads : 1; }
    template <bool PACKED> __host__ __device__ int rows() const { return PACKED ? work.tq : Bwd<DH>::IT; }
    template <bool PACKED> __host__ __device__ int used() const { return PACKED ? work.heads * work.tq : Bwd<DH>::IT; }
    template <bool PACKED> __host__ __device__ int tokens() const { return PACKED ? TILE / work.heads : TILE; }
};

// 32 fp32 sums of one row to where the gradient goes
__device__ __forceinline__ void put32(void *dst, long long at, const uint32_t (&r)[32], int mode) {
    if (mode == GRAD_BF16_SET) {
        bf16 *d = static_cast<bf16 *>(dst) + at;
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
            uint32_t wd[4];
#pragma unroll
            for (int t = 0; t < 4; t++) wd[t] = pack_bf16(__uint_as_float(r[e + 2 * t]), __uint_as_float(r[e + 2 * t + 1]));
            *reinterpret_cast<uint4 *>(d + e) = make_uint4(wd[0], wd[1], wd[2], wd[3]);
        }
    } else {
        float *d = static_cast<float *>(dst) + at;
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
            float4 a = make_float4(__uint_as_float(r[e]), __uint_as_float(r[e + 1]), __uint_as_float(r[e + 2]), __uint_as_float(r[e + 3]));
            if (mode == GRAD_F32_ADD) {
                const float4 b = *reinterpret_cast<const float4 *>(d + e);
                a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
            }
            *reinterpret_cast<float4 *>(d + e) = a;
        }
    }
}

// The same for a warp's 32 rows through a block of shared memory and a TMA store (or add), which clips the rows behind the
// last.  Written by the lanes themselves, 16 bytes of 32 rows at a time, the epilogue of a CTA took 4000 - 8000 cycles.
template <typename Store>
__device__ __forceinline__ void put_block(uint32_t at, const uint32_t (&r)[32], int lane, int mode, Store store) {
    if (mode == GRAD_BF16_SET) {                            // rows of 64 bytes, 64-byte swizzle
#pragma unroll
        for (int j = 0; j < 4; j++) {
            uint32_t wd[4];
#pragma unroll
            for (int t = 0; t < 4; t++) wd[t] = pack_bf16(__uint_as_float(r[8 * j + 2 * t]), __uint_as_float(r[8 * j + 2 * t + 1]));
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)), "r"(wd[0]),
                         "r"(wd[1]), "r"(wd[2]), "r"(wd[3]) : "memory");
        }
    } else {                                                // rows of 128 bytes, 128-byte swizzle
#pragma unroll
        for (int j = 0; j < 8; j++)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(r[4 * j]),
                         "r"(r[4 * j + 1]), "r"(r[4 * j + 2]), "r"(r[4 * j + 3]) : "memory");
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        store();
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
__device__ __forceinline__ void put_block(const CUtensorMap *map, uint32_t at, const uint32_t (&r)[32], int lane, int col, int row0, int mode) {
    put_block(at, r, lane, mode, [&] {
        if (mode == GRAD_F32_ADD) tma_reduce_add_2d(map, at, col, row0);
        else tma_store_2d(map, at, col, row0);
    });
}
// rows [rows][heads] of a tile of DH columns
template <int DH, int SUB>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap *map, uint32_t bar, int head, int row) {
#pragma unroll
    for (int c = 0; c < DH / 64; c++) tma_load_3d(dst + c * SUB, map, bar, c * 64, head, row);
}

template <int DH, bool PACKED>
__device__ __forceinline__ void dkdv_body(const CUtensorMap &map_q, const CUtensorMap &map_k, const CUtensorMap &map_v,
                                          const CUtensorMap &map_do, const CUtensorMap &map_dk, const CUtensorMap &map_dv,
                                          const CUtensorMap &map_part, const BwdParams<DH> &p, uint8_t *smem_raw, int item, int g) {
    typedef Bwd<DH> W;
    constexpr int T = W::kIn, QS = W::kQStages, IT = W::IT;
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    const uint32_t sK = base, sV = sK + W::kOut, sQ = sV + W::kOut, sdO = sQ + QS * T;
    uint8_t *tail = smem_raw + (base - raw) + W::kTiles;
    float *s_lse = reinterpret_cast<float *>(tail);           // [2][IT], -lse * log2(e)
    float *s_delta = s_lse + 2 * IT;                          // [2][IT], -delta * scale
    uint8_t *aux = tail + 4 * IT * 4;
    const uint32_t bars = smem_u32(aux);
    const uint32_t kv_full = bars, q_full = bars + 8, q_empty = bars + 32, do_full = bars + 56, do_empty = bars + 72,
                   rows_empty = bars + 88, s_full = bars + 104, dp_full = bars + 112, loaded = bars + 120,
                   p1_full = bars + 128, p2_full = bars + 136, acc_full = bars + 144;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(aux + 152);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(aux + 160);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.w.Hq / p.w.Hkv;
    int kt, qt_begin, qt_end, seg;
    p.work.item(p.w, item, kt, qt_begin, qt_end, seg);
    const int k_abs0 = kt * TILE;
    const int iters = G / p.template heads<PACKED>() * (qt_end - qt_begin);     // the query heads of the group, `heads` at a time, over the item's query tiles

    if (threadIdx.x == 0) {
        mbar_init(kv_full, 1);
        for (int s = 0; s < QS; s++) {
            mbar_init(q_full + 8 * s, 1);
            mbar_init(q_empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; s++) {
            mbar_init(do_full + 8 * s, 1);
            mbar_init(do_empty + 8 * s, 1);
            mbar_init(rows_empty + 8 * s, 1);
        }
        mbar_init(s_full, 1);
        mbar_init(dp_full, 1);
        mbar_init(loaded, 4 * W::kGroups);
        mbar_init(p1_full, 4 * W::kGroups);
        mbar_init(p2_full, 4 * W::kGroups);
        mbar_init(acc_full, 1);
        // a base that needs more alignment than the carve-out leaves cannot be used
        *abort_flag = (int)(base - raw) > W::kSlack ? 1 : 0;
        if (*abort_flag) atomicExch(&g_tc_fault, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (p.template used<PACKED>() < IT) {       // rows that no copy reaches are factors of the products: zeros
        for (int i = threadIdx.x; i < (QS + 2) * (DH / 64) * (IT - p.template used<PACKED>()) * 8; i += W::kThreads) {
            const int sub = i / ((IT - p.template used<PACKED>()) * 8), at = i % ((IT - p.template used<PACKED>()) * 8);
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sQ + sub * W::kInSub + p.template used<PACKED>() * 128 + at * 16), "r"(0) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(tmem_slot), W::kCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // columns: S^T; dP^T, later P^T (packed) in the first and dS^T (packed) in the second 16 columns of every 32-column
    // group; dV; dK
    const uint32_t tST = tmem, tDPT = tST + IT, tDV = tDPT + IT, tDK = tDV + DH;
    const bool usable = *abort_flag == 0;
    bool done = false;                     // softmax warps: the sums of this CTA are complete

    if (!usable) {
        // nothing was issued: fall through to the common exit
    } else if (warp == 0) {
        if (lane == 0 && iters > 0) {
            mbar_expect_tx(kv_full, 2 * W::kOut);
            load_tile<DH>(sK, &map_k, kv_full, g, k_abs0);
            load_tile<DH>(sV, &map_v, kv_full, g, k_abs0);
        }
        uint32_t sq = 0, qph = 0;
        int h = g * G, qt = qt_begin;
        const uint32_t bytes = (uint32_t)(p.template used<PACKED>() * DH * 2);
        int col_row[IT / 32], col_head[IT / 32];
#pragma unroll
        for (int e = 0; e < IT / 32; e++) {
            col_row[e] = (lane * (IT / 32) + e) / p.template heads<PACKED>();
            col_head[e] = (lane * (IT / 32) + e) % p.template heads<PACKED>();
        }
        for (int it = 0; it < iters; it++) {
            const int qt0 = qt * p.template rows<PACKED>();
            const uint32_t sd = it & 1, dph = (it >> 1) & 1;
            int ok = 1;
            if (lane == 0) {
                ok = mbar_wait(q_empty + 8 * sq, qph ^ 1u, abort_flag) ? 1 : 0;          // dK of the stage's last user
                if (ok) {
                    mbar_expect_tx(q_full + 8 * sq, bytes);
                    load_rows<DH, W::kInSub>(sQ + sq * T, &map_q, q_full + 8 * sq, h, qt0);
                    ok = mbar_wait(do_empty + 8 * sd, dph ^ 1u, abort_flag) ? 1 : 0;     // dV of the stage's last user
                }
                if (ok) {
                    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(do_full + 8 * sd), "r"(bytes) : "memory");
                    load_rows<DH, W::kInSub>(sdO + sd * T, &map_do, do_full + 8 * sd, h, qt0);
                    ok = mbar_wait(rows_empty + 8 * sd, dph ^ 1u, abort_flag) ? 1 : 0;   // delta rows: read until dS^T is packed
                }
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
#pragma unroll
            for (int e = 0; e < IT / 32; e++) {
                const int col = lane * (IT / 32) + e, r = qt0 + col_row[e];
                const bool used = col < p.template used<PACKED>() && r < p.w.n;
                const long long at = (long long)(h + col_head[e]) * p.w.n + r;
                s_lse[sd * IT + col] = used ? -p.lse[at] * kLog2e : 0.f;
                s_delta[sd * IT + col] = used ? -p.delta[at] * p.scale : 0.f;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(do_full + 8 * sd);   // publishes the rows; the phase completes when dO has landed too
            if (++sq == QS) { sq = 0; qph ^= 1u; }
            if (++qt == qt_end) { qt = qt_begin; h += p.template heads<PACKED>(); }
        }
    } else if (warp == 1) {
        // the whole warp runs the issue loop; each MMA / commit executes in one elected lane
        constexpr uint32_t idesc_kk = make_idesc(TILE, IT, false, false);       // both operands K-major
        constexpr uint32_t idesc_acc = make_idesc(TILE, DH, false, true);       // B MN-major (N = head dims)
        bool alive = iters == 0 || mbar_wait_warp(kv_full, 0, abort_flag);
        const uint32_t k_lo = klo(sK), v_lo = klo(sV);
        uint32_t sq_s = 0, qph_s = 0;      // Q stage / phase of the next S^T
        uint32_t sq_k = 0;                 // Q stage of the next dK
        auto issue_st = [&]() -> bool {    // S^T = K Q^T for the next iteration
            if (!mbar_wait_warp(q_full + 8 * sq_s, qph_s, abort_flag)) return false;
            tc_fence_after();
            const uint32_t q_lo = klo(sQ + sq_s * T);
#pragma unroll
            for (int kk = 0; kk < DH / 16; kk++) umma_ss_w(tST, k_lo + kstep(kk), q_lo + W::step(kk), idesc_kk, kk != 0);
            umma_commit_w(s_full);
            if (++sq_s == QS) { sq_s = 0; qph_s ^= 1u; }
            return true;
        };
        auto issue_dpt = [&](int it) -> bool {     // dP^T = V dO^T of iteration `it`
            if (!mbar_wait_warp(do_full + 8 * (it & 1), (it >> 1) & 1, abort_flag)) return false;
            tc_fence_after();
            const uint32_t do_lo = klo(sdO + (it & 1) * T);
#pragma unroll
            for (int kk = 0; kk < DH / 16; kk++) umma_ss_w(tDPT, v_lo + kstep(kk), do_lo + W::step(kk), idesc_kk, kk != 0);
            umma_commit_w(dp_full);
            return true;
        };
        if (alive && iters > 0) alive = issue_st() && issue_dpt(0);
        for (int it = 0; it < iters && alive; it++) {
            const uint32_t sd = it & 1;
            // the softmax warps hold S^T of this iteration in registers: its columns take the next one's at once
            if (it + 1 < iters) {
                if (!mbar_wait_warp(loaded, it & 1, abort_flag)) { alive = false; break; }
                tc_fence_after();
                if (!issue_st()) { alive = false; break; }
            }
            // dV += P^T dO as soon as P^T is packed (first 16 columns of each group of the dP^T region)
            if (!mbar_wait_warp(p1_full, it & 1, abort_flag)) { alive = false; break; }
            tc_fence_after();
            const uint32_t do_mn = desc_lo(sdO + sd * T, W::kInSub);
#pragma unroll
            for (int kk = 0; kk < IT / 16; kk++)
                umma_ts_w(tDV, tDPT + (kk >> 1) * 32 + (kk & 1) * 8, do_mn + mnstep(kk), idesc_acc, (it | kk) != 0);
            umma_commit_w(do_empty + 8 * sd);            // dO of this stage is consumed (dP^T was issued earlier)
            // dK += dS^T Q (second 16 columns of each group)
            if (!mbar_wait_warp(p2_full, it & 1, abort_flag)) { alive = false; break; }
            tc_fence_after();
            const uint32_t q_mn = desc_lo(sQ + sq_k * T, W::kInSub);
#pragma unroll
            for (int kk = 0; kk < IT / 16; kk++)
                umma_ts_w(tDK, tDPT + (kk >> 1) * 32 + 16 + (kk & 1) * 8, q_mn + mnstep(kk), idesc_acc, (it | kk) != 0);
            umma_commit_w(q_empty + 8 * sq_k);           // Q of this stage is consumed
            umma_commit_w(rows_empty + 8 * sd);          // and so are the lse / delta rows
            if (++sq_k == QS) sq_k = 0;
            // the dP^T region is free once dV and dK have read it (in order): next iteration's dP^T
            if (it + 1 < iters && !issue_dpt(it + 1)) { alive = false; break; }
        }
        if (alive && iters > 0) umma_commit_w(acc_full);
    } else {
        const int quarter = warp & 3;
        const int wg = (warp - 2) >> 2;                           // 32-query group of the tile
        const int col_base = wg * 32;
        const int row = quarter * 32 + lane;                      // key row within the tile
        const int k_abs = k_abs0 + row;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        // The group reads its 32 fp32 columns of S^T and of dP^T into registers, then writes the packed bf16 pairs of P^T
        // over the first and of dS^T over the second 16 of ITS OWN dP^T columns; the MMA warp addresses each 16-query
        // slice of those A operands separately.  S^T's columns are never written by these warps.
        const uint32_t tS_g = tST + col_base + lane_base, tP_g = tDPT + col_base + lane_base;
        bool alive = true;
        int qt = qt_begin;
        for (int it = 0; it < iters && alive; it++) {
            const int q_abs0 = p.w.q0 + qt * p.template rows<PACKED>();
            const uint32_t sd = it & 1;
            if (!mbar_wait(s_full, it & 1, abort_flag)) { alive = false; break; }
            tc_fence_after();
            uint32_t rs[32];
            tmem_ld32(tS_g, rs);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(loaded);
            // the producer's lse / delta rows of this stage are published together with the dO tile
            if (!mbar_wait(do_full + 8 * sd, (it >> 1) & 1, abort_flag)) { alive = false; break; }
            const uint32_t see = p.template used<PACKED>() < IT || mixed(p.w, q_abs0, p.template rows<PACKED>(), k_abs0, TILE) ? visible_columns(p.w, k_abs, q_abs0, p.template heads<PACKED>(), p.template used<PACKED>(), col_base) : 0xffffffffu;
            if (!__any_sync(0xffffffffu, see != 0u)) {     // P and dS of all of the warp's pairs are zero
                if (!mbar_wait(dp_full, it & 1, abort_flag)) { alive = false; break; }
                tc_fence_after();
                uint32_t zero[16];
#pragma unroll
                for (int e = 0; e < 16; e++) zero[e] = 0u;
                tmem_st16(tP_g, zero);
                tmem_st16(tP_g + 16, zero);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(p1_full);
                    mbar_arrive(p2_full);
                }
                if (++qt == qt_end) qt = qt_begin;
                continue;
            }
            const f32x2 *lse2 = reinterpret_cast<const f32x2 *>(s_lse + sd * IT + col_base);
            const f32x2 *dl = reinterpret_cast<const f32x2 *>(s_delta + sd * IT + col_base);
            // phase 1: P^T = exp2(S^T * scale - lse), all the dV product needs
            f32x2 pv[16];
            auto shift = [&](int e) { return lse2[e]; };
            if (see == 0xffffffffu) exponentials<false>(rs, p.scale_log2, see, shift, pv);
            else exponentials<true>(rs, p.scale_log2, see, shift, pv);
            // dP^T of this iteration was queued a whole iteration ago; its columns become P^T and dS^T
            uint32_t pp[16];
#pragma unroll
            for (int e = 0; e < 16; e++) pp[e] = pack_pair(pv[e]);
            if (!mbar_wait(dp_full, it & 1, abort_flag)) { alive = false; break; }
            tc_fence_after();
            uint32_t rp[32];
            tmem_ld32(tP_g, rp);
            {
                tmem_st16(tP_g, pp);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p1_full);
            }
            // phase 2: dS^T = P^T * (dP^T * scale - delta * scale)
            {
                uint32_t ds[16];
                const f32x2 sc = pair(p.scale, p.scale);
#pragma unroll
                for (int e = 0; e < 16; e++)
                    ds[e] = pack_pair(mul2(pv[e], fma2(pair(__uint_as_float(rp[2 * e]), __uint_as_float(rp[2 * e + 1])), sc, dl[e])));
                tmem_st16(tP_g + 16, ds);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p2_full);
            }
            if (++qt == qt_end) qt = qt_begin;
        }
        done = alive && (iters == 0 || mbar_wait(acc_full, 0, abort_flag));
    }

    __syncwarp();
    const int wg = (warp - 2) >> 2, row = (warp & 3) * 32 + lane, col_base = wg * 32;
    if (done && wg < DH / 32) {                          // group wg holds head dims 32 * wg .. of every key
        tc_fence_after();
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        uint32_t rv[32], rk[32];
        if (iters > 0) {
            tmem_ld32(tDV + lane_base + col_base, rv);
            tmem_ld32(tDK + lane_base + col_base, rk);
        } else {
#pragma unroll
            for (int e = 0; e < 32; e++) rv[e] = rk[e] = 0u;
        }
        if (p.w.unseen(k_abs0 + row)) {                   // a row of its own, whatever K and V hold there
#pragma unroll
            for (int e = 0; e < 32; e++) rv[e] = rk[e] = 0u;
        }
        if (seg < 0) {                                    // the tiles are through with their products: room for two blocks a warp
            const uint32_t at = base + (uint32_t)(warp - 2) * 8192u;
            const int row0 = k_abs0 + (warp & 3) * 32;
            if (row0 < p.w.q0 + p.w.n) {
                put_block(&map_dv, at, rv, lane, g * DH + col_base, row0, p.mode);
                put_block(&map_dk, at + 4096u, rk, lane, g * DH + col_base, row0, p.mode);
                if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            }
        } else if (p.work.full()) {                       // this segment's share of the sums, all rows of the tile
            const uint32_t at = base + (uint32_t)(warp - 2) * 8192u;
            const int row0 = ((item * p.w.Hkv + g) * 2) * TILE + (warp & 3) * 32;
            put_block(&map_part, at, rk, lane, col_base, row0, GRAD_F32_SET);
            put_block(&map_part, at + 4096u, rv, lane, col_base, row0 + TILE, GRAD_F32_SET);
            if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        } else if (row < p.work.joined_rows(p.w, kt)) {   // the same of a sink tile's sinks
            float *part = p.part + (((long long)item * p.w.Hkv + g) * 2 * p.part_rows + row) * DH + col_base;
            put32(part, 0, rk, GRAD_F32_SET);
            put32(part, (long long)p.part_rows * DH, rv, GRAD_F32_SET);
        } else if (seg == 0 && k_abs0 + row < p.w.q0 + p.w.n) {   // segments behind the first have nothing for these rows
            const long long at = ((long long)(k_abs0 + row) * p.w.Hkv + g) * DH + col_base;
            put32(p.dv, at, rv, p.mode);
            put32(p.dk, at, rk, p.mode);
        }
    }

    __syncwarp();
    leave(abort_flag);
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, W::kCols);
    }
}

template <int DH, bool PACKED, bool CLEAR>
__device__ __forceinline__ void dq_body(const CUtensorMap &map_q, const CUtensorMap &map_k, const CUtensorMap &map_v,
                                        const CUtensorMap &map_do, const CUtensorMap &map_ke, const CUtensorMap &map_ve,
                                        const CUtensorMap &map_kg, const CUtensorMap &map_vg, const CUtensorMap &map_dq, const BwdParams<DH> &p, uint8_t *smem_raw, int block_x, int h0) {
    typedef Bwd<DH> W;
    constexpr int T = W::kIn, KS = W::kKStages, IT = W::IT;
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    // K tiles live from S_j to dQ_j, so their ring has three stages; V tiles are released right after dP_j (two stages)
    const uint32_t sQ = base, sdO = sQ + W::kOut, sK = sdO + W::kOut, sV = sK + KS * T;
    uint8_t *aux = smem_raw + (base - raw) + W::kTiles + 4 * IT * 4;
    const uint32_t bars = smem_u32(aux);
    const uint32_t q_full = bars, k_full = bars + 8, k_empty = bars + 32, v_full = bars + 56, v_empty = bars + 72,
                   s_full = bars + 88, dp_full = bars + 96, s_free = bars + 104, p2_full = bars + 112,
                   acc_full = bars + 120;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(aux + 128);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(aux + 136);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = h0 / (p.w.Hq / p.w.Hkv);
    const int qt0 = block_x * p.template tokens<PACKED>();
    const int q_abs0 = p.w.q0 + qt0;
    const int rows_here = (p.w.n - qt0) < p.template tokens<PACKED>() ? (p.w.n - qt0) : p.template tokens<PACKED>();
    const KeySpan span = key_span<IT>(p.w, q_abs0, q_abs0 + rows_here - 1);
    // the key tiles of this CTA: all of the span, or its share of them
    const int count = span.count(), rank = PACKED && p.split > 1 ? (int)cluster_cta_rank() : 0;
    const int j0 = PACKED ? (int)((long long)count * rank / p.split) : 0;
    const int nkv = PACKED ? (int)((long long)count * (rank + 1) / p.split) - j0 : count;
    auto keys_of = [&](int j) { return j0 + j < span.ns && j0 + j == p.edge ? p.edge_keys : IT; };

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        for (int s = 0; s < KS; s++) {
            mbar_init(k_full + 8 * s, 1);
            mbar_init(k_empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; s++) {
            mbar_init(v_full + 8 * s, 1);
            mbar_init(v_empty + 8 * s, 1);
        }
        mbar_init(s_full, 1);
        mbar_init(dp_full, 1);
        mbar_init(s_free, 4 * W::kGroups);
        mbar_init(p2_full, 4 * W::kGroups);
        mbar_init(acc_full, 1);
        // a base that needs more alignment than the carve-out leaves cannot be used
        *abort_flag = (int)(base - raw) > W::kSlack ? 1 : 0;
        if (*abort_flag) atomicExch(&g_tc_fault, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(tmem_slot), W::kCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // columns: S, dP, dQ
    const uint32_t tS = tmem, tDP = tS + IT, tDQ = tDP + IT;
    const bool usable = *abort_flag == 0;

    if (!usable) {
        // nothing was issued: fall through to the common exit
    } else if (warp == 0) {
        if (lane == 0 && nkv > 0) {
            mbar_expect_tx(q_full, (uint32_t)(2 * p.template heads<PACKED>() * p.template tokens<PACKED>() * DH * 2));
            load_rows<DH, SUB_BYTES>(sQ, &map_q, q_full, h0, qt0);
            load_rows<DH, SUB_BYTES>(sdO, &map_do, q_full, h0, qt0);
            uint32_t ks = 0, kph = 0;
            for (int j = 0; j < nkv; j++) {
                const int tile = span.tile(j0 + j), keys = keys_of(j);
                const bool part = j0 + j < span.ns && j0 + j == p.edge, gap = tile == p.gap.tile;
                const int row = tile * IT - (gap ? p.gap.from : 0);
                const uint32_t bytes = (uint32_t)keys * DH * 2u;
                if (!mbar_wait(k_empty + 8 * ks, kph ^ 1u, abort_flag)) break;
                mbar_expect_tx(k_full + 8 * ks, bytes);
                load_tile<DH, W::kInSub>(sK + ks * T, part ? &map_ke : gap ? &map_kg : &map_k, k_full + 8 * ks, g, row);
                if (++ks == KS) { ks = 0; kph ^= 1u; }
                const uint32_t vs = j & 1, vph = (j >> 1) & 1;
                if (!mbar_wait(v_empty + 8 * vs, vph ^ 1u, abort_flag)) break;
                mbar_expect_tx(v_full + 8 * vs, bytes);
                load_tile<DH, W::kInSub>(sV + vs * T, part ? &map_ve : gap ? &map_vg : &map_v, v_full + 8 * vs, g, row);
            }
        }
    } else if (warp == 1) {
        // the whole warp runs the issue loop; each MMA / commit executes in one elected lane
        constexpr uint32_t idesc_acc = make_idesc(TILE, DH, false, true);
        bool alive = nkv > 0 && mbar_wait_warp(q_full, 0, abort_flag);
        const uint32_t q_lo = klo(sQ), do_lo = klo(sdO);
        // K stage and phase of the tile whose S is issued next / whose dQ is issued next
        uint32_t ks_s = 0, kph_s = 0, ks_q = 0;
        auto issue_s = [&](int j) -> bool {        // S = Q K^T
            if (!mbar_wait_warp(k_full + 8 * ks_s, kph_s, abort_flag)) return false;
            if (CLEAR) clear_unseen<DH, IT, W::kInSub>(p.w, sK + ks_s * T, span.tile(j0 + j) * IT, lane);
            tc_fence_after();
            const uint32_t k_lo = klo(sK + ks_s * T);
#pragma unroll
            for (int kk = 0; kk < DH / 16; kk++) umma_ss_w(tS, q_lo + kstep(kk), k_lo + W::step(kk), make_idesc(TILE, keys_of(j), false, false), kk != 0);
            umma_commit_w(s_full);
            if (++ks_s == KS) { ks_s = 0; kph_s ^= 1u; }
            return true;
        };
        auto issue_dp = [&](int j) -> bool {       // dP = dO V^T
            const uint32_t vs = j & 1;
            if (!mbar_wait_warp(v_full + 8 * vs, (j >> 1) & 1, abort_flag)) return false;
            if (CLEAR) clear_unseen<DH, IT, W::kInSub>(p.w, sV + vs * T, span.tile(j0 + j) * IT, lane);
            tc_fence_after();
            const uint32_t v_lo = klo(sV + vs * T);
#pragma unroll
            for (int kk = 0; kk < DH / 16; kk++) umma_ss_w(tDP, do_lo + kstep(kk), v_lo + W::step(kk), make_idesc(TILE, keys_of(j), false, false), kk != 0);
            umma_commit_w(v_empty + 8 * vs);             // V of this stage is consumed
            umma_commit_w(dp_full);
            return true;
        };
        if (alive) alive = issue_s(0) && issue_dp(0);
        for (int j = 0; j < nkv && alive; j++) {
            if (j + 1 < nkv) {
                // next tile's S as soon as the softmax warps have read this tile's S into registers
                if (!mbar_wait_warp(s_free, j & 1, abort_flag)) { alive = false; break; }
                tc_fence_after();
                if (!issue_s(j + 1)) { alive = false; break; }
            }
            if (!mbar_wait_warp(p2_full, j & 1, abort_flag)) { alive = false; break; }
            tc_fence_after();
            const uint32_t k_mn = desc_lo(sK + ks_q * T, W::kInSub);
            const int slices = keys_of(j) / 16;
#pragma unroll
            for (int kk = 0; kk < IT / 16; kk++)
                if (kk < slices) umma_ts_w(tDQ, tDP + (kk >> 1) * 32 + (kk & 1) * 8, k_mn + mnstep(kk), idesc_acc, (j | kk) != 0);
            umma_commit_w(k_empty + 8 * ks_q);           // K of this stage is consumed
            if (++ks_q == KS) ks_q = 0;
            // the dP columns are free once dQ has read dS (in order)
            if (j + 1 < nkv && !issue_dp(j + 1)) { alive = false; break; }
        }
        if (alive) umma_commit_w(acc_full);
    } else {
        const int quarter = warp & 3;
        const int wg = (warp - 2) >> 2;                           // 32-key group of the tile
        const int key_base = wg * 32;
        const int row = quarter * 32 + lane;
        const int token = row / p.template heads<PACKED>(), h = h0 + row % p.template heads<PACKED>();
        const int qr = qt0 + token;
        const int q_abs = q_abs0 + (token < p.template tokens<PACKED>() ? token : p.template tokens<PACKED>() - 1);    // rows that are none of the tile's see as its last
        const bool used = token < p.template tokens<PACKED>() && qr < p.w.n;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tS_g = tS + key_base + lane_base, tP_g = tDP + key_base + lane_base;
        const float neg_lse2 = used ? -p.lse[(long long)h * p.w.n + qr] * kLog2e : 0.f;
        const float neg_delta_s = used ? -p.delta[(long long)h * p.w.n + qr] * p.scale : 0.f;
        bool alive = true;
        for (int j = 0; j < nkv && alive; j++) {
            const int k_abs0 = span.tile(j0 + j) * IT;
            if (!mbar_wait(s_full, j & 1, abort_flag)) { alive = false; break; }
            tc_fence_after();
            const uint32_t see = mixed(p.w, q_abs0, p.template tokens<PACKED>(), k_abs0, IT) ? visible_keys(p.w, q_abs, k_abs0, key_base) : 0xffffffffu;
            if (!__any_sync(0xffffffffu, see != 0u)) {     // dS of all of the warp's pairs is zero
                __syncwarp();
                if (lane == 0) mbar_arrive(s_free);
                if (!mbar_wait(dp_full, j & 1, abort_flag)) { alive = false; break; }
                tc_fence_after();
                uint32_t zero[16];
#pragma unroll
                for (int e = 0; e < 16; e++) zero[e] = 0u;
                tmem_st16(tP_g, zero);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p2_full);
                continue;
            }
            // phase 1: P from S; the S columns are handed back to the tensor pipe right after the load
            f32x2 pv[16];
            {
                uint32_t rs[32];
                tmem_ld32(tS_g, rs);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(s_free);
                auto shift = [&](int) { return pair(neg_lse2, neg_lse2); };
                if (see == 0xffffffffu) exponentials<false>(rs, p.scale_log2, see, shift, pv);
                else exponentials<true>(rs, p.scale_log2, see, shift, pv);
            }
            // phase 2: dS = P * (dP * scale - delta * scale), packed in place
            if (!mbar_wait(dp_full, j & 1, abort_flag)) { alive = false; break; }
            tc_fence_after();
            {
                uint32_t rp[32], ds[16];
                tmem_ld32(tP_g, rp);
                const f32x2 sc = pair(p.scale, p.scale), dl = pair(neg_delta_s, neg_delta_s);
#pragma unroll
                for (int e = 0; e < 16; e++)
                    ds[e] = pack_pair(mul2(pv[e], fma2(pair(__uint_as_float(rp[2 * e]), __uint_as_float(rp[2 * e + 1])), sc, dl)));
                tmem_st16(tP_g, ds);       // front of the group's own fp32 columns
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p2_full);
            }
        }
        if (alive && nkv > 0 && mbar_wait(acc_full, 0, abort_flag) && wg < DH / 32) {
            tc_fence_after();
            uint32_t r[32];
            tmem_ld32(tDQ + lane_base + key_base, r);
            const int mode = p.mode == GRAD_BF16_SET ? GRAD_BF16_SET : GRAD_F32_SET;
            if (PACKED && p.split > 1) {                      // this CTA's sum, 16-byte groups of eight rows on different banks
#pragma unroll
                for (int e = 0; e < 8; e++)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                                 ::"r"(sK + (uint32_t)(row * DH * 4 + (((wg * 8 + e) ^ (row & 7)) << 4))), "r"(r[4 * e]), "r"(r[4 * e + 1]),
                                 "r"(r[4 * e + 2]), "r"(r[4 * e + 3]) : "memory");
            } else if (32 % p.template heads<PACKED>() == 0) {                            // whole rows to a warp
                const int row0 = qt0 + quarter * (32 / p.template heads<PACKED>());
                if (row0 < p.w.n) {                           // the tiles are through with their products
                    const uint32_t at = base + (uint32_t)(warp - 2) * 4096u;
                    put_block(at, r, lane, mode, [&] { tma_store_3d(&map_dq, at, key_base, h0, row0); });
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
                }
            } else if (used) {                                // few rows
                put32(p.dq, ((long long)qr * p.w.Hq + h) * DH + key_base, r, mode);
            }
        }
    }

    if (PACKED && p.split > 1) {
        __syncwarp();
        cluster_sync_all();
        if (!*abort_flag) {                                   // the sums of the CTAs in order, rows dealt to the warps of all
            constexpr int NC = DH / 32, WARPS = W::kThreads / 32;
            const int rows = rows_here * p.work.heads;
            for (int r = rank * WARPS + warp; r < rows; r += p.split * WARPS) {
                float acc[NC];
#pragma unroll
                for (int e = 0; e < NC; e++) acc[e] = 0.f;
#pragma unroll
                for (int c = 0; c < 8; c++) {
                    if (c >= p.split || (long long)count * c / p.split == (long long)count * (c + 1) / p.split) continue;   // had none
                    float x[NC];
                    ld_cluster<NC>(map_to_cta(sK, (uint32_t)c) + (uint32_t)(r * DH * 4 + (((lane * NC >> 2) ^ (r & 7)) << 4) + (lane * NC & 3) * 4), x);
#pragma unroll
                    for (int e = 0; e < NC; e++) acc[e] += x[e];
                }
                const long long at = ((long long)(qt0 + r / p.work.heads) * p.w.Hq + h0 + r % p.work.heads) * DH + lane * NC;
#pragma unroll
                for (int e = 0; e < NC; e += 2) {
                    if (p.mode == GRAD_BF16_SET) *reinterpret_cast<uint32_t *>(static_cast<bf16 *>(p.dq) + at + e) = pack_bf16(acc[e], acc[e + 1]);
                    else *reinterpret_cast<float2 *>(static_cast<float *>(p.dq) + at + e) = make_float2(acc[e], acc[e + 1]);
                }
            }
        }
    }
    __syncwarp();
    leave(abort_flag);
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, W::kCols);
    }
    if (PACKED && p.split > 1) {
        __syncwarp();
        cluster_sync_all();                                   // no CTA leaves while another may read its sums
    }
}

template <int DH, bool PACKED, bool CLEAR>
__global__ void __launch_bounds__(Bwd<DH>::kThreads, Bwd<DH>::kBlocks)
    attn_window_bwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                           const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do,
                           const __grid_constant__ CUtensorMap map_qi, const __grid_constant__ CUtensorMap map_ki,
                           const __grid_constant__ CUtensorMap map_vi, const __grid_constant__ CUtensorMap map_doi,
                           const __grid_constant__ CUtensorMap map_ke, const __grid_constant__ CUtensorMap map_ve,
                           const __grid_constant__ CUtensorMap map_kg, const __grid_constant__ CUtensorMap map_vg,
                           const __grid_constant__ CUtensorMap map_dq, const __grid_constant__ CUtensorMap map_dk,
                           const __grid_constant__ CUtensorMap map_dv, const __grid_constant__ CUtensorMap map_part,
                           const __grid_constant__ BwdParams<DH> p) {
    pdl_enter();
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    // dispatch order: n_dq_first dQ CTAs (all of them or none), then the dK/dV CTAs, then the rest.  Where clusters share a dQ
    // item: the dQ CTAs, then the dK/dV CTAs, and as many more as fill the last cluster
    const int b = (int)blockIdx.x;
    const bool dq_role = b < p.n_dq_first || b >= p.n_dq_first + p.n_dkdv && !(PACKED && p.split > 1);
    if (!dq_role) {
        const int c = b - p.n_dq_first;                       // no cluster holds both roles: the dQ CTAs fill theirs
        if (!PACKED || c < p.n_dkdv)
            dkdv_body<DH, PACKED>(map_qi, map_k, map_v, map_doi, map_dk, map_dv, map_part, p, smem_raw, c / p.w.Hkv, c % p.w.Hkv);
    } else {
        const int i = b < p.n_dq_first ? b : b - p.n_dkdv, tiles = (p.w.n + p.template tokens<PACKED>() - 1) / p.template tokens<PACKED>();
        const int c = PACKED ? i / p.split : i;
        dq_body<DH, PACKED, CLEAR>(map_q, map_ki, map_vi, map_do, map_ke, map_ve, map_kg, map_vg, map_dq, p, smem_raw, tiles - 1 - c % tiles, c / tiles * p.template heads<PACKED>());
    }
}

// delta[h, i] = sum_j dO[i, h, j] O[i, h, j]: one 16-byte load of each per thread, DH / 8 threads to a row.  O is the stored one,
// so delta carries its rounding, which is what remains where a row sees few keys and dP - delta cancels; sum_j P dP in 32 bits
// would need the products of a pass of its own.
template <int DH>
__global__ void __launch_bounds__(256) window_delta_kernel(const bf16 *o, const bf16 *dout, int n, int Hq, float *delta, WsHeader *hdr,
                                                           void *dk, void *dv, long long unseen16) {
    pdl_enter();
    if (blockIdx.x == 0 && threadIdx.x == 0) clear_status(hdr);
    // rows of dk and dv that no query of the chunk sees have no owner among the key tiles: their gradients are zero (sink rows
    // among them are written later in the stream)
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < unseen16; i += (long long)gridDim.x * 256) {
        static_cast<uint4 *>(dk)[i] = make_uint4(0u, 0u, 0u, 0u);
        static_cast<uint4 *>(dv)[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    constexpr int kLanes = DH / 8;
    const long long rows = (long long)n * Hq, step = (long long)gridDim.x * (256 / kLanes);
    const int sub = threadIdx.x % kLanes;
    for (long long r = (long long)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes; r - threadIdx.x / kLanes < rows; r += step) {
        float s = 0.f;
        if (r < rows) {
            Vec<bf16> a, b;
            a.load(o + r * DH + sub * 8);
            b.load(dout + r * DH + sub * 8);
#pragma unroll
            for (int e = 0; e < 8; e++) s = fmaf(a.v[e], b.v[e], s);
        }
#pragma unroll
        for (int w = kLanes / 2; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
        if (sub == 0 && r < rows) delta[(r % Hq) * n + r / Hq] = s;
    }
}

template <typename K>
bool opt_in_smem(K kernel, int bytes) {
    return cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
}

// [rows, heads, DH] as tiles of `box` rows and 64 columns
template <int DH>
bool tile_map(CUtensorMap *m, const bf16 *p, int64_t rows, int heads, uint32_t box) {
    return make_tensor_map(m, p, rows, (int64_t)heads * DH, (int64_t)heads * DH, 64, box, false);
}
// The sink tile (of T keys) whose last rows are no sinks is read, multiplied and exponentiated only as far as its sinks go.
// `unit`: 16, or 32 where a warp reads all of the 32 columns that it sees some of.
template <int T>
void edge_of(const WindowShape &w, int unit, int &edge, int &keys) {
    edge = w.sinks % T ? w.sinks / T : -1;
    keys = edge < 0 ? unit : (w.sinks % T + unit - 1) / unit * unit;
}

// The two maps of k or v that end with the sinks and begin with the windows' first row; `all`, unused, where no tile needs them.
template <int DH>
bool key_maps(CUtensorMap *edge, CUtensorMap *gap, const CUtensorMap &all, const bf16 *x, const WindowShape &w, int edge_tile, uint32_t edge_keys,
              Gap g, uint32_t tile) {
    *edge = *gap = all;
    return (edge_tile < 0 || tile_map<DH>(edge, x, w.sinks, w.Hkv, edge_keys)) &&
           (g.tile < 0 || tile_map<DH>(gap, x + (int64_t)g.from * w.Hkv * DH, (int64_t)w.q0 + w.n - g.from, w.Hkv, tile));
}

template <int DH>
int fwd_any(const bf16 *q, const bf16 *k, const bf16 *v, const WindowShape &w, bf16 *o, float *lse, cudaStream_t st) {
    typedef Fwd<DH> F;
    FwdParams p;
    memset(&p, 0, sizeof(p));
    p.w = w;
    p.lse = lse;
    p.scale_log2 = kLog2e / sqrtf((float)DH);
    p.o = o;
    const int64_t kv = (int64_t)w.q0 + w.n;
    const int G = w.Hq / w.Hkv, slots = 2 * sm_count();
    // Rows of a tile come from all heads of a group, as far as that divides up: the fewer query rows in a tile, the fewer key
    // tiles it spans, and a handful of rows fills tiles that would be read for each head by itself.
    auto tile_of = [&](int heads) {
        p.heads = heads;
        p.tokens = TILE / heads;
        p.q_tiles = (w.n + p.tokens - 1) / p.tokens;
        return (int64_t)p.q_tiles * (w.Hq / heads);
    };
    int heads = 1;
    while (heads < 32 && G % (2 * heads) == 0) heads *= 2;          // whole rows to a warp, which stores its 32 by itself
    int64_t items = tile_of(heads);
    p.split = 1;
    bool clear;
    p.gap = gap_of<KT>(w, clear);
    if (2 * items <= slots && !clear) {
        // few rows: any divisor of the group, and clusters that share an item's key tiles
        int best = 1;
        for (int d = 2; d <= G && d <= TILE; d++)
            if (G % d == 0 && tile_of(d) <= tile_of(best)) best = d;
        const int64_t few = tile_of(best);
        const int count = key_span<KT>(w, w.q0 + (p.q_tiles - 1) * p.tokens, w.q0 + w.n - 1).count();
        int64_t split = slots / few < 8 ? slots / few : 8;
        if (split > count) split = count;
        // Joining costs as much as 2 steps of a CTA (128 x 64 scores, 0.76 us) and one more for each 16 rows.  At heads of 128,
        // split against one CTA an item: one row of 28:4 heads, window 1024: 8.9 us against 17.6, window 64: 6.2 and 6.1; 32
        // rows of 32:8 heads, window 1024: 13.1 and 17.2, window 512: 12.5 and 11.1.
        const int joined = (w.n < p.tokens ? w.n : p.tokens) * best;
        if (split > 1 && count - (count + split - 1) / split > 2 + joined / 16) {
            items = few;
            p.split = (int)split;
        } else {
            tile_of(heads);
        }
    }
    if (items > 0x7fffffff / 2) return STREAMBP_E_SHAPE;
    p.items = (int)items;
    edge_of<KT>(w, 16, p.edge, p.edge_keys);
    CUtensorMap mq, mk, mv, ke, ve, kg, vg, mo;
    if (!make_heads_map(&mq, q, w.n, w.Hq, DH, 64, (uint32_t)p.heads, (uint32_t)p.tokens, false) || !tile_map<DH>(&mk, k, kv, w.Hkv, KT) ||
        !tile_map<DH>(&mv, v, kv, w.Hkv, KT) || !key_maps<DH>(&ke, &kg, mk, k, w, p.edge, (uint32_t)p.edge_keys, p.gap, KT) ||
        !key_maps<DH>(&ve, &vg, mv, v, w, p.edge, (uint32_t)p.edge_keys, p.gap, KT))
        return STREAMBP_E_CUDA;
    if (p.split > 1) {
        static PerDevice configured;
        if (!configured.get([] { return opt_in_smem(attn_window_fwd_kernel<DH, true, false>, F::kSmem) ? 1 : 0; })) return STREAMBP_E_CUDA;
        return launch_clusters(attn_window_fwd_kernel<DH, true, false>, dim3((unsigned)(p.items * p.split)), F::kThreads, F::kSmem, p.split, 1, st, mq, mk, mv,
                               ke, ve, kg, vg, mk, p);
    }
    if (!make_heads_map(&mo, o, w.n, w.Hq, DH, 32, (uint32_t)p.heads, 32u / (uint32_t)p.heads, false, CU_TENSOR_MAP_SWIZZLE_64B)) return STREAMBP_E_CUDA;
    void (*kernel)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap,
                   const CUtensorMap, const CUtensorMap, const FwdParams) =
        clear ? attn_window_fwd_kernel<DH, false, true> : attn_window_fwd_kernel<DH, false, false>;
    static PerDevice configured[2];
    if (!configured[clear].get([&] { return opt_in_smem(kernel, F::kSmem) ? 1 : 0; })) return STREAMBP_E_CUDA;
    SBP_LAUNCH(kernel, p.items < slots ? p.items : slots, F::kThreads, F::kSmem, st, mq, mk, mv, ke, ve, kg, vg, mo, p);
    return STREAMBP_OK;
}

template <int DH>
int bwd_any(const bf16 *q, const bf16 *k, const bf16 *v, const bf16 *o, const bf16 *dout, const float *lse, const WindowShape &w,
            int mode, void *dq, void *dk, void *dv, float *delta, float *part, WsHeader *hdr, cudaStream_t st) {
    typedef Bwd<DH> W;
    constexpr int IT = W::IT;
    BwdParams<DH> p;
    memset(&p, 0, sizeof(p));
    p.w = w;
    p.work = key_work<TILE>(w, IT, bwd_heads(w, IT), DH == 64 ? kBwdSlots64 : kBwdSlots128);
    const uint32_t heads = (uint32_t)p.work.heads, tokens = TILE / heads;
    edge_of<IT>(w, 32, p.edge, p.edge_keys);
    bool clear;
    p.gap = gap_of<IT>(w, clear);
    const int64_t kv = (int64_t)w.q0 + w.n;
    const uint32_t edge = (uint32_t)p.edge_keys;
    // resident tiles of q, k, v, dO; inner tiles of the same; edge and gap tiles of k, v; blocks of dq, dk, dv, part
    CUtensorMap m[16];
    auto rows_map = [&](CUtensorMap *x, const bf16 *a, uint32_t rows) { return make_heads_map(x, a, w.n, w.Hq, DH, 64, heads, rows, false); };
    if (!rows_map(&m[0], q, tokens) || !tile_map<DH>(&m[1], k, kv, w.Hkv, TILE) || !tile_map<DH>(&m[2], v, kv, w.Hkv, TILE) ||
        !rows_map(&m[3], dout, tokens) || !rows_map(&m[4], q, (uint32_t)p.work.tq) || !tile_map<DH>(&m[5], k, kv, w.Hkv, IT) ||
        !tile_map<DH>(&m[6], v, kv, w.Hkv, IT) || !rows_map(&m[7], dout, (uint32_t)p.work.tq) || !key_maps<DH>(&m[8], &m[14], m[5], k, w, p.edge, edge, p.gap, IT) ||
        !key_maps<DH>(&m[9], &m[15], m[6], v, w, p.edge, edge, p.gap, IT))
        return STREAMBP_E_CUDA;
    const bool f32 = mode != GRAD_BF16_SET;
    const CUtensorMapSwizzle swizzle = f32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
    auto block_map = [&](CUtensorMap *x, void *g, int64_t rows, int heads) {
        return make_tensor_map(x, g, rows, (int64_t)heads * DH, (int64_t)heads * DH, 32, 32, f32, swizzle);
    };
    if (!block_map(&m[11], dk, kv, w.Hkv) || !block_map(&m[12], dv, kv, w.Hkv)) return STREAMBP_E_CUDA;
    m[10] = m[11];           // unused where a row's heads straddle warps
    if (32 % heads == 0 && !make_heads_map(&m[10], dq, w.n, w.Hq, DH, 32, heads, 32 / heads, f32, swizzle)) return STREAMBP_E_CUDA;
    m[13] = m[12];
    if (p.work.full() && !make_tensor_map(&m[13], part, (int64_t)p.work.items() * w.Hkv * 2 * TILE, DH, DH, 32, 32, true)) return STREAMBP_E_CUDA;
    {
        const int64_t unseen16 = mode == GRAD_F32_ADD ? 0 : (int64_t)p.work.lo * TILE * w.Hkv * DH * (mode == GRAD_BF16_SET ? 2 : 4) / 16;
        const int64_t rows = (int64_t)w.n * w.Hq * (DH / 8), work = rows > unseen16 ? rows : unseen16;
        const int64_t blocks = (work + 255) / 256, most = (int64_t)sm_count() * 8;
        SBP_LAUNCH(window_delta_kernel<DH>, (unsigned)(blocks < most ? blocks : most), 256, 0, st, o, dout, w.n, w.Hq, delta, hdr, dk, dv,
                   (long long)unseen16);
    }
    const float scale = 1.f / sqrtf((float)DH);
    p.lse = lse; p.delta = delta;
    p.dq = dq; p.dk = dk; p.dv = dv;
    p.part = part;
    p.part_rows = p.work.slot_rows(w);
    p.mode = mode;
    p.scale = scale;
    p.scale_log2 = scale * kLog2e;
    // The role with the longer walks is dispatched first (a dK/dV tile takes ~1.25x a dQ tile: four products against three)
    const int q_tiles = (w.n + (int)tokens - 1) / (int)tokens;
    const int64_t span = ((w.window < kv ? w.window : kv) + IT - 1) / IT + 1 + (w.sinks + IT - 1) / IT;
    const int64_t walk = p.work.wlen < p.work.q_tiles ? p.work.wlen : p.work.q_tiles;
    const int64_t n_dkdv = (int64_t)p.work.items() * w.Hkv, n_dq = (int64_t)q_tiles * (w.Hq / p.work.heads);
    if (n_dkdv + n_dq > 0x7fffffff / 8) return STREAMBP_E_SHAPE;
    // Few dQ items: clusters that share their key tiles, on the SMs that the dK/dV CTAs leave free or on a quarter of them.  Joining
    // costs as much as two iterations, and one for each 16 rows; what is gained ends where the dK/dV walks do (28:4 heads of 128, window 1024, 5 rows: 20.1 us with one
    // CTA an item, 14.0; 20 rows of 16:1 heads of 64, window 4000: 62 and 22).
    const int64_t count = key_span<IT>(w, w.q0 + (q_tiles - 1) * (int)tokens, w.q0 + w.n - 1).count(), slots = W::kBlocks * sm_count();
    const int64_t joined = (w.n < (int)tokens ? w.n : (int)tokens) * p.work.heads;
    const int64_t room = slots - n_dkdv > slots / 4 ? slots - n_dkdv : slots / 4;
    int64_t split = room / n_dq < 8 ? room / n_dq : 8;
    if (split > count) split = count;
    const int64_t other = 5 * (w.Hq / w.Hkv / p.work.heads) * walk / 4;
    const int64_t left = split > 1 && (count + split - 1) / split > other ? (count + split - 1) / split : other;
    p.split = split > 1 && count - left > 2 + joined / 16 ? (int)split : 1;
    p.n_dkdv = (int)n_dkdv;
    p.n_dq_first = p.split > 1 ? (int)n_dq * p.split : 4 * span > 5 * (w.Hq / w.Hkv / p.work.heads) * walk ? (int)n_dq : 0;
    const int variant = clear ? 2 : heads > 1 || p.split > 1 ? 1 : 0;
    void (*kernel)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap,
                   const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap,
                   const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const BwdParams<DH>) =
        variant == 2 ? attn_window_bwd_kernel<DH, true, true> : variant == 1 ? attn_window_bwd_kernel<DH, true, false> : attn_window_bwd_kernel<DH, false, false>;
    static PerDevice configured[3];
    if (!configured[variant].get([&] { return opt_in_smem(kernel, W::kSmem) ? 1 : 0; })) return STREAMBP_E_CUDA;
    if (p.split > 1) {
        const int64_t ctas = (n_dkdv + n_dq * p.split + p.split - 1) / p.split * p.split;
        const int st_ = launch_clusters(kernel, dim3((unsigned)ctas), W::kThreads, W::kSmem, p.split, 1, st, m[0], m[1], m[2], m[3], m[4], m[5], m[6], m[7],
                                        m[8], m[9], m[14], m[15], m[10], m[11], m[12], m[13], p);
        if (st_ != STREAMBP_OK) return st_;
    } else {
        SBP_LAUNCH(kernel, (unsigned)(n_dkdv + n_dq), W::kThreads, W::kSmem, st, m[0], m[1], m[2], m[3], m[4], m[5], m[6], m[7], m[8], m[9],
                   m[14], m[15], m[10], m[11], m[12], m[13], p);
    }
    return attention_window_join(part, p.work, w, DH, mode, dk, dv, st);
}

}  // namespace

bool attention_window_tc_available() { return tensor_maps_available(); }

int attention_window_fwd_tc(const bf16 *q, const bf16 *k, const bf16 *v, const WindowShape &w, int dh, bf16 *o, float *lse,
                            cudaStream_t st) {
    return dh == 64 ? fwd_any<64>(q, k, v, w, o, lse, st) : fwd_any<128>(q, k, v, w, o, lse, st);
}
int attention_window_bwd_tc(const bf16 *q, const bf16 *k, const bf16 *v, const bf16 *o, const bf16 *dout, const float *lse,
                            const WindowShape &w, int dh, int mode, void *dq, void *dk, void *dv, float *delta, float *part,
                            WsHeader *hdr, cudaStream_t st) {
    return dh == 64 ? bwd_any<64>(q, k, v, o, dout, lse, w, mode, dq, dk, dv, delta, part, hdr, st)
                    : bwd_any<128>(q, k, v, o, dout, lse, w, mode, dq, dk, dv, delta, part, hdr, st);
}
int attention_window_take_fault() { return take_fault_local(); }

}  // namespace sbp
