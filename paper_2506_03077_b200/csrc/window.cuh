// Geometry of attention with a sliding window and a few first keys that stay visible ("sinks"), shared by the kernels and
// the host code that sizes their grids.
//   visible(t, j) = j <= t and (t - j < window or j < sinks)        t, j: absolute rows, queries q0 .. q0 + n - 1
// All rows are below 2^31 (checked at the entry), so positions are ints; element offsets are 64-bit.
#pragma once

#include <cstddef>
#include <cstdint>

namespace sbp {

#ifdef __CUDACC__
#define SBP_HD __host__ __device__ __forceinline__
#else
#define SBP_HD inline
#endif

struct WindowShape {
    int n, q0;            // query rows of the chunk and the absolute row of the first; keys are 0 .. q0 + n - 1
    int Hq, Hkv;
    int window;           // >= 1, at most q0 + n
    int sinks;            // >= 0, at most q0 + n
    // Rows of k and v that no query of the chunk sees may hold anything.  They are sinks .. seen_from() - 1, where there are any.
    SBP_HD int seen_from() const { return q0 - window + 1; }
    SBP_HD bool unseen(int j) const { return j >= sinks && j < seen_from(); }
};

// Key tiles of T keys that some query of rows first .. last (absolute) sees: the sink tiles 0 .. ns - 1, then lo .. hi.
struct KeySpan {
    int ns, lo, hi;
    SBP_HD int count() const { return ns + hi - lo + 1; }
    SBP_HD int tile(int j) const { return j < ns ? j : lo + j - ns; }
};
template <int T>
SBP_HD KeySpan key_span(const WindowShape &w, int first, int last) {
    KeySpan s;
    s.hi = last / T;
    const int from = first - w.window + 1;
    s.lo = from > 0 ? from / T : 0;
    const int st = (w.sinks + T - 1) / T;
    s.ns = st < s.lo ? st : s.lo;
    return s;
}

// The work of the key-tile owners (dK, dV): key tiles of TK keys against query tiles of `tq` rows (of `heads` heads each).  Tiles below `lo` hold
// sinks only, or nothing that a query of the chunk sees.
//   sink tiles 0 .. st - 1 : every later query adds to them; their query tiles are cut into `segs` segments of `len` tiles
//   window tiles wt0 .. kv_tiles - 1 : over the query tiles the window reaches, cut into `wsegs` segments of `wlen`
// One owner per segment; where there are several, fp32 sums meet in a workspace and are joined in the order of the
// segments.  wsegs > 1 (a short chunk: few owners, each with a long walk over its group's heads): all rows of every tile go
// through the workspace (`full`).  Else a sink tile's first segment covers every query that sees a key of the tile
// through the window, and only the sinks' rows do.
template <int TK> struct KeyWork {
    int tq, heads, kv_tiles, q_tiles, lo, st, segs, len, wt0, wsegs, wlen;
    SBP_HD int items() const { return st * segs + (kv_tiles - wt0) * wsegs; }
    SBP_HD bool full() const { return wsegs > 1; }
    // item -> key tile, query tiles [begin, end), segment (-1: the item writes its result itself)
    SBP_HD void item(const WindowShape &w, int i, int &kt, int &begin, int &end, int &seg) const {
        const bool sink = i < st * segs;
        const int n = sink ? segs : wsegs, j = sink ? i : i - st * segs, step = sink ? len : wlen;
        kt = (sink ? 0 : wt0) + j / n;
        const int s = j % n;
        // the last query that sees the tile's last key: any for a sink, else through the window
        const long long last = (long long)kt * TK + TK - 1 + w.window - 1 - w.q0;
        const int all = sink ? q_tiles : (last < 0 ? 0 : (last / tq + 1 < q_tiles ? (int)(last / tq) + 1 : q_tiles));
        begin = first(w, kt) + s * step;
        end = n == 1 || begin + step > all ? all : begin + step;
        if (end < begin) end = begin;
        seg = n > 1 ? s : -1;
    }
    // first query tile that holds a row at or behind the tile's first key
    SBP_HD int first(const WindowShape &w, int kt) const {
        const long long k0 = (long long)kt * TK;
        return k0 > w.q0 ? (int)((k0 - w.q0) / tq) : 0;
    }
    // rows of tile kt whose sums go through the workspace where its work is cut, and the rows of a workspace slot
    SBP_HD int joined_rows(const WindowShape &w, int kt) const {
        const int r = full() ? TK : w.sinks - kt * TK;
        return r < TK ? (r > 0 ? r : 0) : TK;
    }
    // Keys whose sums are joined: the first join_lead, of the sink tiles (all of their rows, or the sinks), and the join_behind
    // from tile wt0 on
    SBP_HD long long join_lead(const WindowShape &w) const {
        const long long kv = (long long)w.q0 + w.n, whole = (long long)st * TK < kv ? (long long)st * TK : kv;
        return segs > 1 ? (full() ? whole : w.sinks) : 0;
    }
    SBP_HD long long join_behind(const WindowShape &w) const {
        const long long behind = (long long)w.q0 + w.n - (long long)wt0 * TK;
        return full() && behind > 0 ? behind : 0;          // none where the sink tiles are all the tiles, the last of them a short one
    }
    SBP_HD int slot_rows(const WindowShape &w) const { return full() || w.sinks > TK ? TK : w.sinks; }
    // floats of the workspace: [item][Hkv][dK, dV][slot_rows][dh]
    size_t part_floats(const WindowShape &w, int dh) const {
        if (segs == 1 && wsegs == 1) return 0;
        return (size_t)(full() ? items() : st * segs) * w.Hkv * 2 * slot_rows(w) * dh;
    }
};
// Inner tiles hold `it` rows: it / heads query rows of `heads` heads of a group, or `it` keys of the dQ role's walk.
// `slots`: CTAs of the kernel that the 148 SMs hold at a time (0: windows are not cut).  A function of the sizes alone, so
// that workspace queries need no GPU and the order of the sums is the same everywhere.
template <int TK>
inline KeyWork<TK> key_work(const WindowShape &w, int it, int heads, int slots) {
    KeyWork<TK> k;
    const int kv = w.q0 + w.n, turns = w.Hq / w.Hkv / heads, TQ = it / heads;
    k.tq = TQ;
    k.heads = heads;
    k.kv_tiles = (kv + TK - 1) / TK;
    k.q_tiles = (w.n + TQ - 1) / TQ;
    const int from = w.q0 - w.window + 1;
    k.lo = from > 0 ? from / TK : 0;
    const int sink_tiles = (w.sinks + TK - 1) / TK;
    k.st = sink_tiles < k.kv_tiles ? sink_tiles : k.kv_tiles;
    k.wt0 = k.st > k.lo ? k.st : k.lo;
    // walk of a window tile; as a sink segment's length it covers the window's part of a sink tile
    k.len = (w.window + TK + 2 * TQ - 2) / TQ;
    const int walk = k.len < k.q_tiles ? k.len : k.q_tiles;
    k.wsegs = 1;
    k.wlen = k.len;
    if (slots > 0) {
        // costs in units of a quarter of a dQ tile of the same launch (`it` keys; a dK/dV one takes ~1.25x: four products
        // against three): what a slot has to do on average, and the longest owner's walk
        const long long span = ((w.window < kv ? w.window : kv) + it - 1) / it + 1 + (w.sinks + it - 1) / it;
        const long long owners = (long long)(k.kv_tiles - k.wt0 + k.st) * w.Hkv, longest = 5ll * turns * walk;
        const long long each = (owners * longest + 4 * span * ((w.n + 128 / heads - 1) / (128 / heads)) * (w.Hq / heads)) / slots;
        // cut while the longest owner has more to do than a slot has on average (2000 rows, 16 heads to one key head, 128:
        // 381 us uncut, 82 us; 4000 rows at heads of 64, window 300: 176 and 74), unless the owners are many already or the
        // walk is too short to pay for the join (3 us, or two to three iterations)
        while (k.wsegs < 16 && 2 * k.wsegs <= walk && (k.wsegs > 1 || turns * walk > 4) && longest > each * k.wsegs && owners * k.wsegs <= 2 * slots) k.wsegs *= 2;
        k.wlen = (walk + k.wsegs - 1) / k.wsegs;
    }
    if (k.full()) k.len = k.wlen;
    else if (k.len < 8 * heads) k.len = 8 * heads;
    k.segs = k.st > 0 ? (k.q_tiles + k.len - 1) / k.len : 1;
    // no more owners of sink tiles than four for each of 148 SMs: that many keep the GPU busy, and they bound the workspace
    // (many sinks need no segments at all)
    const int most = k.st > 0 ? 592 / (k.st * w.Hkv < 592 ? k.st * w.Hkv : 592) : 1;
    if (k.segs > most) {
        k.len = (k.q_tiles + most - 1) / most;
        k.segs = (k.q_tiles + k.len - 1) / k.len;
    }
    if (k.segs < 1) k.segs = 1;
    return k;
}
// rows of an inner tile of the tensor-core backward, by head_dim
constexpr int kBwdRows64 = 64, kBwdRows128 = 128;
// its CTAs on 148 SMs
constexpr int kBwdSlots64 = 296, kBwdSlots128 = 148;

// Heads of a group that share the rows of a tile: the fewer query rows a tile has, the fewer key tiles it spans.  As many as
// divide up into whole rows of 32, or for few rows, that one tile holds, all that it holds; but one where that saves less
// than a fifth of the (query tile, key tile) pairs: the rows' bookkeeping costs more then (8191 rows, window 512, heads of
// 64, 4 to a group: 223 us with one, 226 with 4; 180 rows behind 900, window 300, heads of 128: 28.3 and 21.8; 30 rows, 16
// heads to a group: 19 and 9.4).
inline int bwd_heads(const WindowShape &w, int it) {
    const int G = w.Hq / w.Hkv, kv = w.q0 + w.n;
    int p = 1;
    while (p < 32 && G % (2 * p) == 0) p *= 2;
    for (int d = p + 1; d <= G && d <= it; d++)
        if (G % d == 0 && w.n <= it / d) p = d;
    auto pairs = [&](int heads) {            // in keys, the partly used tiles at the ends of a span counted half
        const long long rows = 128 / heads;
        return ((w.n + rows - 1) / rows) * (G / heads) * ((w.window < kv ? w.window : kv) + rows + it / 2);
    };
    return 5 * pairs(p) <= 4 * pairs(1) ? p : 1;
}

// Where gradients go: fp32 added to or overwritten, or bf16 overwritten.
enum GradMode { GRAD_F32_ADD = 0, GRAD_F32_SET = 1, GRAD_BF16_SET = 2 };

}  // namespace sbp
