// Geometry of attention with a sliding window and a few first keys that stay visible ("sinks"), shared by the kernels and
// the host code that sizes their grids.
//   visible(t, j) = j <= t and (t - j < window or j < sinks)        t, j: absolute rows, queries q0 .. q0 + n - 1
// All rows are below 2^31 (checked at the entry), so positions are ints; element offsets are 64-bit.
#pragma once

#include <cstdint>

namespace sbp {

struct WindowShape {
    int n, q0;            // query rows of the chunk and the absolute row of the first; keys are 0 .. q0 + n - 1
    int Hq, Hkv;
    int window;           // >= 1, at most q0 + n
    int sinks;            // >= 0, at most q0 + n
};

#ifdef __CUDACC__
#define SBP_HD __host__ __device__ __forceinline__
#else
#define SBP_HD inline
#endif

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
// Whether rows first .. last see anything of tile kt <= their own (the span of two row tiles may hold tiles only one sees).
template <int T>
SBP_HD bool sees(const WindowShape &w, int kt, int first, int last) {
    const int from = first - w.window + 1;
    return kt <= last / T && (kt >= (from > 0 ? from / T : 0) || kt * T < w.sinks);
}

// The work of the key-tile owners (dK, dV): key tiles of TK keys against query tiles of TQ rows.  Tiles below `lo` hold
// sinks only, or nothing that a query of the chunk sees.
//   sink tiles 0 .. st - 1 : every later query adds to them; their query tiles are cut into `segs` segments of `len`
//                            tiles, one owner each, whose sums are joined afterwards in the order of the segments
//   window tiles wt0 .. kv_tiles - 1 : one owner each, over the query tiles the window reaches
template <int TK, int TQ = TK> struct KeyWork {
    int kv_tiles, q_tiles, lo, st, segs, len, wt0;
    SBP_HD int items() const { return st * segs + (kv_tiles - wt0); }
    // item -> key tile, query tiles [begin, end), segment (-1: the item writes its result itself)
    SBP_HD void item(const WindowShape &w, int i, int &kt, int &begin, int &end, int &seg) const {
        if (i < st * segs) {
            kt = i / segs;
            seg = i - kt * segs;
            const int f = first(w, kt);
            begin = f + seg * len;
            end = begin + len < q_tiles ? begin + len : q_tiles;
            if (segs == 1) { seg = -1; end = q_tiles; }
        } else {
            kt = wt0 + i - st * segs;
            seg = -1;
            begin = first(w, kt);
            // the last query that sees the tile's last key through the window
            const long long last = (long long)kt * TK + TK - 1 + w.window - 1 - w.q0;
            end = last < 0 ? 0 : (last / TQ + 1 < q_tiles ? (int)(last / TQ) + 1 : q_tiles);
        }
        if (end < begin) end = begin;
    }
    // first query tile that holds a row at or behind the tile's first key
    SBP_HD static int first(const WindowShape &w, int kt) {
        const long long k0 = (long long)kt * TK;
        return k0 > w.q0 ? (int)((k0 - w.q0) / TQ) : 0;
    }
};
template <int TK, int TQ = TK>
inline KeyWork<TK, TQ> key_work(const WindowShape &w) {
    KeyWork<TK, TQ> k;
    const int kv = w.q0 + w.n;
    k.kv_tiles = (kv + TK - 1) / TK;
    k.q_tiles = (w.n + TQ - 1) / TQ;
    const int from = w.q0 - w.window + 1;
    k.lo = from > 0 ? from / TK : 0;
    const int sink_tiles = (w.sinks + TK - 1) / TK;
    k.st = sink_tiles < k.kv_tiles ? sink_tiles : k.kv_tiles;
    k.wt0 = k.st > k.lo ? k.st : k.lo;
    // a segment is as long as a window tile's walk, and the first one covers every query that sees a key of the tile
    // through the window: in the later ones only the sinks have anything to add
    k.len = (w.window + TK + 2 * TQ - 2) / TQ;
    if (k.len < 8) k.len = 8;
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
// query rows to a tile of the tensor-core backward's key-tile owners, by head_dim
constexpr int kBwdRows64 = 64, kBwdRows128 = 128;

// rows of a sink tile whose sums go through the workspace
template <int T>
SBP_HD int sink_rows(const WindowShape &w, int kt) {
    const int r = w.sinks - kt * T;
    return r < T ? (r > 0 ? r : 0) : T;
}

// Where gradients go: fp32 added to or overwritten, or bf16 overwritten.
enum GradMode { GRAD_F32_ADD = 0, GRAD_F32_SET = 1, GRAD_BF16_SET = 2 };

}  // namespace sbp
