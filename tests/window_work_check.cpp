// Host check of the geometry of the windowed backward (window.cuh): which keys and which (query, key) pairs the owners of key
// tiles take, and what the joining kernel adds up.
//   window_work_check sweep                                             every shape of a grid of short calls, and a few long ones
//   window_work_check shape n q0 Hq Hkv head_dim window sinks           one shape
// Prints the first fault of a shape and exits with 1.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "window.cuh"

using namespace sbp;

static const char *g_fault = nullptr;
static long long g_at = 0;
static bool fault(const char *what, long long at) {
    g_fault = what;
    g_at = at;
    return false;
}
static bool visible(const WindowShape &w, int t, int j) { return j <= t && (t - j < w.window || j < w.sinks); }

template <int TK>
static bool check(const WindowShape &w, int dh, const KeyWork<TK> &k) {
    const int kv = w.q0 + w.n;
    // how often a key's gradients are written by an owner, and by the joining kernel
    std::vector<int> direct(kv, 0), joined(kv, 0);
    const long long lead = k.join_lead(w), behind = k.join_behind(w);
    if (lead < 0 || behind < 0 || lead + behind > kv) return fault("keys of the joining kernel", lead + behind);
    for (long long i = 0; i < lead + behind; i++) {
        const long long key = i < lead ? i : (long long)k.wt0 * TK + i - lead;
        if (key >= kv) return fault("the joining kernel is past the last key", key);
        joined[key]++;
        const int kt = (int)(key / TK), row = (int)(key % TK), n = i < lead ? k.segs : k.wsegs;
        const int item0 = i < lead ? kt * k.segs : k.st * k.segs + (kt - k.wt0) * k.wsegs;
        if (row >= k.joined_rows(w, kt) || row >= k.slot_rows(w)) return fault("a joined row that no owner leaves", key);
        if (n < 2 || item0 + n > k.items()) return fault("segments of a joined key", key);
        // the last float of its last slot
        const size_t last = ((((size_t)(item0 + n - 1) * w.Hkv + w.Hkv - 1) * 2 + 1) * k.slot_rows(w) + row) * dh + dh - 1;
        if (last >= k.part_floats(w, dh)) return fault("a slot behind the workspace", key);
    }
    std::vector<int> begin(k.items()), end(k.items()), tile(k.items()), seg(k.items());
    for (int i = 0; i < k.items(); i++) {
        k.item(w, i, tile[i], begin[i], end[i], seg[i]);
        if (tile[i] < 0 || tile[i] >= k.kv_tiles || begin[i] > end[i] || (end[i] > begin[i] && end[i] > k.q_tiles)) return fault("item", i);
        for (int r = 0; r < TK && tile[i] * TK + r < kv; r++) {
            if (seg[i] < 0 || (!k.full() && r >= k.joined_rows(w, tile[i]) && seg[i] == 0)) direct[tile[i] * TK + r]++;
            else if ((k.full() || r < k.joined_rows(w, tile[i])) && joined[tile[i] * TK + r] != 1)
                return fault("an owner's sum that is not joined", tile[i] * TK + r);
        }
    }
    for (int j = 0; j < kv; j++) {
        if (direct[j] + joined[j] > 1) return fault("key written twice", j);
        if (direct[j] + joined[j] == 0 && (j >= (long long)k.lo * TK || j < w.sinks)) return fault("key never written", j);
        if (direct[j] + joined[j] == 0 && !w.unseen(j)) return fault("key that is seen, never written", j);
    }
    // every visible pair by one owner that counts for the key
    std::vector<std::vector<int>> owners_of(k.kv_tiles);
    for (int i = 0; i < k.items(); i++) owners_of[tile[i]].push_back(i);
    for (int j = 0; j < kv; j += j + 40 < kv && kv > 300 ? 37 : 1)
        for (int t = j > w.q0 ? j : w.q0; t < kv; t++) {
            if (!visible(w, t, j)) continue;
            int owners = 0;
            const int qt = (t - w.q0) / k.tq;
            for (int i : owners_of[j / TK])
                if (begin[i] <= qt && qt < end[i]) owners += joined[j] || seg[i] <= 0;
            if (owners != 1) return fault("owners of a pair", j);
        }
    return true;
}

// the entry's reading of its arguments
static WindowShape shape(int n, int q0, int Hq, int Hkv, int window, int sinks) {
    const int kv = q0 + n;
    WindowShape w = {n, q0, Hq, Hkv, window < kv ? window : kv, sinks < kv ? sinks : kv};
    if (w.window == kv || w.sinks == kv) {
        w.window = kv;
        w.sinks = 0;
    }
    return w;
}
static bool check_all(int n, int q0, int Hq, int Hkv, int dh, int window, int sinks) {
    const WindowShape w = shape(n, q0, Hq, Hkv, window, sinks);
    const int it = dh == 64 ? kBwdRows64 : kBwdRows128;
    if (check<128>(w, dh, key_work<128>(w, it, bwd_heads(w, it), dh == 64 ? kBwdSlots64 : kBwdSlots128)) &&
        check<32>(w, dh, key_work<32>(w, 32, 1, 0)))
        return true;
    printf("n %d q0 %d heads %d:%d of %d window %d sinks %d: %s (%lld)\n", n, q0, Hq, Hkv, dh, window, sinks, g_fault, g_at);
    return false;
}

int main(int argc, char **argv) {
    if (argc == 9 && !strcmp(argv[1], "shape")) {
        int a[7];
        for (int i = 0; i < 7; i++) a[i] = atoi(argv[2 + i]);
        return check_all(a[0], a[1], a[2], a[3], a[4], a[5], a[6]) ? 0 : 1;
    }
    if (argc != 2 || strcmp(argv[1], "sweep")) return 2;
    const int heads[][2] = {{16, 1}, {32, 8}, {28, 4}, {12, 4}, {4, 2}, {1, 1}, {47, 1}};
    bool good = true;
    long long shapes = 0;
    for (auto &h : heads)
        for (int dh = 64; dh <= 128; dh += 64) {
            for (int n : {1, 2, 7, 17, 20, 49, 64, 71, 100, 127, 128, 129, 151, 200, 255, 333, 520})
                for (int q0 : {0, 1, 50, 127, 128, 129, 300})
                    for (int window : {1, 8, 64, 100, 129, 1000})
                        for (int sinks : {0, 1, 4, 33, 100, 127, 128, 129, 200, 300}) {
                            good = check_all(n, q0, h[0], h[1], dh, window, sinks) && good;
                            shapes++;
                        }
            for (int n : {1500, 2048, 4097})
                for (int sinks : {0, 3, 140, 2100}) {
                    good = check_all(n, 5, h[0], h[1], dh, 100, sinks) && good;
                    shapes++;
                }
        }
    printf("%lld shapes\n", shapes);
    return good ? 0 : 1;
}
