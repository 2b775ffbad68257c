// Rows of logits that start anywhere: a row as 16-byte groups of memory, and the values' order.
#pragma once

#include "sm100.cuh"

namespace sbp {

// Up to kScanMost ids one block of a call looks through, which saves a launch that clears the status; more are looked at by the
// blocks that use them, behind such a launch (clear_status_launch).
constexpr int64_t kScanMost = 1 << 14, kScanRow = 4096;     // (however many, where each stands for so many bytes of a row: then the rest of the call takes longer)
// That block's look through `count` ids, several loads in flight: the first i for which bad(ids[i], i) goes into the header as
// E_BAD_LABEL with detail i / per, or OK.
template <typename F>
__device__ __forceinline__ void report_first(const int64_t *__restrict__ ids, int64_t count, int64_t per, WsHeader *hdr, F bad) {
    __shared__ unsigned long long s_first;
    constexpr unsigned long long kNone = ~0ull;
    if (threadIdx.x == 0) s_first = kNone;
    __syncthreads();
    unsigned long long first = kNone;
    for (int64_t i0 = threadIdx.x; i0 < count; i0 += 8 * (int64_t)blockDim.x) {
        int64_t id[8];
#pragma unroll
        for (int u = 0; u < 8; u++) {
            const int64_t i = i0 + u * (int64_t)blockDim.x;
            id[u] = ids[i < count ? i : i0];
        }
#pragma unroll
        for (int u = 0; u < 8; u++) {
            const int64_t i = i0 + u * (int64_t)blockDim.x;
            if (i < count && bad(id[u], i) && (unsigned long long)i < first) first = (unsigned long long)i;
        }
    }
    if (first != kNone) atomicMin(&s_first, first);
    __syncthreads();
    if (threadIdx.x == 0) {
        hdr->status = s_first == kNone ? STREAMBP_OK : STREAMBP_E_BAD_LABEL;
        hdr->detail = s_first == kNone ? 0 : (int)(s_first / (unsigned long long)per);
    }
    __syncthreads();
}

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// the larger of two; NaN where one is
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Two fp32 operations in one instruction.
struct Pair {
    unsigned long long v;
    __device__ __forceinline__ Pair() {}
    __device__ __forceinline__ Pair(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ void get(float &a, float &b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// 16 bytes of a row as they came, their largest and smallest value (NaN left out), and their values as pairs.
template <typename T> struct Raw;
template <> struct Raw<float> {
    uint4 w;
    __device__ __forceinline__ float largest() const {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
    __device__ __forceinline__ float smallest() const {
        return fminf(fminf(__uint_as_float(w.x), __uint_as_float(w.y)), fminf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
    __device__ __forceinline__ void fill(float v) { w = make_uint4(__float_as_uint(v), __float_as_uint(v), __float_as_uint(v), __float_as_uint(v)); }
    __device__ __forceinline__ void pairs(Pair (&p)[2]) const {
        p[0] = Pair(__uint_as_float(w.x), __uint_as_float(w.y));
        p[1] = Pair(__uint_as_float(w.z), __uint_as_float(w.w));
    }
};
template <> struct Raw<bf16> {
    uint4 w;
    static __device__ __forceinline__ __nv_bfloat162 two(uint32_t u) { return *reinterpret_cast<__nv_bfloat162 *>(&u); }
    __device__ __forceinline__ float largest() const {
        const __nv_bfloat162 a = __hmax2(__hmax2(two(w.x), two(w.y)), __hmax2(two(w.z), two(w.w)));
        return fmaxf(__low2float(a), __high2float(a));
    }
    __device__ __forceinline__ float smallest() const {
        const __nv_bfloat162 a = __hmin2(__hmin2(two(w.x), two(w.y)), __hmin2(two(w.z), two(w.w)));
        return fminf(__low2float(a), __high2float(a));
    }
    __device__ __forceinline__ void fill(float v) {
        const uint32_t h = __float_as_uint(v) >> 16, u = h << 16 | h;        // (v is a bf16 value)
        w = make_uint4(u, u, u, u);
    }
    __device__ __forceinline__ void pairs(Pair (&p)[4]) const {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; i++) p[i] = Pair(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xFFFF0000u));
    }
};

// Row of n elements at p, seen as aligned 16-byte groups: group v holds the elements v N - off .. v N - off + N - 1, of
// which the first and the last group may hold some only.  Those are read element by element: nothing outside the row is read.
template <typename T>
struct RowGroups {
    static constexpr int N = Vec<T>::N;
    const T *base;       // p, aligned down (never read in front of p)
    int off, n, groups;
    __device__ __forceinline__ RowGroups(const T *p, int n_) {
        off = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
        base = p - off;
        n = n_;
        groups = (int)(((int64_t)off + n + N - 1) / N);
    }
    __device__ __forceinline__ int first(int v) const { return v * N - off; }                      // element index of the group
    __device__ __forceinline__ bool whole(int v) const { return first(v) >= 0 && first(v) <= n - N; }
    // the groups that the row fills: whole_begin .. whole_end - 1 (none where the second is not larger)
    __device__ __forceinline__ int whole_begin() const { return off ? 1 : 0; }
    __device__ __forceinline__ int whole_end() const { return (int)(((int64_t)off + n) / N); }
    __device__ __forceinline__ void load_whole(int v, Raw<T> &x) const { x.w = *reinterpret_cast<const uint4 *>(base + (int64_t)v * N); }
    // group v as it is, -inf where the row has no element
    __device__ __forceinline__ void load(int v, Raw<T> &x) const {
        if (whole(v)) {
            x.w = *reinterpret_cast<const uint4 *>(base + (int64_t)v * N);
        } else {
            T t[N];
#pragma unroll
            for (int i = 0; i < N; i++) {
                const int e = first(v) + i;
                t[i] = e >= 0 && e < n ? base[(int64_t)v * N + i] : from_f32<T>(-INFINITY);
            }
            memcpy(&x.w, t, 16);
        }
    }
    // values of group v, `fill` where the row has none
    __device__ __forceinline__ void load(int v, float (&x)[N], float fill) const {
        if (whole(v)) {
            Vec<T> a;
            a.load(base + (int64_t)v * N);
#pragma unroll
            for (int i = 0; i < N; i++) x[i] = a.v[i];
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) {
                const int e = first(v) + i;
                x[i] = e >= 0 && e < n ? to_f32(base[(int64_t)v * N + i]) : fill;
            }
        }
    }
};

// A temperature's reciprocal in two floats: x / tau as x hi + x lo loses no more than the rounding of the result.
struct Heat {
    float hi, lo;
};
inline Heat make_heat(float temperature) {
    const double r = 1.0 / (double)temperature;
    Heat h;
    h.hi = (float)r;
    h.lo = (float)(r - (double)h.hi);
    return h;
}

// The order of a list of alternatives as one number: larger values first, of equal ones (the two zeros are equal) the lower
// index first.  No two elements of a row share a number; 0 stands for none.  The value must not be NaN.
__device__ __forceinline__ unsigned long long order_of(float value, int index) {
    const uint32_t u = __float_as_uint(value + 0.f);
    const uint32_t key = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return (unsigned long long)key << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float value_of(unsigned long long o) {
    const uint32_t key = (uint32_t)(o >> 32);
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ int index_of(unsigned long long o) { return (int)~(uint32_t)o; }

// Softmax statistics of a set of logits: their maximum m, S = sum of exp((z - m) / tau), and W = sum of the same times
// (z - m).  All terms of S are positive and all of W negative, so neither loses digits; an empty set has m = -inf, S = W = 0.
// A NaN or +inf among the logits makes S NaN.
struct RowStats {
    float m, S, W;
};
// Distances below a maximum count as at most this far (their exponential is 0 at every temperature that is allowed), so that
// logits of -inf or of the type's lowest value add 0 to W and not 0 times an infinity.
constexpr float kDeep = -1e30f;
__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ RowStats join(const RowStats &a, const RowStats &b, float c) {
    RowStats r;
    r.m = fmaxf(a.m, b.m);
    const float m = finite_or_zero(r.m), da = a.m - m, db = b.m - m;
    const float fa = exp2_approx(da * c), fb = exp2_approx(db * c);
    r.S = a.S * fa + b.S * fb;
    r.W = fa * fmaf(fmaxf(da, kDeep), a.S, a.W) + fb * fmaf(fmaxf(db, kDeep), b.S, b.W);
    return r;
}

// Adds the values of x (all at or below m) to the sums of a thread.
template <typename T, bool ENT, int U>
__device__ __forceinline__ void add_batch(const Raw<T> (&x)[U], float c, Pair &S, Pair &W, float m) {
    constexpr int H = RowGroups<T>::N / 2;
    const Pair minus(-m, -m), cc(c, c);
#pragma unroll
    for (int u = 0; u < U; u++) {
        Pair p[H];
        x[u].pairs(p);
#pragma unroll
        for (int i = 0; i < H; i++) {
            const Pair d = p[i] + minus, t = d * cc;
            float a, b;
            t.get(a, b);
            const Pair e(exp2_approx(a), exp2_approx(b));
            S = S + e;
            if (ENT) W = fma2(e, d, W);
        }
    }
}
// The same where some are so far below it that e * d is not the 0 it has to be.
template <typename T, int U>
__device__ __forceinline__ void add_deep_batch(const Raw<T> (&x)[U], float c, Pair &S, Pair &W, float m) {
    constexpr int H = RowGroups<T>::N / 2;
#pragma unroll
    for (int u = 0; u < U; u++) {
        Pair p[H];
        x[u].pairs(p);
#pragma unroll
        for (int i = 0; i < H; i++) {
            float a, b;
            p[i].get(a, b);
            a -= m;
            b -= m;
            const Pair e(exp2_approx(a * c), exp2_approx(b * c));
            S = S + e;
            W = fma2(e, Pair(fmaxf(a, kDeep), fmaxf(b, kDeep)), W);
        }
    }
}

// A thread's running maximum and sums.
template <typename T, bool ENT>
struct Running {
    float m = -INFINITY, largest = -INFINITY;        // of all, and of the part
    Pair S = Pair(0.f, 0.f), W = Pair(0.f, 0.f);
    template <int U> __device__ __forceinline__ void add(const Raw<T> (&x)[U], float c) {
        float mx = x[0].largest(), mn = x[0].smallest();
#pragma unroll
        for (int u = 1; u < U; u++) {
            mx = fmaxf(mx, x[u].largest());
            if (ENT) mn = fminf(mn, x[u].smallest());
        }
        largest = fmaxf(largest, mx);
        if (mx > m) {
            if (m > -INFINITY) {
                const float dm = fmaxf(m - mx, kDeep), f = exp2_approx(dm * c);
                const Pair ff(f, f);
                if (ENT) W = ff * fma2(Pair(dm, dm), S, W);
                S = S * ff;
            }
            m = mx;
        }
        const float at = finite_or_zero(m);
        if (ENT && !(mn - at > kDeep)) add_deep_batch<T, U>(x, c, S, W, at);
        else add_batch<T, ENT, U>(x, c, S, W, at);
    }
};

}  // namespace sbp
