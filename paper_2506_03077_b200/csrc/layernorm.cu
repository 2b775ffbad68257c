// Layer norm: y = (x - mean) rstd gain + bias over the columns of each row, and its gradient with the sums of gain and bias.
//
//   xhat = (x - mean) rstd,  g = dy gain,  dx = (g - mean(g) - xhat mean(g xhat)) rstd (+ add)
//   dgain = sum over rows of dy xhat,  dbias = sum over rows of dy
// A row's values stay in registers between the passes over it, so that all tensors cross HBM once: memory is the bound.  Rows go
// to a warp, or to blocks of as many threads as hold them; the column sums stay in the threads that own the columns while a block
// walks its rows, and the blocks' sums are joined in their order by a second launch (no atomics: equal inputs give equal bits).
// Statistics and sums are fp32, the variance from the differences to the mean; y and dx are rounded once.
//
// Measured at 16384 x 4096 bf16: forward 49 us (5.5 TB/s; 84 % of a copy's rate), gradient with a residual's gradient added and
// both sums 90 us (5.9 TB/s; 91 %), by two fp32 operations to an instruction: by one each 99, as without the residual, so that
// instructions weigh as much as memory there; forward that changes nothing.  fp32, 8192 x 4096 without a residual: 42 and 71 us.
// Rows that start anywhere are moved by single elements and bound by their instructions: 8192 x 4097 bf16 in 50 and 104 us (2.7
// and 1.9 TB/s), the gradient in fp32 with a residual 120 us (4.5 TB/s).  (Loading the two aligned groups around such a thread's
// columns and shifting them into place: 63 and 162 us.)
#include <algorithm>
#include <type_traits>

#include "vocab_rows.cuh"

namespace sbp {

namespace {
constexpr int kMaxThreads = 512, kWideThreads = 1024, kMaxWarps = kWideThreads / 32;

__device__ __forceinline__ float sum_of(Pair p) {
    float a, b;
    p.get(a, b);
    return a + b;
}

// N elements at a time: 16 bytes, or one where a pointer, a leading dimension or the width is not made of 16-byte groups.
// They stay in their storage type while they wait.
template <typename T, int N> struct Pack {
    uint4 w;
    __device__ __forceinline__ void load(const T *p) { w = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void clear() { w = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&x)[N]) const {
        Vec<T> a;
        a.load(reinterpret_cast<const T *>(&w));
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = a.v[i];
    }
    __device__ __forceinline__ void get(Pair (&x)[N / 2]) const {
        Raw<T> r;
        r.w = w;
        r.pairs(x);
    }
    static __device__ __forceinline__ void store(T *p, const Pair (&x)[N / 2]) {
        float v[N];
#pragma unroll
        for (int i = 0; i < N / 2; i++) x[i].get(v[2 * i], v[2 * i + 1]);
        store(p, v);
    }
    __device__ __forceinline__ void set(const float (&x)[N]) {
        Vec<T> a;
#pragma unroll
        for (int i = 0; i < N; i++) a.v[i] = x[i];
        a.store(reinterpret_cast<T *>(&w));
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[N]) {
        Pack q;
        q.set(x);
        *reinterpret_cast<uint4 *>(p) = q.w;
    }
};
template <typename T> struct Pack<T, 1> {
    T w;
    __device__ __forceinline__ void load(const T *p) { w = *p; }
    __device__ __forceinline__ void clear() { w = from_f32<T>(0.f); }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = to_f32(w); }
    static __device__ __forceinline__ void store(T *p, const float (&x)[1]) { *p = from_f32<T>(x[0]); }
};

// Columns of a thread, `step` apart from `first` on.  In 16-byte groups the threads of a row hold neighbouring groups; single
// elements are a warp's own 32 NV neighbouring columns, 32 apart, so that a thread's addresses are one register and constants
// (with as many addresses and bounds as columns a row of 4097 took 96 instructions an element, and 4 times as long).
template <int N, int NV> struct Columns {
    int first, step, left;      // left: from the first to the row's end
    bool all;                   // the warp's columns are all the row's: its loops ask nothing
    __device__ __forceinline__ Columns(int thread, int threads, int d)
        : first(N == 1 ? (thread >> 5) * 32 * NV + (thread & 31) : thread * N), step(N == 1 ? 32 : threads * N), left(d - first),
          all(N == 1 && ((thread >> 5) + 1) * 32 * NV <= d) {}
    __device__ __forceinline__ int at(int j) const { return j * step; }         // from the first
    __device__ __forceinline__ bool has(int j) const { return j * step < left; }
    // f(a constant), true where each j has its column
    template <typename F> __device__ __forceinline__ void each(F f) const {
        if (N == 1 && all) f(std::true_type());
        else f(std::false_type());
    }
};

// Sums of two values over the threads of a row: one warp (no barrier), or the block (one barrier; `slot` alternates).
template <bool WARP>
__device__ __forceinline__ float2 row_sum(float a, float b, float2 (*red)[kMaxWarps], int slot) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if (WARP) return make_float2(a, b);
    if ((threadIdx.x & 31) == 0) red[slot][threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    float2 s = make_float2(0.f, 0.f);
    for (int w = 0; w < (int)(blockDim.x >> 5); w++) {
        s.x += red[slot][w].x;
        s.y += red[slot][w].y;
    }
    return s;
}

template <typename T>
struct NormArgs {
    const T *x, *gain, *bias;           // gain and bias are optional
    T *y;
    float *mean, *rstd;                 // optional
    int64_t rows, ldx, ldy;
    int d;
    float eps;
};

// WARP: a warp to a row, else a block
template <typename T, int N, int NV, bool WARP>
__global__ void __launch_bounds__(N == 1 ? kWideThreads : kMaxThreads) norm_fwd_kernel(NormArgs<T> a) {
    pdl_enter();
    __shared__ float2 red[2][kMaxWarps];
    const int lane = WARP ? threadIdx.x & 31 : threadIdx.x;
    const int64_t r = WARP ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    if (r >= a.rows) return;
    const Columns<N, NV> col(lane, WARP ? 32 : blockDim.x, a.d);
    const T *x = a.x + r * a.ldx + col.first;
    Pack<T, N> p[NV];
    col.each([&](auto all) {
#pragma unroll
        for (int j = 0; j < NV; j++) {
            p[j].clear();
            if (all.value || col.has(j)) p[j].load(x + col.at(j));
        }
    });
    float s = 0.f, v[N];
#pragma unroll
    for (int j = 0; j < NV; j++) {
        p[j].get(v);
#pragma unroll
        for (int i = 0; i < N; i++) s += v[i];
    }
    const float mean = row_sum<WARP>(s, 0.f, red, 0).x / (float)a.d;
    s = 0.f;
    col.each([&](auto all) {
#pragma unroll
        for (int j = 0; j < NV; j++) {
            if (!all.value && !col.has(j)) continue;
            p[j].get(v);
#pragma unroll
            for (int i = 0; i < N; i++) s = fmaf(v[i] - mean, v[i] - mean, s);
        }
    });
    const float rstd = rsqrtf(row_sum<WARP>(s, 0.f, red, 1).x / (float)a.d + a.eps);
    if (lane == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    const T *gain = a.gain + col.first, *bias = a.bias + col.first;
    T *y = a.y + r * a.ldy + col.first;
    col.each([&](auto all) {
#pragma unroll
        for (int j = 0; j < NV; j++) {
            if (!all.value && !col.has(j)) continue;
            float g[N];
            Pack<T, N> q;
            p[j].get(v);
#pragma unroll
            for (int i = 0; i < N; i++) v[i] = (v[i] - mean) * rstd;
            if (a.gain) {
                q.load(gain + col.at(j));
                q.get(g);
#pragma unroll
                for (int i = 0; i < N; i++) v[i] *= g[i];
            }
            if (a.bias) {
                q.load(bias + col.at(j));
                q.get(g);
#pragma unroll
                for (int i = 0; i < N; i++) v[i] += g[i];
            }
            Pack<T, N>::store(y + col.at(j), v);
        }
    });
}

// rows too wide for registers: the row is read three times (the second and third time from L2)
template <typename T, int N>
__global__ void __launch_bounds__(kWideThreads) norm_fwd_wide_kernel(NormArgs<T> a) {
    pdl_enter();
    __shared__ float2 red[2][kMaxWarps];
    const int64_t r = blockIdx.x;
    const T *x = a.x + r * a.ldx;
    const int first = threadIdx.x * N, step = kWideThreads * N;
    Pack<T, N> p;
    float s = 0.f, v[N];
#pragma unroll 4
    for (int c = first; c < a.d; c += step) {
        p.load(x + c);
        p.get(v);
#pragma unroll
        for (int i = 0; i < N; i++) s += v[i];
    }
    const float mean = row_sum<false>(s, 0.f, red, 0).x / (float)a.d;
    s = 0.f;
#pragma unroll 4
    for (int c = first; c < a.d; c += step) {
        p.load(x + c);
        p.get(v);
#pragma unroll
        for (int i = 0; i < N; i++) s = fmaf(v[i] - mean, v[i] - mean, s);
    }
    const float rstd = rsqrtf(row_sum<false>(s, 0.f, red, 1).x / (float)a.d + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    for (int c = first; c < a.d; c += step) {
        float g[N];
        p.load(x + c);
        p.get(v);
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = (v[i] - mean) * rstd;
        if (a.gain) {
            p.load(a.gain + c);
            p.get(g);
#pragma unroll
            for (int i = 0; i < N; i++) v[i] *= g[i];
        }
        if (a.bias) {
            p.load(a.bias + c);
            p.get(g);
#pragma unroll
            for (int i = 0; i < N; i++) v[i] += g[i];
        }
        Pack<T, N>::store(a.y + r * a.ldy + c, v);
    }
}

template <typename T>
struct NormGradArgs {
    const T *dy, *x, *gain, *add;       // gain and add are optional
    const float *mean, *rstd;
    T *dx;                              // optional
    float *partials;                    // [blocks][2][d], null where no sums are wanted
    int64_t rows, lddy, ldx, ldadd, lddx;
    int d;
};

// rows that start anywhere, element by element: sixteen columns a thread (8192 x 4097 bf16 in 104 us, with eight 114)
template <typename T, int NV>
__global__ void __launch_bounds__(kMaxThreads) norm_bwd_kernel(NormGradArgs<T> a) {
    pdl_enter();
    __shared__ float2 red[2][kMaxWarps];
    const Columns<1, NV> col(threadIdx.x, blockDim.x, a.d);
    float sg[NV], sb[NV], gain[NV];
#pragma unroll
    for (int j = 0; j < NV; j++) {
        sg[j] = sb[j] = 0.f;
        gain[j] = a.gain && col.has(j) ? to_f32(a.gain[col.first + col.at(j)]) : 1.f;
    }
    int slot = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, slot ^= 1) {
        const T *pdy = a.dy + r * a.lddy + col.first, *px = a.x + r * a.ldx + col.first, *padd = a.add + r * a.ldadd + col.first;
        T dy[NV], x[NV], add[NV];
        col.each([&](auto all) {
#pragma unroll
            for (int j = 0; j < NV; j++) {
                dy[j] = x[j] = from_f32<T>(0.f);
                if (!all.value && !col.has(j)) continue;
                dy[j] = pdy[col.at(j)];
                x[j] = px[col.at(j)];
            }
#pragma unroll
            for (int j = 0; j < NV; j++) add[j] = from_f32<T>(0.f);
            if (!a.add) return;
#pragma unroll
            for (int j = 0; j < NV; j++)
                if (all.value || col.has(j)) add[j] = padd[col.at(j)];
        });
        const float mean = a.mean[r], rstd = a.rstd[r];
        float s1 = 0.f, s2 = 0.f, g[NV], h[NV];
#pragma unroll
        for (int j = 0; j < NV; j++) {              // (dy is 0 behind the last column)
            g[j] = to_f32(dy[j]);
            h[j] = (to_f32(x[j]) - mean) * rstd;
            sg[j] = fmaf(g[j], h[j], sg[j]);
            sb[j] += g[j];
            g[j] *= gain[j];
            s1 += g[j];
            s2 = fmaf(g[j], h[j], s2);
        }
        if (!a.dx) continue;
        const float2 s = row_sum<false>(s1, s2, red, slot);
        const float m1 = s.x / (float)a.d, m2 = s.y / (float)a.d;
        T *dx = a.dx + r * a.lddx + col.first;
        col.each([&](auto all) {
#pragma unroll
            for (int j = 0; j < NV; j++)
                if (all.value || col.has(j)) dx[col.at(j)] = from_f32<T>(fmaf(g[j] - m1 - h[j] * m2, rstd, to_f32(add[j])));
        });
    }
    if (!a.partials) return;
    float *out = a.partials + (int64_t)blockIdx.x * 2 * a.d + col.first;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        if (!col.has(j)) continue;
        out[col.at(j)] = sg[j];
        out[a.d + col.at(j)] = sb[j];
    }
}

__device__ __forceinline__ float4 four(Pair a, Pair b) {
    float4 f;
    a.get(f.x, f.y);
    b.get(f.z, f.w);
    return f;
}

// The same for rows of whole 16-byte groups, brought into shared memory by the copy engine `stages` rows ahead: the sums of the
// columns take most of the registers, so rows that wait there would be few.  A row's place is free again when all threads have
// taken their part into registers, which the barrier of the row's sums tells.
// TEAMS > 1: that many warps to a block, each with rows and a ring of its own (narrow rows, whose barriers would cost most).
template <typename T, int NV, int TEAMS>
__global__ void __launch_bounds__(TEAMS > 1 ? TEAMS * 32 : kMaxThreads) norm_bwd_ring_kernel(NormGradArgs<T> a, int stages) {
    pdl_enter();
    constexpr int N = Vec<T>::N, H = N / 2, kMaxStages = 8;
    constexpr bool WARP = TEAMS > 1;
    extern __shared__ __align__(128) unsigned char s_raw[];
    __shared__ float2 red[2][kMaxWarps];
    __shared__ __align__(8) unsigned long long s_full[TEAMS][kMaxStages];
    __shared__ int s_abort;
    const int lanes = WARP ? 32 : blockDim.x, lane = WARP ? threadIdx.x & 31 : threadIdx.x, team = WARP ? threadIdx.x >> 5 : 0;
    const int row_bytes = a.d * (int)sizeof(T), streams = a.add ? 3 : 2;
    const int64_t first = (int64_t)blockIdx.x * TEAMS + team, step = (int64_t)gridDim.x * TEAMS;       // rows
    auto stage = [&](int s, int stream) { return s_raw + (size_t)((team * stages + s) * streams + stream) * row_bytes; };
    auto fetch = [&](int64_t r, int s) {            // by lane 0
        const uint32_t bar = smem_u32(&s_full[team][s]);
        mbar_expect_tx(bar, (uint32_t)(streams * row_bytes));
        auto copy = [&](const T *p, int stream) {
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                             smem_u32(stage(s, stream))), "l"(p), "r"(row_bytes), "r"(bar)
                         : "memory");
        };
        copy(a.dy + r * a.lddy, 0);
        copy(a.x + r * a.ldx, 1);
        if (a.add) copy(a.add + r * a.ldadd, 2);
    };
    if (threadIdx.x == 0) s_abort = 0;
    if (lane == 0) {
        for (int s = 0; s < stages; s++) mbar_init(smem_u32(&s_full[team][s]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int s = 0; s < stages; s++)
            if (first + s * step < a.rows) fetch(first + s * step, s);
    }
    Pair sg[NV][H], sb[NV][H];
    Pack<T, N> gain[NV];
#pragma unroll
    for (int j = 0; j < NV; j++) {
#pragma unroll
        for (int i = 0; i < H; i++) sg[j][i] = sb[j][i] = Pair(0.f, 0.f);
        const int c = (lane + j * lanes) * N;
        gain[j].clear();
        if (a.gain && c < a.d) gain[j].load(a.gain + c);
    }
    float mean = first < a.rows ? a.mean[first] : 0.f, rstd = first < a.rows ? a.rstd[first] : 0.f;
    __syncthreads();
    int slot = 0, at = 0, phase = 0;
    for (int64_t r = first; r < a.rows; r += step, slot ^= 1) {
        const bool more = r + step < a.rows;
        const float mean_next = more ? a.mean[r + step] : 0.f, rstd_next = more ? a.rstd[r + step] : 0.f;
        mbar_wait_warp(smem_u32(&s_full[team][at]), phase, &s_abort);
        Pack<T, N> dy[NV], x[NV], add[NV];
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (lane + j * lanes) * N;
            dy[j].clear();
            x[j].clear();
            add[j].clear();
            if (c >= a.d) continue;
            dy[j].load(reinterpret_cast<const T *>(stage(at, 0)) + c);
            x[j].load(reinterpret_cast<const T *>(stage(at, 1)) + c);
            if (a.add) add[j].load(reinterpret_cast<const T *>(stage(at, 2)) + c);
        }
        const Pair minus_mean(-mean, -mean), rstd2(rstd, rstd);
        Pair s1(0.f, 0.f), s2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < NV; j++) {
            if ((lane + j * lanes) * N >= a.d) continue;
            Pair g[H], h[H], w[H];
            dy[j].get(g);
            x[j].get(h);
            gain[j].get(w);
#pragma unroll
            for (int i = 0; i < H; i++) {
                h[i] = (h[i] + minus_mean) * rstd2;
                sg[j][i] = fma2(g[i], h[i], sg[j][i]);
                sb[j][i] = sb[j][i] + g[i];
                if (a.gain) g[i] = g[i] * w[i];
                s1 = s1 + g[i];
                s2 = fma2(g[i], h[i], s2);
            }
        }
        const float2 s = row_sum<WARP>(sum_of(s1), sum_of(s2), red, slot);
        if (WARP) __syncwarp();
        if (lane == 0 && r + stages * step < a.rows && *(volatile int *)&s_abort == 0) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            fetch(r + stages * step, at);
        }
        if (++at == stages) {
            at = 0;
            phase ^= 1;
        }
        if (a.dx) {
            const float m1 = s.x / (float)a.d, m2 = s.y / (float)a.d;
            const Pair minus_m1(-m1, -m1), minus_m2(-m2, -m2);
#pragma unroll
            for (int j = 0; j < NV; j++) {
                const int c = (lane + j * lanes) * N;
                if (c >= a.d) continue;
                Pair g[H], h[H], w[H], t[H];
                dy[j].get(g);
                x[j].get(h);
                gain[j].get(w);
                add[j].get(t);
#pragma unroll
                for (int i = 0; i < H; i++) {
                    if (a.gain) g[i] = g[i] * w[i];
                    g[i] = fma2(fma2((h[i] + minus_mean) * rstd2, minus_m2, g[i] + minus_m1), rstd2, t[i]);
                }
                Pack<T, N>::store(a.dx + r * a.lddx + c, g);
            }
        }
        mean = mean_next;
        rstd = rstd_next;
    }
    if (*(volatile int *)&s_abort) {        // give copies that are still in flight time to land before shared memory is released
        const unsigned long long t0 = global_timer();
        while (global_timer() - t0 < 200000ull) {}
    }
    if (!a.partials) return;
    float *out = a.partials + (int64_t)blockIdx.x * 2 * a.d;
    // the warps' sums, one on another in the rings' place, the last warp's on all
    float *own = reinterpret_cast<float *>(s_raw);
    for (int t = 0; t < TEAMS; t++) {
        if (WARP) __syncthreads();
        if (t != team) continue;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (lane + j * lanes) * N;
            if (c >= a.d) continue;
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                float4 g = four(sg[j][i / 2], sg[j][i / 2 + 1]), b = four(sb[j][i / 2], sb[j][i / 2 + 1]);
                auto add = [](float4 x, const float *y) {
                    const float4 z = *reinterpret_cast<const float4 *>(y);
                    return make_float4(x.x + z.x, x.y + z.y, x.z + z.z, x.w + z.w);
                };
                if (t > 0) {
                    g = add(g, own + c + i);
                    b = add(b, own + a.d + c + i);
                }
                float *to = t == TEAMS - 1 ? out : own;
                *reinterpret_cast<float4 *>(to + c + i) = g;
                *reinterpret_cast<float4 *>(to + a.d + c + i) = b;
            }
        }
    }
}

// Rows wider than registers hold, in a block of up to 1024 threads: only the columns' sums stay there, and a row is read from the
// ring once for its sums and again for dx (2048 x 16384 bf16 in 70 us; dx and the sums by a launch each, rows from memory, 126).
// Its place is filled again behind the barrier of the next row's sums.
template <typename T>
__global__ void __launch_bounds__(kWideThreads) norm_bwd_wide_ring_kernel(NormGradArgs<T> a, int stages) {
    pdl_enter();
    constexpr int N = Vec<T>::N, NV = 16 / N, H = N / 2, kMaxStages = 8;
    extern __shared__ __align__(128) unsigned char s_raw[];
    __shared__ float2 red[2][kMaxWarps];
    __shared__ __align__(8) unsigned long long s_full[kMaxStages];
    __shared__ int s_abort;
    const int lanes = blockDim.x, lane = threadIdx.x, row_bytes = a.d * (int)sizeof(T), streams = a.add ? 3 : 2;
    const int64_t step = gridDim.x;
    auto stage = [&](int s, int stream) { return s_raw + (size_t)(s * streams + stream) * row_bytes; };
    auto fetch = [&](int64_t r, int s) {            // by thread 0
        const uint32_t bar = smem_u32(&s_full[s]);
        mbar_expect_tx(bar, (uint32_t)(streams * row_bytes));
        auto copy = [&](const T *p, int stream) {
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                             smem_u32(stage(s, stream))), "l"(p), "r"(row_bytes), "r"(bar)
                         : "memory");
        };
        copy(a.dy + r * a.lddy, 0);
        copy(a.x + r * a.ldx, 1);
        if (a.add) copy(a.add + r * a.ldadd, 2);
    };
    if (lane == 0) {
        s_abort = 0;
        for (int s = 0; s < stages; s++) mbar_init(smem_u32(&s_full[s]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int s = 0; s < stages; s++)
            if (blockIdx.x + s * step < a.rows) fetch(blockIdx.x + s * step, s);
    }
    Pair sg[NV][H], sb[NV][H];
#pragma unroll
    for (int j = 0; j < NV; j++)
#pragma unroll
        for (int i = 0; i < H; i++) sg[j][i] = sb[j][i] = Pair(0.f, 0.f);
    __syncthreads();
    int slot = 0, at = 0, phase = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += step, slot ^= 1) {
        const float mean = a.mean[r], rstd = a.rstd[r];
        mbar_wait_warp(smem_u32(&s_full[at]), phase, &s_abort);
        const T *dy = reinterpret_cast<const T *>(stage(at, 0)), *x = reinterpret_cast<const T *>(stage(at, 1));
        const Pair minus_mean(-mean, -mean), rstd2(rstd, rstd);
        auto both = [&](int c, Pair (&g)[H], Pair (&h)[H]) {       // dy and xhat
            Pack<T, N> p;
            p.load(dy + c);
            p.get(g);
            p.load(x + c);
            p.get(h);
#pragma unroll
            for (int i = 0; i < H; i++) h[i] = (h[i] + minus_mean) * rstd2;
        };
        auto times_gain = [&](int c, Pair (&g)[H]) {
            if (!a.gain) return;
            Pair w[H];
            Pack<T, N> p;
            p.load(a.gain + c);
            p.get(w);
#pragma unroll
            for (int i = 0; i < H; i++) g[i] = g[i] * w[i];
        };
        Pair s1(0.f, 0.f), s2(0.f, 0.f), g[H], h[H];
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (lane + j * lanes) * N;
            if (c >= a.d) continue;
            both(c, g, h);
#pragma unroll
            for (int i = 0; i < H; i++) {
                sg[j][i] = fma2(g[i], h[i], sg[j][i]);
                sb[j][i] = sb[j][i] + g[i];
            }
            times_gain(c, g);
#pragma unroll
            for (int i = 0; i < H; i++) {
                s1 = s1 + g[i];
                s2 = fma2(g[i], h[i], s2);
            }
        }
        const float2 s = row_sum<false>(sum_of(s1), sum_of(s2), red, slot);
        if (lane == 0 && r != blockIdx.x && r + (stages - 1) * step < a.rows && *(volatile int *)&s_abort == 0) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            fetch(r + (stages - 1) * step, at == 0 ? stages - 1 : at - 1);
        }
        if (a.dx) {
            const float m1 = s.x / (float)a.d, m2 = s.y / (float)a.d;
            const Pair minus_m1(-m1, -m1), minus_m2(-m2, -m2);
#pragma unroll
            for (int j = 0; j < NV; j++) {
                const int c = (lane + j * lanes) * N;
                if (c >= a.d) continue;
                both(c, g, h);
                times_gain(c, g);
                Pair t[H];
#pragma unroll
                for (int i = 0; i < H; i++) t[i] = Pair(0.f, 0.f);
                if (a.add) {
                    Pack<T, N> p;
                    p.load(reinterpret_cast<const T *>(stage(at, 2)) + c);
                    p.get(t);
                }
#pragma unroll
                for (int i = 0; i < H; i++) g[i] = fma2(fma2(h[i], minus_m2, g[i] + minus_m1), rstd2, t[i]);
                Pack<T, N>::store(a.dx + r * a.lddx + c, g);
            }
        }
        if (++at == stages) {
            at = 0;
            phase ^= 1;
        }
    }
    if (*(volatile int *)&s_abort) {        // give copies that are still in flight time to land before shared memory is released
        const unsigned long long t0 = global_timer();
        while (global_timer() - t0 < 200000ull) {}
    }
    if (!a.partials) return;
    float *out = a.partials + (int64_t)blockIdx.x * 2 * a.d;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (lane + j * lanes) * N;
        if (c >= a.d) continue;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            *reinterpret_cast<float4 *>(out + c + i) = four(sg[j][i / 2], sg[j][i / 2 + 1]);
            *reinterpret_cast<float4 *>(out + a.d + c + i) = four(sb[j][i / 2], sb[j][i / 2 + 1]);
        }
    }
}

// wide rows: dx row by row, the row read twice
template <typename T, int N>
__global__ void __launch_bounds__(kWideThreads) norm_bwd_wide_kernel(NormGradArgs<T> a) {
    pdl_enter();
    __shared__ float2 red[2][kMaxWarps];
    const int64_t r = blockIdx.x;
    const float mean = a.mean[r], rstd = a.rstd[r];
    const T *dy = a.dy + r * a.lddy, *x = a.x + r * a.ldx;
    const int first = threadIdx.x * N, step = kWideThreads * N;
    auto both = [&](int c, float (&g)[N], float (&h)[N]) {       // dy gain and xhat
        Pack<T, N> p, q;
        p.load(dy + c);
        q.load(x + c);
        p.get(g);
        q.get(h);
        if (a.gain) {
            float w[N];
            p.load(a.gain + c);
            p.get(w);
#pragma unroll
            for (int i = 0; i < N; i++) g[i] *= w[i];
        }
#pragma unroll
        for (int i = 0; i < N; i++) h[i] = (h[i] - mean) * rstd;
    };
    float s1 = 0.f, s2 = 0.f, g[N], h[N];
#pragma unroll 2
    for (int c = first; c < a.d; c += step) {
        both(c, g, h);
#pragma unroll
        for (int i = 0; i < N; i++) {
            s1 += g[i];
            s2 = fmaf(g[i], h[i], s2);
        }
    }
    const float2 s = row_sum<false>(s1, s2, red, 0);
    const float m1 = s.x / (float)a.d, m2 = s.y / (float)a.d;
    for (int c = first; c < a.d; c += step) {
        both(c, g, h);
        float t[N];
#pragma unroll
        for (int i = 0; i < N; i++) t[i] = 0.f;
        if (a.add) {
            Pack<T, N> p;
            p.load(a.add + r * a.ldadd + c);
            p.get(t);
        }
#pragma unroll
        for (int i = 0; i < N; i++) g[i] = fmaf(g[i] - m1 - h[i] * m2, rstd, t[i]);
        Pack<T, N>::store(a.dx + r * a.lddx + c, g);
    }
}
// wide rows: column sums of a split of the rows, four rows of loads at a time
template <typename T, int N>
__global__ void __launch_bounds__(128) norm_bwd_wide_sums_kernel(NormGradArgs<T> a, int splits) {
    pdl_enter();
    constexpr int U = 4;
    const int c = (blockIdx.x * 128 + threadIdx.x) * N;
    if (c >= a.d) return;
    float sg[N], sb[N];
#pragma unroll
    for (int i = 0; i < N; i++) sg[i] = sb[i] = 0.f;
    for (int64_t r = blockIdx.y; r < a.rows; r += U * (int64_t)splits) {
        Pack<T, N> dy[U], x[U];
        float mean[U], rstd[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t q = r + u * (int64_t)splits;
            if (q >= a.rows) continue;
            dy[u].load(a.dy + q * a.lddy + c);
            x[u].load(a.x + q * a.ldx + c);
            mean[u] = a.mean[q];
            rstd[u] = a.rstd[q];
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (r + u * (int64_t)splits >= a.rows) continue;
            float g[N], h[N];
            dy[u].get(g);
            x[u].get(h);
#pragma unroll
            for (int i = 0; i < N; i++) {
                sg[i] = fmaf(g[i], (h[i] - mean[u]) * rstd[u], sg[i]);
                sb[i] += g[i];
            }
        }
    }
    float *out = a.partials + (int64_t)blockIdx.y * 2 * a.d;
#pragma unroll
    for (int i = 0; i < N; i++) {
        out[c + i] = sg[i];
        out[a.d + c + i] = sb[i];
    }
}

// dgain, dbias (+)= the blocks' sums, added in their order: 32 columns and 32 sections of the blocks to a block
__global__ void __launch_bounds__(1024) norm_join_kernel(const float *__restrict__ partials, int blocks, int d, float *dgain,
                                                         float *dbias, int accumulate, WsHeader *hdr) {
    pdl_enter();
    __shared__ float s_part[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    if (blockIdx.x == 0 && threadIdx.x == 0) clear_status(hdr);
    const int64_t c = (int64_t)blockIdx.x * 32 + x;         // of both sums, one behind the other
    const int per = (blocks + 31) / 32, b0 = y * per, b1 = min(b0 + per, blocks);
    float s = 0.f;
    if (c < 2 * (int64_t)d) {
#pragma unroll 8
        for (int b = b0; b < b1; b++) s += partials[(int64_t)b * 2 * d + c];
    }
    s_part[y][x] = s;
    __syncthreads();
    if (y || c >= 2 * (int64_t)d) return;
    for (int i = 1; i < 32; i++) s += s_part[i][x];
    float *to = c < d ? (dgain ? dgain + c : nullptr) : (dbias ? dbias + (c - d) : nullptr);
    if (to) *to = accumulate ? *to + s : s;
}

template <typename T>
bool grouped(const void *p, int64_t ld) {
    return p == nullptr || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % Vec<T>::N == 0);
}
constexpr int64_t kNarrow = 4096;   // rows of few groups from which on each is a warp's (65536 x 768 bf16 in 69 us, as a block's 116; 8192 in 17 and 25)
constexpr int64_t kWide = 8192;     // columns above which a gradient's rows are not held by a block

template <typename T, int N, int NV>
int launch_fwd_warps(const NormArgs<T> &a, cudaStream_t st) {
    SBP_LAUNCH((norm_fwd_kernel<T, N, NV, true>), (unsigned)((a.rows + 7) / 8), 256, 0, st, a);
    return STREAMBP_OK;
}
template <typename T, int N, int NV>
int launch_fwd(const NormArgs<T> &a, cudaStream_t st) {
    const int groups = (a.d + N - 1) / N;
    if (groups <= 32 * NV) return launch_fwd_warps<T, N, NV>(a, st);
    SBP_LAUNCH((norm_fwd_kernel<T, N, NV, false>), (unsigned)a.rows, (unsigned)(((groups + NV - 1) / NV + 31) / 32 * 32), 0, st, a);
    return STREAMBP_OK;
}
// Shared memory of an SM for the rows under way, and blocks that share it
constexpr int kRingBytes = 208 << 10;
template <typename T, int NV, int TEAMS = 1>
int launch_ring(const NormGradArgs<T> &a, int blocks, cudaStream_t st) {
    const int groups = a.d / Vec<T>::N, threads = TEAMS > 1 ? TEAMS * 32 : ((groups + NV - 1) / NV + 31) / 32 * 32;
    const int each = (blocks + 147) / 148, row = TEAMS * (a.add ? 3 : 2) * a.d * (int)sizeof(T);
    const int64_t turns = (a.rows + TEAMS * (int64_t)blocks - 1) / (TEAMS * (int64_t)blocks);
    const int stages = (int)std::max<int64_t>(1, std::min<int64_t>({8, turns, kRingBytes / (each * row)}));
    static PerDevice ready;
    auto kernel = norm_bwd_ring_kernel<T, NV, TEAMS>;
    if (!ready.get([&] { return cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes)) ? 1 : 0; }))
        return STREAMBP_E_CUDA;
    SBP_LAUNCH(kernel, (unsigned)blocks, threads, stages * row, st, a, stages);
    return STREAMBP_OK;
}
template <typename T>
int launch_wide_ring(const NormGradArgs<T> &a, int blocks, int row, cudaStream_t st) {
    static PerDevice ready;
    auto kernel = norm_bwd_wide_ring_kernel<T>;
    if (!ready.get([&] { return cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes)) ? 1 : 0; }))
        return STREAMBP_E_CUDA;
    const int stages = std::min(8, kRingBytes / row);
    SBP_LAUNCH(kernel, (unsigned)blocks, (unsigned)((a.d + 511) / 512 * 32), stages * row, st, a, stages);
    return STREAMBP_OK;
}
}  // namespace

int layernorm_take_fault() { return take_fault_local(); }

// Blocks that walk the rows of a backward pass (a function of the sizes alone, so that the order of the sums is the same
// everywhere and the workspace query needs no GPU).
int layernorm_blocks(int64_t rows, int64_t d) {
    // (at least four rows each, so that there are not more sums to join than rows that made them)
    const int64_t most = d > kWide ? std::max<int64_t>(16, 148 * 16 * 1024 / d) : 148 * std::min<int64_t>(32, std::max<int64_t>(2, kWide / d));
    return (int)std::max<int64_t>(std::min<int64_t>(rows, 148), std::min<int64_t>((rows + 3) / 4, most));
}

template <typename T>
int layernorm_fwd(const T *x, int64_t ldx, const T *gain, const T *bias, float eps, int64_t rows, int64_t d, T *y, int64_t ldy,
                  float *mean, float *rstd, cudaStream_t st) {
    const NormArgs<T> a{x, gain, bias, y, mean, rstd, rows, ldx, ldy, (int)d, eps};
    constexpr int N = Vec<T>::N;
    const bool whole = d % N == 0 && grouped<T>(x, ldx) && grouped<T>(y, ldy) && grouped<T>(gain, 0) && grouped<T>(bias, 0);
    // (held by blocks of up to 512 threads: 2048 x 16384 bf16 in 31 us, read three times 51; by 1024 threads 1024 x 32768 in 42, read
    // three times 36)
    if (d > kMaxThreads * (whole ? 4 * N : 16)) {
        if (whole) SBP_LAUNCH((norm_fwd_wide_kernel<T, N>), (unsigned)rows, kWideThreads, 0, st, a);
        else SBP_LAUNCH((norm_fwd_wide_kernel<T, 1>), (unsigned)rows, kWideThreads, 0, st, a);
        return STREAMBP_OK;
    }
    const int64_t groups = d / N;
    // (element by element: 8192 x 4097 bf16 in 50 us with sixteen a thread, with eight 67; 4 rows in 5.5 and 4.0)
    if (!whole && d <= 128) return launch_fwd_warps<T, 1, 4>(a, st);
    if (!whole) return rows < 4 * 148 ? launch_fwd<T, 1, 8>(a, st) : launch_fwd<T, 1, 16>(a, st);
    // (four groups a thread where rows fill the GPU: 16384 x 4096 bf16 in 50 us and 4 rows in 3.0, with two 58 and 2.4)
    if (groups <= 32) return launch_fwd_warps<T, N, 1>(a, st);
    if (groups <= 1024 && a.rows < 4 * 148) return launch_fwd<T, N, 2>(a, st);
    return launch_fwd<T, N, 4>(a, st);
}

template <typename T>
int layernorm_bwd(const T *dy, int64_t lddy, const T *x, int64_t ldx, const T *gain, const float *mean, const float *rstd,
                  const T *add, int64_t ldadd, int64_t rows, int64_t d, T *dx, int64_t lddx, float *dgain, float *dbias,
                  bool accumulate, float *partials, WsHeader *hdr, cudaStream_t st) {
    const bool sums = dgain || dbias;
    const NormGradArgs<T> a{dy, x, gain, add, mean, rstd, dx, sums ? partials : nullptr, rows, lddy, ldx, ldadd, lddx, (int)d};
    int blocks = layernorm_blocks(rows, d);
    constexpr int N = Vec<T>::N;
    const bool whole = d % N == 0 && grouped<T>(x, ldx) && grouped<T>(dy, lddy) && grouped<T>(add, ldadd) && grouped<T>(dx, lddx) &&
                       grouped<T>(gain, 0);
    const int64_t row = (add ? 3 : 2) * d * (int64_t)sizeof(T);
    if (whole && d > kWide && d <= 16 * kWideThreads && 2 * row <= kRingBytes) {
        blocks = std::min(blocks, 148);
        SBP_TRY((launch_wide_ring<T>(a, blocks, (int)row, st)));
    } else if (d > kWide) {
        // (the sums first: dx may lie where dy or x does)
        const int64_t strips = (d / (whole ? N : 1) + 127) / 128;
        if (sums) {
            if (whole) SBP_LAUNCH((norm_bwd_wide_sums_kernel<T, N>), dim3((unsigned)strips, (unsigned)blocks), 128, 0, st, a, blocks);
            else SBP_LAUNCH((norm_bwd_wide_sums_kernel<T, 1>), dim3((unsigned)strips, (unsigned)blocks), 128, 0, st, a, blocks);
        }
        if (dx) {
            if (whole) SBP_LAUNCH((norm_bwd_wide_kernel<T, N>), (unsigned)rows, kWideThreads, 0, st, a);
            else SBP_LAUNCH((norm_bwd_wide_kernel<T, 1>), (unsigned)rows, kWideThreads, 0, st, a);
        }
    } else if (whole) {
        // sixteen columns a thread (their sums take 32 registers), fewer where a row is short
        const int64_t groups = d / N;
        if (groups <= (N == 4 ? 128 : 96) && rows >= kNarrow) {
            // (the sums of four bf16 groups a lane leave too few warps an SM)
            blocks = std::min(blocks, 148 * (groups <= 64 ? 6 : 3));
            if (groups <= 32) SBP_TRY((launch_ring<T, 1, 4>(a, blocks, st)));
            else if (groups <= 64) SBP_TRY((launch_ring<T, 2, 4>(a, blocks, st)));
            else if (N > 4 || groups <= 96) SBP_TRY((launch_ring<T, 3, 4>(a, blocks, st)));
            else SBP_TRY((launch_ring<T, 16 / N, 4>(a, blocks, st)));
        } else if (groups <= 128) SBP_TRY((launch_ring<T, 1>(a, blocks, st)));
        else SBP_TRY((launch_ring<T, 16 / N>(a, blocks, st)));
    } else {
        SBP_LAUNCH((norm_bwd_kernel<T, 16>), (unsigned)blocks, (unsigned)((d + 511) / 512 * 32), 0, st, a);
    }
    if (sums)
        SBP_LAUNCH(norm_join_kernel, (unsigned)((2 * d + 31) / 32), 1024, 0, st, partials, blocks, (int)d, dgain, dbias,
                   accumulate ? 1 : 0, hdr);
    return STREAMBP_OK;
}

template int layernorm_fwd<float>(const float *, int64_t, const float *, const float *, float, int64_t, int64_t, float *, int64_t,
                                  float *, float *, cudaStream_t);
template int layernorm_fwd<bf16>(const bf16 *, int64_t, const bf16 *, const bf16 *, float, int64_t, int64_t, bf16 *, int64_t,
                                 float *, float *, cudaStream_t);
template int layernorm_bwd<float>(const float *, int64_t, const float *, int64_t, const float *, const float *, const float *,
                                  const float *, int64_t, int64_t, int64_t, float *, int64_t, float *, float *, bool, float *,
                                  WsHeader *, cudaStream_t);
template int layernorm_bwd<bf16>(const bf16 *, int64_t, const bf16 *, int64_t, const bf16 *, const float *, const float *,
                                 const bf16 *, int64_t, int64_t, int64_t, bf16 *, int64_t, float *, float *, bool, float *,
                                 WsHeader *, cudaStream_t);

}  // namespace sbp
