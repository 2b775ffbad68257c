// Gradient of the product epilogue C = act(z) + residual, z = A W^T + bias: dz = dC * act'(z), dbias = column sums of dz
// (the residual's gradient is dC itself; dA = dz W and dW = dz^T A are products).
//
// HBM-bound: dC and z are read once, dz is written once.  A block owns a strip of 64 columns (a 128-byte row segment in
// bf16, eight threads of one 16-byte load each) and walks its rows 32 at a time, keeping the sums of its columns in
// registers; a grid of (strips, row splits) fills the GPU.  The splits of a strip leave their sums in `partials`, which a second
// small kernel adds in their order, or for small products are a cluster that adds them itself: no atomics, the same inputs
// give the same bits.  What bounds it: four rows in flight a thread as raw 16-byte words and four blocks an SM read at 4.2 -
// 4.7 TB/s (2048 x 14336 with GELU: 42 us for 176 MB, its tanh form 39; 8192 x 4096 with SiLU: 43 us for 201 MB); unpacked as they arrive they
// cost twice the registers and half the blocks.
#include <type_traits>

#include "activation.cuh"
#include "sm100.cuh"

namespace sbp {
namespace {

constexpr int kStrip = 64, kRowsAtOnce = 32, kClusterSplits = 8;

// Where a block's sums of its 64 columns go (threads 0 .. 63): the workspace, or through the cluster to dbias.
struct Sums {
    float *partials;          // [splits][N], or [2 splits][N] of the word kernel's two classes; null: no sums are wanted, or a cluster joins them
    float *dbias;             // cluster
    int accumulate;
    WsHeader *hdr;
};
__device__ __forceinline__ void put_sums(const Sums &to, float s, int col, int N, float *joined) {
    if (!to.dbias) {
        if (threadIdx.x < kStrip && col < N) to.partials[(int64_t)blockIdx.y * N + col] = s;
        return;
    }
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) clear_status(to.hdr);
    if (threadIdx.x < kStrip) joined[threadIdx.x] = s;
    __syncthreads();
    cluster_sync_all();
    if (blockIdx.y == 0 && threadIdx.x < kStrip && col < N) {
        float t = 0.f;
        for (unsigned i = 0; i < gridDim.y; i++) t += ld_cluster_f32(map_to_cta(smem_u32(joined + threadIdx.x), i));
        to.dbias[col] = to.accumulate ? to.dbias[col] + t : t;
    }
    cluster_sync_all();                       // no block leaves while another may read its sums
}

// rows and strips of any alignment: a lane per column (consecutive addresses), four rows at a time, eight in flight
template <typename T, int ACT>
__global__ void __launch_bounds__(256)
    epilogue_bwd_any_kernel(const T *dC, int64_t ldd, const T *pre, int64_t ldp, int64_t M, int N, int64_t rows_per_split, T *dZ,
                            int64_t ldz, Sums to) {
    pdl_enter();
    constexpr bool FAST = sizeof(T) == 2;
    __shared__ float s_sum[4][kStrip], joined[kStrip];
    const int tc = threadIdx.x & 63, tr = threadIdx.x >> 6, col = blockIdx.x * kStrip + tc;
    const int64_t first = blockIdx.y * rows_per_split, end = first + rows_per_split < M ? first + rows_per_split : M;
    float sum = 0.f;
    if (col < N) {
        constexpr int kAhead = 8;
        for (int64_t r0 = first + tr; r0 < end; r0 += 4 * kAhead) {
            T d[kAhead], z[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; a++) {
                const int64_t r = r0 + 4 * a < end ? r0 + 4 * a : r0;        // past the end: the first row again, not used
                d[a] = dC[r * ldd + col];
                if (ACT != STREAMBP_ACT_NONE) z[a] = pre[r * ldp + col];
            }
#pragma unroll
            for (int a = 0; a < kAhead; a++) {
                const int64_t r = r0 + 4 * a;
                if (r >= end) break;
                float x = to_f32(d[a]);
                // a product of its own, never part of an fma with the sum: the sums do not depend on whether dZ is wanted
                if (ACT != STREAMBP_ACT_NONE) x = __fmul_rn(x, slope<ACT, FAST>(to_f32(z[a])));
                sum += x;
                if (dZ) dZ[r * ldz + col] = from_f32<T>(x);
            }
        }
    }
    if (!to.partials && !to.dbias) return;
    s_sum[tr][tc] = sum;
    __syncthreads();
    put_sums(to, (s_sum[0][tc] + s_sum[1][tc]) + (s_sum[2][tc] + s_sum[3][tc]), col, N, joined);
}

// bf16 rows that start anywhere, those of all matrices alike: a warp to a row, a lane to two columns, read and written as the
// 4-byte word they make.  In rows that start on a word (class 0) a strip's words hold columns 64 b .. 64 b + 63, in the others
// (class 1) columns 64 b - 1 .. 64 b + 62; a warp's rows are eight apart and so of one class, and the classes' sums are rows
// of `partials` of their own.  A lane per column has half as much under way (5000 x 19001 with SiLU: 168 us against 130; 2048 x
// 8191: 38.6 and 32.4).
template <bool WORD>
__device__ __forceinline__ uint32_t load_two(const bf16 *p, bool lo, bool hi) {
    if (WORD) return *reinterpret_cast<const uint32_t *>(p);
    const uint16_t *u = reinterpret_cast<const uint16_t *>(p);
    return (lo ? (uint32_t)u[0] : 0u) | (hi ? (uint32_t)u[1] << 16 : 0u);
}
template <int ACT>
__global__ void __launch_bounds__(256, 4)
    epilogue_bwd_words_kernel(const bf16 *dC, int64_t ldd, const bf16 *pre, int64_t ldp, int64_t M, int N, int64_t rows_per_split,
                              bf16 *dZ, int64_t ldz, Sums to) {
    pdl_enter();
    constexpr int kAhead = 8, kWarps = 8;
    __shared__ float s_sum[kWarps][kStrip];
    __shared__ int s_class[kWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t first = blockIdx.y * rows_per_split, end = first + rows_per_split < M ? first + rows_per_split : M, row0 = first + warp;
    const int cls = (int)((reinterpret_cast<uintptr_t>(dC) >> 1) + (uint64_t)row0 * (uint64_t)ldd) & 1;
    const int col = blockIdx.x * kStrip + 2 * lane - cls;
    const bool lo = col >= 0 && col < N, hi = col + 1 < N;
    float sum_lo = 0.f, sum_hi = 0.f;
    auto rows = [&](auto whole) {                     // one loop without a branch between its loads for warps of whole words
        constexpr bool kWord = decltype(whole)::value;
        for (int64_t r0 = row0; r0 < end; r0 += kWarps * kAhead) {
            uint32_t d[kAhead], z[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; a++) {
                const int64_t r = r0 + kWarps * a < end ? r0 + kWarps * a : r0;      // past the end: the first row again, not used
                d[a] = load_two<kWord>(dC + r * ldd + col, lo, hi);
                if (ACT != STREAMBP_ACT_NONE) z[a] = load_two<kWord>(pre + r * ldp + col, lo, hi);
            }
#pragma unroll
            for (int a = 0; a < kAhead; a++) {
                const int64_t r = r0 + kWarps * a;
                if (r >= end) break;
                float x = __uint_as_float(d[a] << 16), y = __uint_as_float(d[a] & 0xFFFF0000u);
                if (ACT != STREAMBP_ACT_NONE) {
                    x = __fmul_rn(x, slope<ACT, true>(__uint_as_float(z[a] << 16)));
                    y = __fmul_rn(y, slope<ACT, true>(__uint_as_float(z[a] & 0xFFFF0000u)));
                }
                sum_lo += x;
                sum_hi += y;
                if (dZ) {
                    bf16 *at = dZ + r * ldz + col;
                    if (kWord) *reinterpret_cast<__nv_bfloat162 *>(at) = __floats2bfloat162_rn(x, y);
                    else {
                        if (lo) at[0] = __float2bfloat16_rn(x);
                        if (hi) at[1] = __float2bfloat16_rn(y);
                    }
                }
            }
        }
    };
    if (__all_sync(0xffffffffu, lo && hi)) rows(std::true_type());
    else rows(std::false_type());
    if (!to.partials) return;
    s_sum[warp][2 * lane] = sum_lo;
    s_sum[warp][2 * lane + 1] = sum_hi;
    if (lane == 0) s_class[warp] = cls;
    __syncthreads();
    const int of = threadIdx.x / kStrip, j = threadIdx.x % kStrip, c = blockIdx.x * kStrip + j - of;
    if (of < 2 && c >= 0 && c < N) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; w++) t += s_class[w] == of ? s_sum[w][j] : 0.f;
        to.partials[((int64_t)blockIdx.y * 2 + of) * N + c] = t;
    }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(256, 4)
    epilogue_bwd_kernel(const T *dC, int64_t ldd, const T *pre, int64_t ldp, int64_t M, int N, int64_t rows_per_split, T *dZ,
                        int64_t ldz, Sums to) {
    pdl_enter();
    constexpr bool FAST = sizeof(T) == 2;
    __shared__ float s_sum[8][kStrip + 1], joined[kStrip];
    const int tc = threadIdx.x & 7, tr = threadIdx.x >> 3;
    const int col0 = blockIdx.x * kStrip + tc * 8;
    const int64_t first = blockIdx.y * rows_per_split, end = first + rows_per_split < M ? first + rows_per_split : M;
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; e++) sum[e] = 0.f;
    if (col0 < N) {                                              // N is a multiple of 8
        constexpr int kAhead = sizeof(T) == 2 ? 4 : 2, V = 8 / Vec<T>::N;           // rows in flight per thread
        // loads stay as they came (four registers for 16 bytes) until their row's turn
        auto some = [&](int64_t r0, auto count) {
            constexpr int n = decltype(count)::value;
            uint4 d[n][V], z[n][V];
#pragma unroll
            for (int a = 0; a < n; a++)
#pragma unroll
                for (int v = 0; v < V; v++) {
                    d[a][v] = *reinterpret_cast<const uint4 *>(dC + (r0 + a * kRowsAtOnce) * ldd + col0 + v * Vec<T>::N);
                    if (ACT != STREAMBP_ACT_NONE)
                        z[a][v] = *reinterpret_cast<const uint4 *>(pre + (r0 + a * kRowsAtOnce) * ldp + col0 + v * Vec<T>::N);
                }
#pragma unroll
            for (int a = 0; a < n; a++)
#pragma unroll
                for (int v = 0; v < V; v++) {
                    Vec<T> x, y;
                    x.load(reinterpret_cast<const T *>(&d[a][v]));
                    if (ACT != STREAMBP_ACT_NONE) y.load(reinterpret_cast<const T *>(&z[a][v]));
#pragma unroll
                    for (int e = 0; e < Vec<T>::N; e++) {
                        if (ACT != STREAMBP_ACT_NONE) x.v[e] = __fmul_rn(x.v[e], slope<ACT, FAST>(y.v[e]));
                        sum[v * Vec<T>::N + e] += x.v[e];
                    }
                    if (dZ) x.store(dZ + (r0 + a * kRowsAtOnce) * ldz + col0 + v * Vec<T>::N);
                }
        };
        int64_t r = first + tr;
        for (; r + (kAhead - 1) * kRowsAtOnce < end; r += kAhead * kRowsAtOnce) some(r, std::integral_constant<int, kAhead>());
        for (; r < end; r += kRowsAtOnce) some(r, std::integral_constant<int, 1>());
    }
    if (!to.partials && !to.dbias) return;
    // the 32 row threads of a column: four of a warp by shuffles (lanes 8 apart), then the eight warps
#pragma unroll
    for (int e = 0; e < 8; e++) {
        sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 8);
        sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 16);
    }
    if ((threadIdx.x & 31) < 8) {
#pragma unroll
        for (int e = 0; e < 8; e++) s_sum[threadIdx.x >> 5][tc * 8 + e] = sum[e];
    }
    __syncthreads();
    const int c = blockIdx.x * kStrip + threadIdx.x;
    float s = 0.f;
    if (threadIdx.x < kStrip) {
#pragma unroll
        for (int w = 0; w < 8; w++) s += s_sum[w][threadIdx.x];
    }
    put_sums(to, s, c, N, joined);
}

__global__ void __launch_bounds__(256) epilogue_sum_kernel(const float *partials, int splits, int N, float *dbias, int accumulate, WsHeader *hdr) {
    pdl_enter();
    if (blockIdx.x == 0 && threadIdx.x == 0) clear_status(hdr);
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= N) return;
    float s = 0.f;
    for (int i = 0; i < splits; i++) s += partials[(int64_t)i * N + c];
    dbias[c] = accumulate ? dbias[c] + s : s;
}

// One launch, the splits of a strip a cluster: where the second launch would cost more than blocks that wait for one another
// do (333 x 2731: 8.3 -> 7.1 us, and 4 us less of the host's time; 1500 x 2000: 11.8 -> 8.5; 2048 x 14336: 43 -> 49, left).
bool small_product(int64_t M, int64_t N) { return M <= 2048 && M * N <= (4 << 20); }

template <typename T, int ACT>
int launch(const T *dC, int64_t ldd, const T *pre, int64_t ldp, int64_t M, int64_t N, T *dZ, int64_t ldz, float *dbias,
           bool accumulate, float *partials, WsHeader *hdr, cudaStream_t st) {
    auto rows16 = [](const void *q, int64_t ld) {
        return !q || ((reinterpret_cast<uintptr_t>(q) & 15u) == 0 && (ld * (int64_t)sizeof(T)) % 16 == 0);
    };
    const int splits = gemm_epilogue_splits(M, N);
    const int64_t per = (M + splits - 1) / splits;
    const dim3 grid((unsigned)((N + kStrip - 1) / kStrip), (unsigned)splits);
    const bool vec = N % 8 == 0 && rows16(dC, ldd) && rows16(ACT != STREAMBP_ACT_NONE ? pre : nullptr, ldp) && rows16(dZ, ldz);
    void (*kernel)(const T *, int64_t, const T *, int64_t, int64_t, int, int64_t, T *, int64_t, Sums) =
        vec ? epilogue_bwd_kernel<T, ACT> : epilogue_bwd_any_kernel<T, ACT>;
    Sums to = {nullptr, nullptr, accumulate ? 1 : 0, hdr};
    if (dbias && small_product(M, N)) {
        to.dbias = dbias;
        return launch_clusters(kernel, grid, 256, 0, 1, splits, st, dC, ldd, pre, ldp, M, (int)N, per, dZ, ldz, to);
    }
    if (dbias) to.partials = partials;
    if constexpr (std::is_same<T, bf16>::value) {
        auto start = [](const void *q, int64_t ld) { return (int)((reinterpret_cast<uintptr_t>(q) >> 1) & 1) + 2 * (int)(ld & 1); };
        if (!vec && (ACT == STREAMBP_ACT_NONE || start(pre, ldp) == start(dC, ldd)) && (!dZ || start(dZ, ldz) == start(dC, ldd))) {
            // one strip more where N is a multiple of its width: class 1 ends a column short
            SBP_LAUNCH(epilogue_bwd_words_kernel<ACT>, dim3((unsigned)(N / kStrip + 1), (unsigned)splits), 256, 0, st, dC, ldd, pre, ldp, M, (int)N,
                       per, dZ, ldz, to);
            if (!dbias) return STREAMBP_OK;
            SBP_LAUNCH(epilogue_sum_kernel, (unsigned)((N + 255) / 256), 256, 0, st, partials, 2 * splits, (int)N, dbias, accumulate ? 1 : 0, hdr);
            return STREAMBP_OK;
        }
    }
    SBP_LAUNCH(kernel, grid, 256, 0, st, dC, ldd, pre, ldp, M, (int)N, per, dZ, ldz, to);
    if (dbias)
        SBP_LAUNCH(epilogue_sum_kernel, (unsigned)((N + 255) / 256), 256, 0, st, partials, splits, (int)N, dbias, accumulate ? 1 : 0, hdr);
    return STREAMBP_OK;
}

}  // namespace

// Row splits: about twelve blocks (three waves of four) for each of the 148 SMs, at least 32 rows each; small products no
// more than a cluster holds.  A function of the sizes alone, so that the workspace query needs no GPU and the order of the
// sums is the same everywhere.
int gemm_epilogue_splits(int64_t M, int64_t N) {
    const int64_t strips = (N + kStrip - 1) / kStrip, rows = (M + kRowsAtOnce - 1) / kRowsAtOnce;
    int64_t s = (148 * 12 + strips - 1) / strips;
    if (s > rows) s = rows;
    if (s > kClusterSplits && small_product(M, N)) s = kClusterSplits;
    return s < 1 ? 1 : (int)s;
}

template <typename T>
int gemm_epilogue_bwd(const T *dC, int64_t ldd, const T *pre, int64_t ldp, int act, int64_t M, int64_t N, T *dZ, int64_t ldz,
                      float *dbias, bool accumulate, float *partials, WsHeader *hdr, cudaStream_t st) {
    switch (act) {
        case STREAMBP_ACT_NONE: return launch<T, STREAMBP_ACT_NONE>(dC, ldd, pre, ldp, M, N, dZ, ldz, dbias, accumulate, partials, hdr, st);
        case STREAMBP_ACT_RELU: return launch<T, STREAMBP_ACT_RELU>(dC, ldd, pre, ldp, M, N, dZ, ldz, dbias, accumulate, partials, hdr, st);
        case STREAMBP_ACT_GELU: return launch<T, STREAMBP_ACT_GELU>(dC, ldd, pre, ldp, M, N, dZ, ldz, dbias, accumulate, partials, hdr, st);
        case STREAMBP_ACT_GELU_TANH:
            return launch<T, STREAMBP_ACT_GELU_TANH>(dC, ldd, pre, ldp, M, N, dZ, ldz, dbias, accumulate, partials, hdr, st);
        case STREAMBP_ACT_SILU: return launch<T, STREAMBP_ACT_SILU>(dC, ldd, pre, ldp, M, N, dZ, ldz, dbias, accumulate, partials, hdr, st);
        default: return STREAMBP_E_SHAPE;
    }
}
template int gemm_epilogue_bwd<float>(const float *, int64_t, const float *, int64_t, int, int64_t, int64_t, float *, int64_t,
                                      float *, bool, float *, WsHeader *, cudaStream_t);
template int gemm_epilogue_bwd<bf16>(const bf16 *, int64_t, const bf16 *, int64_t, int, int64_t, int64_t, bf16 *, int64_t,
                                     float *, bool, float *, WsHeader *, cudaStream_t);

}  // namespace sbp
