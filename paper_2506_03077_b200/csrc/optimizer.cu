// What applies the gradients of the streamed backward: the norm of all gradients with its clip factor, and one AdamW
// step over many tensors per launch, with moments in 32 bits or in 8.
//
// Both kernels read a list of tensors from their launch parameters (no table in device memory, nothing to allocate or
// to copy, so a captured graph replays them as they are) and walk it in pieces of kPiece elements: piece -> tensor by a
// binary search over the running piece counts, the same for the whole block.  Every element is read once and written
// once; what bounds them is HBM.
//
// Moments in 8 bits: blocks of 32 consecutive elements of a tensor share a power of two 2^(s - 127) (one byte s) and
// hold e4m3 codes.  s = (biased exponent of the block's largest magnitude) - 7, at least 1: the largest code is then
// below 256 and never saturates, and decoding is exact in fp32, and in bf16 for s of 3 and more (below, the smallest codes are
// finer than bf16's 2^-133: rounded).  The second moment is held as its ROOT,
// which halves the exponent range it needs (17 octaves from the smallest code to the largest are 34 of v), and a root
// that is not zero is held as at least the smallest code 2^-9: a second moment rounded to zero beside a first moment
// that is not would make the next step's quotient jump by 1 / sqrt(1 - beta2).
#include <cuda_fp8.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "common.cuh"
#include "sm100.cuh"

namespace sbp {
namespace {

constexpr int kThreads = 256, kGroup = 4;                 // a thread's unit: 4 consecutive elements (16 bytes of fp32)
constexpr int kUnroll = 4;                                // units per thread and piece, all loaded before the first is used
constexpr int kPiece = kThreads * kGroup * kUnroll;       // 4096 elements; a multiple of the 32 of a block of codes
constexpr int kBlock = STREAMBP_MX8_BLOCK;
static_assert(kPiece % kBlock == 0 && kBlock == 8 * kGroup, "eight neighbouring threads hold a block of codes");

template <int CAP>
struct StepParams {
    streambp_adamw_tensor t[CAP];
    int piece_begin[CAP + 1];        // pieces of tensor i: piece_begin[i] .. piece_begin[i + 1] - 1
    int n;
    double lr64, beta1_64, beta2_64; // for a step number on the device
    float lr, beta1, beta2, rest1, rest2;           // rest: 1 - beta
    // power times eps, lr / (1 - beta1^step) and 1 / sqrt(1 - beta2^step): a power of two that keeps the divisor in the range of
    // the reciprocal, which reads subnormal numbers as zero and gives zero for results that are some (1 but for extreme eps)
    double power;
    float eps, step_size, inv_root_bc2;
    const float *grad_scale;         // optional
    const int64_t *step;             // optional: the step number is read from the device
};

// the tensor that piece `b` belongs to: largest i with piece_begin[i] <= b
__device__ __forceinline__ int find_tensor(const int *begin, int n, int b) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (begin[mid] <= b) lo = mid; else hi = mid;
    }
    return lo;
}

// Four elements from `p`, or the first `valid` of them and zeros.
__device__ __forceinline__ void load4(const float *p, int valid, float (&v)[4]) {
    if (valid >= 4) {
        const float4 t = *reinterpret_cast<const float4 *>(p);
        v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = e < valid ? p[e] : 0.f;
    }
}
__device__ __forceinline__ void load4(const bf16 *p, int valid, float (&v)[4]) {
    if (valid >= 4) {
        const uint2 t = *reinterpret_cast<const uint2 *>(p);
        v[0] = __uint_as_float(t.x << 16); v[1] = __uint_as_float(t.x & 0xFFFF0000u);
        v[2] = __uint_as_float(t.y << 16); v[3] = __uint_as_float(t.y & 0xFFFF0000u);
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = e < valid ? __bfloat162float(p[e]) : 0.f;
    }
}
__device__ __forceinline__ void store4(float *p, int valid, const float (&v)[4]) {
    if (valid >= 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (e < valid) p[e] = v[e];
    }
}
__device__ __forceinline__ void store4(bf16 *p, int valid, const float (&v)[4]) {
    if (valid >= 4) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
        *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (e < valid) p[e] = __float2bfloat16_rn(v[e]);
    }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t *p, int valid) {
    if (valid >= 4) return *reinterpret_cast<const uint32_t *>(p);
    uint32_t w = 0;
    for (int e = 0; e < valid; e++) w |= (uint32_t)p[e] << (8 * e);
    return w;
}
__device__ __forceinline__ void store_codes(uint8_t *p, int valid, uint32_t w) {
    if (valid >= 4) {
        *reinterpret_cast<uint32_t *>(p) = w;
    } else {
        for (int e = 0; e < valid; e++) p[e] = (uint8_t)(w >> (8 * e));
    }
}

// 2^(s - 127) and its inverse; s = 255 stands for NaN (a block that held an infinity or a NaN)
__device__ __forceinline__ float scale_value(uint32_t s) { return s == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(s << 23); }
__device__ __forceinline__ void decode4(uint32_t codes, float scale, float (&v)[4]) {
#pragma unroll
    for (int e = 0; e < 2; e++) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes >> (16 * e)), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        v[2 * e] = f.x * scale;
        v[2 * e + 1] = f.y * scale;
    }
}
// the larger magnitude, a NaN if either is one
__device__ __forceinline__ float max_abs(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}
// biased exponent of the largest magnitude of four values, as the block scale sees it (255: an infinity or a NaN)
__device__ __forceinline__ uint32_t exponent_of(const float (&v)[4]) {
    return __float_as_uint(max_abs(max_abs(v[0], v[1]), max_abs(v[2], v[3]))) << 1 >> 24;
}
__device__ __forceinline__ uint32_t scale_byte(uint32_t exponent) {
    return exponent == 255u ? 255u : (exponent > 8u ? exponent - 7u : 1u);
}
// KEEP (values that are not negative): what `nonzero(e)` says is not zero becomes at least the smallest code
template <bool KEEP, typename F>
__device__ __forceinline__ uint32_t encode4(const float (&v)[4], uint32_t s, F nonzero) {
    const float inv = s == 255u ? 0.f : __uint_as_float((254u - s) << 23);
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; e++) y[e] = v[e] * inv;
    if (KEEP && fminf(fminf(y[0], y[1]), fminf(y[2], y[3])) < 0.001953125f) {      // rare, or a block that holds zeros
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (nonzero(e)) y[e] = fmaxf(y[e], 0.001953125f);
    }
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y[0], y[1]), __NV_SATFINITE, __NV_E4M3) |
           (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y[2], y[3]), __NV_SATFINITE, __NV_E4M3) << 16;
}
// the largest of two 16-bit fields over the eight neighbouring threads that hold a block
__device__ __forceinline__ uint32_t block_max2(uint32_t v) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) v = __vmaxu2(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

struct Rates {
    float gs, lr, b1, b2, rest1, rest2, eps, step_size, inv_root_bc2;
};
// Roots of N values, each rounded to nearest: from an approximate inverse root y, the root v y corrected by its exact
// residual (Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990).  The residual is
// exact where it is no subnormal number: values of which one is too small (or 0) or too large go through powers of four, so that
// subnormal second moments (gradients around 1e-19) have their roots too.
__device__ __forceinline__ float corrected_root(float v) {
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(v));
    const float s = v * y;
    return fmaf(fmaf(-s, s, v), 0.5f * y, s);
}
template <int N>
__device__ __forceinline__ void roots(float (&v)[N]) {
    constexpr uint32_t kLeast = 0x11000000u, kMost = 0x7d000000u;     // 2^-93 and 2^123 as bits, which order like the values
    bool odd = false;
#pragma unroll
    for (int e = 0; e < N; e++) odd |= __float_as_uint(v[e]) - kLeast > kMost - kLeast;
    if (!odd) {
#pragma unroll
        for (int e = 0; e < N; e++) v[e] = corrected_root(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < N; e++) {
            const bool small = v[e] < 1.f;
            const float w = corrected_root(v[e] * (small ? 0x1p96f : 0x1p-32f)) * (small ? 0x1p-48f : 0x1p16f);
            v[e] = isinf(v[e]) || v[e] == 0.f ? v[e] : w;
        }
    }
}
__device__ __forceinline__ float fast_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// the parameter from the new moment m and root u (quotient to 2 ulp, far below the rounding of the result)
__device__ __forceinline__ float moved(const Rates &r, float p, float decay, float m, float u) {
    return fmaf(-r.step_size, m * fast_rcp(fmaf(u, r.inv_root_bc2, r.eps)), p * decay);
}

// One piece of one tensor.  FULL: all of its kPiece elements exist, so that every load is unconditional and all of them
// are issued before the first is used (with the tests for a tensor's end between them the loads went out one by one).
template <typename P, bool MASTER, bool FULL>
__device__ __forceinline__ void step_piece_f32(const streambp_adamw_tensor &t, long long base, const Rates &r) {
    const long long left = t.count - base;
    P *param = static_cast<P *>(t.param) + base;
    float *master = t.master + base;
    const float *grad = t.grad + base;
    float *mp = static_cast<float *>(t.m) + base, *vp = static_cast<float *>(t.v) + base;
    const float decay = 1.f - r.lr * t.weight_decay;
    float g[kUnroll][4], p[kUnroll][4], m[kUnroll][4], v[kUnroll][4];
    int valid[kUnroll], off[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; k++) {
        off[k] = (k * kThreads + (int)threadIdx.x) * kGroup;
        const long long rest = left - off[k];
        valid[k] = FULL || rest >= 4 ? 4 : (rest > 0 ? (int)rest : 0);
    }
#pragma unroll
    for (int k = 0; k < kUnroll; k++) {
        load4(grad + off[k], valid[k], g[k]);
        if constexpr (MASTER) load4(master + off[k], valid[k], p[k]);
        else load4(param + off[k], valid[k], p[k]);
        load4(mp + off[k], valid[k], m[k]);
        load4(vp + off[k], valid[k], v[k]);
    }
#pragma unroll
    for (int k = 0; k < kUnroll; k++) {
        float u[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float x = g[k][e] * r.gs;
            m[k][e] = fmaf(r.b1, m[k][e], r.rest1 * x);
            u[e] = v[k][e] = fmaf(r.b2, v[k][e], r.rest2 * x * x);
        }
        roots(u);
#pragma unroll
        for (int e = 0; e < 4; e++) p[k][e] = moved(r, p[k][e], decay, m[k][e], u[e]);
        store4(mp + off[k], valid[k], m[k]);
        store4(vp + off[k], valid[k], v[k]);
        if constexpr (MASTER) store4(master + off[k], valid[k], p[k]);
        store4(param + off[k], valid[k], p[k]);
    }
}

// Moments in 8 bits: a thread takes eight consecutive elements (8 bytes of codes), four threads hold a block.
template <typename P, bool MASTER, bool FULL>
__device__ __forceinline__ void step_piece_mx8(const streambp_adamw_tensor &t, long long base, const Rates &r) {
    constexpr int kEach = 8;
    P *param = static_cast<P *>(t.param) + base;
    float *master = t.master + base;
    const float *grad = t.grad + base;
    uint8_t *mc = static_cast<uint8_t *>(t.m) + base, *vc = static_cast<uint8_t *>(t.v) + base;
    uint8_t *ms = t.m_scale + base / kBlock, *vs = t.v_scale + base / kBlock;
    const float decay = 1.f - r.lr * t.weight_decay;
#pragma unroll 1
    for (int k = 0; k < kPiece / (kThreads * kEach); k++) {
        const int off = (k * kThreads + (int)threadIdx.x) * kEach;
        const long long rest = t.count - base - off;
        const int valid = FULL || rest >= 8 ? 8 : (rest > 0 ? (int)rest : 0);
        const int lo = FULL ? 4 : (valid < 4 ? valid : 4), hi = valid - lo;
        float g[8], p[8], m[8], u[8];
        uint32_t cm[2], cv[2];
        auto half = [](float (&a)[8], int h) -> float(&)[4] { return *reinterpret_cast<float(*)[4]>(a + 4 * h); };
        load4(grad + off, lo, half(g, 0));
        load4(grad + off + 4, hi, half(g, 1));
        if constexpr (MASTER) {
            load4(master + off, lo, half(p, 0));
            load4(master + off + 4, hi, half(p, 1));
        } else if constexpr (FULL && std::is_same<P, bf16>::value) {
            Vec<bf16> x;
            x.load(reinterpret_cast<const bf16 *>(param) + off);
#pragma unroll
            for (int e = 0; e < 8; e++) p[e] = x.v[e];
        } else {
            load4(param + off, lo, half(p, 0));
            load4(param + off + 4, hi, half(p, 1));
        }
        if constexpr (FULL) {
            const uint2 a = *reinterpret_cast<const uint2 *>(mc + off), b = *reinterpret_cast<const uint2 *>(vc + off);
            cm[0] = a.x; cm[1] = a.y; cv[0] = b.x; cv[1] = b.y;
        } else {
            cm[0] = load_codes(mc + off, lo); cm[1] = load_codes(mc + off + 4, hi);
            cv[0] = load_codes(vc + off, lo); cv[1] = load_codes(vc + off + 4, hi);
        }
        const uint32_t sm = FULL || valid > 0 ? ms[off / kBlock] : 1u, sv = FULL || valid > 0 ? vs[off / kBlock] : 1u;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            decode4(cm[h], scale_value(sm), half(m, h));
            decode4(cv[h], scale_value(sv), half(u, h));
        }
        // every operation rounded by itself, the root to the nearest: a code that another evaluation of the formula in fp32
        // would round the other way changes what it stands for by up to an eighth, and with it the next step
#pragma unroll
        for (int e = 0; e < 8; e++) {
            g[e] *= r.gs;
            m[e] = __fadd_rn(__fmul_rn(r.b1, m[e]), __fmul_rn(r.rest1, g[e]));
            u[e] = __fadd_rn(__fmul_rn(r.b2, __fmul_rn(u[e], u[e])), __fmul_rn(__fmul_rn(r.rest2, g[e]), g[e]));
        }
        roots(u);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            p[e] = moved(r, p[e], decay, m[e], u[e]);
            if (!FULL && e >= valid) m[e] = u[e] = 0.f;
        }
        const uint32_t em = max(exponent_of(half(m, 0)), exponent_of(half(m, 1))),
                       eu = max(exponent_of(half(u, 0)), exponent_of(half(u, 1)));
        uint32_t big = em | (eu << 16);
        big = __vmaxu2(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = __vmaxu2(big, __shfl_xor_sync(0xffffffffu, big, 2));
        const uint32_t nm = scale_byte(big & 0xffffu), nv = scale_byte(big >> 16);
        uint32_t wm[2], wv[2];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            wm[h] = encode4<false>(half(m, h), nm, [](int) { return false; });
            // not zero is decided from what the root is made of: its square may have vanished in fp32
            wv[h] = encode4<true>(half(u, h), nv, [&](int e) {
                return 4 * h + e < valid && (g[4 * h + e] != 0.f || (cv[h] >> (8 * e) & 0x7fu) != 0u);
            });
        }
        if constexpr (FULL) {
            *reinterpret_cast<uint2 *>(mc + off) = make_uint2(wm[0], wm[1]);
            *reinterpret_cast<uint2 *>(vc + off) = make_uint2(wv[0], wv[1]);
        } else {
            store_codes(mc + off, lo, wm[0]); store_codes(mc + off + 4, hi, wm[1]);
            store_codes(vc + off, lo, wv[0]); store_codes(vc + off + 4, hi, wv[1]);
        }
        if ((FULL || valid > 0) && (threadIdx.x & 3) == 0) {
            ms[off / kBlock] = (uint8_t)nm;
            vs[off / kBlock] = (uint8_t)nv;
        }
        if constexpr (MASTER) {
            store4(master + off, lo, half(p, 0));
            store4(master + off + 4, hi, half(p, 1));
        }
        if constexpr (FULL && std::is_same<P, bf16>::value) {
            Vec<bf16> x;
#pragma unroll
            for (int e = 0; e < 8; e++) x.v[e] = p[e];
            x.store(reinterpret_cast<bf16 *>(param) + off);
        } else {
            store4(param + off, lo, half(p, 0));
            store4(param + off + 4, hi, half(p, 1));
        }
    }
}
template <typename P, bool MX8, bool MASTER, bool FULL>
__device__ __forceinline__ void step_piece(const streambp_adamw_tensor &t, long long base, const Rates &r) {
    if constexpr (MX8) step_piece_mx8<P, MASTER, FULL>(t, base, r);
    else step_piece_f32<P, MASTER, FULL>(t, base, r);
}

// Blocks per SM: moments in 8 bits are bound by the issue rate and by the loads in flight together, four blocks of 64
// registers take 0.56 ms for 233 M bf16 parameters (5.0 TB/s), five of 48 0.57, three of 80 0.65; moments in 32 bits need
// nothing but loads in flight, three blocks with four units of them a thread run at the copy rate (40 M parameters with a
// master copy: 0.186 ms, 6.4 TB/s).
// P: parameter type, MX8: moments in 8 bits.  With a master copy the parameter is the rounded master and is not read.
template <typename P, bool MX8, int CAP>
__global__ void __launch_bounds__(kThreads, MX8 ? 4 : 3) adamw_kernel(const __grid_constant__ StepParams<CAP> a) {
    pdl_enter();
    __shared__ float s_rate[2];
    Rates r{a.grad_scale ? *a.grad_scale : 1.f, a.lr, a.beta1, a.beta2, a.rest1, a.rest2, a.eps, a.step_size, a.inv_root_bc2};
    if (!isfinite(r.gs)) return;              // the gradients were not finite: the step is left out, the same for every block
    if (a.step) {
        if (threadIdx.x == 0) {
            const long long t = *a.step;
            const double n = t < 1 ? 1.0 : (double)t;
            s_rate[0] = (float)(a.power * a.lr64 / (1.0 - pow(a.beta1_64, n)));
            s_rate[1] = (float)(a.power / sqrt(1.0 - pow(a.beta2_64, n)));
        }
        __syncthreads();
        r.step_size = s_rate[0];
        r.inv_root_bc2 = s_rate[1];
    }
    const int pieces = a.piece_begin[a.n];
    for (int piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
        const int i = find_tensor(a.piece_begin, a.n, piece);
        const streambp_adamw_tensor &t = a.t[i];
        const long long base = (long long)(piece - a.piece_begin[i]) * kPiece;
        const bool full = t.count - base >= kPiece;
        if (std::is_same<P, bf16>::value && t.master) {
            if (full) step_piece<P, MX8, true, true>(t, base, r);
            else step_piece<P, MX8, true, false>(t, base, r);
        } else {
            if (full) step_piece<P, MX8, false, true>(t, base, r);
            else step_piece<P, MX8, false, false>(t, base, r);
        }
    }
}

// ---- norm of all gradients -----------------------------------------------------------------------------------
// Block b sums the squares of its pieces into partial[b]; one block then adds the partials in their order.  No atomics:
// the same gradients give the same bits.  A thread forms the squares of eight elements at a time in fp32 and adds them
// up in 64 bits (every square in 64 bits made the fp64 units the bound: 287 us for 233 M elements against 145 us of
// reading).  Where such a sum leaves the range in which fp32 squares are exact to a rounding -- gradients above 1e19, or
// all below 1e-13 -- the eight are squared again in 64 bits, so no norm of fp32 values overflows or vanishes.
template <int CAP>
struct NormParams {
    const float *grad[CAP];
    long long count[CAP];
    int piece_begin[CAP + 1];
    int n;
    int first;                       // 0: add to what an earlier launch of the same call left in the partials
    double *partial;
};
constexpr int kNormUnroll = 8, kNormPiece = kThreads * kGroup * kNormUnroll, kSmallPieces = 32;

__device__ __forceinline__ double block_sum_f64(double v, double *red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x < 32) {
        t = threadIdx.x < (blockDim.x >> 5) ? red[threadIdx.x] : 0.0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    }
    return t;                        // complete in warp 0
}

__device__ __forceinline__ double squares8(const float (&a)[4], const float (&b)[4]) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 4; e++) s = fmaf(a[e], a[e], fmaf(b[e], b[e], s));
    if (s < 1e30f && s > 1e-26f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int e = 0; e < 4; e++) d += (double)a[e] * a[e] + (double)b[e] * b[e];
    return d;
}

// `tid`: of kThreads that share the piece
template <bool FULL>
__device__ __forceinline__ double norm_piece(const float *g, long long left, int tid) {
    float x[kNormUnroll][4];
#pragma unroll
    for (int k = 0; k < kNormUnroll; k++) {
        const int off = (k * kThreads + tid) * kGroup;
        const long long rest = left - off;
        load4(g + off, FULL || rest >= 4 ? 4 : (rest > 0 ? (int)rest : 0), x[k]);
    }
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kNormUnroll; k += 2) sum += squares8(x[k], x[k + 1]);
    return sum;
}

// the thread's share of pieces first, first + step, ..
template <int CAP>
__device__ __forceinline__ double norm_share(const NormParams<CAP> &a, int first, int step, int tid) {
    double sum = 0.0;
    const int pieces = a.piece_begin[a.n];
    for (int piece = first; piece < pieces; piece += step) {
        const int i = find_tensor(a.piece_begin, a.n, piece);
        const long long base = (long long)(piece - a.piece_begin[i]) * kNormPiece, left = a.count[i] - base;
        sum += left >= kNormPiece ? norm_piece<true>(a.grad[i] + base, left, tid) : norm_piece<false>(a.grad[i] + base, left, tid);
    }
    return sum;
}
template <int CAP>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const __grid_constant__ NormParams<CAP> a) {
    pdl_enter();
    __shared__ double red[32];
    const double s = block_sum_f64(norm_share(a, blockIdx.x, gridDim.x, threadIdx.x), red);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = a.first ? s : a.partial[blockIdx.x] + s;
}
__device__ __forceinline__ void put_norm(double squares, float max_norm, float *norm, float *scale) {
    const double s = sqrt(squares);
    const float n = (float)s;
    *norm = n;
    if (!scale) return;
    // of the norm as it is given, in fp32: whoever forms the factor from it has the same
    if (!isfinite(s)) *scale = __uint_as_float(0x7fc00000u);
    else if (isinf(n)) *scale = fminf(1.f, (float)((double)max_norm / s));      // (max_norm may be infinite)
    else *scale = fminf(1.f, __fmul_rn(__frcp_rn(__fadd_rn(n, 1e-6f)), max_norm));
}
// Few pieces, one to each team of kThreads in a cluster, whose blocks' shares are added in their order.  One launch where the
// other way takes two: 20 tensors of 60 000 elements in all, norm and step, 13.4 us of the host's time against 15.1, the
// device's much the same (8 - 10 us).
__global__ void __launch_bounds__(1024) grad_norm_small_kernel(const __grid_constant__ NormParams<32> a, float max_norm, float *norm,
                                                               float *scale, WsHeader *hdr) {
    pdl_enter();
    if (blockIdx.x == 0 && threadIdx.x == 0) clear_status(hdr);
    __shared__ double red[32], share;
    constexpr int kTeams = 1024 / kThreads;
    const double s = block_sum_f64(norm_share(a, blockIdx.x * kTeams + threadIdx.x / kThreads, gridDim.x * kTeams, threadIdx.x % kThreads), red);
    if (threadIdx.x == 0) share = s;
    __syncthreads();
    cluster_sync_all();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        double t = 0.0;
        for (unsigned i = 0; i < gridDim.x; i++) t += ld_cluster_f64(map_to_cta(smem_u32(&share), i));
        put_norm(t, max_norm, norm, scale);
    }
    cluster_sync_all();                       // no block leaves while another may read its share
}

__global__ void __launch_bounds__(1024) grad_norm_finish_kernel(const double *partial, int n, float max_norm, float *norm,
                                                                float *scale, WsHeader *hdr) {
    pdl_enter();
    if (threadIdx.x == 0) clear_status(hdr);
    __shared__ double red[32];
    double v = 0.0;
    for (int i = threadIdx.x; i < n; i += blockDim.x) v += partial[i];
    const double s = block_sum_f64(v, red);
    if (threadIdx.x == 0) put_norm(s, max_norm, norm, scale);
}

// ---- moments in 8 bits <-> values -----------------------------------------------------------------------------
template <bool KEEP>
__global__ void __launch_bounds__(kThreads) mx8_encode_kernel(const float *x, long long count, uint8_t *codes, uint8_t *scale) {
    pdl_enter();
    const long long step = (long long)gridDim.x * kThreads * kGroup;
    // every thread of a warp runs the same number of turns: the block maximum is exchanged between neighbours
    for (long long base = (long long)blockIdx.x * kThreads * kGroup; base < count; base += step) {
        const long long at = base + (long long)threadIdx.x * kGroup, rest = count - at;
        const int valid = rest >= 4 ? 4 : (rest > 0 ? (int)rest : 0);
        float v[4];
        load4(x + at, valid, v);
        const uint32_t s = scale_byte(block_max2(exponent_of(v)));
        store_codes(codes + at, valid, encode4<KEEP>(v, s, [&](int e) { return v[e] > 0.f; }));
        if (valid > 0 && (threadIdx.x & 7) == 0) scale[at / kBlock] = (uint8_t)s;
    }
}
// 16 codes (one 16-byte load, half a block) per thread and turn, two turns in flight
template <typename T>
__global__ void __launch_bounds__(kThreads) mx8_decode_kernel(const uint8_t *codes, const uint8_t *scale, long long count, T *out) {
    pdl_enter();
    const long long step = (long long)gridDim.x * kThreads * 16;
    for (long long at = ((long long)blockIdx.x * kThreads + threadIdx.x) * 16; at < count; at += 2 * step) {
        uint4 w[2];
        uint32_t s[2];
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const long long o = at + k * step;
            if (o + 16 <= count) w[k] = *reinterpret_cast<const uint4 *>(codes + o);
            if (o < count) s[k] = scale[o / kBlock];
        }
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const long long o = at + k * step;
            if (o + 16 <= count) {
                const uint32_t q[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
                float v[16];
#pragma unroll
                for (int e = 0; e < 4; e++) decode4(q[e], scale_value(s[k]), *reinterpret_cast<float(*)[4]>(v + 4 * e));
#pragma unroll
                for (int e = 0; e < 16; e += Vec<T>::N) {
                    Vec<T> x;
#pragma unroll
                    for (int i = 0; i < Vec<T>::N; i++) x.v[i] = v[e + i];
                    x.store(out + o + e);
                }
            } else {
                for (long long e = o; e < count; e += 4) {
                    const int valid = count - e < 4 ? (int)(count - e) : 4;
                    float v[4];
                    decode4(load_codes(codes + e, valid), scale_value(s[k]), v);
                    store4(out + e, valid, v);
                }
            }
        }
    }
}

bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int begin_call() {
    call_state().cuda_error = 0;
    call_state().launches = 0;
    return STREAMBP_OK;
}

int grid_for(int64_t pieces, int per_sm) {
    const int64_t most = (int64_t)sm_count() * per_sm;
    return (int)(pieces < most ? pieces : most);
}

// Launches over `n` tensors of up to CAP at a time.  Two capacities: launch parameters are copied by the driver for every
// launch, and the usual layer of a dozen tensors should not pay for two hundred.
template <typename P, bool MX8, int CAP>
int launch_adamw(const streambp_adamw_cfg &c, const streambp_adamw_tensor *tensors, int n, const float *grad_scale,
                 const int64_t *step, double power, double step_size, double inv_root_bc2, cudaStream_t st) {
    StepParams<CAP> a;
    int i = 0;
    while (i < n) {
        a.n = 0;
        int64_t pieces = 0;
        for (; i < n && a.n < CAP; i++) {
            if (tensors[i].count == 0) continue;
            const int64_t more = (tensors[i].count + kPiece - 1) / kPiece;
            if (pieces + more > 0x40000000) break;
            a.t[a.n] = tensors[i];
            a.piece_begin[a.n++] = (int)pieces;
            pieces += more;
        }
        if (a.n == 0) break;
        a.piece_begin[a.n] = (int)pieces;
        a.lr64 = c.lr; a.beta1_64 = c.beta1; a.beta2_64 = c.beta2;
        a.lr = (float)c.lr; a.beta1 = (float)c.beta1; a.beta2 = (float)c.beta2;
        a.rest1 = (float)(1.0 - c.beta1); a.rest2 = (float)(1.0 - c.beta2);
        a.power = power;
        a.eps = (float)power * (float)c.eps;           // of eps in 32 bits, as the rest of the step takes it
        a.step_size = (float)(power * step_size);
        a.inv_root_bc2 = (float)(power * inv_root_bc2);
        a.grad_scale = grad_scale;
        a.step = step;
        SBP_LAUNCH((adamw_kernel<P, MX8, CAP>), grid_for(pieces, 8), kThreads, 0, st, a);
    }
    return STREAMBP_OK;
}
// Tensors i .. of the list into the parameters of one launch, as many as it holds; their pieces.
template <int CAP>
int64_t fill_norm(NormParams<CAP> &a, const float *const *grads, const int64_t *counts, int n, int &i) {
    a.n = 0;
    int64_t pieces = 0;
    for (; i < n && a.n < CAP; i++) {
        if (counts[i] == 0) continue;
        const int64_t more = (counts[i] + kNormPiece - 1) / kNormPiece;
        if (pieces + more > 0x40000000) break;
        a.grad[a.n] = grads[i];
        a.count[a.n] = counts[i];
        a.piece_begin[a.n++] = (int)pieces;
        pieces += more;
    }
    a.piece_begin[a.n] = (int)pieces;
    return pieces;
}
template <int CAP>
int launch_norm(const float *const *grads, const int64_t *counts, int n, double *partial, int *used, cudaStream_t st) {
    NormParams<CAP> a;
    a.partial = partial;
    const int most = sm_count() * 4 < 4096 ? sm_count() * 4 : 4096;   // blocks of a launch: those of a call share the partials
    int i = 0;
    *used = 0;
    while (i < n) {
        const int64_t pieces = fill_norm(a, grads, counts, n, i);
        if (a.n == 0) break;
        a.first = *used == 0;
        // the first launch of a call that needs more than one sets every partial, the others add to them
        const bool one = a.first && i == n;
        const int grid = one && pieces < most ? (int)pieces : most;
        *used = grid;
        SBP_LAUNCH(grad_norm_kernel<CAP>, grid, kThreads, 0, st, a);
    }
    return STREAMBP_OK;
}
template <typename P, bool MX8>
int launch_adamw_any(const streambp_adamw_cfg &c, const streambp_adamw_tensor *tensors, int n, const float *grad_scale,
                     const int64_t *step, double power, double step_size, double inv_root_bc2, cudaStream_t st) {
    if (n <= 32) return launch_adamw<P, MX8, 32>(c, tensors, n, grad_scale, step, power, step_size, inv_root_bc2, st);
    return launch_adamw<P, MX8, 256>(c, tensors, n, grad_scale, step, power, step_size, inv_root_bc2, st);
}

}  // namespace
}  // namespace sbp

using namespace sbp;

extern "C" {

int streambp_adamw_step(const streambp_adamw_cfg *cfg, const streambp_adamw_tensor *tensors, int32_t n,
                        const float *grad_scale, const int64_t *step, void *cuda_stream) {
    if (!cfg || (n > 0 && !tensors)) return STREAMBP_E_NULL;
    if (n < 0) return STREAMBP_E_SHAPE;
    if (cfg->param_dtype != STREAMBP_F32 && cfg->param_dtype != STREAMBP_BF16) return STREAMBP_E_DTYPE;
    if (cfg->state_dtype != STREAMBP_STATE_F32 && cfg->state_dtype != STREAMBP_STATE_MX8) return STREAMBP_E_DTYPE;
    if (!(cfg->lr >= 0.0) || !(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0) ||
        !(cfg->eps >= 0.0) || std::isinf((float)cfg->lr) || std::isinf((float)cfg->eps) || (!step && cfg->step < 1))
        return STREAMBP_E_SHAPE;
    if ((grad_scale && (reinterpret_cast<uintptr_t>(grad_scale) & 3u)) || (step && (reinterpret_cast<uintptr_t>(step) & 7u)))
        return STREAMBP_E_ALIGN;
    const bool mx8 = cfg->state_dtype == STREAMBP_STATE_MX8;
    for (int i = 0; i < n; i++) {
        const streambp_adamw_tensor &t = tensors[i];
        if (t.count < 0 || t.count > (1ll << 40) || !(t.weight_decay >= 0.f) || std::isinf(t.weight_decay)) return STREAMBP_E_SHAPE;
        if (t.count == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v || (mx8 && (!t.m_scale || !t.v_scale))) return STREAMBP_E_NULL;
        if (!al16(t.param) || !al16(t.master) || !al16(t.grad) || !al16(t.m) || !al16(t.v)) return STREAMBP_E_ALIGN;
        if (t.master && cfg->param_dtype != STREAMBP_BF16) return STREAMBP_E_DTYPE;
    }
    begin_call();
    const double t = step ? 1.0 : (double)cfg->step;
    const double step_size = cfg->lr / (1.0 - std::pow(cfg->beta1, t));
    const double inv_root_bc2 = 1.0 / std::sqrt(1.0 - std::pow(cfg->beta2, t));
    // a root is at most 2^64 and its factor below 2^30, so only eps takes a divisor out of 2^-126 .. 2^126 (a root that is not zero is
    // at least 2^-75), and 2^24 brings the smallest one back (a rate that this would overflow keeps its own power)
    const double power = cfg->eps > 0x1p125 ? 0x1p-8 : (cfg->eps > 0.0 && cfg->eps < 0x1p-126 && step_size < 0x1p100 ? 0x1p24 : 1.0);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    NvtxRange range("streambp_adamw_step");
    if (cfg->param_dtype == STREAMBP_F32)
        return mx8 ? launch_adamw_any<float, true>(*cfg, tensors, n, grad_scale, step, power, step_size, inv_root_bc2, st)
                   : launch_adamw_any<float, false>(*cfg, tensors, n, grad_scale, step, power, step_size, inv_root_bc2, st);
    return mx8 ? launch_adamw_any<bf16, true>(*cfg, tensors, n, grad_scale, step, power, step_size, inv_root_bc2, st)
               : launch_adamw_any<bf16, false>(*cfg, tensors, n, grad_scale, step, power, step_size, inv_root_bc2, st);
}

size_t streambp_grad_norm_workspace_bytes(void) { return kHeaderBytes + sizeof(double) * 4096; }

int streambp_grad_norm(const float *const *grads, const int64_t *counts, int32_t n, float max_norm, float *norm,
                       float *scale, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!norm || !workspace || (n > 0 && (!grads || !counts))) return STREAMBP_E_NULL;
    if (n < 0 || (scale && !(max_norm > 0.f))) return STREAMBP_E_SHAPE;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) || (reinterpret_cast<uintptr_t>(norm) & 3u) ||
        (reinterpret_cast<uintptr_t>(scale) & 3u))
        return STREAMBP_E_ALIGN;
    for (int i = 0; i < n; i++) {
        if (counts[i] < 0 || counts[i] > (1ll << 40)) return STREAMBP_E_SHAPE;
        if (counts[i] > 0 && !grads[i]) return STREAMBP_E_NULL;
        if (counts[i] > 0 && !al16(grads[i])) return STREAMBP_E_ALIGN;
    }
    if (workspace_bytes < streambp_grad_norm_workspace_bytes()) return STREAMBP_E_WORKSPACE;
    begin_call();
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    NvtxRange range("streambp_grad_norm");
    double *partial = reinterpret_cast<double *>(static_cast<char *>(workspace) + kHeaderBytes);
    WsHeader *hdr = static_cast<WsHeader *>(workspace);
    if (n <= 32) {
        NormParams<32> a;
        int i = 0;
        const int64_t pieces = fill_norm(a, grads, counts, n, i);
        if (i == n && pieces <= kSmallPieces) {
            const int blocks = pieces > 4 ? (int)(pieces + 3) / 4 : 1;
            return launch_clusters(grad_norm_small_kernel, dim3((unsigned)blocks), 1024, 0, blocks, 1, st, a, max_norm, norm, scale, hdr);
        }
    }
    int used = 0;
    if (n <= 32) SBP_TRY(launch_norm<32>(grads, counts, n, partial, &used, st));
    else SBP_TRY(launch_norm<512>(grads, counts, n, partial, &used, st));
    SBP_LAUNCH(grad_norm_finish_kernel, 1, 1024, 0, st, partial, used, max_norm, norm, scale, hdr);
    return STREAMBP_OK;
}

int streambp_mx8_encode(const float *values, int64_t count, int32_t keep_nonzero, uint8_t *codes, uint8_t *scales,
                        void *cuda_stream) {
    if (count < 0 || count > (1ll << 40)) return STREAMBP_E_SHAPE;
    if (count == 0) return STREAMBP_OK;
    if (!values || !codes || !scales) return STREAMBP_E_NULL;
    if (!al16(values) || !al16(codes)) return STREAMBP_E_ALIGN;
    begin_call();
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int grid = grid_for((count + kThreads * kGroup - 1) / (kThreads * kGroup), 8);
    if (keep_nonzero) SBP_LAUNCH(mx8_encode_kernel<true>, grid, kThreads, 0, st, values, (long long)count, codes, scales);
    else SBP_LAUNCH(mx8_encode_kernel<false>, grid, kThreads, 0, st, values, (long long)count, codes, scales);
    return STREAMBP_OK;
}

int streambp_mx8_decode(const uint8_t *codes, const uint8_t *scales, int64_t count, void *out, int32_t out_dtype,
                        void *cuda_stream) {
    if (count < 0 || count > (1ll << 40)) return STREAMBP_E_SHAPE;
    if (out_dtype != STREAMBP_F32 && out_dtype != STREAMBP_BF16) return STREAMBP_E_DTYPE;
    if (count == 0) return STREAMBP_OK;
    if (!codes || !scales || !out) return STREAMBP_E_NULL;
    if (!al16(codes) || !al16(out)) return STREAMBP_E_ALIGN;
    begin_call();
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int grid = grid_for((count + kThreads * 32 - 1) / (kThreads * 32), 8);
    if (out_dtype == STREAMBP_F32) SBP_LAUNCH(mx8_decode_kernel<float>, grid, kThreads, 0, st, codes, scales, (long long)count, (float *)out);
    else SBP_LAUNCH(mx8_decode_kernel<bf16>, grid, kThreads, 0, st, codes, scales, (long long)count, (bf16 *)out);
    return STREAMBP_OK;
}

}  // extern "C"
