// C = act(A W^T + bias) + residual on tcgen05 (bf16 operands, fp32 accumulation), the sum before act kept on request.
//
// Two kernels, chosen by the number of rows:
//   gemm_act_pair_kernel : persistent CTA pairs (cta_group::2) over output tiles of 256 rows x `bn` columns.  Per CTA one
//                          producer warp (TMA), one issuing warp and EIGHT epilogue warps: an epilogue that reads a
//                          residual, evaluates an activation and writes two matrices takes longer than four warps have
//                          while the next tile's products run (K = 512: 304 us with four warps for a problem that takes
//                          the products 60 us).  `bn` is chosen so that the tiles fill the last wave of pairs.
//   gemm_act_rows_kernel : up to 128 rows a tile.  The roles of the operands are exchanged -- 128 rows of W are the M side of
//                          the product, the few rows of A its N side -- because a product's rate is bound by the
//                          shared memory it reads, which a 256-row tile of mostly missing rows spends in full (35 us for
//                          ONE row of a 4096 x 4096 product).  K is split over a cluster of up to eight CTAs so that all
//                          SMs stream W; their sums meet through distributed shared memory, in a fixed order.
// Every wait is bounded (sm100.cuh); on expiry the roles leave their loops, tensor memory is freed and the kernel returns.
#include <cstring>

#include "activation.cuh"
#include "sm100.cuh"

namespace sbp {
namespace {

constexpr int BK = 64;
constexpr uint32_t kTmemCols = 512;

struct EpiParams {
    CUtensorMap map_a, map_w, map_c, map_pre;     // map_c, map_pre: 32 x 32 blocks (vec only)
    int M, N, nkb;
    const bf16 *bias, *residual;
    bf16 *C, *pre;
    long long ldr, ldc, ldp;
    int vec;                 // rows of C, residual and pre and the bias start on 16-byte boundaries
    int bn, tiles_m, tiles;  // pair kernel
};

// ---------------------------------------------------------------------------------------------------------------
// CTA pairs
// ---------------------------------------------------------------------------------------------------------------
constexpr int PM = 256, PBN = 256, P_STAGES = 6;
constexpr int P_A_BYTES = 128 * BK * 2, P_STAGE_BYTES = P_A_BYTES + (PBN / 2) * BK * 2;      // 16 + 16 KiB
constexpr int P_EPI_WARPS = 8, P_THREADS = 64 + 32 * P_EPI_WARPS;
constexpr int P_STAGING = P_EPI_WARPS * 32 * 32 * 4;                                          // 4 KiB a warp
constexpr int P_SMEM = P_STAGES * P_STAGE_BYTES + P_STAGING + 1024 + 256;
static_assert(P_SMEM <= 232448, "pair kernel exceeds the shared memory of an SM");

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ void st_shared_v4(uint32_t at, const uint32_t (&w)[4]) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}

// 32 rows (one per lane) x 32 columns of the tile: z = accumulator + bias, then pre, activation, residual, C.  The blocks
// of pre and C leave through shared memory (rows of 64 bytes, 64-byte swizzle: no bank conflicts) as TMA stores, which also
// clip the rows behind the matrix and whole groups of 8 columns (of a group that the matrix ends in they write all 16 bytes:
// such a block goes through finish_rows).  As 16-byte stores of 32 different rows they took the memory pipe four times as many
// accesses as they have lines.
template <int ACT>
__device__ __forceinline__ void finish_vec(const EpiParams &p, const uint32_t (&r)[32], const uint4 (&rs)[4], uint32_t stage,
                                           int lane, int row0, int col0) {
    // the previous block's stores have read the staging
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const uint32_t at = stage + (uint32_t)lane * 64u + ((uint32_t)(j ^ ((lane >> 1) & 3)) << 4);
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; e++) z[e] = __uint_as_float(r[8 * j + e]);
        if (p.bias && col0 + 8 * j < p.N) {            // no group ends outside the matrix
            Vec<bf16> b;
            b.load(p.bias + col0 + 8 * j);
#pragma unroll
            for (int e = 0; e < 8; e++) z[e] += b.v[e];
        }
        uint32_t w[4];
        if (p.pre) {
#pragma unroll
            for (int e = 0; e < 4; e++) w[e] = pack2(z[2 * e], z[2 * e + 1]);
            st_shared_v4(at + 2048u, w);
        }
        const uint32_t q[4] = {rs[j].x, rs[j].y, rs[j].z, rs[j].w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            float a = activate<ACT, true>(z[2 * e]), b = activate<ACT, true>(z[2 * e + 1]);
            if (p.residual) {
                a += __uint_as_float(q[e] << 16);
                b += __uint_as_float(q[e] & 0xFFFF0000u);
            }
            w[e] = pack2(a, b);
        }
        st_shared_v4(at, w);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        tma_store_2d(&p.map_c, stage, col0, row0);
        if (p.pre) tma_store_2d(&p.map_pre, stage + 2048u, col0, row0);
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
// The same where rows do not start on 16-byte boundaries, or the columns end inside a group of 8: the block is transposed
// through shared memory (16-byte groups exchanged with the row's bits, so that neither side has bank conflicts) and walked
// row by row with a lane per column: consecutive addresses instead of one element of each of 32 rows.  Eight rows at a time,
// without a branch among them, and the residuals of the next eight under way: 8000 x 1997 x 1024 with a residual 107 -> 68 us,
// with GELU and z kept 94 -> 70 (2000 columns: 47).
template <int ACT, bool RES>
__device__ __forceinline__ void finish_rows(const EpiParams &p, const uint32_t (&r)[32], float *stage, int lane, int row0, int col0) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");        // of blocks that went as TMA stores
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const uint32_t w[4] = {r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]};
        st_shared_v4(smem_u32(stage) + (uint32_t)(lane * 128 + ((j ^ (lane & 7)) << 4)), w);
    }
    __syncwarp();
    const int col = col0 + lane;
    if (col < p.N) {
        const float b = p.bias ? __bfloat162float(p.bias[col]) : 0.f;
        const int rows = p.M - row0 < 32 ? p.M - row0 : 32;
        const bf16 *res_at = RES ? p.residual + (long long)row0 * p.ldr + col : nullptr;
        bf16 *pre_at = p.pre ? p.pre + (long long)row0 * p.ldp + col : nullptr, *c_at = p.C + (long long)row0 * p.ldc + col;
        bf16 ahead[8];
        auto request = [&](int i) {
#pragma unroll
            for (int k = 0; k < 8; k++) ahead[k] = i + k < rows ? res_at[(i + k) * p.ldr] : __float2bfloat16_rn(0.f);
        };
        if (RES) request(0);
#pragma unroll 1
        for (int i = 0; i < rows; i += 8) {         // eight rows at a time, the residuals of the next ones requested first
            float res[8], z[8];
#pragma unroll
            for (int k = 0; k < 8; k++) res[k] = RES ? __bfloat162float(ahead[k]) : 0.f;
            if (RES) request(i + 8);
#pragma unroll
            for (int k = 0; k < 8; k++) z[k] = stage[(i + k) * 32 + (((lane >> 2) ^ k) << 2) + (lane & 3)] + b;
            if (pre_at)
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (i + k < rows) pre_at[(i + k) * p.ldp] = __float2bfloat16_rn(z[k]);
#pragma unroll
            for (int k = 0; k < 8; k++) z[k] = activate<ACT, true>(z[k]) + res[k];
#pragma unroll
            for (int k = 0; k < 8; k++)
                if (i + k < rows) c_at[(i + k) * p.ldc] = __float2bfloat16_rn(z[k]);
        }
    }
    __syncwarp();
}

template <int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(P_THREADS, 1) gemm_act_pair_kernel(const __grid_constant__ EpiParams p) {
    pdl_enter();
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t tiles = (raw + 1023u) & ~1023u;
    uint8_t *base = smem_raw + (tiles - raw);
    float *staging = reinterpret_cast<float *>(base + P_STAGES * P_STAGE_BYTES);
    uint8_t *aux = base + P_STAGES * P_STAGE_BYTES + P_STAGING;
    const uint32_t bar_full = smem_u32(aux);                  // P_STAGES, used in the even CTA
    const uint32_t bar_empty = bar_full + 8 * P_STAGES;       // P_STAGES, in both
    const uint32_t bar_tfull = bar_empty + 8 * P_STAGES;      // 2, in both
    const uint32_t bar_tempty = bar_tfull + 16;               // 2, even CTA: the epilogue warps of both arrive
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(aux + 16 * P_STAGES + 32);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(aux + 16 * P_STAGES + 40);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_cta_rank();
    const int pair = (int)(blockIdx.x >> 1), pairs = (int)(gridDim.x >> 1);

    if (threadIdx.x == 0) {
        for (int s = 0; s < P_STAGES; s++) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; b++) {
            mbar_init(bar_tfull + 8 * b, 1);
            mbar_init(bar_tempty + 8 * b, 2 * P_EPI_WARPS);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(tmem_slot), kTmemCols);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();            // both CTAs' barriers exist before anything arrives at them
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t stage = 0, phase = 0;
            const uint32_t bytes = 2u * (uint32_t)(P_A_BYTES + p.bn * BK);      // both CTAs: A, and half of bn rows of W
            bool alive = true;
            for (int tile = pair; tile < p.tiles && alive; tile += pairs) {
                const int m = (tile % p.tiles_m) * PM + 128 * (int)rank, n = (tile / p.tiles_m) * p.bn + (p.bn / 2) * (int)rank;
                for (int kb = 0; kb < p.nkb; kb++) {
                    if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag)) { alive = false; break; }
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * stage, bytes);
                    const uint32_t full = map_to_cta(bar_full + 8 * stage, 0), sa = tiles + stage * P_STAGE_BYTES;
                    tma_load_2d_pair(sa, &p.map_a, full, kb * BK, m);
                    tma_load_2d_pair(sa + P_A_BYTES, &p.map_w, full, kb * BK, n);
                    if (++stage == P_STAGES) { stage = 0; phase ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = make_idesc(PM, p.bn, false, false);
            uint32_t stage = 0, phase = 0, local = 0;
            bool alive = true;
            for (int tile = pair; tile < p.tiles && alive; tile += pairs, local++) {
                const uint32_t buf = local & 1u, use = local >> 1;
                if (!mbar_wait_cluster(bar_tempty + 8 * buf, (use & 1u) ^ 1u, abort_flag)) break;
                tc_fence_after();
                const uint32_t d = tmem + buf * PBN;
                for (int kb = 0; kb < p.nkb; kb++) {
                    if (!mbar_wait_cluster(bar_full + 8 * stage, phase, abort_flag)) { alive = false; break; }
                    tc_fence_after();
                    const uint32_t sa = tiles + stage * P_STAGE_BYTES;
                    const uint32_t a_lo = desc_lo(sa, 16u), b_lo = desc_lo(sa + P_A_BYTES, 16u);
#pragma unroll
                    for (int kk = 0; kk < BK / 16; kk++) umma_ss_pair(d, a_lo + kk * 2, b_lo + kk * 2, idesc, (uint32_t)(kb | kk));
                    umma_commit_pair(bar_empty + 8 * stage);
                    if (++stage == P_STAGES) { stage = 0; phase ^= 1u; }
                }
                if (alive) umma_commit_pair(bar_tfull + 8 * buf);
            }
        }
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;         // 32 rows; blocks of 32 columns half, half + 2, ...
        float *stage = staging + (warp - 2) * 1024;
        uint32_t local = 0;
        for (int tile = pair; tile < p.tiles; tile += pairs, local++) {
            const uint32_t buf = local & 1u, use = local >> 1;
            const int row0 = (tile % p.tiles_m) * PM + 128 * (int)rank + quarter * 32, n0 = (tile / p.tiles_m) * p.bn;
            const int row = row0 + lane;
            const uint32_t acc = tmem + buf * PBN + ((uint32_t)(quarter * 32) << 16);
            // blocks of whole groups of 8 columns; the residual of such a block is requested one block ahead (the first before
            // the products are done)
            auto groups = [&](int col0) { return p.vec && (col0 + 32 <= p.N || (p.N & 7) == 0); };
            uint4 rs[4];
            auto fetch = [&](int c) {
                const int col0 = n0 + c * 32;
                if (p.residual && groups(col0) && row < p.M && c < p.bn / 32) {
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        if (col0 + 8 * j < p.N) rs[j] = *reinterpret_cast<const uint4 *>(p.residual + (long long)row * p.ldr + col0 + 8 * j);
                }
            };
            fetch(half);
            if (!mbar_wait(bar_tfull + 8 * buf, use & 1u, abort_flag)) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = half; c < p.bn / 32; c += 2) {
                const int col0 = n0 + c * 32;
                if (col0 >= p.N || row0 >= p.M) break;                // uniform across the warp
                uint32_t r[32];
                tmem_ld32(acc + c * 32, r);
                if (groups(col0)) {
                    const uint4 now[4] = {rs[0], rs[1], rs[2], rs[3]};
                    fetch(c + 2);
                    finish_vec<ACT>(p, r, now, smem_u32(stage), lane, row0, col0);
                } else {
                    if (p.residual) finish_rows<ACT, true>(p, r, stage, lane, row0, col0);
                    else finish_rows<ACT, false>(p, r, stage, lane, row0, col0);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (rank == 0) mbar_arrive(bar_tempty + 8 * buf);
                else mbar_arrive_remote(map_to_cta(bar_tempty + 8 * buf, 0));
            }
        }
    }

    if (warp >= 2 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
    if (*abort_flag) {      // give copies that are still in flight time to land before shared memory is released
        const unsigned long long t0 = global_timer();
        while (global_timer() - t0 < 200000ull) { }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();            // neither CTA's shared or tensor memory goes away while the other may still reach it
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, kTmemCols);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// Few rows
// ---------------------------------------------------------------------------------------------------------------
constexpr int R_THREADS = 192;
template <int NP> struct Rows {                          // NP: rows of A per tile (the N side of the product)
    static constexpr int kA = NP * BK * 2, kStage = 128 * BK * 2 + kA;
    static constexpr int kStages = NP <= 32 ? 9 : (NP <= 64 ? 8 : 6);
    static constexpr int kSmem = kStages * kStage + 1024 + 256;
    static constexpr uint32_t kCols = NP < 32 ? 32 : NP;
    static_assert(kSmem <= 232448 && NP * 512 <= kStages * kStage, "stages hold the sums of a tile after the products");
};

// grid (n tiles x S, m tiles), clusters of S along x: CTA `rank` of a cluster sums its share of the K blocks
template <int ACT, int NP>
__global__ void __launch_bounds__(R_THREADS, 1) gemm_act_rows_kernel(const __grid_constant__ EpiParams p, int S) {
    pdl_enter();
    typedef Rows<NP> R;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t tiles = (raw + 1023u) & ~1023u;
    uint8_t *aux = smem_raw + (tiles - raw) + R::kStages * R::kStage;
    const uint32_t bar_full = smem_u32(aux), bar_empty = bar_full + 8 * R::kStages, bar_done = bar_empty + 8 * R::kStages;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(aux + 16 * R::kStages + 8);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(aux + 16 * R::kStages + 16);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = S == 1 ? 0 : (int)cluster_cta_rank();
    const int n0 = (int)(blockIdx.x / S) * 128, m0 = (int)blockIdx.y * NP;
    const int kb0 = (int)((long long)p.nkb * rank / S), kb1 = (int)((long long)p.nkb * (rank + 1) / S);

    if (threadIdx.x == 0) {
        for (int s = 0; s < R::kStages; s++) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, 1);
        }
        mbar_init(bar_done, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(tmem_slot), R::kCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t stage = 0, phase = 0;
            for (int kb = kb0; kb < kb1; kb++) {
                if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag)) break;
                const uint32_t full = bar_full + 8 * stage, s = tiles + stage * R::kStage;
                mbar_expect_tx(full, R::kStage);
                tma_load_2d(s, &p.map_w, full, kb * BK, n0);
                tma_load_2d(s + 128 * BK * 2, &p.map_a, full, kb * BK, m0);
                if (++stage == R::kStages) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = make_idesc(128, NP, false, false);
            uint32_t stage = 0, phase = 0;
            bool alive = true;
            for (int kb = kb0; kb < kb1; kb++) {
                if (!mbar_wait(bar_full + 8 * stage, phase, abort_flag)) { alive = false; break; }
                tc_fence_after();
                const uint32_t s = tiles + stage * R::kStage, w_lo = desc_lo(s, 16u), a_lo = desc_lo(s + 128 * BK * 2, 16u);
#pragma unroll
                for (int kk = 0; kk < BK / 16; kk++) umma_ss(tmem, w_lo + kk * 2, a_lo + kk * 2, idesc, (uint32_t)((kb - kb0) | kk));
                umma_commit(bar_empty + 8 * stage);
                if (++stage == R::kStages) { stage = 0; phase ^= 1u; }
            }
            if (alive) umma_commit(bar_done);
        }
    }
    // sums [NP rows][128 columns] of this CTA, in the operand stages (all products have read theirs)
    float *sums = reinterpret_cast<float *>(smem_raw + (tiles - raw));
    const int col_in = (warp & 3) * 32 + lane, col = n0 + col_in;
    const bool epi = warp >= 2;
    bool good = true;
    if (epi) {
        good = mbar_wait(bar_done, 0, abort_flag);
        if (good) {
            tc_fence_after();
            const uint32_t acc = tmem + ((uint32_t)((warp & 3) * 32) << 16);
#pragma unroll 1
            for (int c = 0; c < (int)R::kCols; c += 32) {
                uint32_t r[32];
                tmem_ld32(acc + c, r);
#pragma unroll
                for (int e = 0; e < 32; e++)
                    if (c + e < NP) sums[(c + e) * 128 + col_in] = __uint_as_float(r[e]);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (S > 1) cluster_sync_all();
    if (epi && !*abort_flag && col < p.N) {
        const float b = p.bias ? __bfloat162float(p.bias[col]) : 0.f;
        const uint32_t own = smem_u32(sums);
        // rows rank, rank + S, ... of the tile: the CTAs of a cluster share the work of the epilogue
        const int rows = p.M - m0 < NP ? p.M - m0 : NP;
#pragma unroll 1
        for (int i0 = rank; i0 < rows; i0 += 4 * S) {           // four rows' loads in flight
            float res[4], z[4];
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const int i = i0 + k * S < rows ? i0 + k * S : i0;
                res[k] = p.residual ? __bfloat162float(p.residual[(long long)(m0 + i) * p.ldr + col]) : 0.f;
                z[k] = S == 1 ? sums[i * 128 + col_in] : 0.f;
            }
            if (S > 1)
                for (int s = 0; s < S; s++) {
                    const uint32_t from = map_to_cta(own, (uint32_t)s) + (uint32_t)col_in * 4u;
#pragma unroll
                    for (int k = 0; k < 4; k++) z[k] += ld_cluster_f32(from + (uint32_t)(i0 + k * S < rows ? i0 + k * S : i0) * 512u);
                }
#pragma unroll
            for (int k = 0; k < 4; k++) {
                if (i0 + k * S >= rows) break;
                const long long row = m0 + i0 + k * S;
                z[k] += b;
                if (p.pre) p.pre[row * p.ldp + col] = __float2bfloat16_rn(z[k]);
                p.C[row * p.ldc + col] = __float2bfloat16_rn(activate<ACT, true>(z[k]) + res[k]);
            }
        }
    }
    __syncwarp();
    if (*abort_flag) {
        const unsigned long long t0 = global_timer();
        while (global_timer() - t0 < 200000ull) { }
    }
    __syncthreads();
    if (S > 1) cluster_sync_all();          // no CTA leaves while another may read its sums
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, R::kCols);
    }
}

template <int ACT, int NP>
int launch_rows(EpiParams p, const GemmEpilogue<bf16> &g, cudaStream_t st) {
    typedef Rows<NP> R;
    static PerDevice configured;
    if (!configured.get([] {
            return cuda_ok(cudaFuncSetAttribute(gemm_act_rows_kernel<ACT, NP>, cudaFuncAttributeMaxDynamicSharedMemorySize, R::kSmem)) ? 1 : 0;
        }))
        return STREAMBP_E_CUDA;
    if (!make_tensor_map(&p.map_a, g.A, g.M, g.K, g.lda, BK, NP, false) ||
        !make_tensor_map(&p.map_w, g.W, g.N, g.K, g.ldw, BK, 128, false))
        return STREAMBP_E_CUDA;
    const int64_t nt = (g.N + 127) / 128, mt = (g.M + NP - 1) / NP;
    if (mt > 65535) return STREAMBP_E_SHAPE;
    // as many CTAs to a cluster as the SMs allow, each with at least four K blocks to stream
    int S = 1;
    while (S < 8 && nt * mt * S * 2 <= sm_count() && p.nkb >= 8 * S) S *= 2;
    return launch_clusters(gemm_act_rows_kernel<ACT, NP>, dim3((unsigned)(nt * S), (unsigned)mt), R_THREADS, R::kSmem, S, 1, st, p, S);
}

// 32 x 32 blocks of a bf16 matrix, rows of 64 bytes swizzled in shared memory
bool make_store_map(CUtensorMap *map, const bf16 *base, int64_t rows, int64_t cols, int64_t ld) {
    return make_tensor_map(map, base, rows, cols, ld, 32, 32, false, CU_TENSOR_MAP_SWIZZLE_64B);
}

template <int ACT>
int launch_pair(EpiParams p, const GemmEpilogue<bf16> &g, cudaStream_t st) {
    static PerDevice configured;
    if (!configured.get([] {
            return cuda_ok(cudaFuncSetAttribute(gemm_act_pair_kernel<ACT>, cudaFuncAttributeMaxDynamicSharedMemorySize, P_SMEM)) ? 1 : 0;
        }))
        return STREAMBP_E_CUDA;
    const int pairs = sm_count() / 2 > 0 ? sm_count() / 2 : 1;
    p.tiles_m = (int)((g.M + PM - 1) / PM);
    // 256 columns a tile, or 224 where those need no more waves of pairs than the wider ones (each wave is then shorter:
    // 1500 x 5325 x 4096, two waves either way: 92 us against 98; the time of a wave falls by 2-6 %, so never for more waves)
    auto tiles_of = [&](int bn) { return (int64_t)p.tiles_m * ((g.N + bn - 1) / bn); };
    const int64_t wide = tiles_of(256), narrow = tiles_of(224);
    p.bn = wide > pairs && (narrow + pairs - 1) / pairs == (wide + pairs - 1) / pairs ? 224 : 256;
    const int64_t tiles = p.bn == 256 ? wide : narrow;
    if (tiles > (1ll << 30)) return STREAMBP_E_SHAPE;
    p.tiles = (int)tiles;
    if (!make_tensor_map(&p.map_a, g.A, g.M, g.K, g.lda, BK, 128, false) ||
        !make_tensor_map(&p.map_w, g.W, g.N, g.K, g.ldw, BK, (uint32_t)p.bn / 2, false))
        return STREAMBP_E_CUDA;
    if (p.vec && (!make_store_map(&p.map_c, g.C, g.M, g.N, g.ldc) || (g.pre && !make_store_map(&p.map_pre, g.pre, g.M, g.N, g.ldp))))
        return STREAMBP_E_CUDA;
    SBP_LAUNCH(gemm_act_pair_kernel<ACT>, 2 * (p.tiles < pairs ? p.tiles : pairs), P_THREADS, P_SMEM, st, p);
    return STREAMBP_OK;
}

template <int ACT>
int launch_any(const EpiParams &p, const GemmEpilogue<bf16> &g, cudaStream_t st) {
    // one tile of up to 128 rows: 4096 x 14336 with 128 rows takes 39 us against 82 by pairs, 1 row of 4096 x 4096 14 us
    // against 31; two tiles of 128 rows (256 x 4096 x 4096) take what one pair tile does
    if (gemm_tc_variant() == 2 && g.M > 128) return launch_pair<ACT>(p, g, st);
    if (g.M <= 16) return launch_rows<ACT, 16>(p, g, st);
    if (g.M <= 32) return launch_rows<ACT, 32>(p, g, st);
    if (g.M <= 64) return launch_rows<ACT, 64>(p, g, st);
    return launch_rows<ACT, 128>(p, g, st);
}

}  // namespace

bool gemm_tc_epilogue_supported(const GemmEpilogue<bf16> &g) {
    // the outputs are written by plain stores of any alignment: only the operands have rules
    return gemm_tc_supported(OP_NT, g.M, g.N, g.K, g.lda, g.ldw, 8, g.A, g.W, g.A, false);
}

int gemm_tc_epilogue(const GemmEpilogue<bf16> &g, cudaStream_t st) {
    if (!gemm_tc_epilogue_supported(g)) return STREAMBP_E_SHAPE;
    EpiParams p;
    memset(&p, 0, sizeof(p));
    p.M = (int)g.M;
    p.N = (int)g.N;
    p.nkb = (int)((g.K + BK - 1) / BK);
    p.bias = g.bias;
    p.residual = g.residual;
    p.C = g.C;
    p.pre = g.pre;
    p.ldr = g.ldr;
    p.ldc = g.ldc;
    p.ldp = g.ldp;
    auto rows16 = [](const void *q, int64_t ld) { return !q || ((reinterpret_cast<uintptr_t>(q) & 15u) == 0 && ld % 8 == 0); };
    p.vec = rows16(g.C, g.ldc) && rows16(g.residual, g.ldr) && rows16(g.pre, g.ldp) && rows16(g.bias, 8);
    switch (g.act) {
        case STREAMBP_ACT_NONE: return launch_any<STREAMBP_ACT_NONE>(p, g, st);
        case STREAMBP_ACT_RELU: return launch_any<STREAMBP_ACT_RELU>(p, g, st);
        case STREAMBP_ACT_GELU: return launch_any<STREAMBP_ACT_GELU>(p, g, st);
        case STREAMBP_ACT_GELU_TANH: return launch_any<STREAMBP_ACT_GELU_TANH>(p, g, st);
        case STREAMBP_ACT_SILU: return launch_any<STREAMBP_ACT_SILU>(p, g, st);
        default: return STREAMBP_E_SHAPE;
    }
}

int gemm_epilogue_take_fault() { return take_fault_local(); }

}  // namespace sbp
