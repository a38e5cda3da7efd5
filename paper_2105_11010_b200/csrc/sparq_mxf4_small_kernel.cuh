// Products of 4-bit microscaled operands (sparq_gemm_mxf4) for few rows: tokens that are decoded, small batches.
//
//   out[m][n] = sum_k A[m][k] B[n][k]
//
// A tile is 128 rows of B (a layer's weights) x BN rows of A (tokens): the weights take the MMA's 128-row side, so that one
// token costs one pass over the weights and BN = 16 columns of tensor memory.  Lane l of the accumulator is output column n0 + l, and
// a warp's store of one token's outputs is contiguous.
//
// A cluster of `split` CTAs shares a tile where the tiles leave SMs idle: each takes an equal run of reduction
// steps and sends its partial sums to the CTA that owns a token (groups of four) through distributed shared memory;
// the owner adds them in rank order, so that the result does not depend on timing.
//
// Warps: 0 producer, 1 tensor memory and MMA issue, 2..5 epilogue (lane quarter warp % 4).
#pragma once

#include "sparq_mx_tc.cuh"

namespace sparq {

struct MxGemmArgs {
    int64_t M, N;               // tokens, output columns
    int k_mmas, k_blocks;       // reduction steps of 64 and of 256 elements
    int scale_tiles;            // tiles of a row block's scales in memory
    const uint8_t *a_scales, *b_scales;
    const float *a_max, *b_max; // NVFP4
    const float *bias;
    int relu;
    float *f32_out;
    uint16_t *bf16_out;
    unsigned int *status;
    long long wait_limit;
    int stages, split;
};

constexpr int kMxSmallThreads = 192;

__device__ __forceinline__ float mx_alpha(const MxGemmArgs &g)
{
    if (!g.a_max) return 1.0f;
    return __fmul_rn(__fdiv_rn(nvfp4_largest(__ldg(g.a_max)), 2688.0f), __fdiv_rn(nvfp4_largest(__ldg(g.b_max)), 2688.0f));
}

__device__ __forceinline__ float mx_finish(float acc, float alpha, float bias, int relu)
{
    float y = __fadd_rn(__fmul_rn(acc, alpha), bias);
    if (relu) y = y > 0.0f ? y : 0.0f;
    return y;
}

__host__ __device__ constexpr int mx_small_stage(int bn, bool nv) { return (128 + bn) * kMxBK + (1 + (bn + 127) / 128) * scale_tiles(nv) * kScaleTile; }
// Groups of four tokens that each CTA of a cluster finishes, and its room for their partial sums.
__host__ __device__ inline int mx_own_groups(int64_t tokens, int split) { return (int)((tokens + 3) / 4 + split - 1) / split; }
__host__ __device__ inline int mx_recv_bytes(int groups, int split) { return split > 1 ? split * groups * 128 * 16 : 0; }

template <int BN, bool NV>
struct Mxf4Small : MxCta {
    static constexpr int T = scale_tiles(NV), kABlocks = (BN + 127) / 128;
    static constexpr int kStage = mx_small_stage(BN, NV), kWeights = 128 * kMxBK, kTokens = BN * kMxBK;
    static constexpr uint32_t kColsB = BN, kColsA = BN + 4 * T;       // columns of the scales, behind the accumulator's
    static constexpr uint32_t kCols = tmem_columns(BN + 4 * T + 4 * T * kABlocks);
    uint32_t recv, nt;
    int64_t n0, m0;
    int tokens, kb_first, groups, own, own_valid;

    __device__ void produce(const CUtensorMap &map_b, const CUtensorMap &map_a, const MxGemmArgs &g) const
    {
        if (lane == 0) {
            dep_launch();
            const int64_t b_row = (int64_t)nt * g.scale_tiles * kScaleTile;
            const int64_t a_row = m0 / 128 * g.scale_tiles * kScaleTile;
            const int a_blocks = kABlocks == 2 && tokens > 128 ? 2 : 1;
            int it = 0, s = 0;
            uint32_t ph = 1;
            for (; it < steps; ++it) {
                if (it >= S && !mbar_wait(empty_bar(s), ph, abort_flag, g.status, g.wait_limit)) break;
                const uint32_t full = full_bar(s), at = smem + (uint32_t)(s * kStage);
                const int kb = kb_first + it, t0 = kb * T;
                const uint32_t sf = (uint32_t)(g.scale_tiles - t0 < T ? g.scale_tiles - t0 : T) * kScaleTile;
                mbar_expect_tx(full, kWeights + kTokens + sf * (1 + a_blocks));
                tma_load_2d(at, &map_b, full, kb * kMxBK, (int)n0);
                tma_load_2d(at + kWeights, &map_a, full, kb * kMxBK, (int)m0);
                tma_load_bytes(at + kWeights + kTokens, g.b_scales + b_row + (int64_t)t0 * kScaleTile, sf, full);
                for (int b = 0; b < a_blocks; ++b)
                    tma_load_bytes(at + kWeights + kTokens + (uint32_t)((1 + b) * T * kScaleTile),
                                   g.a_scales + a_row + ((int64_t)b * g.scale_tiles + t0) * kScaleTile, sf, full);
                if (++s == S) { s = 0; ph ^= 1u; }
            }
            if (*abort_flag)       // none of this thread's copies may land after the CTA has exited
                for (int j = it > S ? it - S : 0; j < it; ++j)
                    mbar_wait(full_bar(j % S), (uint32_t)(j / S) & 1u, abort_flag, g.status, g.wait_limit, true);
        }
        __syncwarp();
    }

    __device__ void issue(const MxGemmArgs &g) const
    {
        const uint32_t elected = elect_one();
        int s = 0;
        uint32_t ph = 0;
        for (int it = 0; it < steps; ++it) {
            mbar_wait(full_bar(s), ph, abort_flag, g.status, g.wait_limit);
            tc_fence_after();
            if (elected) {
                const uint32_t at = smem + (uint32_t)(s * kStage), sf = at + kWeights + kTokens;
                const int kb = kb_first + it, mmas = g.k_mmas - kb * kMxSteps < kMxSteps ? g.k_mmas - kb * kMxSteps : kMxSteps;
                const uint64_t bdesc = make_smem_desc<kMxBK>(at), adesc = make_smem_desc<kMxBK>(at + kWeights);
#pragma unroll
                for (int k = 0; k < kMxSteps; ++k) {
                    if (k >= mmas) continue;
                    const int t = NV ? k : k >> 1;
                    if (NV || (k & 1) == 0) {
                        tc_copy_scales(tmem + kColsB + 4 * t, scale_desc(sf + t * kScaleTile));
#pragma unroll
                        for (int b = 0; b < kABlocks; ++b)
                            tc_copy_scales(tmem + kColsA + 4 * (kABlocks * t + b), scale_desc(sf + ((1 + b) * T + t) * kScaleTile));
                    }
                    const uint32_t id = make_idesc_f4(BN, 128, NV, NV ? 0u : (k & 1) * 2u);
                    tc_mma_f4<NV>(tmem, bdesc + (uint64_t)(k * 2), adesc + (uint64_t)(k * 2), id, tmem + kColsB + 4 * t,
                                  tmem + kColsA + 4 * kABlocks * t, (it > 0 || k > 0) ? 1u : 0u);
                }
                tc_commit(empty_bar(s));
            }
            __syncwarp();
            if (++s == S) { s = 0; ph ^= 1u; }
        }
        if (elected) tc_commit(acc_bar());
        __syncwarp();
        mbar_wait(acc_bar(), 0, abort_flag, g.status, g.wait_limit, true);
        __syncwarp();
    }

    __device__ void finish(const MxGemmArgs &g) const
    {
        const int quarter = warp & 3;
        const int64_t n = n0 + quarter * 32 + lane;
        const bool live = n < g.N;
        const float alpha = mx_alpha(g), bias = g.bias && live ? __ldg(g.bias + n) : 0.0f;
        auto put = [&](int token, float acc) {
            if (!live) return;
            const float y = mx_finish(acc, alpha, bias, g.relu);
            const int64_t at = (m0 + token) * g.N + n;
            if (g.f32_out) g.f32_out[at] = y;
            if (g.bf16_out) g.bf16_out[at] = (uint16_t)bf16x2_of(y, 0.0f);
        };
        mbar_wait(acc_bar(), 0, abort_flag, g.status, g.wait_limit);
        tc_fence_after();
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16);
        constexpr int kChunk = BN < 32 ? 16 : 32;
        if (split > 1) {
            __syncwarp();
            cluster_wait();        // every CTA of the cluster has its barriers ready
        }
#pragma unroll 1
        for (int c0 = 0; c0 < tokens; c0 += kChunk) {
            uint32_t v[32];
            if (kChunk == 32) tmem_ld_32x32_issue(taddr + c0, v);
            else tmem_ld_32x16_issue(taddr + c0, v);
            tmem_ld_wait();
            if (split == 1) {
#pragma unroll
                for (int j = 0; j < kChunk; ++j)
                    if (c0 + j < tokens) put(c0 + j, __uint_as_float(v[j]));
            } else {
#pragma unroll
                for (int q = 0; q < kChunk / 4; ++q) {
                    const int grp = c0 / 4 + q;
                    if (grp >= groups) continue;
                    const int owner = grp / own, local = grp - owner * own;
                    const uint32_t dst = recv + (uint32_t)(((rank * own + local) * 128 + quarter * 32 + lane) * 16);
                    store_remote16(map_to_rank(dst, owner), map_to_rank(recv_bar(), owner), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                }
            }
        }
        if (split > 1) {
            mbar_wait(recv_bar(), 0, abort_flag, g.status, g.wait_limit);
            for (int local = 0; local < own_valid; ++local) {
                float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                for (uint32_t q = 0; q < split; ++q) {
                    uint4 p;
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(p.x), "=r"(p.y), "=r"(p.z), "=r"(p.w)
                                 : "r"(recv + (uint32_t)((((int)q * own + local) * 128 + quarter * 32 + lane) * 16)));
                    a[0] += __uint_as_float(p.x);
                    a[1] += __uint_as_float(p.y);
                    a[2] += __uint_as_float(p.z);
                    a[3] += __uint_as_float(p.w);
                }
                const int token = (rank * own + local) * 4;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (token + j < tokens) put(token + j, a[j]);
            }
        }
        tc_fence_before();
    }
};

template <int BN, bool NV>
__global__ void __launch_bounds__(kMxSmallThreads)
sparq_mxf4_small_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a, const MxGemmArgs g)
{
    using Cta = Mxf4Small<BN, NV>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) MxBars bars;
    __shared__ uint32_t tmem_base_slot;
    __shared__ uint32_t abort_word;

    Cta c;
    const int warp = c.warp = threadIdx.x >> 5, lane = c.lane = threadIdx.x & 31;
    c.abort_flag = &abort_word;
    c.S = g.stages;
    c.smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    c.bars = smem_u32(&bars);
    c.recv = c.smem + (uint32_t)(c.S * Cta::kStage);
    const uint32_t split = c.split = (uint32_t)g.split, tile = blockIdx.x / split;
    c.rank = (int)(blockIdx.x - tile * split);
    const uint32_t n_tiles = (uint32_t)((g.N + 127) / 128), mt = tile / n_tiles;
    c.nt = tile - mt * n_tiles;
    c.n0 = (int64_t)c.nt * 128;
    c.m0 = (int64_t)mt * BN;
    c.tokens = g.M - c.m0 < BN ? (int)(g.M - c.m0) : BN;
    c.kb_first = (int)((int64_t)c.rank * g.k_blocks / split);
    c.steps = (int)((int64_t)(c.rank + 1) * g.k_blocks / split) - c.kb_first;
    c.groups = (c.tokens + 3) / 4;
    c.own = mx_own_groups(c.tokens, (int)split);
    const int rest = c.groups - c.rank * c.own;
    c.own_valid = rest < 0 ? 0 : rest < c.own ? rest : c.own;

    if (warp == 0) {
        if (lane == 0) {
            prefetch_tensormap(&map_b);
            prefetch_tensormap(&map_a);
            for (int s = 0; s < c.S; ++s) {
                mbar_init(c.full_bar(s), 1);
                mbar_init(c.empty_bar(s), 1);
            }
            mbar_init(c.acc_bar(), 1);
            mbar_init(c.recv_bar(), 1);
            abort_word = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    } else if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&tmem_base_slot)), "r"(Cta::kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    c.tmem = tmem_base_slot;
    if (split > 1) {
        if (threadIdx.x == 0) mbar_expect_tx(c.recv_bar(), split * (uint32_t)c.own_valid * (128 * 16));
        __syncwarp();
        cluster_arrive();       // "barriers ready": waited for before the first remote store
    }
    dep_wait();
    switch (warp) {
    case 0: c.produce(map_b, map_a, g); break;
    case 1: c.issue(g); break;
    default: c.finish(g);
    }
    if (split > 1 && warp < 2) {
        __syncwarp();
        cluster_wait();            // matches the arrival above
    }
    __syncthreads();
    // No CTA leaves while a peer may still write to its shared memory.  In a normal run its barrier has counted every byte
    // by now; after a wait that gave up it stays until every other CTA has sent its rows, and those have landed.
    if (split > 1 && *c.abort_flag) {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        mx_wait_landed(c, g.status, g.wait_limit);
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(c.tmem), "r"(Cta::kCols) : "memory");
    }
}

}  // namespace sparq
