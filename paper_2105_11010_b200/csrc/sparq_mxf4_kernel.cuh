// Products of 4-bit microscaled operands (sparq_gemm_mxf4), large: out[m][n] = sum_k A[m][k] B[n][k].
//
// A persistent pair of CTAs walks tiles of 256 x 256: one MMA (cta_group::2) multiplies 256 rows of A by 256 of B, each CTA
// holds half of either operand's rows and its 128 rows of the accumulator.  A step of 64 elements takes the tensor cores
// 128 cycles, in which each SM's shared memory takes in 8 KB and gives 8 KB of operands: all of its bandwidth.  One CTA by
// itself (128 x 256) would need half as much again.
//
// Scales: each CTA brings those of its 128 rows of A and of all 256 rows of B, as tiles that one tcgen05.cp lays into
// tensor memory in front of the MMAs that use them.
//
// Tensor memory: 464 columns of accumulators, 48 of scales.  Two accumulators of 256 columns do not fit, so they share 48
// columns: the epilogue empties those first (columns 208..255), and the next tile's first MMA waits for no more than that.
//
// Warps: 0 producer, 1 tensor memory and (leader) MMA issue, 2..9 epilogue (lane quarter warp % 4, every second run of 16
// columns).
#pragma once

#include "sparq_mxf4_small_kernel.cuh"

namespace sparq {

constexpr int kPairTile = 256;
constexpr int kPairThreads = 320;
constexpr int kPairEpiWarps = 8;
constexpr uint32_t kPairSecond = 208;           // first column of the odd tiles' accumulator
constexpr uint32_t kPairScales = 464;           // first column of the scales

__host__ __device__ constexpr int pair_stage(bool nv) { return 2 * 128 * kMxBK + 3 * scale_tiles(nv) * kScaleTile; }
// Stages start on 1024-byte boundaries.
__host__ __device__ constexpr int pair_stage_room(bool nv) { return (pair_stage(nv) + 1023) / 1024 * 1024; }
__host__ __device__ constexpr int pair_stages(bool nv) { return (232448 - 4096) / pair_stage_room(nv) < kMaxStages ? (232448 - 4096) / pair_stage_room(nv) : kMaxStages; }

struct MxPairArgs {
    MxGemmArgs g;
    int m_tiles, n_tiles, pairs;
};

// Tile t in an order that keeps eight rows of tiles together: their operands and the column's stay in L2.
__device__ __forceinline__ void pair_tile(const MxPairArgs &p, int t, int &mt, int &nt)
{
    const int per_group = 8 * p.n_tiles, group = t / per_group, first = group * 8;
    const int rows = p.m_tiles - first < 8 ? p.m_tiles - first : 8, in = t - group * per_group;
    nt = in / rows;
    mt = first + in - nt * rows;
}

template <bool NV>
struct Mxf4Pair : MxCta {
    static constexpr int T = scale_tiles(NV), kHalf = 128 * kMxBK, kScalesAt = 2 * kHalf;
    static constexpr int kBytes = pair_stage(NV), kRoom = pair_stage_room(NV), kStages = pair_stages(NV);
    int tiles, pair;

    __device__ void produce(const CUtensorMap &map_a, const CUtensorMap &map_b, const CUtensorMap &map_sa, const CUtensorMap &map_sb, const MxPairArgs &p) const
    {
        if (lane == 0) {
            dep_launch();
            const MxGemmArgs &g = p.g;
            int s = 0, used = 0;
            uint32_t ph = 1;
            bool live = true;
            for (int t = pair; t < tiles && live; t += p.pairs) {
                int mt, nt;
                pair_tile(p, t, mt, nt);
                const int a_row = mt * kPairTile + rank * 128, b_row = nt * kPairTile + rank * 128;
                const int a_tile = (mt * 2 + rank) * g.scale_tiles, b_tile = nt * 2 * g.scale_tiles;
                for (int kb = 0; kb < g.k_blocks; ++kb) {
                    if (used >= kStages && !mbar_wait(empty_bar(s), ph, abort_flag, g.status, g.wait_limit)) { live = false; break; }
                    const uint32_t at = smem + (uint32_t)(s * kRoom), bar = map_to_rank(full_bar(s), 0);
                    if (rank == 0) mbar_expect_tx(full_bar(s), 2 * kBytes);
                    tma_load_pair_2d(at, &map_a, bar, kb * kMxBK, a_row);
                    tma_load_pair_2d(at + kHalf, &map_b, bar, kb * kMxBK, b_row);
                    tma_load_pair_2d(at + kScalesAt, &map_sa, bar, 0, a_tile + kb * T);
                    tma_load_pair_2d(at + kScalesAt + T * kScaleTile, &map_sb, bar, 0, b_tile + kb * T);
                    tma_load_pair_2d(at + kScalesAt + 2 * T * kScaleTile, &map_sb, bar, 0, b_tile + g.scale_tiles + kb * T);
                    if (used < kStages) ++used;
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
            // After a wait that gave up no copy may land when the CTAs have left: the leader waits for what both announced, the
            // other CTA for the leader at the cluster's barrier.
            if (*abort_flag && rank == 0) {
                for (int j = 0; j < used; ++j) {
                    const int q = s - 1 - j < 0 ? s - 1 - j + kStages : s - 1 - j;
                    // ph is flipped whenever the ring starts over: the parity of the last phase announced on stage q
                    mbar_wait(full_bar(q), q < s ? ph ^ 1u : ph, abort_flag, g.status, g.wait_limit, true);
                }
            }
        }
        __syncwarp();
    }

    __device__ void issue(const MxPairArgs &p) const
    {
        if (rank == 0) {
            const MxGemmArgs &g = p.g;
            const uint32_t elected = elect_one();
            int s = 0, i = 0;
            uint32_t ph = 0;
            for (int t = pair; t < tiles; t += p.pairs, ++i) {
                const uint32_t d = tmem + (i & 1) * kPairSecond;
                if (i > 0) mbar_wait(freed_bar(0), (uint32_t)(i - 1) & 1u, abort_flag, g.status, g.wait_limit);
                for (int kb = 0; kb < g.k_blocks; ++kb) {
                    mbar_wait(full_bar(s), ph, abort_flag, g.status, g.wait_limit);
                    tc_fence_after();
                    if (elected) {
                        const uint32_t at = smem + (uint32_t)(s * kRoom), sf = at + kScalesAt, ta = tmem + kPairScales, tb = ta + 4 * T;
                        const uint64_t adesc = make_smem_desc<kMxBK>(at), bdesc = make_smem_desc<kMxBK>(at + kHalf);
                        const int mmas = g.k_mmas - kb * kMxSteps;
#pragma unroll
                        for (int k = 0; k < kMxSteps; ++k) {
                            if (k >= mmas) continue;
                            const int q = NV ? k : k >> 1;
                            if (NV || (k & 1) == 0) {
                                tc_copy_scales_pair(ta + 4 * q, scale_desc(sf + q * kScaleTile));
                                tc_copy_scales_pair(tb + 8 * q, scale_desc(sf + (T + q) * kScaleTile));
                                tc_copy_scales_pair(tb + 8 * q + 4, scale_desc(sf + (2 * T + q) * kScaleTile));
                            }
                            tc_mma_f4_pair<NV>(d, adesc + (uint64_t)(k * 2), bdesc + (uint64_t)(k * 2), make_idesc_f4(kPairTile, 256, NV, NV ? 0u : (k & 1) * 2u),
                                               ta + 4 * q, tb + 8 * q, (kb > 0 || k > 0) ? 1u : 0u);
                        }
                        tc_commit_pair(empty_bar(s));
                        if (kb == g.k_blocks - 1) tc_commit_pair(acc_bar(i & 1));
                    }
                    __syncwarp();
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
            // every MMA has retired before the warp goes on
            if (i > 0) mbar_wait(acc_bar((i - 1) & 1), (uint32_t)((i - 1) >> 1) & 1u, abort_flag, g.status, g.wait_limit, true);
        }
        __syncwarp();
    }

    // 16 columns of a row.  WHOLE: all of them exist, outputs and bias on 32-byte boundaries.
    template <bool WHOLE>
    __device__ void put(const MxGemmArgs &g, const uint32_t *v, int64_t m, int64_t n, float alpha) const
    {
        if (m >= g.M || (!WHOLE && n >= g.N)) return;
        const int cols = WHOLE || g.N - n >= 16 ? 16 : (int)(g.N - n);
        float y[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = __fmul_rn(__uint_as_float(v[j]), alpha);
        if (g.bias) {
            float b[16];
            load_run<false, WHOLE ? 32 : 0>(b, g.bias + n, cols);
#pragma unroll
            for (int j = 0; j < 16; ++j) y[j] = __fadd_rn(y[j], b[j]);
        }
        if (g.relu) {
#pragma unroll
            for (int j = 0; j < 16; ++j) y[j] = y[j] > 0.0f ? y[j] : 0.0f;
        }
        const int64_t at = m * g.N + n;
        if (g.f32_out) store_run<false, WHOLE ? 32 : 0>(g.f32_out + at, y, cols);
        if (g.bf16_out) store_run<true, WHOLE ? 32 : 0>(g.bf16_out + at, y, cols);
    }

    __device__ void finish(const MxPairArgs &p) const
    {
        const MxGemmArgs &g = p.g;
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const float alpha = mx_alpha(g);
        const bool aligned = (g.N & (g.bf16_out ? 15 : 7)) == 0 &&
                             ((reinterpret_cast<uintptr_t>(g.f32_out) | reinterpret_cast<uintptr_t>(g.bf16_out) | reinterpret_cast<uintptr_t>(g.bias)) & 31u) == 0;
        const uint32_t freed = map_to_rank(freed_bar(0), 0);
        int i = 0;
        for (int t = pair; t < tiles; t += p.pairs, ++i) {
            int mt, nt;
            pair_tile(p, t, mt, nt);
            const int64_t m = (int64_t)mt * kPairTile + rank * 128 + quarter * 32 + lane, n0 = (int64_t)nt * kPairTile;
            mbar_wait(acc_bar(i & 1), (uint32_t)(i >> 1) & 1u, abort_flag, g.status, g.wait_limit);
            tc_fence_after();
            const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (i & 1) * kPairSecond;
            const bool whole = aligned && n0 + kPairTile <= g.N;
            // run r of 16 columns; the ones that the next tile's accumulator shares come first: 13, 14, 15 of the even tiles, 0, 1, 2 of the odd
            auto run_of = [&](int q) { return (i & 1) ? q : q < 3 ? 13 + q : q - 3; };
#pragma unroll 1
            for (int q = half; q < 16; q += 4) {
                const int ra = run_of(q), rb = run_of(q + 2);
                uint32_t va[32], vb[32];
                tmem_ld_32x16_issue(taddr + ra * 16, va);
                tmem_ld_32x16_issue(taddr + rb * 16, vb);
                tmem_ld_wait();
                if (q == half) {            // both of this warp's runs among the first three are in registers
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_remote(freed);
                }
                if (whole) {
                    put<true>(g, va, m, n0 + ra * 16, alpha);
                    put<true>(g, vb, m, n0 + rb * 16, alpha);
                } else {
                    put<false>(g, va, m, n0 + ra * 16, alpha);
                    put<false>(g, vb, m, n0 + rb * 16, alpha);
                }
            }
        }
        tc_fence_before();
    }
};

template <bool NV>
__global__ void __launch_bounds__(kPairThreads)
sparq_mxf4_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_sa,
                  const __grid_constant__ CUtensorMap map_sb, const MxPairArgs p)
{
    using Cta = Mxf4Pair<NV>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) MxBars bars;
    __shared__ uint32_t tmem_base_slot;
    __shared__ uint32_t abort_word;

    Cta c;
    const int warp = c.warp = threadIdx.x >> 5, lane = c.lane = threadIdx.x & 31;
    c.abort_flag = &abort_word;
    c.smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    c.bars = smem_u32(&bars);
    c.rank = (int)(blockIdx.x & 1u);
    c.pair = (int)(blockIdx.x >> 1);
    c.tiles = p.m_tiles * p.n_tiles;

    if (warp == 0) {
        if (lane == 0) {
            prefetch_tensormap(&map_a);
            prefetch_tensormap(&map_b);
            prefetch_tensormap(&map_sa);
            prefetch_tensormap(&map_sb);
            for (int s = 0; s < Cta::kStages; ++s) {
                mbar_init(c.full_bar(s), 1);
                mbar_init(c.empty_bar(s), 1);
            }
            mbar_init(c.acc_bar(0), 1);
            mbar_init(c.acc_bar(1), 1);
            mbar_init(c.freed_bar(0), 2 * kPairEpiWarps);
            abort_word = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    } else if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&tmem_base_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive();          // both CTAs have their barriers and their tensor memory
    cluster_wait();
    tc_fence_after();
    c.tmem = tmem_base_slot;
    dep_wait();
    switch (warp) {
    case 0: c.produce(map_a, map_b, map_sa, map_sb, p); break;
    case 1: c.issue(p); break;
    default: c.finish(p);
    }
    // Neither CTA leaves, or gives its tensor memory back, while the pair's MMAs or the other's arrivals may reach it.
    tc_fence_before();
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(c.tmem), "r"(512u) : "memory");
    }
}

}  // namespace sparq
