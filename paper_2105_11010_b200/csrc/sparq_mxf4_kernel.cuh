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
// 16384 x 4096 x 4096 NVFP4 to bf16 109 us call after call, 127 with L2 emptied in between; 8192 x 8192 x 8192 201 us, 5.5 PFLOP/s, 0.84
// of four times cuBLAS's bf16 rate in a burst.  What bounds it is the way from L2 to the SMs: 8192 x 4096 x 4096 takes in 638 MB of
// operands (29 MB of them from HBM) in 57 us, 11 TB/s or 7 KB a cycle, with the tensor pipe 62 % active; and the power cap.
//
// Warps: 0 producer of the codes, 10 of the scales, 1 tensor memory and (leader) MMA issue, 2..9 epilogue (lane quarter warp % 4, two spans of 64 columns).
#pragma once

#include "sparq_mxf4_small_kernel.cuh"

namespace sparq {

constexpr int kPairTile = 256;
constexpr int kPairEpiWarps = 8;
constexpr int kPairScaleWarp = 2 + kPairEpiWarps;
constexpr int kPairThreads = 32 * (kPairScaleWarp + 1);
constexpr uint32_t kPairSecond = 208;           // first column of the odd tiles' accumulator
constexpr uint32_t kPairScales = 464;           // first column of the scales

__host__ __device__ constexpr int pair_stage(bool nv) { return 2 * 128 * kMxBK + 3 * scale_tiles(nv) * kScaleTile; }
// Stages start on 1024-byte boundaries.
__host__ __device__ constexpr int pair_stage_room(bool nv) { return (pair_stage(nv) + 1023) / 1024 * 1024; }
__host__ __device__ constexpr int pair_stages(bool nv) { return (232448 - 1024 - 512 - kPairEpiWarps * kMxStaging) / pair_stage_room(nv); }
__host__ __device__ constexpr int pair_smem(bool nv) { return 1024 + pair_stages(nv) * pair_stage_room(nv) + kPairEpiWarps * kMxStaging; }

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

    // Two producers, one for the codes and one for the scales, on the same barriers: one thread that issued all four copies of a
    // step took longer than the step's MMAs (16 pairs, K 32768: 0.36 us a step, 0.28 without the scales' copies).
    template <bool CODES>
    __device__ void produce(const CUtensorMap &map_a, const CUtensorMap &map_b, const MxPairArgs &p) const
    {
        if (lane == 0) {
            if (CODES) dep_launch();
            const MxGemmArgs &g = p.g;
            const uint32_t leader_full = map_to_rank(full_bar(0), 0);
            int s = 0;
            uint32_t ph = 1, n = 0;
            bool live = true;
            for (int t = pair; t < tiles && live; t += p.pairs) {
                int mt, nt;
                pair_tile(p, t, mt, nt);
                const int a_row = mt * kPairTile + rank * 128, b_row = nt * kPairTile + rank * 128;
                for (int kb = 0; kb < g.k_blocks; ++kb) {
                    if (n >= kStages && !mbar_wait(empty_bar(s), ph, abort_flag, g.status, g.wait_limit)) { live = false; break; }
                    const uint32_t at = smem + (uint32_t)(s * kRoom), bar = leader_full + 8u * (uint32_t)s;
                    if (CODES) {
                        if (rank == 0) mbar_expect_tx(full_bar(s), 2 * kBytes);
                        tma_load_pair_2d(at, &map_a, bar, kb * kMxBK, a_row);
                        tma_load_pair_2d(at + kHalf, &map_b, bar, kb * kMxBK, b_row);
                    } else {
                        tma_load_pair_3d(at + kScalesAt, &map_a, bar, 0, kb * T, mt * 2 + rank);
                        tma_load_pair_3d(at + kScalesAt + T * kScaleTile, &map_b, bar, 0, kb * T, nt * 2);
                    }
                    ++n;
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
            store_remote(map_to_rank(smem_u32((const void *)(issued + 2 * rank + (CODES ? 0 : 1))), 0), n);
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
            bool live = true;
            for (int t = pair; t < tiles && live; t += p.pairs, ++i) {
                const uint32_t d = tmem + (i & 1) * kPairSecond;
                if (i > 0) live = mbar_wait_warp(elected, freed_bar(0), (uint32_t)(i - 1) & 1u, abort_flag, g.status, g.wait_limit);
                if (!live) break;
                for (int kb = 0; kb < g.k_blocks; ++kb) {
                    live = mbar_wait_warp(elected, full_bar(s), ph, abort_flag, g.status, g.wait_limit);
                    if (!live) {
                        tc_commit_pair(acc_bar(i & 1), elected);        // what there is of the tile
                        break;
                    }
                    tc_fence_after();
                    const uint32_t at = smem + (uint32_t)(s * kRoom), sf = at + kScalesAt, ta = tmem + kPairScales, tb = ta + 4 * T;
                    const uint64_t adesc = make_smem_desc<kMxBK>(at), bdesc = make_smem_desc<kMxBK>(at + kHalf);
                    const int mmas = g.k_mmas - kb * kMxSteps;
#pragma unroll
                    for (int k = 0; k < kMxSteps; ++k) {
                        if (k >= mmas) continue;
                        const int q = NV ? k : k >> 1;
                        if (NV || (k & 1) == 0) {
                            tc_copy_scales_pair(ta + 4 * q, scale_desc(sf + q * kScaleTile), elected);
                            tc_copy_scales_pair(tb + 8 * q, scale_desc(sf + (T + q) * kScaleTile), elected);
                            tc_copy_scales_pair(tb + 8 * q + 4, scale_desc(sf + (2 * T + q) * kScaleTile), elected);
                        }
                        tc_mma_f4_pair<NV>(d, adesc + (uint64_t)(k * 2), bdesc + (uint64_t)(k * 2), make_idesc_f4(kPairTile, 256, NV, NV ? 0u : (k & 1) * 2u),
                                           ta + 4 * q, tb + 8 * q, (kb > 0 || k > 0) ? 1u : 0u, elected);
                    }
                    tc_commit_pair(empty_bar(s), elected);
                    if (kb == g.k_blocks - 1) tc_commit_pair(acc_bar(i & 1), elected);
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
            // every MMA has retired before the warp goes on
            if (i > 0) mbar_wait(acc_bar((i - 1) & 1), (uint32_t)((i - 1) >> 1) & 1u, abort_flag, g.status, g.wait_limit, true);
            if (!live && lane == 0) {
                store_remote(map_to_rank(smem_u32((const void *)abort_flag), 1), 1u);        // the other CTA's producers stop, too
                drain_pair(full_bar(0), kStages, issued, 2 * kHalf, 3 * T * kScaleTile, abort_flag, g.status, g.wait_limit);
            }
        }
        __syncwarp();
    }

    __device__ void finish(const CUtensorMap &map_f, const CUtensorMap &map_h, const MxPairArgs &p) const
    {
        const MxGemmArgs &g = p.g;
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const float alpha = mx_alpha(g);
        const uint32_t freed = map_to_rank(freed_bar(0), 0);
        int i = 0;
        for (int t = pair; t < tiles; t += p.pairs, ++i) {
            int mt, nt;
            pair_tile(p, t, mt, nt);
            const int64_t m0 = (int64_t)mt * kPairTile + rank * 128 + quarter * 32, n0 = (int64_t)nt * kPairTile;
            mbar_wait(acc_bar(i & 1), (uint32_t)(i >> 1) & 1u, abort_flag, g.status, g.wait_limit);
            tc_fence_after();
            const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (i & 1) * kPairSecond;
            // Spans of 64 columns, two for each half of the warps.  The one that holds the columns which the next tile's accumulator
            // shares comes first: 3 of the even tiles, 0 of the odd ones.
            const int first = (i & 1) ? 2 * half : 3 - 2 * half, second = (i & 1) ? first + 1 : first - 1;
#pragma unroll 1
            for (int q = 0; q < 2; ++q) {
                const int span = q ? second : first;
                uint32_t v[2][32];
                tmem_ld_32x32_issue(taddr + span * 64, v[0]);
                tmem_ld_32x32_issue(taddr + span * 64 + 32, v[1]);
                tmem_ld_wait();
                if (q == 0) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_remote(freed);
                }
                mx_put_span(map_f, map_h, g, v, smem + (uint32_t)(kStages * kRoom + (warp - 2) * kMxStaging), m0, n0 + span * 64, alpha);
            }
        }
        if (lane == 0) tma_store_wait_all();
        __syncwarp();
        tc_fence_before();
    }
};

template <bool NV>
__global__ void __launch_bounds__(kPairThreads)
sparq_mxf4_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_sa,
                  const __grid_constant__ CUtensorMap map_sb, const __grid_constant__ CUtensorMap map_f, const __grid_constant__ CUtensorMap map_h,
                  const MxPairArgs p)
{
    using Cta = Mxf4Pair<NV>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) MxBars bars;
    __shared__ uint32_t tmem_base_slot;
    __shared__ uint32_t abort_word;
    __shared__ volatile uint32_t issued[4];

    Cta c;
    const int warp = c.warp = threadIdx.x >> 5, lane = c.lane = threadIdx.x & 31;
    c.abort_flag = &abort_word;
    c.issued = issued;
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
            for (int q = 0; q < 4; ++q) issued[q] = kStillIssuing;
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
    case 0: c.template produce<true>(map_a, map_b, p); break;
    case 1: c.issue(p); break;
    case kPairScaleWarp: c.template produce<false>(map_sa, map_sb, p); break;
    default: c.finish(map_f, map_h, p);
    }
    // Neither CTA leaves, or gives its tensor memory back, while the pair's MMAs, the other's arrivals or a copy may reach it.
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
