// Linear layers in bf16 and fp16 (sparq_linear) for launches of few tiles or few rows: tokens that are decoded, small batches, experts
// with a few rows each.
//
// A tile is 128 rows of one operand (the MMA's M side, accumulator lanes) x BN rows of the other (columns).
//   SWAP     lanes are 128 columns of the output (rows of the weights), columns 16, 32 or 64 tokens: one token costs one pass over the weights and
//            16 columns of tensor memory, and a warp's store of one token's outputs is contiguous.
//   else     lanes are 128 tokens, columns 128 columns of the output.
//
// A cluster of `split` CTAs shares a tile where the tiles leave SMs idle: each takes an equal run of reduction steps and sends its
// partial sums to the CTA that owns a group of columns through distributed shared memory; the owner adds them in rank order, so that
// the result does not depend on timing.  Where there are more tiles than SMs, two CTAs share an SM, so that one's start and end run beside the other's
// copies.
//
// 1 x 4096 x 4096 bf16 8.6 us (weights 33.5 MB, 5.1 us of HBM), 250 x 1001 x 1000 9.3 (a chain: launch, first operands, four steps, sums over the
// cluster, rows that start anywhere), 8 rows of 7 of 16 experts, 2048 x 1408, 8.1 (40 MB, 6.2).
//
// Warps: 0 producer of x, the last of w, 1 tensor memory and MMA issue, the others epilogue (lane quarter warp % 4; of eight, every other
// group of columns).
#pragma once

#include "sparq_linear_kernel.cuh"

namespace sparq {

struct LinSmallArgs {
    LinArgs g;
    int stages, split;
};

__host__ __device__ constexpr int lin_small_epi(bool swap) { return swap ? 4 : 8; }
__host__ __device__ constexpr int lin_small_threads(bool swap) { return 32 * (3 + lin_small_epi(swap)); }
__host__ __device__ constexpr int lin_small_stage(int bn) { return (128 + bn) * kLinBK * 2; }
static_assert(lin_small_stage(128) >= 8 * kMxStaging, "the epilogue's staging memory lies where the ring was");
// Columns that change hands together (without SWAP a block of MXINT8); groups that each CTA of a cluster finishes; its room for their partial sums.
__host__ __device__ constexpr int lin_group(bool swap) { return swap ? 4 : 32; }
__host__ __device__ inline int lin_own_groups(int cols, int split, bool swap) { return ((cols + lin_group(swap) - 1) / lin_group(swap) + split - 1) / split; }
__host__ __device__ inline int lin_recv_bytes(int groups, int split, bool swap) { return split > 1 ? split * groups * lin_group(swap) * 128 * 4 : 0; }

// z of a warp's 32 neighbouring columns (n is the lane's) as one block of MXINT8.
__device__ __forceinline__ void lin_keep_across(const LinArgs &g, float z, int64_t row, int64_t n)
{
    const uint32_t mb = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(z) & 0x7FFFFFFFu), code = e8m0_code(mb, 0u);
    if ((n & ~INT64_C(31)) >= g.N) return;
    float f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = z;
    const uint4 w = int8_codes(f, code, mb);
    g.z_codes[row * g.z_pitch + n] = mb >= kInfBits ? 0 : (int8_t)(w.x & 0xFFu);
    if ((n & 31) == 0) {
        uint8_t *sc = g.z_scales + row * g.z_spitch + n / 32;
        *sc = (uint8_t)code;
        if (n + 32 >= g.N)
            for (int64_t c = n / 32 + 1; c < g.z_spitch; ++c) *++sc = 0;
    }
}

template <int BN, bool SWAP, bool W_KN, bool F32, bool KEEP>
struct LinSmall : MxCta {
    static constexpr int kEpi = lin_small_epi(SWAP), kGroup = lin_group(SWAP);
    static constexpr int kStage = lin_small_stage(BN), kLaneBytes = 128 * kLinBK * 2;
    static constexpr uint32_t kCols = tmem_columns(2 * BN);         // two accumulators, for sums in pieces
    uint32_t recv;
    int64_t m0, end;            // first row and end of the expert's
    int e, n0, rows, cols, kb_first, own, own_valid;

    template <bool X>
    __device__ void produce(const CUtensorMap &map, const LinArgs &g) const
    {
        if (lane == 0) {
            if (X) dep_launch();
            constexpr bool kLanes = X != SWAP;
            constexpr uint32_t kBytes = kLanes ? kLaneBytes : BN * kLinBK * 2;
            int it = 0, s = 0;
            uint32_t ph = 1;
            for (; it < steps; ++it) {
                if (it >= S && !mbar_wait(empty_bar(s), ph, abort_flag, g.status, g.wait_limit)) break;
                const uint32_t full = full_bar(s), at = smem + (uint32_t)(s * kStage) + (kLanes ? 0u : (uint32_t)kLaneBytes);
                const int k = (kb_first + it) * kLinBK;
                mbar_expect_tx(full, kBytes);
                if (X) {
                    tma_load_2d(at, &map, full, k, (int)m0);
                } else if (W_KN) {
                    tma_load_3d(at, &map, full, n0, k, e);
                    tma_load_3d(at + kBytes / 2, &map, full, n0 + 64, k, e);
                } else {
                    tma_load_3d(at, &map, full, k, n0, e);
                }
                if (++s == S) { s = 0; ph ^= 1u; }
            }
            issued[X ? 0 : 1] = (uint32_t)it;
        }
        __syncwarp();
    }

    __device__ void issue(const LinArgs &g) const
    {
        constexpr bool kRowsMn = SWAP && W_KN, kColsMn = !SWAP && W_KN;
        const uint32_t elected = elect_one(), id = make_idesc_16(BN, 128, (uint32_t)g.bf16, kRowsMn, kColsMn);
        int s = 0, n = 0, in = 0;           // piece, and its steps; piece n adds up in accumulator n & 1
        uint32_t ph = 0;
        bool live = true;
        for (int it = 0; it < steps; ++it, ++in) {
            if (in == g.piece) {
                tc_commit_if(acc_bar(n & 1), elected);
                ++n;
                in = 0;
                if (n > 1) live = mbar_wait_warp(elected, freed_bar(n & 1), (uint32_t)((n >> 1) - 1) & 1u, abort_flag, g.status, g.wait_limit);
                if (!live) break;
            }
            if (!mbar_wait_warp(elected, full_bar(s), ph, abort_flag, g.status, g.wait_limit)) { live = false; break; }
            tc_fence_after();
            const uint32_t at = smem + (uint32_t)(s * kStage);
            const int mmas = g.k_mmas - (kb_first + it) * kLinSteps;
            const uint64_t rdesc = kRowsMn ? mn_major_desc(at, kLaneBytes / 2) : make_smem_desc<128>(at);
            const uint64_t cdesc = kColsMn ? mn_major_desc(at + kLaneBytes, kLaneBytes / 2) : make_smem_desc<128>(at + kLaneBytes);
#pragma unroll
            for (int k = 0; k < kLinSteps; ++k) {
                if (k >= mmas) continue;
                tc_mma_bf16(tmem + (uint32_t)((n & 1) * BN), rdesc + (uint64_t)(k * (kRowsMn ? 128 : 2)), cdesc + (uint64_t)(k * (kColsMn ? 128 : 2)), id, (in > 0 || k > 0) ? 1u : 0u, elected);
            }
            tc_commit_if(empty_bar(s), elected);
            if (++s == S) { s = 0; ph ^= 1u; }
        }
        tc_commit_if(acc_bar(n & 1), elected);
        mbar_wait(acc_bar(n & 1), (uint32_t)(n >> 1) & 1u, abort_flag, g.status, g.wait_limit, true);
        if (!live && lane == 0) drain_two(full_bar(0), (uint32_t)S, issued, abort_flag, g.status, g.wait_limit);
        __syncwarp();
    }

    // kGroup columns of this lane from `col` on; a warp's lanes call it together.  SWAP: the outputs of kGroup tokens; else a block of a row.
    __device__ void put(const LinArgs &g, int col, const float (&acc)[kGroup], float lane_bias) const
    {
        const int r = (warp & 3) * 32 + lane;
        if constexpr (SWAP) {
            const int count = cols - col < kGroup ? cols - col : kGroup;
            const int64_t n = n0 + r, first = m0 + col;
            const bool live = r < rows;
            float y[kGroup], res[kGroup];
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                y[j] = g.bias ? __fadd_rn(acc[j], lane_bias) : acc[j];
                res[j] = 0.0f;
                if (g.residual && live && j < count) {
                    const int64_t at = (first + j) * g.ldr + n;
                    if (F32) {
                        res[j] = reinterpret_cast<const float *>(g.residual)[at];
                    } else {
                        const uint32_t h = reinterpret_cast<const uint16_t *>(g.residual)[at];
                        float lo = __uint_as_float(h << 16), hi;
                        if (!g.bf16) floats_of_f16x2(h, lo, hi);
                        res[j] = lo;
                    }
                }
            }
            if (KEEP) {
#pragma unroll
                for (int j = 0; j < kGroup; ++j)
                    if (j < count) lin_keep_across(g, y[j], first + j, n);
            }
            lin_act<!F32, false>(y, g.act);
#pragma unroll
            for (int j = 0; j < kGroup; ++j) {
                if (g.residual) y[j] = __fadd_rn(y[j], res[j]);
                if (!live || j >= count) continue;
                const int64_t at = (first + j) * g.ldo + n;
                if (F32) reinterpret_cast<float *>(g.out)[at] = y[j];
                else reinterpret_cast<uint16_t *>(g.out)[at] = (uint16_t)(g.bf16 ? bf16x2_of(y[j], 0.0f) : f16x2_of(y[j], 0.0f));
            }
        } else {
            const int64_t n = n0 + col, m = m0 + (warp & 3) * 32;
            const int live = end - m < 0 ? 0 : end - m < 32 ? (int)(end - m) : 32, count = cols - col < 32 ? cols - col : 32;
            const uint32_t stage = smem + (uint32_t)((warp - 2) * kMxStaging);        // the ring is free, its last MMA has read it
            uint32_t v[32];
            float y[32];
            LinFetch<F32> fetch;
            const float bias = lin_bias(g, e, n);
            if (g.residual) fetch.issue(g, m, live, n, n + count);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(acc[j]);
            uint32_t scale = 0u;
            lin_value<F32, KEEP>(g, y, v, bias, m0 + r, r < rows, n, scale);
            if (KEEP && r < rows) lin_keep_scales<1>(g, scale, m0 + r, n);
            __syncwarp();
            if (g.residual) fetch.land(stage);
            if (F32) lin_stage_f32(g, y, stage);
            else if (g.bf16) lin_stage_row<true>(g, y, stage, 0);
            else lin_stage_row<false>(g, y, stage, 0);
            constexpr int width = F32 ? 4 : 2;
            lin_flush_rows<F32>(reinterpret_cast<uint8_t *>(g.out) + (m * g.ldo + n) * width, g.ldo * width, stage, live, count * width);
        }
    }

    // Sums in several pieces, of the columns that the warp reads in finish(): back into the first accumulator, whence they are taken as one piece is.  (No third one for them: where CTAs of several launches share an
    // SM, one would wait for tensor memory while its cluster waits for it, and may wait for another cluster that waits likewise.)
    __device__ __forceinline__ void add_pieces(const LinArgs &g, uint32_t taddr, int half) const
    {
        constexpr int C = SWAP ? BN : 64;
        float sum[C];
        int n = 0;
        auto at = [&](int b, int h) { return taddr + (uint32_t)(b * BN + h + (SWAP ? 0 : split == 1 ? half * 64 : half * 32 + (h & 32))); };
        lin_add_pieces(*this, g, (steps + g.piece - 1) / g.piece, n, sum, at, [&](int b) { mbar_arrive(freed_bar(b)); });
#pragma unroll
        for (int h = 0; h < C; h += 16) {
            uint4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float *s = sum + h + 4 * j;
                v[j] = make_uint4(__float_as_uint(s[0]), __float_as_uint(s[1]), __float_as_uint(s[2]), __float_as_uint(s[3]));
            }
            tmem_st_32x16(at(0, h), v);
        }
        tmem_st_wait();
    }

    __device__ void finish(const CUtensorMap &map, const LinArgs &g) const
    {
        const int quarter = warp & 3, half = (warp - 2) >> 2, r = quarter * 32 + lane;
        const float lane_bias = SWAP && g.bias && r < rows ? __ldg(g.bias + e * g.N + n0 + r) : 0.0f;
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16);
        if (steps > g.piece) {
            add_pieces(g, taddr, half);
        } else {
            mbar_wait(acc_bar(), 0, abort_flag, g.status, g.wait_limit);
            tc_fence_after();
        }
        if (split > 1) {
            __syncwarp();
            cluster_wait();        // every CTA of the cluster has its barriers ready
        }
        if constexpr (!SWAP) {
            if (split == 1) {       // 64 columns to a warp; the ring is free, its last MMA has read it
                if (half * 64 < cols) {
                    const int64_t m = m0 + quarter * 32, n = n0 + half * 64;
                    const int live = end - m < 0 ? 0 : end - m < 32 ? (int)(end - m) : 32;
                    LinFetch<F32> fetch;
                    if (g.residual && !F32) fetch.issue(g, m, live, n, g.N);
                    uint32_t scales = 0u;
                    lin_put_span<F32, KEEP>(map, g, smem + (uint32_t)((warp - 2) * kMxStaging), m, live, end == g.M, n, lin_bias(g, e, n), lin_bias(g, e, n + 32), fetch, scales,
                                            [&](int h, uint32_t(&v)[32]) {
                                                tmem_ld_32x32_issue(taddr + half * 64 + h * 32, v);
                                                tmem_ld_wait();
                                            });
                    if (KEEP && lane < live) lin_keep_scales<2>(g, scales, m + lane, n);
                    if (lane == 0) tma_store_wait_all();
                    __syncwarp();
                }
                tc_fence_before();
                return;
            }
        }
        // partial sums: per rank and group, 16-byte pieces of all lanes one after the other
        auto piece = [&](int from, int local, int q) { return recv + (uint32_t)((((from * own + local) * (kGroup / 4) + q) * 128 + r) * 16); };
        if (SWAP && split == 1) {
#pragma unroll 1
            for (int c = 0; c < cols; c += 4) {
                uint32_t v[4];
                tmem_ld_32x4_issue(taddr + c, v);
                tmem_ld_wait();
                float a[kGroup];
#pragma unroll
                for (int j = 0; j < kGroup; ++j) a[j] = __uint_as_float(v[j % 4]);
                put(g, c, a, lane_bias);
            }
            tc_fence_before();
            return;
        }
        constexpr int kAtOnce = SWAP ? 16 : 32;       // columns of a turn
#pragma unroll 1
        for (int c = half * kAtOnce; c < cols; c += kEpi / 4 * kAtOnce) {
            uint32_t v[32];
            if constexpr (SWAP) tmem_ld_32x16_issue(taddr + c, v);
            else tmem_ld_32x32_issue(taddr + c, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < kAtOnce / kGroup; ++i) {
                const int col = c + kGroup * i;
                if (col >= cols || r >= rows) continue;
                const int grp = col / kGroup, owner = grp / own, local = grp - owner * own;
                const uint32_t bar = map_to_rank(recv_bar(), owner);
#pragma unroll
                for (int q = 0; q < kGroup / 4; ++q) {
                    const int at = kGroup * i + 4 * q;
                    store_remote16(map_to_rank(piece(rank, local, q), owner), bar, v[at], v[at + 1], v[at + 2], v[at + 3]);
                }
            }
            __syncwarp();
        }
        if (split > 1) {
            mbar_wait(recv_bar(), 0, abort_flag, g.status, g.wait_limit);
            __syncwarp();
#pragma unroll 1
            for (int local = half; local < own_valid; local += kEpi / 4) {
                float a[kGroup];
#pragma unroll
                for (int j = 0; j < kGroup; ++j) a[j] = 0.0f;
                if (r < rows) {
#pragma unroll 2
                    for (int from = 0; from < (int)split; ++from)
#pragma unroll
                        for (int q = 0; q < kGroup / 4; ++q) {
                            uint32_t p[4];
                            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(p[0]), "=r"(p[1]), "=r"(p[2]), "=r"(p[3]) : "r"(piece(from, local, q)));
#pragma unroll
                            for (int j = 0; j < 4; ++j) a[4 * q + j] = __fadd_rn(a[4 * q + j], __uint_as_float(p[j]));
                        }
                }
                __syncwarp();
                put(g, (rank * own + local) * kGroup, a, lane_bias);
            }
        }
        tc_fence_before();
    }
};

template <int BN, bool SWAP, bool W_KN, bool F32, bool KEEP>
__global__ void __launch_bounds__(lin_small_threads(SWAP), SWAP ? 2 : 1)
sparq_linear_small_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_out,
                          const LinSmallArgs p)
{
    using Cta = LinSmall<BN, SWAP, W_KN, F32, KEEP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) MxBars bars;
    __shared__ uint32_t tmem_base_slot;
    __shared__ uint32_t abort_word;
    __shared__ volatile uint32_t issued[2];

    const LinArgs &g = p.g;
    Cta c;
    const int warp = c.warp = threadIdx.x >> 5, lane = c.lane = threadIdx.x & 31;
    c.abort_flag = &abort_word;
    c.issued = issued;
    c.S = p.stages;
    c.smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    c.bars = smem_u32(&bars);
    c.recv = c.smem + (uint32_t)(c.S * Cta::kStage);
    const uint32_t split = c.split = (uint32_t)p.split, at = blockIdx.x / split;
    c.rank = (int)(blockIdx.x - at * split);
    c.kb_first = (int)((int64_t)c.rank * g.k_blocks / split);
    c.steps = (int)((int64_t)(c.rank + 1) * g.k_blocks / split) - c.kb_first;

    if (warp == 0) {
        if (lane == 0) {
            prefetch_tensormap(&map_x);
            prefetch_tensormap(&map_w);
            for (int s = 0; s < c.S; ++s) {
                mbar_init(c.full_bar(s), 2);
                mbar_init(c.empty_bar(s), 1);
            }
            for (int b = 0; b < 2; ++b) {
                mbar_init(c.acc_bar(b), 1);
                mbar_init(c.freed_bar(b), Cta::kEpi);
            }
            mbar_init(c.recv_bar(), 1);
            abort_word = 0;
            issued[0] = issued[1] = kStillIssuing;
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
    dep_wait();
    // The tile; a cluster behind the last one has nothing to do.
    LinTile tile;
    LinWalk<SWAP ? BN : 128> walk(g, lane);
    if (walk.find(at, tile)) {
        c.e = tile.e;
        c.m0 = tile.m0;
        c.end = tile.end;
        c.n0 = tile.nt * 128;
        const int tokens = tile.end - tile.m0 < (SWAP ? BN : 128) ? (int)(tile.end - tile.m0) : (SWAP ? BN : 128);
        const int outputs = g.N - c.n0 < 128 ? (int)(g.N - c.n0) : 128;
        c.rows = SWAP ? outputs : tokens;
        c.cols = SWAP ? tokens : outputs;
        const int groups = (c.cols + Cta::kGroup - 1) / Cta::kGroup;
        c.own = lin_own_groups(c.cols, (int)split, SWAP);
        const int rest = groups - c.rank * c.own;
        c.own_valid = rest < 0 ? 0 : rest < c.own ? rest : c.own;
        if (split > 1) {
            if (threadIdx.x == 0) mbar_expect_tx(c.recv_bar(), split * (uint32_t)(c.own_valid * c.rows) * (Cta::kGroup * 4));
            __syncwarp();
            cluster_arrive();       // "barriers ready": waited for before the first remote store
        }
        constexpr int kLast = 2 + Cta::kEpi;
        switch (warp) {
        case 0: c.template produce<true>(map_x, g); break;
        case 1: c.issue(g); break;
        case kLast: c.template produce<false>(map_w, g); break;
        default: c.finish(map_out, g);
        }
        if (split > 1 && (warp < 2 || warp == kLast)) {
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
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(c.tmem), "r"(Cta::kCols) : "memory");
    }
}

}  // namespace sparq
