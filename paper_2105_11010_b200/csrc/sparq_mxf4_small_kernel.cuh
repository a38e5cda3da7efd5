// Products of 4-bit microscaled operands (sparq_gemm_mxf4) for launches whose tiles all run at once: tokens that are decoded, small
// batches.
//
//   out[m][n] = sum_k A[m][k] B[n][k]
//
// A tile is 128 rows of one operand (the MMA's M side, accumulator lanes) x BN rows of the other (columns).
//   SWAP     lanes are rows of B (a layer's weights), columns 16 or 32 rows of A: one token costs one pass over the weights and
//            16 columns of tensor memory, and a warp's store of one token's outputs is contiguous.  1 x 8192 x 8192 NVFP4 7.8 us,
//            4.8 TB/s of weights; 1 x 16384 x 8192 11.9, 6.3 TB/s.
//   else     lanes are rows of A, columns 128 rows of B: a lane holds runs of an output row, stored 32 bytes at a time.
//            (64 tokens as columns: 64 x 2048, K 512, 4.8 us, 128 tokens 7.2, most of it two-byte stores.)
//
// A cluster of `split` CTAs shares a tile where the tiles leave SMs idle: each takes an equal run of reduction steps
// and sends its partial sums to the CTA that owns a group of columns through distributed shared memory; the owner adds
// them in rank order, so that the result does not depend on timing.
//
// Warps: 0 and the last producers (of either operand: one thread that issues all four copies of a step takes 0.35 us for it), 1 tensor
// memory and MMA issue, the others epilogue (lane quarter warp % 4; of eight, every other 16 columns).
#pragma once

#include "sparq_mx_tc.cuh"

namespace sparq {

struct MxGemmArgs {
    int64_t M, N;               // rows of A and of B
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
    int staged;                 // outputs go out through shared memory, in boxes: their rows start on 16-byte boundaries
};

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

// 32 columns of an output row from their accumulators.
__device__ __forceinline__ void mx_finish_row(const MxGemmArgs &g, float (&y)[32], const uint32_t (&v)[32], int64_t n, float alpha)
{
#pragma unroll
    for (int j = 0; j < 32; ++j) y[j] = __fmul_rn(__uint_as_float(v[j]), alpha);
    if (g.bias) {
        if (n + 32 <= g.N && (reinterpret_cast<uintptr_t>(g.bias + n) & 15u) == 0) {
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 b = __ldg(reinterpret_cast<const float4 *>(g.bias + n + j));
                y[j] = __fadd_rn(y[j], b.x);
                y[j + 1] = __fadd_rn(y[j + 1], b.y);
                y[j + 2] = __fadd_rn(y[j + 2], b.z);
                y[j + 3] = __fadd_rn(y[j + 3], b.w);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) y[j] = __fadd_rn(y[j], n + j < g.N ? __ldg(g.bias + n + j) : 0.0f);
        }
    }
    if (g.relu) {
#pragma unroll
        for (int j = 0; j < 32; ++j) y[j] = y[j] > 0.0f ? y[j] : 0.0f;
    }
}

// 32 rows x 128 bytes of one output through a warp's staging memory (rows of 128 bytes, swizzled as TMA does).  Rows of 32 lanes
// stored straight from registers are 32 lines to an instruction: 128 x 512, K 512, 5.3 us.
constexpr int kMxStaging = 32 * 128;
__device__ __forceinline__ void mx_stage_row(const uint32_t (&w)[32], uint32_t stage)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" :: "r"(stage + (uint32_t)(lane * 128 + ((j ^ (lane & 7)) << 4))), "r"(w[4 * j]),
                     "r"(w[4 * j + 1]), "r"(w[4 * j + 2]), "r"(w[4 * j + 3]) : "memory");
}
__device__ __forceinline__ void mx_store_box(const CUtensorMap &map, const uint32_t (&w)[32], uint32_t stage, int64_t m, int64_t n, const MxGemmArgs &g)
{
    const int lane = threadIdx.x & 31;
    if (lane == 0) tma_store_wait_read<0>();        // the box before has left
    __syncwarp();
    mx_stage_row(w, stage);
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0 && m < g.M && n < g.N) {
        tma_store_2d(&map, stage, (int)n, (int)m);
        tma_store_commit();
    }
}
// The same for rows that TMA cannot address (odd lengths): the warp stores one row after the other, lane by lane.
template <bool BF16>
__device__ __forceinline__ void mx_store_rows(void *out, const uint32_t (&w)[32], uint32_t stage, int64_t m, int64_t n, const MxGemmArgs &g)
{
    const int lane = threadIdx.x & 31, col = BF16 ? 2 * lane : lane;
    __syncwarp();
    mx_stage_row(w, stage);
    __syncwarp();
    const int rows = g.M - m < 32 ? (int)(g.M - m) : 32, cols = g.N - n - col < 2 ? (int)(g.N - n - col) : 2;
    const uint32_t src = stage + (uint32_t)((lane & 3) * 4);
    const int64_t at = m * g.N + n + col;
    if (BF16) {
        uint16_t *h = reinterpret_cast<uint16_t *>(out) + at;
        const bool pairs = (g.N & 1) == 0 && (reinterpret_cast<uintptr_t>(h) & 3u) == 0;
#pragma unroll 4
        for (int r = 0; r < rows; ++r, h += g.N) {
            uint32_t v;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(src + (uint32_t)(r * 128 + (((lane >> 2) ^ (r & 7)) << 4))));
            if (cols == 2 && pairs) {
                *reinterpret_cast<uint32_t *>(h) = v;
            } else {
                if (cols > 0) h[0] = (uint16_t)v;
                if (cols > 1) h[1] = (uint16_t)(v >> 16);
            }
        }
    } else {
        uint32_t *f = reinterpret_cast<uint32_t *>(out) + at;
#pragma unroll 4
        for (int r = 0; r < rows; ++r, f += g.N) {
            uint32_t v;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(src + (uint32_t)(r * 128 + (((lane >> 2) ^ (r & 7)) << 4))));
            if (cols > 0) *f = v;
        }
    }
}

// 64 columns of a warp's 32 rows: row m0 + lane, columns n .. n + 63 from v.
__device__ __forceinline__ void mx_put_span(const CUtensorMap &map_f, const CUtensorMap &map_h, const MxGemmArgs &g, const uint32_t (&v)[2][32],
                                            uint32_t stage, int64_t m0, int64_t n, float alpha)
{
    uint32_t h[32];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float y[32];
        mx_finish_row(g, y, v[q], n + 32 * q, alpha);
        if (g.f32_out) {
            uint32_t f[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) f[j] = __float_as_uint(y[j]);
            if (g.staged) mx_store_box(map_f, f, stage, m0, n + 32 * q, g);
            else mx_store_rows<false>(g.f32_out, f, stage, m0, n + 32 * q, g);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) h[16 * q + j] = bf16x2_of(y[2 * j], y[2 * j + 1]);
    }
    if (g.bf16_out) {
        if (g.staged) mx_store_box(map_h, h, stage, m0, n, g);
        else mx_store_rows<true>(g.bf16_out, h, stage, m0, n, g);
    }
}

__host__ __device__ constexpr int mx_small_epi(bool swap) { return swap ? 4 : 8; }
__host__ __device__ constexpr int mx_small_threads(bool swap) { return 32 * (3 + mx_small_epi(swap)); }
__host__ __device__ constexpr int mx_small_stage(int bn, bool nv) { return (128 + bn) * kMxBK + 2 * scale_tiles(nv) * kScaleTile; }
// Columns that change hands together; groups that each CTA of a cluster finishes of a tile with `cols` columns, and its room
// for their partial sums.
__host__ __device__ constexpr int mx_group(bool swap) { return swap ? 4 : 16; }
__host__ __device__ inline int mx_own_groups(int64_t cols, int split, bool swap) { return ((int)((cols + mx_group(swap) - 1) / mx_group(swap)) + split - 1) / split; }
__host__ __device__ inline int mx_recv_bytes(int groups, int split, bool swap) { return split > 1 ? split * groups * mx_group(swap) * 128 * 4 : 0; }

template <int BN, bool NV, bool SWAP>
struct Mxf4Small : MxCta {
    static constexpr int kEpi = mx_small_epi(SWAP), T = scale_tiles(NV), kGroup = mx_group(SWAP);
    static constexpr int kStage = mx_small_stage(BN, NV), kRows = 128 * kMxBK, kScalesAt = (128 + BN) * kMxBK;
    static constexpr uint32_t kColsR = BN, kColsC = BN + 4 * T;       // columns of the scales, behind the accumulator's
    static constexpr uint32_t kCols = tmem_columns(BN + 8 * T);
    uint32_t recv;
    int64_t r0, c0;             // first row of either operand
    int rows, cols, kb_first, groups, own, own_valid;

    // The codes of one operand's rows and their scales (of whole blocks of 128 rows).
    template <bool LANES>
    __device__ void produce(const CUtensorMap &map, const uint8_t *scales, const MxGemmArgs &g) const
    {
        if (lane == 0) {
            if (LANES) dep_launch();
            const int row = (int)(LANES ? r0 : c0);
            const uint8_t *src = scales + (int64_t)(row / 128) * g.scale_tiles * kScaleTile;
            int it = 0, s = 0;
            uint32_t ph = 1;
            for (; it < steps; ++it) {
                if (it >= S && !mbar_wait(empty_bar(s), ph, abort_flag, g.status, g.wait_limit)) break;
                const uint32_t full = full_bar(s), at = smem + (uint32_t)(s * kStage);
                const int kb = kb_first + it, t0 = kb * T;
                const uint32_t sf = (uint32_t)(g.scale_tiles - t0 < T ? g.scale_tiles - t0 : T) * kScaleTile;
                mbar_expect_tx(full, (LANES ? kRows : BN * kMxBK) + sf);
                tma_load_2d(at + (LANES ? 0 : kRows), &map, full, kb * kMxBK, row);
                tma_load_bytes(at + kScalesAt + (LANES ? 0 : T * kScaleTile), src + (int64_t)t0 * kScaleTile, sf, full);
                if (++s == S) { s = 0; ph ^= 1u; }
            }
            issued[LANES ? 0 : 1] = (uint32_t)it;
        }
        __syncwarp();
    }

    __device__ void issue(const MxGemmArgs &g) const
    {
        const uint32_t elected = elect_one();
        int s = 0;
        uint32_t ph = 0;
        bool live = true;
        for (int it = 0; it < steps; ++it) {
            if (!mbar_wait_warp(elected, full_bar(s), ph, abort_flag, g.status, g.wait_limit)) { live = false; break; }
            tc_fence_after();
            const uint32_t at = smem + (uint32_t)(s * kStage), sf = at + kScalesAt;
            const int mmas = g.k_mmas - (kb_first + it) * kMxSteps;
            const uint64_t rdesc = make_smem_desc<kMxBK>(at), cdesc = make_smem_desc<kMxBK>(at + kRows);
#pragma unroll
            for (int k = 0; k < kMxSteps; ++k) {
                if (k >= mmas) continue;
                const int t = NV ? k : k >> 1;
                if (NV || (k & 1) == 0) {
                    tc_copy_scales(tmem + kColsR + 4 * t, scale_desc(sf + t * kScaleTile), elected);
                    tc_copy_scales(tmem + kColsC + 4 * t, scale_desc(sf + (T + t) * kScaleTile), elected);
                }
                tc_mma_f4<NV>(tmem, rdesc + (uint64_t)(k * 2), cdesc + (uint64_t)(k * 2), make_idesc_f4(BN, 128, NV, NV ? 0u : (k & 1) * 2u),
                              tmem + kColsR + 4 * t, tmem + kColsC + 4 * t, (it > 0 || k > 0) ? 1u : 0u, elected);
            }
            tc_commit_if(empty_bar(s), elected);
            if (++s == S) { s = 0; ph ^= 1u; }
        }
        tc_commit_if(acc_bar(), elected);
        mbar_wait(acc_bar(), 0, abort_flag, g.status, g.wait_limit, true);
        if (!live && lane == 0) drain_two(full_bar(0), (uint32_t)S, issued, abort_flag, g.status, g.wait_limit);
        __syncwarp();
    }

    // kGroup columns of this lane from `col` on.  SWAP: the outputs of kGroup tokens, in columns of `out`; else a run of a row.
    __device__ void put(const MxGemmArgs &g, int col, const float (&acc)[kGroup], float alpha, float lane_bias) const
    {
        const int r = (warp & 3) * 32 + lane;
        if (r >= rows) return;
        const int count = cols - col < kGroup ? cols - col : kGroup;
        float y[kGroup];
        if (SWAP) {
#pragma unroll
            for (int j = 0; j < kGroup; ++j) y[j] = mx_finish(acc[j], alpha, lane_bias, g.relu);
            const int64_t at = (c0 + col) * g.N + r0 + r;
            if (g.f32_out) {
                float *f = g.f32_out + at;
#pragma unroll
                for (int j = 0; j < kGroup; ++j, f += g.N)
                    if (j < count) *f = y[j];
            }
            if (g.bf16_out) {
                uint16_t *h = g.bf16_out + at;
#pragma unroll
                for (int j = 0; j < kGroup; ++j, h += g.N)
                    if (j < count) *h = (uint16_t)bf16x2_of(y[j], 0.0f);
            }
            return;
        }
        const int64_t n = c0 + col, at = (r0 + r) * g.N + n;
#pragma unroll
        for (int j = 0; j < kGroup; ++j) y[j] = mx_finish(acc[j], alpha, g.bias && j < count ? __ldg(g.bias + n + j) : 0.0f, g.relu);
        if (g.f32_out) store_row<false>(g.f32_out + at, y, count);
        if (g.bf16_out) store_row<true>(g.bf16_out + at, y, count);
    }

    template <bool BF16>
    __device__ void store_row(void *out, const float (&y)[kGroup], int count) const
    {
        constexpr int W = BF16 ? kGroup / 2 : kGroup;
        uint32_t v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = BF16 ? bf16x2_of(y[2 * i % kGroup], y[(2 * i + 1) % kGroup]) : __float_as_uint(y[i]);
        uint8_t *b = reinterpret_cast<uint8_t *>(out);
        const uint32_t low = (uint32_t)reinterpret_cast<uintptr_t>(b);
        if (count == kGroup && (low & 31u) == 0) {
#pragma unroll
            for (int i = 0; i < W; i += 8) st_v8(b + 4 * i, v + i);
        } else if (count == kGroup && (low & 15u) == 0) {
#pragma unroll
            for (int i = 0; i < W; i += 4) st_v4(b + 4 * i, v + i);
        } else {
#pragma unroll
            for (int i = 0; i < kGroup; ++i) {
                if (i >= count) continue;
                if (BF16) reinterpret_cast<uint16_t *>(b)[i] = (uint16_t)(v[i / 2 % W] >> (16 * (i & 1)));
                else reinterpret_cast<uint32_t *>(b)[i] = v[i % W];
            }
        }
    }

    __device__ void finish(const CUtensorMap &map_f, const CUtensorMap &map_h, const MxGemmArgs &g) const
    {
        const int quarter = warp & 3, half = (warp - 2) >> 2, r = quarter * 32 + lane;
        const float alpha = mx_alpha(g), lane_bias = SWAP && g.bias && r < rows ? __ldg(g.bias + r0 + r) : 0.0f;
        mbar_wait(acc_bar(), 0, abort_flag, g.status, g.wait_limit);
        tc_fence_after();
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16);
        if (split > 1) {
            __syncwarp();
            cluster_wait();        // every CTA of the cluster has its barriers ready
        }
        if (!SWAP && split == 1) {     // 64 columns to a warp; the ring is free, its last MMA has read it
            if (half * 64 < cols) {
                uint32_t v[2][32];
                tmem_ld_32x32_issue(taddr + half * 64, v[0]);
                tmem_ld_32x32_issue(taddr + half * 64 + 32, v[1]);
                tmem_ld_wait();
                mx_put_span(map_f, map_h, g, v, smem + (uint32_t)((warp - 2) * kMxStaging), r0 + quarter * 32, c0 + half * 64, alpha);
                if (lane == 0) tma_store_wait_all();
                __syncwarp();
            }
            tc_fence_before();
            return;
        }
        // partial sums: per rank and group, 16-byte pieces of all lanes one after the other
        auto piece = [&](int from, int local, int q) { return recv + (uint32_t)((((from * own + local) * (kGroup / 4) + q) * 128 + r) * 16); };
#pragma unroll 1
        for (int c = half * 16; c < cols; c += kEpi / 4 * 16) {
            uint32_t v[32];
            tmem_ld_32x16_issue(taddr + c, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16 / kGroup; ++i) {
                const int col = c + kGroup * i;
                if (col >= cols) continue;
                if (split == 1) {
                    float a[kGroup];
#pragma unroll
                    for (int j = 0; j < kGroup; ++j) a[j] = __uint_as_float(v[kGroup * i + j]);
                    put(g, col, a, alpha, lane_bias);
                } else if (r < rows) {
                    const int grp = col / kGroup, owner = grp / own, local = grp - owner * own;
                    const uint32_t bar = map_to_rank(recv_bar(), owner);
#pragma unroll
                    for (int q = 0; q < kGroup / 4; ++q) {
                        const int e = kGroup * i + 4 * q;
                        store_remote16(map_to_rank(piece(rank, local, q), owner), bar, v[e], v[e + 1], v[e + 2], v[e + 3]);
                    }
                }
            }
        }
        if (split > 1) {
            mbar_wait(recv_bar(), 0, abort_flag, g.status, g.wait_limit);
#pragma unroll 1
            for (int local = half; local < own_valid; local += kEpi / 4) {
                float a[kGroup];
#pragma unroll
                for (int j = 0; j < kGroup; ++j) a[j] = 0.0f;
#pragma unroll 2
                for (int from = 0; from < (int)split; ++from)
#pragma unroll
                    for (int q = 0; q < kGroup / 4; ++q) {
                        uint32_t p[4];
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(p[0]), "=r"(p[1]), "=r"(p[2]), "=r"(p[3]) : "r"(piece(from, local, q)));
#pragma unroll
                        for (int j = 0; j < 4; ++j) a[4 * q + j] = __fadd_rn(a[4 * q + j], __uint_as_float(p[j]));
                    }
                put(g, (rank * own + local) * kGroup, a, alpha, lane_bias);
            }
        }
        tc_fence_before();
    }
};

template <int BN, bool NV, bool SWAP>
__global__ void __launch_bounds__(mx_small_threads(SWAP))
sparq_mxf4_small_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_f,
                        const __grid_constant__ CUtensorMap map_h, const MxGemmArgs g)
{
    using Cta = Mxf4Small<BN, NV, SWAP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) MxBars bars;
    __shared__ uint32_t tmem_base_slot;
    __shared__ uint32_t abort_word;
    __shared__ volatile uint32_t issued[2];

    Cta c;
    const int warp = c.warp = threadIdx.x >> 5, lane = c.lane = threadIdx.x & 31;
    c.abort_flag = &abort_word;
    c.issued = issued;
    c.S = g.stages;
    c.smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    c.bars = smem_u32(&bars);
    c.recv = c.smem + (uint32_t)(c.S * Cta::kStage);
    const uint32_t split = c.split = (uint32_t)g.split, tile = blockIdx.x / split;
    c.rank = (int)(blockIdx.x - tile * split);
    const int64_t R = SWAP ? g.N : g.M, C = SWAP ? g.M : g.N;
    const uint32_t n_tiles = (uint32_t)((g.N + 127) / 128), mt = tile / n_tiles, nt = tile - mt * n_tiles;
    c.r0 = (int64_t)(SWAP ? nt : mt) * 128;
    c.c0 = (int64_t)(SWAP ? mt : nt) * BN;
    c.rows = R - c.r0 < 128 ? (int)(R - c.r0) : 128;
    c.cols = C - c.c0 < BN ? (int)(C - c.c0) : BN;
    c.kb_first = (int)((int64_t)c.rank * g.k_blocks / split);
    c.steps = (int)((int64_t)(c.rank + 1) * g.k_blocks / split) - c.kb_first;
    c.groups = (c.cols + Cta::kGroup - 1) / Cta::kGroup;
    c.own = mx_own_groups(c.cols, (int)split, SWAP);
    const int rest = c.groups - c.rank * c.own;
    c.own_valid = rest < 0 ? 0 : rest < c.own ? rest : c.own;

    if (warp == 0) {
        if (lane == 0) {
            prefetch_tensormap(&map_a);
            prefetch_tensormap(&map_b);
            for (int s = 0; s < c.S; ++s) {
                mbar_init(c.full_bar(s), 2);
                mbar_init(c.empty_bar(s), 1);
            }
            mbar_init(c.acc_bar(), 1);
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
    if (split > 1) {
        if (threadIdx.x == 0) mbar_expect_tx(c.recv_bar(), split * (uint32_t)(c.own_valid * c.rows) * (Cta::kGroup * 4));
        __syncwarp();
        cluster_arrive();       // "barriers ready": waited for before the first remote store
    }
    dep_wait();
    constexpr int kLast = 2 + Cta::kEpi;
    switch (warp) {
    case 0: c.template produce<true>(SWAP ? map_b : map_a, SWAP ? g.b_scales : g.a_scales, g); break;
    case 1: c.issue(g); break;
    case kLast: c.template produce<false>(SWAP ? map_a : map_b, SWAP ? g.a_scales : g.b_scales, g); break;
    default: c.finish(map_f, map_h, g);
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
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(c.tmem), "r"(Cta::kCols) : "memory");
    }
}

}  // namespace sparq
