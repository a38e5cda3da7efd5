// Weight gradients from inputs that were kept in 8 bits (sparq_wgrad_mx8).
//
//   dw[n][k] (+)= sum_m dy[m][n] X[m][k],   X[m][k] = q * 2^-6 * 2^e
//
// q has at most seven significant bits and its scale is a power of two, so X is exact in bf16 (down to 2^-133, bf16's
// last subnormal): the products are those of a bf16 contraction that would have been given X itself, at half its bytes.
//
// The sum runs over the rows of both matrices, so both operands lie along the output axes in shared memory (MN-major): dy as
// TMA brings it, X as the transform warps write it, from codes and scales that TMA brings beside it.
#pragma once

#include "sparq_mx_tc.cuh"

namespace sparq {

struct WgradArgs {
    int64_t M, N, K;
    int blocks;                 // reduction steps of kWgTokens
    int accumulate;
    float *dw;
    unsigned int *status;
    long long wait_limit;
    int stages, split;
};

constexpr int kWgTokens = 64;                    // per reduction step: four MMAs of 16
constexpr int kWgBox = kWgTokens * 128;          // 64 tokens x 64 bf16 columns

// Scale 2^(code - 127 - 6) as a pair of equal bf16 values; NaN for the scale's NaN.
__device__ __forceinline__ uint32_t bf16_scale_pair(uint32_t code)
{
    const uint32_t b = code == kNanE8M0 ? 0x7FC0u : code > 6u ? (code - 6u) << 7 : 0x40u >> (6u - code);
    return b * 0x00010001u;
}

// Four codes of one block as bf16 values.  As bit patterns in bf16, whose steps are 1 in [128, 256) and 2 in [256, 512):
//     0x4300 | (b & 0x7F) = 128 + (b & 0x7F),   0x4300 | (b & 0x80) = 128 or 256,
// and their difference is the two's complement value; difference and product with a power of two are exact.
__device__ __forceinline__ void codes_to_bf16(uint32_t w, uint32_t scale, uint32_t &lo, uint32_t &hi)
{
    auto two = [&](uint32_t p) {
        const uint32_t v = (p & 0x007F007Fu) | 0x43004300u, c = (p & 0x00800080u) | 0x43004300u;
        uint32_t d;
        asm("{\n\t.reg .b32 t;\n\tsub.rn.bf16x2 t, %1, %2;\n\tmul.rn.bf16x2 %0, t, %3;\n\t}" : "=r"(d) : "r"(v), "r"(c), "r"(scale));
        return d;
    };
    lo = two(prmt(w, 0u, 0x4140u));
    hi = two(prmt(w, 0u, 0x4342u));
}

// The tensor cores cut a running sum off where fp32 would round it, so its error grows with the number of additions and
// has a sign: 16384 tokens in one sum were off by 5e-6, 100352 by 9e-6 (2-norm).  A sum therefore runs over kWgChunk tokens in
// tensor memory and is then added, rounded to nearest, to one that the worker warps hold in registers, while the next one runs in
// the other half of the accumulators.
constexpr int kWgChunkSteps = 8;                 // 512 tokens

// ---- few output tiles, or little work ------------------------------------------------------------------
// Tiles of 128 x 128, a cluster of `split` CTAs on each that take equal runs of tokens: their partial sums go to the CTA that
// owns a group of four columns through distributed shared memory (the operand ring's, once every CTA of the cluster is
// done with it), and are added in rank order.
// Warps: 0 producer, 1 tensor memory and MMA issue, 2..9 workers: they transform every stage, and after a chunk's last one add up
// the chunk before (warp w: lane quarter w % 4, half of the columns).

constexpr int kWgBN = 128;
constexpr int kWgWorkers = 8;
constexpr int kWgThreads = 32 * (2 + kWgWorkers);
constexpr int kWgOwn = kWgBN / 2;                                   // columns of a worker thread's row
constexpr int kWgRaw = 2 * kWgBox;                                  // dy: two boxes
constexpr int kWgCodes = kWgRaw, kWgScales = kWgCodes + kWgTokens * kWgBN, kWgX = kWgScales + kWgTokens * 16;
constexpr int kWgStage = kWgX + 2 * kWgBox;                         // 41 KB
constexpr int kWgStages = 5;
static_assert(kWgX % 1024 == 0 && kWgStage % 1024 == 0, "operand tiles start on 1024-byte boundaries");
static_assert(kWgStages * kWgStage >= (128 + 8) * kWgBN * 4 && kWgStages <= kMaxStages, "the ring has room for a tile of partial sums");

struct WgradSmall : MxCta {
    int64_t n0, k0;
    int first, cols, groups, own, own_valid;

    __device__ void produce(const CUtensorMap &map_dy, const CUtensorMap &map_codes, const CUtensorMap &map_scales, const WgradArgs &g) const
    {
        if (lane == 0) {
            dep_launch();
            int it = 0, s = 0;
            uint32_t ph = 1;
            for (; it < steps; ++it) {
                if (it >= S && !mbar_wait(empty_bar(s), ph, abort_flag, g.status, g.wait_limit)) break;
                const uint32_t full = full_bar(s), at = smem + (uint32_t)(s * kWgStage);
                const int m = (first + it) * kWgTokens;
                mbar_expect_tx(full, kWgX);
                tma_load_2d(at, &map_dy, full, (int)n0, m);
                tma_load_2d(at + kWgBox, &map_dy, full, (int)n0 + 64, m);
                tma_load_2d(at + kWgCodes, &map_codes, full, (int)k0, m);
                tma_load_2d(at + kWgScales, &map_scales, full, (int)(k0 / 32) & ~15, m);
                if (++s == S) { s = 0; ph ^= 1u; }
            }
            if (*abort_flag)       // none of this thread's copies may land after the CTA has exited
                for (int j = it > S ? it - S : 0; j < it; ++j)
                    mbar_wait(full_bar(j % S), (uint32_t)(j / S) & 1u, abort_flag, g.status, g.wait_limit, true);
        }
        __syncwarp();
    }

    // Chunk c adds up in accumulator c & 1; acc says that it is complete, freed that the workers have read it.
    __device__ void issue(const WgradArgs &g) const
    {
        const uint32_t elected = elect_one();
        constexpr uint32_t id = make_idesc_bf16_mn(kWgBN, 128);
        int s = 0, c = 0;
        uint32_t ph = 0;
        for (int it = 0; it < steps; ++it) {
            const int in = it & (kWgChunkSteps - 1);
            if (in == 0 && c >= 2) mbar_wait(freed_bar(c & 1), (uint32_t)((c >> 1) - 1) & 1u, abort_flag, g.status, g.wait_limit);
            mbar_wait(full_bar(s), ph, abort_flag, g.status, g.wait_limit);
            mbar_wait(xf_bar(s), ph, abort_flag, g.status, g.wait_limit);
            tc_fence_after();
            const bool chunk_ends = in == kWgChunkSteps - 1 || it == steps - 1;
            if (elected) {
                const uint32_t at = smem + (uint32_t)(s * kWgStage), d = tmem + (uint32_t)((c & 1) * kWgBN);
                const uint64_t adesc = mn_major_desc(at, kWgBox), bdesc = mn_major_desc(at + kWgX, kWgBox);
#pragma unroll
                for (int k = 0; k < kWgTokens / 16; ++k)
                    tc_mma_bf16(d, adesc + (uint64_t)(k * 128), bdesc + (uint64_t)(k * 128), id, (in > 0 || k > 0) ? 1u : 0u);
                tc_commit(empty_bar(s));
                if (chunk_ends) tc_commit(acc_bar(c & 1));
            }
            __syncwarp();
            if (chunk_ends) ++c;
            if (++s == S) { s = 0; ph ^= 1u; }
        }
        // every MMA has retired before the warp goes on
        mbar_wait(acc_bar((c - 1) & 1), (uint32_t)((c - 1) >> 1) & 1u, abort_flag, g.status, g.wait_limit, true);
        __syncwarp();
    }

    __device__ void add_chunk(const WgradArgs &g, int c, float (&sum)[kWgOwn]) const
    {
        mbar_wait(acc_bar(c & 1), (uint32_t)(c >> 1) & 1u, abort_flag, g.status, g.wait_limit);
        tc_fence_after();
        const uint32_t taddr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((c & 1) * kWgBN + ((warp - 2) >> 2) * kWgOwn);
#pragma unroll
        for (int h = 0; h < kWgOwn / 32; ++h) {
            uint32_t v[32];
            tmem_ld_32x32_issue(taddr + h * 32, v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) sum[h * 32 + j] = __fadd_rn(sum[h * 32 + j], __uint_as_float(v[j]));
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(freed_bar(c & 1));
    }

    __device__ void work(const WgradArgs &g, float (&sum)[kWgOwn]) const
    {
        const int wt = threadIdx.x - 64, chunk = wt & 15, t0 = wt >> 4;       // eight codes of every sixteenth token
        const uint32_t src = kWgCodes + (uint32_t)(t0 * kWgBN + chunk * 8);
        const uint32_t sc = kWgScales + (uint32_t)(t0 * 16 + ((int)(k0 / 32) & 15) + (chunk >> 2));
        const uint32_t dst = kWgX + (uint32_t)((chunk >> 3) * kWgBox + t0 * 128 + (((chunk & 7) ^ (t0 & 7)) << 4));
#pragma unroll
        for (int j = 0; j < kWgOwn; ++j) sum[j] = 0.0f;
        int s = 0, c = 0;
        uint32_t ph = 0;
        for (int it = 0; it < steps; ++it) {
            mbar_wait(full_bar(s), ph, abort_flag, g.status, g.wait_limit);
            const uint32_t at = smem + (uint32_t)(s * kWgStage);
#pragma unroll
            for (int j = 0; j < kWgTokens / 16; ++j) {
                uint32_t a, b, code, x0, x1, x2, x3;
                asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(a), "=r"(b) : "r"(at + src + (uint32_t)(j * 16 * kWgBN)));
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(code) : "r"(at + sc + (uint32_t)(j * 16 * 16)));
                const uint32_t scale = bf16_scale_pair(code);
                codes_to_bf16(a, scale, x0, x1);
                codes_to_bf16(b, scale, x2, x3);
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" :: "r"(at + dst + (uint32_t)(j * 16 * 128)), "r"(x0), "r"(x1), "r"(x2), "r"(x3) : "memory");
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(xf_bar(s));
            if (++s == S) { s = 0; ph ^= 1u; }
            if ((it & (kWgChunkSteps - 1)) == kWgChunkSteps - 1 && it < steps - 1) {
                if (c > 0) add_chunk(g, c - 1, sum);
                ++c;
            }
        }
        if (c > 0) add_chunk(g, c - 1, sum);
        add_chunk(g, c, sum);
    }

    __device__ void finish(const WgradArgs &g, const float (&sum)[kWgOwn]) const
    {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const int64_t n = n0 + quarter * 32 + lane;
        auto put = [&](int col, const float (&a)[4]) {
            if (n >= g.N) return;
            float *out = g.dw + n * g.K + k0 + col;
            if (col + 4 <= cols && (reinterpret_cast<uintptr_t>(out) & 15u) == 0) {
                float4 v = make_float4(a[0], a[1], a[2], a[3]);
                if (g.accumulate) {
                    const float4 o = *reinterpret_cast<const float4 *>(out);
                    v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
                }
                *reinterpret_cast<float4 *>(out) = v;
                return;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (col + j < cols) out[j] = g.accumulate ? out[j] + a[j] : a[j];
        };
#pragma unroll
        for (int q = 0; q < kWgOwn / 4; ++q) {
            const int grp = half * (kWgOwn / 4) + q;
            if (grp >= groups) continue;
            const float a[4] = {sum[4 * q], sum[4 * q + 1], sum[4 * q + 2], sum[4 * q + 3]};
            if (split == 1) {
                put(grp * 4, a);
            } else {
                const int owner = grp / own, local = grp - owner * own;
                const uint32_t dst = smem + (uint32_t)(((rank * own + local) * 128 + quarter * 32 + lane) * 16);
                store_remote16(map_to_rank(dst, owner), map_to_rank(recv_bar(), owner), __float_as_uint(a[0]), __float_as_uint(a[1]),
                               __float_as_uint(a[2]), __float_as_uint(a[3]));
            }
        }
        if (split == 1) return;
        mbar_wait(recv_bar(), 0, abort_flag, g.status, g.wait_limit, true);
        for (int local = half; local < own_valid; local += 2) {
            float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (uint32_t q = 0; q < split; ++q) {
                uint4 p;
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(p.x), "=r"(p.y), "=r"(p.z), "=r"(p.w)
                             : "r"(smem + (uint32_t)((((int)q * own + local) * 128 + quarter * 32 + lane) * 16)));
                a[0] += __uint_as_float(p.x);
                a[1] += __uint_as_float(p.y);
                a[2] += __uint_as_float(p.z);
                a[3] += __uint_as_float(p.w);
            }
            put((rank * own + local) * 4, a);
        }
    }
};

__global__ void __launch_bounds__(kWgThreads)
sparq_wgrad_small_kernel(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_codes,
                         const __grid_constant__ CUtensorMap map_scales, const WgradArgs g)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) MxBars bars;
    __shared__ uint32_t tmem_base_slot;
    __shared__ uint32_t abort_word;

    WgradSmall c;
    const int warp = c.warp = threadIdx.x >> 5, lane = c.lane = threadIdx.x & 31;
    c.abort_flag = &abort_word;
    c.S = g.stages;
    c.smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    c.bars = smem_u32(&bars);
    const uint32_t split = c.split = (uint32_t)g.split, tile = blockIdx.x / split;
    c.rank = (int)(blockIdx.x - tile * split);
    const uint32_t k_tiles = (uint32_t)((g.K + kWgBN - 1) / kWgBN), nt = tile / k_tiles;
    c.n0 = (int64_t)nt * 128;
    c.k0 = (int64_t)(tile - nt * k_tiles) * kWgBN;
    c.first = (int)((int64_t)c.rank * g.blocks / split);
    c.steps = (int)((int64_t)(c.rank + 1) * g.blocks / split) - c.first;
    c.cols = g.K - c.k0 < kWgBN ? (int)(g.K - c.k0) : kWgBN;
    c.groups = (c.cols + 3) / 4;
    c.own = (c.groups + (int)split - 1) / (int)split;
    const int rest = c.groups - c.rank * c.own;
    c.own_valid = rest < 0 ? 0 : rest < c.own ? rest : c.own;

    if (warp == 0) {
        if (lane == 0) {
            prefetch_tensormap(&map_dy);
            prefetch_tensormap(&map_codes);
            prefetch_tensormap(&map_scales);
            for (int s = 0; s < c.S; ++s) {
                mbar_init(c.full_bar(s), 1);
                mbar_init(c.xf_bar(s), kWgWorkers);
                mbar_init(c.empty_bar(s), 1);
            }
            for (int b = 0; b < 2; ++b) {
                mbar_init(c.acc_bar(b), 1);
                mbar_init(c.freed_bar(b), kWgWorkers);
            }
            mbar_init(c.recv_bar(), 1);
            abort_word = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    } else if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&tmem_base_slot)), "r"(2u * kWgBN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    c.tmem = tmem_base_slot;
    if (threadIdx.x == 0 && split > 1) mbar_expect_tx(c.recv_bar(), split * (uint32_t)c.own_valid * (128 * 16));
    float sum[kWgOwn];
    dep_wait();
    switch (warp) {
    case 0: c.produce(map_dy, map_codes, map_scales, g); break;
    case 1: c.issue(g); break;
    default: c.work(g, sum);
    }
    // Every MMA of this CTA has retired (or a wait gave up), and none of its copies is on its way: the cluster's rings are
    // free for partial sums once all CTAs are here.
    __syncthreads();
    if (split > 1) {
        cluster_arrive();
        cluster_wait();
    }
    if (warp >= 2) c.finish(g, sum);
    __syncthreads();
    // No CTA leaves while its peers' rows are on their way to it: every CTA sends all of its rows, after a wait that gave up
    // too, and finish() waits for them whether or not the flag is up.
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(c.tmem), "r"(2u * kWgBN) : "memory");
    }
}

}  // namespace sparq
