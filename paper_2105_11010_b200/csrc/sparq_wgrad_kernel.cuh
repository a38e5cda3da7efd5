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

// The tokens are cut into `parts` equal runs of steps whose sums are added in order.  A launch takes `count` of them from `part` on and
// writes each one's sums `part_stride` elements after the one's before: all parts into scratch memory that another launch adds up,
// or one part after the other into dw itself.
struct WgradArgs {
    int64_t M, N, K;
    int blocks;                 // reduction steps of kWgTokens
    int parts, part, count;
    int64_t part_stride;
    int accumulate;
    float *dw;
    unsigned int *status;
    long long wait_limit;
    int split;
};

constexpr int kWgTokens = 64;                    // per reduction step: four MMAs of 16
constexpr int kWgBox = kWgTokens * 128;          // 64 tokens x 64 bf16 columns

// Scale 2^(code - 127 - 6) as a pair of equal bf16 values: an exponent of its own for codes 7 to 254, a subnormal below, NaN
// for the scale's NaN.
__device__ __forceinline__ uint32_t bf16_scale_pair(uint32_t code)
{
    uint32_t b = (code - 6u) << 7;
    if (code - 7u > 247u) b = code == kNanE8M0 ? 0x7FC0u : 0x40u >> (6u - code);
    return prmt(b, b, 0x1010u);
}

// Four codes of one block as bf16 values, in the order 0, 2, 1, 3: the columns of the operand and so of the accumulator, which are put in
// order when they are written out.  As bit patterns in bf16, whose steps are 1 in [128, 256) and 2 in [256, 512):
//     0x4300 | (b & 0x7F) = 128 + (b & 0x7F),   0x4300 | (b & 0x80) = 128 or 256,
// and their difference is the two's complement value; difference and product with a power of two are exact.
__device__ __forceinline__ void codes_to_bf16(uint32_t w, uint32_t scale, uint32_t &even, uint32_t &odd)
{
    auto two = [&](uint32_t p) {
        const uint32_t v = (p & 0x007F007Fu) | 0x43004300u, c = (p & 0x00800080u) | 0x43004300u;
        uint32_t d;
        asm("{\n\t.reg .b32 t;\n\tsub.rn.bf16x2 t, %1, %2;\n\tmul.rn.bf16x2 %0, t, %3;\n\t}" : "=r"(d) : "r"(v), "r"(c), "r"(scale));
        return d;
    };
    even = two(w);
    odd = two(w >> 8);
}
__host__ __device__ constexpr int wgrad_column(int j) { return (j & ~3) | ((j & 1) << 1) | ((j >> 1) & 1); }

// A team of 128 threads turns a raw tile (64 tokens x 128 codes, swizzled by TMA; rows of 16 scales) into an operand tile (two atoms of 64
// columns).  A thread takes 16 codes of every sixteenth token.  Eight neighbouring lanes take half a row each of tokens t and t ^ 5, whose
// swizzles differ in bits 0 and 2: loads and stores of 16 bytes then meet all banks.  All loads go out before the first store.
struct TeamPlace {
    uint32_t src, sc, dst0, dst1;           // offsets in a raw stage, and in an operand tile
    __device__ TeamPlace(int thread, int scale_offset, uint32_t codes_at, uint32_t scales_at, uint32_t x_at)
    {
        const int c4 = thread & 3, atom = (thread >> 3) & 1, u = thread >> 4;
        const int t = ((u & 3) | ((u & 4) << 1)) ^ (thread & 4 ? 5 : 0), x = t & 7;
        src = codes_at + (uint32_t)(t * 128 + (((atom * 4 + c4) ^ x) << 4));
        sc = scales_at + (uint32_t)(t * 16 + scale_offset + atom * 2 + (c4 >> 1));
        dst0 = x_at + (uint32_t)(atom * (64 * 128) + t * 128 + (((2 * c4) ^ x) << 4));
        dst1 = x_at + (uint32_t)(atom * (64 * 128) + t * 128 + (((2 * c4 + 1) ^ x) << 4));
    }
};
__device__ __forceinline__ void transform_stage(uint32_t at, uint32_t to, const TeamPlace &p)
{
    uint32_t w[4][4], code[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[j][0]), "=r"(w[j][1]), "=r"(w[j][2]), "=r"(w[j][3]) : "r"(at + p.src + (uint32_t)(j * 16 * 128)));
        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(code[j]) : "r"(at + p.sc + (uint32_t)(j * 16 * 16)));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t scale = bf16_scale_pair(code[j]);
        uint32_t x[8];
#pragma unroll
        for (int q = 0; q < 4; ++q) codes_to_bf16(w[j][q], scale, x[2 * q], x[2 * q + 1]);
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" :: "r"(to + p.dst0 + (uint32_t)(j * 16 * 128)), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" :: "r"(to + p.dst1 + (uint32_t)(j * 16 * 128)), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]) : "memory");
    }
}

// The tensor cores cut a running sum off where fp32 would round it, so its error grows with the number of additions and
// has a sign: 16384 tokens in one sum were off by 5e-6, 100352 by 9e-6 (2-norm).  A sum therefore runs over kWgChunk tokens in
// tensor memory and is then added, rounded to nearest, to one that the worker warps hold in registers, while the next one runs in
// the other half of the accumulators.
constexpr int kWgChunkSteps = 8;                 // 512 tokens

// C columns of a row (sum[at(j)] is column j) to `out`, the first `cols` of them, added to what is there or not.  Whole vectors
// where they can be: 32 bytes, or behind the row's first 16-byte boundary 16 (rows of a length that is no multiple of four, element by
// element: 316 x 2496 x 3779 67 us).
template <int C, class At>
__device__ __forceinline__ void wgrad_put_row(float *out, const float (&sum)[C], int64_t cols, int accumulate, At at)
{
    if (cols >= C && (reinterpret_cast<uintptr_t>(out) & 31u) == 0) {
#pragma unroll
        for (int j = 0; j < C; j += 8) {
            uint32_t v[8];
            if (accumulate) {
                ld_v8(v, out + j);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(__fadd_rn(__uint_as_float(v[i]), sum[at(j + i)]));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(sum[at(j + i)]);
            }
            st_v8(out + j, v);
        }
        return;
    }
    auto one = [&](int64_t j, float v) { out[j] = accumulate ? __fadd_rn(out[j], v) : v; };
    // columns head .. head + 3, + 4 .. + 7 and so on are vectors; head differs from lane to lane
    const int head = (int)((0u - ((uint32_t)reinterpret_cast<uintptr_t>(out) >> 2)) & 3u);
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (j < head && j < cols) one(j, sum[at(j)]);
#pragma unroll
    for (int j = 0; j < C; j += 4) {
        float t[6], v[4];
#pragma unroll
        for (int i = 0; i < 6; ++i) {
            const float a = j + i < C ? sum[at((j + i) % C)] : 0.0f, b = j + i + 1 < C ? sum[at((j + i + 1) % C)] : 0.0f;
            t[i] = head & 1 ? b : a;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = head & 2 ? t[i + 2] : t[i];
        const int64_t first = j + head;
        if (j + 4 <= C - 4 + (head == 0 ? 4 : 0) && first + 4 <= cols) {
            float4 *to = reinterpret_cast<float4 *>(out + first);
            float4 w = make_float4(v[0], v[1], v[2], v[3]);
            if (accumulate) {
                const float4 o = *to;
                w = make_float4(__fadd_rn(o.x, w.x), __fadd_rn(o.y, w.y), __fadd_rn(o.z, w.z), __fadd_rn(o.w, w.w));
            }
            *to = w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (first + i < cols && first + i < C) one(first + i, v[i]);
        }
    }
}

// ---- few output tiles, or little work ------------------------------------------------------------------
// Tiles of 128 x 128, a cluster of `split` CTAs on each that take equal runs of tokens: their partial sums go to the CTA that
// owns a group of four columns through distributed shared memory (the operand ring's, once every CTA of the cluster is
// done with it), and are added in rank order.
// Warps: 0 producer of dy, 18 of codes and scales, 1 tensor memory and MMA issue, 2..17 workers: they transform the stages, and after a
// chunk's last one add up the chunk before (warp w: lane quarter w % 4, a quarter of the columns).

constexpr int kWgBN = 128;
constexpr int kWgTeams = 4, kWgWorkers = 4 * kWgTeams;
constexpr int kWgThreads = 32 * (3 + kWgWorkers);
constexpr int kWgOwn = kWgBN / kWgTeams;                            // columns of a worker thread's row
constexpr int kWgCodes = 2 * kWgBox, kWgScales = kWgCodes + kWgTokens * kWgBN;      // in a raw stage, behind two boxes of dy
// Two rings: R stages of what TMA brings, and X stages of X in bf16, which the teams write while the MMAs read another.
constexpr int kWgStage = kWgScales + kWgTokens * 16;                // 25 KB
constexpr int kWgXStage = 2 * kWgBox;
static_assert(kWgStage % 1024 == 0, "operand tiles start on 1024-byte boundaries");

// The barriers of the weight gradients' kernels: those of MxBars, of the raw stages, and of free X stages.
struct WgradBars {
    MxBars m;
    uint64_t raw[kMaxStages], x_empty[kMaxStages];
};
template <int R, int X>
struct WgradCta : MxCta {
    static constexpr int kRaw = R, kX = X, kRings = R * kWgStage + X * kWgXStage;
    static_assert(R <= kMaxStages && X <= kMaxStages, "a barrier for each stage");
    // A wait for a step's raw stage comes behind the wait for its X stage, whose MMA is behind that of the raw stage's last use.
    static_assert(X <= R, "the X stage's last step is not older than the raw stage's");
    __device__ uint32_t raw_bar(int s) const { return bars + (uint32_t)sizeof(MxBars) + (uint32_t)s * 8u; }
    __device__ uint32_t x_empty_bar(int q) const { return raw_bar(kMaxStages + q); }
    __device__ uint32_t x_stage(int q) const { return smem + (uint32_t)(R * kWgStage + q * kWgXStage); }
};
// Position in a ring of N stages, and the parity of its phase.
template <int N>
struct RingAt {
    int s = 0;
    uint32_t ph = 0;
    __device__ void next() { if (++s == N) { s = 0; ph ^= 1u; } }
};

// drain_ring as a call: 64 x 512 x 512 4.78 us, inlined into WgradSmall's kernel 4.83.
__device__ __noinline__ void drain_ring_call(uint32_t bar, uint32_t S, uint32_t n, volatile uint32_t *abort_flag, unsigned int *status, long long limit)
{
    drain_ring(bar, S, n, abort_flag, status, limit);
}

struct WgradSmall : WgradCta<6, 4> {
    static_assert(kX % kWgTeams == 0, "an X stage belongs to one team");
    static_assert(kRings >= (128 + 8) * kWgBN * 4, "the rings have room for a tile of partial sums");
    int64_t n0, k0;
    float *dw;
    int first, cols, groups, own, own_valid;

    // Two producers: dy, on the full barriers; codes and scales, on the raw ones.  (One thread takes over 0.4 us to issue all
    // four copies of a step.)
    template <bool DY>
    __device__ void produce(const CUtensorMap &map_a, const CUtensorMap &map_b, const WgradArgs &g) const
    {
        if (lane == 0) {
            if (DY) dep_launch();
            int it = 0, s = 0;
            uint32_t ph = 1;
            for (; it < steps; ++it) {
                if (it >= S && !mbar_wait(empty_bar(s), ph, abort_flag, g.status, g.wait_limit)) { issued[DY ? 0 : 1] = (uint32_t)it; break; }
                const uint32_t bar = DY ? full_bar(s) : raw_bar(s), at = smem + (uint32_t)(s * kWgStage);
                const int m = (first + it) * kWgTokens;
                mbar_expect_tx(bar, DY ? kWgCodes : kWgStage - kWgCodes);
                if (DY) {
                    tma_load_2d(at, &map_a, bar, (int)n0, m);
                    tma_load_2d(at + kWgBox, &map_a, bar, (int)n0 + 64, m);
                } else {
                    tma_load_2d(at + kWgCodes, &map_a, bar, (int)k0, m);
                    tma_load_2d(at + kWgScales, &map_b, bar, (int)(k0 / 32) & ~15, m);
                }
                if (++s == S) { s = 0; ph ^= 1u; }
            }
        }
        __syncwarp();
    }

    // Chunk c adds up in accumulator c & 1; acc says that it is complete, freed that the workers have read it.
    __device__ void issue(const WgradArgs &g) const
    {
        const uint32_t elected = elect_one();
        constexpr uint32_t id = make_idesc_bf16_mn(kWgBN, 128);
        RingAt<kRaw> raw;
        RingAt<kX> x;
        int c = 0;
        for (int it = 0; it < steps; ++it) {
            const int in = it & (kWgChunkSteps - 1);
            if (in == 0 && c >= 2 && !mbar_wait_warp(elected, freed_bar(c & 1), (uint32_t)((c >> 1) - 1) & 1u, abort_flag, g.status, g.wait_limit)) break;
            if (!mbar_wait_warp(elected, full_bar(raw.s), raw.ph, abort_flag, g.status, g.wait_limit) ||
                !mbar_wait_warp(elected, xf_bar(x.s), x.ph, abort_flag, g.status, g.wait_limit)) {
                tc_commit_if(acc_bar(c & 1), elected);          // what there is of the chunk
                ++c;
                break;
            }
            tc_fence_after();
            const bool chunk_ends = in == kWgChunkSteps - 1 || it == steps - 1;
            const uint32_t at = smem + (uint32_t)(raw.s * kWgStage), d = tmem + (uint32_t)((c & 1) * kWgBN);
            const uint64_t adesc = mn_major_desc(at, kWgBox), bdesc = mn_major_desc(x_stage(x.s), kWgBox);
#pragma unroll
            for (int k = 0; k < kWgTokens / 16; ++k)
                tc_mma_bf16(d, adesc + (uint64_t)(k * 128), bdesc + (uint64_t)(k * 128), id, (in > 0 || k > 0) ? 1u : 0u, elected);
            tc_commit_if(empty_bar(raw.s), elected);
            tc_commit_if(x_empty_bar(x.s), elected);
            if (chunk_ends) tc_commit_if(acc_bar(c & 1), elected);
            if (chunk_ends) ++c;
            raw.next();
            x.next();
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
        // A team of four warps takes every fourth stage: a stage's chain of barriers, loads, arithmetic and stores is mostly latency, which the
        // other teams' fill (100352 x 128 x 1152 call after call: four teams 54.8 us, two 59.5, of which 36 are there without any transform).
        const int team = (warp - 2) >> 2;
        const TeamPlace place((threadIdx.x - 64) & 127, (int)(k0 / 32) & 15, kWgCodes, kWgScales, 0);
#pragma unroll
        for (int j = 0; j < kWgOwn; ++j) sum[j] = 0.0f;
        RingAt<kRaw> raw;
        RingAt<kX> x;
        int c = 0;
        for (int it = 0; it < steps; ++it) {
            if (it % kWgTeams == team) {
                // The X stage first: its MMA, of step it - kX, comes behind that of step it - kRaw, whose phase of the raw barrier, another
                // team's to wait for, is complete then.  A barrier tells a phase from the next only, so that before it a wait for this step's
                // would return at once.
                // (A stage whose wait gave up is not handed on.)
                if (it >= kX && !mbar_wait_warp(lane == 0 ? 1u : 0u, x_empty_bar(x.s), x.ph ^ 1u, abort_flag, g.status, g.wait_limit)) return;
                if (!mbar_wait_warp(lane == 0 ? 1u : 0u, raw_bar(raw.s), raw.ph, abort_flag, g.status, g.wait_limit)) return;
                transform_stage(smem + (uint32_t)(raw.s * kWgStage), x_stage(x.s), place);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(xf_bar(x.s));
            }
            raw.next();
            x.next();
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
            float *out = dw + n * g.K + k0 + col;
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
        if (split == 1) {
            if (n < g.N && half * kWgOwn < cols)
                wgrad_put_row(dw + n * g.K + k0 + half * kWgOwn, sum, cols - half * kWgOwn, g.accumulate, [](int j) { return wgrad_column(j); });
            return;
        }
#pragma unroll
        for (int q = 0; q < kWgOwn / 4; ++q) {
            const int grp = half * (kWgOwn / 4) + q;
            if (grp >= groups) continue;
            const float a[4] = {sum[4 * q], sum[4 * q + wgrad_column(1)], sum[4 * q + wgrad_column(2)], sum[4 * q + 3]};
            const int owner = grp / own, local = grp - owner * own;
            const uint32_t dst = smem + (uint32_t)(((rank * own + local) * 128 + quarter * 32 + lane) * 16);
            store_remote16(map_to_rank(dst, owner), map_to_rank(recv_bar(), owner), __float_as_uint(a[0]), __float_as_uint(a[1]),
                           __float_as_uint(a[2]), __float_as_uint(a[3]));
        }
        mbar_wait(recv_bar(), 0, abort_flag, g.status, g.wait_limit, true);
        for (int local = half; local < own_valid; local += kWgTeams) {
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
    __shared__ __align__(8) WgradBars room;
    __shared__ uint32_t tmem_base_slot;
    __shared__ uint32_t abort_word;
    __shared__ volatile uint32_t issued[2];

    WgradSmall c;
    const int warp = c.warp = threadIdx.x >> 5, lane = c.lane = threadIdx.x & 31;
    c.abort_flag = &abort_word;
    c.issued = issued;
    c.S = WgradSmall::kRaw;
    c.smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    c.bars = smem_u32(&room);
    const uint32_t split = c.split = (uint32_t)g.split, item = blockIdx.x / split;
    c.rank = (int)(blockIdx.x - item * split);
    const uint32_t k_tiles = (uint32_t)((g.K + kWgBN - 1) / kWgBN), tiles = k_tiles * (uint32_t)((g.N + 127) / 128);
    const uint32_t in = item / tiles, tile = item - in * tiles, nt = tile / k_tiles;
    c.n0 = (int64_t)nt * 128;
    c.k0 = (int64_t)(tile - nt * k_tiles) * kWgBN;
    c.dw = g.dw + in * g.part_stride;
    // this part's steps, and this CTA's of them
    const int part = g.part + (int)in, part_first = (int)((int64_t)part * g.blocks / g.parts);
    const int part_steps = (int)((int64_t)(part + 1) * g.blocks / g.parts) - part_first;
    c.first = part_first + (int)((int64_t)c.rank * part_steps / split);
    c.steps = part_first + (int)((int64_t)(c.rank + 1) * part_steps / split) - c.first;
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
                mbar_init(c.raw_bar(s), 1);
                mbar_init(c.empty_bar(s), 1);
            }
            for (int q = 0; q < WgradSmall::kX; ++q) {
                mbar_init(c.xf_bar(q), 4);
                mbar_init(c.x_empty_bar(q), 1);
            }
            for (int b = 0; b < 2; ++b) {
                mbar_init(c.acc_bar(b), 1);
                mbar_init(c.freed_bar(b), kWgWorkers);
            }
            mbar_init(c.recv_bar(), 1);
            abort_word = 0;
            issued[0] = issued[1] = (uint32_t)c.steps;      // unless a producer stops in front of one
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
    case 0: c.produce<true>(map_dy, map_dy, g); break;
    case 1: c.issue(g); break;
    case 2 + kWgWorkers: c.produce<false>(map_codes, map_scales, g); break;
    default: c.work(g, sum);
    }
    // Every MMA of this CTA has retired (or a wait gave up), and none of its copies is on its way: the cluster's rings are
    // free for partial sums once all CTAs are here.
    __syncthreads();
    if (threadIdx.x == 32 * (2 + kWgWorkers) && *c.abort_flag) {
        drain_ring_call(c.full_bar(0), WgradSmall::kRaw, issued[0], c.abort_flag, g.status, g.wait_limit);
        drain_ring_call(c.raw_bar(0), WgradSmall::kRaw, issued[1], c.abort_flag, g.status, g.wait_limit);
    }
    __syncwarp();
    if (split > 1) {
        cluster_arrive();
        cluster_wait();
    }
    if (warp >= 2 && warp < 2 + kWgWorkers) c.finish(g, sum);
    __syncthreads();
    // No CTA leaves while its peers' rows are on their way to it: every CTA sends all of its rows, after a wait that gave up
    // too, and finish() waits for them whether or not the flag is up.
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(c.tmem), "r"(2u * kWgBN) : "memory");
    }
}

// ---- many output tiles -----------------------------------------------------------------------------------
// A persistent pair of CTAs walks tiles of 256 x 256: one MMA (cta_group::2) multiplies 256 columns of dy by 256 of X.  Each CTA
// brings its 128 columns of dy, and brings and transforms its 128 columns of X: a value of X is transformed once per row of tiles
// of 256, half as often as with one CTA by itself.  A step of 64 tokens takes 0.50 to 0.55 us: the chain from the codes' arrival
// through the transform to the MMA, more than any pipe.
// X16: X comes as bf16 (the library's own, expanded from the codes by the launch before) and goes from TMA to the MMA, 0.36 us a step;
// the workers only add up.  Same operands, same order of sums, same bits.  16384 x 4096 x 4096 396 to 450 us call after call with
// the expansion's 35 (452 with L2 emptied in between), 1.2 to 1.39 PFLOP/s in all, at the power cap; 8192 tokens: 12 TB/s of operands
// from L2, tensor pipe 81 % active.
// Warps: 0 producer of dy, 2 of codes and scales, 1 tensor memory and (leader) MMA issue, 4..11 workers, each thread with 128
// columns of a row in registers.

constexpr int kWgTile = 256;
constexpr int kWgPairWorkers = 8, kWgPairTeams = kWgPairWorkers / 4;
constexpr int kWgPairOwn = 128;                  // columns of a worker thread's row
constexpr int kWgCodeWarp = 2;
constexpr int kWgFirstWorker = 4;                // whole groups of four warps, for setmaxnreg
constexpr int kWgPairThreads = 32 * (kWgFirstWorker + kWgPairWorkers);

constexpr int kWgStages16 = 7;
// Three X stages are the teams' in turn, so that a barrier for each would hold every other phase for the other team, and a team could take a
// phase for the one that it asks for only from another barrier's arrival, which nothing orders.  So there are two sets of them: step s
// retires on barrier s % 6, which one team asks for, every phase of it.  (Six raw and four X stages, one set: 16384 x 1024 x 1024 in one
// part 144 us instead of 139.)
constexpr int kWgXSets = 2;
using WgradPairRings = WgradCta<7, 3>;
__host__ __device__ constexpr int wgrad_smem(bool x16) { return 1024 + (x16 ? kWgStages16 * 4 * kWgBox : WgradPairRings::kRings); }

// The first `whole` tiles run over all tokens, the others (the tail) over the parts that the launch takes.  Where those follow whole tiles,
// the first part's sums go to dw, the others' into tail_sums, 256 x 256 for each tile, or in launches of their own (skip: of the tail only)
// to dw too.
struct WgradPairArgs {
    WgradArgs g;
    int n_tiles, k_tiles, pairs, whole, skip;
    float *tail_sums;
};

// Steps of part p.
__device__ __forceinline__ int part_begin(const WgradArgs &g, int p) { return (int)((int64_t)p * g.blocks / g.parts); }

// Tile t in an order that keeps eight rows of tiles together.
__device__ __forceinline__ void wgrad_tile(int n_tiles, int k_tiles, int t, int &nt, int &kt)
{
    const int per_group = 8 * k_tiles, group = t / per_group, first = group * 8;
    const int rows = n_tiles - first < 8 ? n_tiles - first : 8, in = t - group * per_group;
    kt = in / rows;
    nt = first + in - kt * rows;
}

// Item t of a launch: its tile, its steps, and which part of the tail's tile `at` it is (whole tiles: part 0).
struct WgradItem {
    int nt, kt, part, at, first, last;
    __device__ WgradItem(const WgradPairArgs &p, int t)
    {
        const int tail = p.n_tiles * p.k_tiles - p.whole, u = p.skip ? t : t - p.whole;
        part = u < 0 ? 0 : u / tail;
        at = u - part * tail;
        wgrad_tile(p.n_tiles, p.k_tiles, p.whole + at, nt, kt);
        part += u < 0 ? 0 : p.g.part;
        first = u < 0 ? 0 : part_begin(p.g, part);
        last = u < 0 ? p.g.blocks : part_begin(p.g, part + 1);
    }
};

// full: dy of both CTAs, in the leader; raw: codes and scales of this CTA; xf: transformed by both CTAs' workers,
// in the leader; empty: the MMAs that read the stage have retired; acc, freed: as above.
template <bool X16>
struct WgradPair : WgradPairRings {
    static constexpr int kXBars = kWgXSets * kX;
    static_assert(kXBars % kWgPairTeams == 0 && kXBars <= kMaxStages, "a barrier belongs to one team");
    static constexpr int kXAt = 2 * kWgBox, kStage = X16 ? kXAt + kWgXStage : kWgStage, kStages = X16 ? kWgStages16 : kRaw;
    int tiles, pair;

    template <bool DY>
    __device__ void produce(const CUtensorMap &map_a, const CUtensorMap &map_b, const WgradPairArgs &p) const
    {
        if (lane == 0) {
            if (DY) dep_launch();
            const WgradArgs &g = p.g;
            const uint32_t leader_full = map_to_rank(full_bar(0), 0);
            int s = 0;
            uint32_t ph = 1, done = 0;
            bool live = true;
            for (int t = pair; t < tiles && live; t += p.pairs) {
                const WgradItem item(p, t);
                const int n = item.nt * kWgTile + rank * 128, k = item.kt * kWgTile + rank * 128, sc = (k / 32) & ~15;
                for (int b = item.first; b < item.last; ++b) {
                    if (done >= kStages && !mbar_wait(empty_bar(s), ph, abort_flag, g.status, g.wait_limit)) { live = false; break; }
                    const uint32_t at = smem + (uint32_t)(s * kStage);
                    const int m = b * kWgTokens;
                    if (DY) {
                        const uint32_t bar = leader_full + 8u * (uint32_t)s;
                        if (rank == 0) mbar_expect_tx(full_bar(s), (X16 ? 8 : 4) * kWgBox);
                        tma_load_pair_2d(at, &map_a, bar, n, m);
                        tma_load_pair_2d(at + kWgBox, &map_a, bar, n + 64, m);
                    } else if (X16) {
                        const uint32_t bar = leader_full + 8u * (uint32_t)s;
                        tma_load_pair_2d(at + kXAt, &map_a, bar, k, m);
                        tma_load_pair_2d(at + kXAt + kWgBox, &map_a, bar, k + 64, m);
                    } else {
                        mbar_expect_tx(raw_bar(s), kWgStage - kWgCodes);
                        tma_load_2d(at + kWgCodes, &map_a, raw_bar(s), k, m);
                        tma_load_2d(at + kWgScales, &map_b, raw_bar(s), sc, m);
                    }
                    ++done;
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
            // (codes and scales count on their own CTA's barriers)
            if (DY || X16) store_remote(map_to_rank(smem_u32((const void *)(issued + 2 * rank + (DY ? 0 : 1))), 0), done);
            else issued[4] = done;
        }
        __syncwarp();
    }

    // Chunks are counted through all tiles: chunk c adds up in accumulator c & 1.
    __device__ void issue(const WgradPairArgs &p) const
    {
        if (rank == 0) {
            const WgradArgs &g = p.g;
            const uint32_t elected = elect_one();
            constexpr uint32_t id = make_idesc_bf16_mn(kWgTile, 256);
            RingAt<kStages> raw;
            RingAt<kX> x;
            RingAt<kXBars> xe;
            int c = 0;
            bool live = true;
            for (int t = pair; t < tiles && live; t += p.pairs) {
                const WgradItem item(p, t);
                const int steps_of = item.last - item.first;
                for (int b = 0; b < steps_of; ++b) {
                    const int in = b & (kWgChunkSteps - 1);
                    if (in == 0 && c >= 2) live = mbar_wait_warp(elected, freed_bar(c & 1), (uint32_t)((c >> 1) - 1) & 1u, abort_flag, g.status, g.wait_limit);
                    if (!live) break;
                    live = mbar_wait_warp(elected, full_bar(raw.s), raw.ph, abort_flag, g.status, g.wait_limit) &&
                           (X16 || mbar_wait_warp(elected, xf_bar(x.s), x.ph, abort_flag, g.status, g.wait_limit));
                    if (!live) {
                        tc_commit_pair(acc_bar(c & 1), elected);        // what there is of the chunk
                        ++c;
                        break;
                    }
                    tc_fence_after();
                    const bool chunk_ends = in == kWgChunkSteps - 1 || b == steps_of - 1;
                    const uint32_t at = smem + (uint32_t)(raw.s * kStage), d = tmem + (uint32_t)((c & 1) * kWgTile);
                    const uint64_t adesc = mn_major_desc(at, kWgBox), bdesc = mn_major_desc(X16 ? at + kXAt : x_stage(x.s), kWgBox);
#pragma unroll
                    for (int k = 0; k < kWgTokens / 16; ++k)
                        tc_mma_bf16_pair(d, adesc + (uint64_t)(k * 128), bdesc + (uint64_t)(k * 128), id, (in > 0 || k > 0) ? 1u : 0u, elected);
                    tc_commit_pair(empty_bar(raw.s), elected);
                    if (!X16) tc_commit_pair(x_empty_bar(xe.s), elected);
                    if (chunk_ends) tc_commit_pair(acc_bar(c & 1), elected);
                    if (chunk_ends) ++c;
                    raw.next();
                    x.next();
                    xe.next();
                }
            }
            // every MMA has retired before the warp goes on
            if (c > 0) mbar_wait(acc_bar((c - 1) & 1), (uint32_t)((c - 1) >> 1) & 1u, abort_flag, g.status, g.wait_limit, true);
            if (!live && lane == 0) {
                store_remote(map_to_rank(smem_u32((const void *)abort_flag), 1), 1u);        // the other CTA's producers stop, too
                drain_pair(full_bar(0), kStages, issued, 2 * kWgBox, X16 ? 2 * kWgBox : 0, abort_flag, g.status, g.wait_limit);
            }
        }
        __syncwarp();
    }

    __device__ void add_chunk(const WgradArgs &g, int c, uint32_t leader_freed, float (&sum)[kWgPairOwn]) const
    {
        mbar_wait(acc_bar(c & 1), (uint32_t)(c >> 1) & 1u, abort_flag, g.status, g.wait_limit);
        tc_fence_after();
        const uint32_t taddr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((c & 1) * kWgTile + ((warp - kWgFirstWorker) >> 2) * kWgPairOwn);
#pragma unroll
        for (int h = 0; h < kWgPairOwn / 16; ++h) {
            uint32_t v[32];
            tmem_ld_32x16_issue(taddr + h * 16, v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[h * 16 + j] = __fadd_rn(sum[h * 16 + j], __uint_as_float(v[j]));
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(leader_freed + 8u * (uint32_t)(c & 1));
    }

    __device__ void write(const WgradPairArgs &p, const WgradItem &item, const float (&sum)[kWgPairOwn]) const
    {
        const WgradArgs &g = p.g;
        const int row = rank * 128 + (warp & 3) * 32 + lane, col = ((warp - kWgFirstWorker) >> 2) * kWgPairOwn;
        const int64_t n = (int64_t)item.nt * kWgTile + row, k = (int64_t)item.kt * kWgTile + col;
        if (n >= g.N || k >= g.K) return;
        const bool aside = p.tail_sums && item.part > 0;
        float *to = aside ? p.tail_sums + (((int64_t)(item.part - 1) * (p.n_tiles * p.k_tiles - p.whole) + item.at) * kWgTile + row) * kWgTile + col
                          : g.dw + (item.part - g.part) * g.part_stride + n * g.K + k;
        wgrad_put_row(to, sum, g.K - k, aside ? 0 : g.accumulate, [](int j) { return X16 ? j : wgrad_column(j); });
    }

    __device__ void work(const WgradPairArgs &p) const
    {
        const WgradArgs &g = p.g;
        // a team of four warps takes every other stage: one's barriers and loads run beside the other's arithmetic
        const int team = (warp - kWgFirstWorker) >> 2;
        const uint32_t leader_xf = map_to_rank(xf_bar(0), 0), leader_freed = map_to_rank(freed_bar(0), 0);
        RingAt<kStages> raw;
        RingAt<kX> x;
        RingAt<kXBars> xe;
        int c = 0, stage = 0;
        for (int t = pair; t < tiles; t += p.pairs) {
            const WgradItem item(p, t);
            const int steps_of = item.last - item.first;
            const TeamPlace place(threadIdx.x & 127, ((item.kt * kWgTile + rank * 128) / 32) & 15, kWgCodes, kWgScales, 0);
            float sum[kWgPairOwn];
#pragma unroll
            for (int j = 0; j < kWgPairOwn; ++j) sum[j] = 0.0f;
            const int c_first = c;
            for (int b = 0; b < steps_of; ++b) {
                if (!X16) {
                    if (stage % kWgPairTeams == team) {
                        const bool wrap = xe.s < kX;            // step - kX: its barrier, and whether that lies in the round before
                        if (stage >= kX && !mbar_wait_warp(lane == 0 ? 1u : 0u, x_empty_bar(wrap ? xe.s + kXBars - kX : xe.s - kX), wrap ? xe.ph ^ 1u : xe.ph, abort_flag, g.status, g.wait_limit)) return;
                        if (!mbar_wait_warp(lane == 0 ? 1u : 0u, raw_bar(raw.s), raw.ph, abort_flag, g.status, g.wait_limit)) return;
                        transform_stage(smem + (uint32_t)(raw.s * kStage), x_stage(x.s), place);
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_remote(leader_xf + 8u * (uint32_t)x.s);
                    }
                    ++stage;
                    raw.next();
                    x.next();
                    xe.next();
                }
                if ((b & (kWgChunkSteps - 1)) == kWgChunkSteps - 1 && b < steps_of - 1) {
                    if (c > c_first) add_chunk(g, c - 1, leader_freed, sum);
                    ++c;
                }
            }
            if (c > c_first) add_chunk(g, c - 1, leader_freed, sum);
            add_chunk(g, c, leader_freed, sum);
            ++c;
            write(p, item, sum);
        }
    }
};

template <bool X16>
__global__ void __launch_bounds__(kWgPairThreads, 1)
sparq_wgrad_kernel(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_codes,
                   const __grid_constant__ CUtensorMap map_scales, const WgradPairArgs p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) WgradBars room;
    __shared__ uint32_t tmem_base_slot;
    __shared__ uint32_t abort_word;
    __shared__ volatile uint32_t issued[5];

    using Cta = WgradPair<X16>;
    Cta c;
    const int warp = c.warp = threadIdx.x >> 5, lane = c.lane = threadIdx.x & 31;
    c.abort_flag = &abort_word;
    c.issued = issued;
    c.smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    c.bars = smem_u32(&room);
    c.rank = (int)(blockIdx.x & 1u);
    c.pair = (int)(blockIdx.x >> 1);
    c.tiles = (p.skip ? 0 : p.whole) + (p.n_tiles * p.k_tiles - p.whole) * p.g.count;

    if (warp == 0) {
        if (lane == 0) {
            prefetch_tensormap(&map_dy);
            prefetch_tensormap(&map_codes);
            prefetch_tensormap(&map_scales);
            for (int s = 0; s < Cta::kStages; ++s) {
                mbar_init(c.full_bar(s), 1);
                mbar_init(c.raw_bar(s), 1);
                mbar_init(c.empty_bar(s), 1);
            }
            for (int q = 0; q < Cta::kX; ++q) mbar_init(c.xf_bar(q), 2 * 4);         // a team of each CTA
            for (int q = 0; q < Cta::kXBars; ++q) mbar_init(c.x_empty_bar(q), 1);
            for (int b = 0; b < 2; ++b) {
                mbar_init(c.acc_bar(b), 1);
                mbar_init(c.freed_bar(b), 2 * kWgPairWorkers);
            }
            abort_word = 0;
            for (int q = 0; q < 5; ++q) issued[q] = X16 || (q & 1) == 0 ? kStillIssuing : 0;
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
    // Registers: 384 threads were launched with 168 each; of the same 64512, the workers take 224 and the first four warps 56.
    if (warp >= kWgFirstWorker) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        c.work(p);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        switch (warp) {
        case 0: c.template produce<true>(map_dy, map_dy, p); break;
        case 1: c.issue(p); break;
        case kWgCodeWarp: c.template produce<false>(map_codes, map_scales, p); break;
        default: break;
        }
    }
    // Neither CTA leaves, or gives its tensor memory back, while the pair's MMAs, the other's arrivals or a copy may reach it.
    tc_fence_before();
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    // (The leader waited for the copies on its barriers.  Those of codes and scales are each CTA's own.)
    if (!X16 && threadIdx.x == 32 * 3 && *c.abort_flag) drain_ring(c.raw_bar(0), Cta::kStages, issued[4], c.abort_flag, p.g.status, p.g.wait_limit);
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(c.tmem), "r"(512u) : "memory");
    }
}

// dw += the sums of the tail's later parts, one after the other; a block takes kWgAddRows rows of a tile.
constexpr int kWgAddRows = 4;
__global__ void __launch_bounds__(kWgTile)
wgrad_add_tail_kernel(const WgradPairArgs p)
{
    const int per_tile = kWgTile / kWgAddRows, at = (int)blockIdx.x / per_tile, row = ((int)blockIdx.x - at * per_tile) * kWgAddRows;
    int nt, kt;
    wgrad_tile(p.n_tiles, p.k_tiles, p.whole + at, nt, kt);
    const int64_t n = (int64_t)nt * kWgTile + row, k = (int64_t)kt * kWgTile + threadIdx.x, part = (int64_t)(p.n_tiles * p.k_tiles - p.whole) * kWgTile * kWgTile;
    const float *from = p.tail_sums + ((int64_t)at * kWgTile + row) * kWgTile + threadIdx.x;
    float *dw = p.g.dw + n * p.g.K + k;
    dep_wait();
    dep_launch();
    if (k >= p.g.K) return;
    float a[kWgAddRows];
#pragma unroll
    for (int r = 0; r < kWgAddRows; ++r) a[r] = n + r < p.g.N ? dw[r * p.g.K] : 0.0f;
#pragma unroll 4
    for (int q = 1; q < p.g.parts; ++q, from += part)
#pragma unroll
        for (int r = 0; r < kWgAddRows; ++r) a[r] = __fadd_rn(a[r], n + r < p.g.N ? from[r * kWgTile] : 0.0f);
#pragma unroll
    for (int r = 0; r < kWgAddRows; ++r)
        if (n + r < p.g.N) dw[r * p.g.K] = a[r];
}

// dw (+)= the parts' sums, one after the other.
__global__ void __launch_bounds__(256)
wgrad_add_parts_kernel(const float *sums, int64_t count, int parts, int accumulate, float *dw)
{
    const bool vec = (count & 3) == 0 && (reinterpret_cast<uintptr_t>(dw) & 15u) == 0;
    const int64_t stride = (int64_t)gridDim.x * 256 * (vec ? 4 : 1);
    dep_wait();
    dep_launch();
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * (vec ? 4 : 1); i < count; i += stride) {
        if (vec) {
            float4 a = *reinterpret_cast<const float4 *>(accumulate ? dw + i : sums + i);
#pragma unroll 4
            for (int p = accumulate ? 0 : 1; p < parts; ++p) {
                const float4 v = *reinterpret_cast<const float4 *>(sums + p * count + i);
                a = make_float4(__fadd_rn(a.x, v.x), __fadd_rn(a.y, v.y), __fadd_rn(a.z, v.z), __fadd_rn(a.w, v.w));
            }
            *reinterpret_cast<float4 *>(dw + i) = a;
        } else {
            float a = accumulate ? dw[i] : sums[i];
            for (int p = accumulate ? 0 : 1; p < parts; ++p) a = __fadd_rn(a, sums[p * count + i]);
            dw[i] = a;
        }
    }
}

}  // namespace sparq
