// Tensor-core instructions of the microscaled contractions: block-scaled 4-bit products (kind::mxf4, kind::mxf4nvf4)
// with their scales in tensor memory, and bf16 products of operands that lie along the output axes.
#pragma once

#include "sparq_gemm_kernel.cuh"
#include "sparq_gemm_small_kernel.cuh"
#include "sparq_mx.cuh"

namespace sparq {

constexpr int kMxBK = 128;               // bytes of a row per reduction step: 256 4-bit elements, four MMAs of 64
constexpr int kMxSteps = 4;
constexpr int kScaleTile = 512;          // 128 rows x 4 scales
// Scale tiles of 128 rows per reduction step.
__host__ __device__ constexpr int scale_tiles(bool nv) { return nv ? 4 : 2; }

// Scales of 128 rows from shared memory (32 rows of 16 bytes, 8-row groups back to back) into four columns of
// tensor memory, the same in every lane quarter.
__device__ __forceinline__ uint64_t scale_desc(uint32_t saddr)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
}
// (This and the instructions below are for a warp that runs its loop converged, as tc_mma_i8_if: one lane issues.  A step's MMAs issued
// inside a branch of that lane took 340 cycles, their operands moved to the uniform registers one by one.)
__device__ __forceinline__ void tc_copy_scales(uint32_t taddr, uint64_t desc, uint32_t elected)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}"
                 :: "r"(taddr), "l"(desc), "r"(elected) : "memory");
}

// Instruction descriptor of a block-scaled product of e2m1 operands; MXFP4 (e8m0 scales) uses the bytes sf, sf + 1 of each
// scale word, NVFP4 all four.
__device__ __forceinline__ constexpr uint32_t make_idesc_f4(int n, int m, bool nv, uint32_t sf)
{
    return (sf << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((nv ? 0u : 1u) << 23) | ((uint32_t)(m >> 4) << 24) | (sf << 29);
}

// D[tmem] (+)= (A * scales) (B * scales), 64 elements of the reduction.
template <bool NV>
__device__ __forceinline__ void tc_mma_f4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate,
                                               uint32_t elected)
{
    if (NV)
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(elected) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(elected) : "memory");
}

// bf16 operands whose rows run along the reduction axis in memory (MN-major): 64 elements of the output axis are a 128-byte
// row, swizzled; 8 reduction steps are 1024 bytes, the next 64 elements `block` bytes further.
__device__ __forceinline__ uint64_t mn_major_desc(uint32_t saddr, uint32_t block)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(block >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | (2ull << 61);
}
__device__ __forceinline__ constexpr uint32_t make_idesc_bf16_mn(int n, int m)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void tc_mma_bf16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate, uint32_t elected)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
}
// 16 columns of each lane's row.
__device__ __forceinline__ void tmem_ld_32x16_issue(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}

// Contiguous bytes (16-byte aligned at both ends) into shared memory.
__device__ __forceinline__ void tma_load_bytes(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

__host__ __device__ constexpr int tmem_columns(int want) { return want <= 32 ? 32 : want <= 64 ? 64 : want <= 128 ? 128 : want <= 256 ? 256 : 512; }

// mbar_wait of a converged warp through one of its lanes.  Every lane's own look at a barrier, complete or not, takes its turn: about
// 130 cycles for 32 of them, which in a loop of a few hundred cycles is what the loop takes.  The lanes decide together, by votes, so
// that the warp stays converged for the instructions behind the wait that need it to be; __syncwarp makes what the one lane has
// seen come before what the others do.
__device__ __forceinline__ bool mbar_try_wait_of(uint32_t mine, uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 q, %3, 0;\n\t"
        "setp.ne.b32 p, 0, 0;\n\t"
        "@q mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity), "r"(mine) : "memory");
    const bool any = __any_sync(0xFFFFFFFFu, ok);
    __syncwarp();
    return any;
}
__device__ __forceinline__ bool mbar_wait_warp(uint32_t mine, uint32_t bar, uint32_t parity, volatile uint32_t *abort_flag, unsigned int *status,
                                               long long limit_cycles)
{
    if (mbar_try_wait_of(mine, bar, parity)) return true;
    if (__any_sync(0xFFFFFFFFu, *abort_flag != 0u)) return false;
    const long long t0 = clock64();
    for (uint32_t it = 1;; ++it) {
        if (mbar_try_wait_of(mine, bar, parity)) return true;
        if ((it & 0x3Fu) == 0) {
            if (__any_sync(0xFFFFFFFFu, *abort_flag != 0u)) return false;
            if (__any_sync(0xFFFFFFFFu, clock64() - t0 > limit_cycles)) {
                if (mine) {
                    *abort_flag = 1u;
                    atomicOr(status, 1u);
                }
                __syncwarp();
                return false;
            }
        }
    }
}

// ---- after a wait that gave up -------------------------------------------------------------------------
// No copy may land when its CTA has left.  So no stage is released that has not landed whole: an issuer or a team whose wait gave up stops, and
// the producers come to a stand a ring behind the last release, at most.  Each says how many stages it issued, and what is on its way is
// waited for.  Where several producers count on one barrier, a stage that only some of them came to would never complete: the issuer, if it
// gave up, makes up for what the others owe it.  (One that did not give up has seen every stage land.  All of it behind the barrier at the
// kernel's end: 0.1 us of every launch of a product.)
constexpr uint32_t kStillIssuing = 0xFFFFFFFFu;

// The last of `n` stages in a ring of S barriers from `bar` on, all of whose producers came to them.
__device__ __forceinline__ void drain_ring(uint32_t bar, uint32_t S, uint32_t n, volatile uint32_t *abort_flag, unsigned int *status, long long limit)
{
#pragma unroll 1
    for (uint32_t j = n > S ? n - S : 0; j < n; ++j) mbar_wait(bar + 8u * (j % S), j / S & 1u, abort_flag, status, limit, true);
}
// Stages of the producer that issued most; kStillIssuing if one has not stopped within the limit.
__device__ __forceinline__ uint32_t most_issued(const volatile uint32_t *issued, int producers, long long limit)
{
    const long long t0 = clock64();
    uint32_t n;
    do {
        n = 0;
#pragma unroll 1
        for (int p = 0; p < producers; ++p) n = issued[p] > n ? issued[p] : n;
    } while (n == kStillIssuing && clock64() - t0 <= limit);
    return n;
}
// Two producers of one CTA that both arrive on a stage's barrier.
__device__ __forceinline__ void drain_two(uint32_t bar, uint32_t S, const volatile uint32_t *issued, volatile uint32_t *abort_flag, unsigned int *status,
                                          long long limit)
{
    const uint32_t n = most_issued(issued, 2, limit);
    if (n == kStillIssuing) return;
#pragma unroll 1
    for (uint32_t j = issued[0] < issued[1] ? issued[0] : issued[1]; j < n; ++j) mbar_arrive(bar + 8u * (j % S));
    drain_ring(bar, S, n, abort_flag, status, limit);
}

// ---- CTA pairs (cta_group::2): one MMA over the operands and tensor memory of both ---------------------
// The even CTA of the pair (the leader) issues; A's and D's rows and B's rows are halved between the two.

// A box into this CTA's shared memory that counts on the leader's barrier (an address from map_to_rank).
__device__ __forceinline__ void tma_load_pair_2d(uint32_t dst, const CUtensorMap *map, uint32_t leader_bar, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 :: "r"(dst), "l"(map), "r"(leader_bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tma_load_pair_3d(uint32_t dst, const CUtensorMap *map, uint32_t leader_bar, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 :: "r"(dst), "l"(map), "r"(leader_bar), "r"(x), "r"(y), "r"(z) : "memory");
}
// Arrives on the same barrier of both CTAs once the MMAs before it have retired.
__device__ __forceinline__ void tc_commit_pair(uint32_t bar, uint32_t elected)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
                 "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
                 :: "r"(bar), "h"((uint16_t)3), "r"(elected) : "memory");
}
// Four producers, two of each CTA, whose copies count on the leader's barriers: bytes 0 and 2 of a stage from producers 0 and 2 (one of each
// CTA), bytes 1 from 1 and 3.  Producer 0, the leader's, announces a stage's bytes for all of them.
__device__ __forceinline__ void mbar_complete_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void drain_pair(uint32_t bar, uint32_t S, const volatile uint32_t *issued, uint32_t bytes0, uint32_t bytes1,
                                           volatile uint32_t *abort_flag, unsigned int *status, long long limit)
{
    const uint32_t n = most_issued(issued, 4, limit);
    if (n == kStillIssuing) return;
#pragma unroll 1
    for (uint32_t j = n > S ? n - S : 0; j < n; ++j) {
        uint32_t on_way = 0;
#pragma unroll 1
        for (int p = 0; p < 4; ++p)
            if (j < issued[p]) on_way += p & 1 ? bytes1 : bytes0;
        const uint32_t at = bar + 8u * (j % S), owed = 2 * (bytes0 + bytes1) - on_way;
        if (j >= issued[0]) mbar_expect_tx(at, on_way);
        else if (owed) mbar_complete_tx(at, owed);
        mbar_wait(at, j / S & 1u, abort_flag, status, limit, true);
    }
}
// A word of another CTA of the cluster (an address from map_to_rank).
__device__ __forceinline__ void store_remote(uint32_t dst, uint32_t v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" :: "r"(dst), "r"(v) : "memory");
}
__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" :: "r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void tc_copy_scales_pair(uint32_t taddr, uint64_t desc, uint32_t elected)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}"
                 :: "r"(taddr), "l"(desc), "r"(elected) : "memory");
}
template <bool NV>
__device__ __forceinline__ void tc_mma_f4_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate,
                                               uint32_t elected)
{
    if (NV)
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(elected) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(elected) : "memory");
}
__device__ __forceinline__ void tc_mma_bf16_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate, uint32_t elected)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
}

// Clusters of 1, 2, 4 and 8 CTAs, one CTA on each SM, that run at once on an SM count like the B200's (148, 74, 33, 15: clusters stay
// within a group of SMs).  On a few SMs (a process may be given a share of them) 0 for sizes that do not fit.
inline int clusters_at_once(int split, int sms) { return split == 1 ? sms : split == 2 ? sms / 2 : split == 4 ? sms * 33 / 148 : sms * 15 / 148; }

// Barriers of a CTA, in shared memory.
struct MxBars {
    uint64_t full[kMaxStages], empty[kMaxStages], xf[kMaxStages], acc[2], freed[2], recv;
};

// One CTA's view of its work; the roles of its warps.
struct MxCta {
    uint32_t smem, bars, tmem;          // operand ring (1024-byte aligned), MxBars, accumulator
    volatile uint32_t *abort_flag, *issued;     // issued: stages of each producer that has stopped; in pairs the leader's words count
    int warp, lane, S, rank, steps;
    uint32_t split;
    __device__ uint32_t full_bar(int s) const { return bars + (uint32_t)s * 8u; }
    __device__ uint32_t empty_bar(int s) const { return bars + (uint32_t)(kMaxStages + s) * 8u; }
    __device__ uint32_t xf_bar(int s) const { return bars + (uint32_t)(2 * kMaxStages + s) * 8u; }
    __device__ uint32_t acc_bar(int i = 0) const { return bars + (uint32_t)(3 * kMaxStages + i) * 8u; }
    __device__ uint32_t freed_bar(int i) const { return bars + (uint32_t)(3 * kMaxStages + 2 + i) * 8u; }
    __device__ uint32_t recv_bar() const { return bars + (uint32_t)(3 * kMaxStages + 4) * 8u; }
};

__device__ __forceinline__ void mx_wait_landed(const MxCta &c, unsigned int *status, long long limit)
{
    mbar_wait(c.recv_bar(), 0, c.abort_flag, status, limit, true);
}

}  // namespace sparq
