// Linear layers in bf16 and fp16 (sparq_linear): out[m][n] = act(sum_k x[m][k] w[n][k] + bias[n]) + residual[m][n], dense or with a
// weight matrix for each expert's run of rows; w as N x K, or as K x N (a layer's own weights in the product of its input's gradient).
//
// A persistent pair of CTAs walks tiles of 256 x 256: one MMA (cta_group::2) multiplies 256 rows of x by 256 columns, each CTA holds half
// of either operand and its 128 rows of the accumulator, in tensor memory beside that of the next tile.
//
// 16384 x 4096 x 4096 bf16 340 to 354 us in runs of milliseconds (1.55 to 1.62 PFLOP/s, one library product 334 to 350), 404 under the power cap (401); with bias, GELU and
// a residual 362 and 438: what bounds it there is the cap.  Short sums are bound by the epilogue, two warps a scheduler whose stalls are dependent
// instructions and instruction fetches: 8192 x 4096 x 1024 50 us, with SiLU 53, with z kept as well, the sum in three pieces, 73.  (Sixteen epilogue warps, for which the ring gives up
// a stage: 359 instead of 346, and z kept no faster.)
#pragma once

#include "sparq_act.cuh"
#include "sparq_half.cuh"
#include "sparq_mxf4_small_kernel.cuh"

namespace sparq {

struct LinArgs {
    int64_t M, N;
    int k_mmas, k_blocks;               // reduction steps of 16 and of 64
    int piece;                          // steps of 64 whose sum tensor memory holds without rounding to nearest
    const int32_t *offsets;             // of experts' rows, or nullptr
    int groups;
    int bf16;                           // operands: bf16, else fp16
    const float *bias;
    int act;
    const void *residual;
    int64_t ldr;
    void *out;
    int64_t ldo;
    int8_t *z_codes;
    uint8_t *z_scales;
    int64_t z_pitch, z_spitch;
    int staged;                         // out goes through shared memory in boxes: its rows start on 16-byte boundaries
    unsigned int *status;
    long long wait_limit;
    int n_tiles, units;                 // column tiles; pairs that walk tiles
};

constexpr int kLinBK = 64;              // elements of the reduction per step: 128 bytes, four MMAs of 16
constexpr int kLinSteps = 4;

// Instruction descriptor of a product of 16-bit operands with fp32 sums; *_mn: the operand's rows run along the reduction axis in memory.
__device__ __forceinline__ constexpr uint32_t make_idesc_16(int n, int m, uint32_t bf16, bool a_mn, bool b_mn)
{
    return (1u << 4) | (bf16 << 7) | (bf16 << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// ---- sums in pieces ------------------------------------------------------------------------------------
// The tensor cores cut a running sum off where fp32 would round it, so that its error grows with the number of additions and has a sign.  A sum therefore runs over a piece of K in
// tensor memory, and pieces are added rounded to nearest in the registers of the warps that need the sum, while the next piece runs in another accumulator.
//
// What a cut-off piece of P terms of mixed signs is off by grows with P, what an fp32 sum of K terms is off by with the root of K.  Sums that fp32 outputs or kept z show take pieces of 12 sqrt(K)
// elements, 1024 at the most (terms of one sign lose up to P / 16 units of 2^-23): fp32 outputs are 1.0 to 1.5 times as far off as an fp32 product, z in 8 bits 1.0 to 1.3 times (K = 64 to 8192; in one piece
// 1.2 to 9.5 and 1.0 to 3.4 times).  16-bit outputs show none of this: pieces of 8192, which lose 2^-14 at the most, a quarter of the least half step that they are rounded by
// (fp16, 2^-12).
inline int lin_piece(int64_t K, bool shown)
{
    if (!shown) return 8192 / kLinBK;
    int p = 1;
    while (p < 1024 / kLinBK && (int64_t)(p + 1) * (p + 1) * 256 <= 9 * K) ++p;        // (64 p = 12 sqrt(K))
    return p;
}

// C columns of a lane, a multiple of 32, or 16, of the `pieces` pieces from the CTA's n-th on, added up: at(b, h) is where the columns from h on of accumulator b are, freed(b) hands b back.
template <int C, class Cta, class At, class Freed>
__device__ __forceinline__ void lin_add_pieces(const Cta &c, const LinArgs &g, int pieces, int &n, float (&sum)[C], const At &at, const Freed &freed)
{
    constexpr int kAtOnce = C < 32 ? 1 : C < 64 ? 2 : 4;       // loads of 16 columns in flight
    auto piece = [&](auto first) {
        mbar_wait(c.acc_bar(n & 1), (uint32_t)(n >> 1) & 1u, c.abort_flag, g.status, g.wait_limit);
        __syncwarp();
        tc_fence_after();
#pragma unroll
        for (int h = 0; h < C; h += 16 * kAtOnce) {
            uint32_t v[kAtOnce][32];
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) tmem_ld_32x16_issue(at(n & 1, h + 16 * q), v[q]);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16 * kAtOnce; ++j) {
                const float p = __uint_as_float(v[j / 16][j % 16]);
                sum[h + j] = decltype(first)::value ? p : __fadd_rn(sum[h + j], p);
            }
        }
        tc_fence_before();
        __syncwarp();
        if (c.lane == 0) freed(n & 1);
        __syncwarp();
        ++n;
    };
    piece(std::true_type{});
#pragma unroll 1
    for (int p = 1; p < pieces; ++p) piece(std::false_type{});
}

// ---- tiles of experts' rows ----------------------------------------------------------------------------
// Rows first .. end - 1 of an expert: bounds outside the tensor are taken as the nearest within, falling ones as those of no rows.
__device__ __forceinline__ void expert_rows(const int32_t *offsets, int groups, int64_t M, int e, int64_t &first, int64_t &end)
{
    first = end = 0;
    if (e >= groups) return;
    const int64_t a = offsets[e], b = offsets[e + 1];
    first = a < 0 ? 0 : a > M ? M : a;
    end = b < first ? first : b > M ? M : b;
}

struct LinTile {
    int e, nt;
    int64_t m0, end;            // first row, end of the expert's rows
};

// Tiles of ROWS rows and a column tile, expert by expert, within one eight rows of tiles at a time: their operands and the column's stay
// in L2.  A warp asks for rising tile numbers, all lanes together: each lane has one expert of a block of 32.  (Runs that overlap may make more
// tiles than there can be; numbers stop at kMostTiles, which no launch comes to otherwise.)
constexpr uint32_t kMostTiles = 1u << 30;
template <int ROWS>
struct LinWalk {
    const LinArgs &g;
    int lane, block;
    uint32_t base, tiles, incl, all;
    int64_t first, end;
    __device__ LinWalk(const LinArgs &g_, int lane_) : g(g_), lane(lane_), block(0), base(0u) { load(); }
    __device__ static uint32_t most(uint64_t v) { return v < kMostTiles ? (uint32_t)v : kMostTiles; }
    __device__ void load()
    {
        if (g.offsets) {
            expert_rows(g.offsets, g.groups, g.M, block * 32 + lane, first, end);
        } else {
            first = 0;
            end = lane == 0 ? g.M : 0;
        }
        tiles = most((uint64_t)((end - first + ROWS - 1) / ROWS) * (uint32_t)g.n_tiles);
        incl = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl = most(incl + v);
        }
        all = __shfl_sync(0xFFFFFFFFu, incl, 31);
    }
    __device__ bool find(uint32_t t, LinTile &out)
    {
        while (t >= base + all) {
            base = most(base + all);
            all = 0u;
            if (t >= kMostTiles || !g.offsets || ++block * 32 >= g.groups) {
                block = g.groups;
                return false;
            }
            load();
        }
        const int at = __popc(__ballot_sync(0xFFFFFFFFu, base + incl <= t));
        const uint32_t before = __shfl_sync(0xFFFFFFFFu, incl, at > 0 ? at - 1 : 0);
        const int in = (int)(t - base - (at > 0 ? before : 0u));
        const int64_t row = __shfl_sync(0xFFFFFFFFu, first, at);
        out.e = block * 32 + at;
        out.end = __shfl_sync(0xFFFFFFFFu, end, at);
        const int m_tiles = (int)((out.end - row + ROWS - 1) / ROWS), per_group = 8 * g.n_tiles, group = in / per_group;
        const int rows = m_tiles - group * 8 < 8 ? m_tiles - group * 8 : 8, in_group = in - group * per_group;
        out.nt = in_group / rows;
        out.m0 = row + (int64_t)(group * 8 + in_group - out.nt * rows) * ROWS;
        return true;
    }
};

// ---- epilogue ----------------------------------------------------------------------------------------------

// SILU and GELU of C columns of a lane's row beside 16-bit outputs.  Powers of two and reciprocals share one unit, 16 lanes a cycle, which is what these functions wait for;
// two reciprocals come from one: 1 / a = b / (a b).  That is in range for z above -43 (a = 1 + exp(-z) below 2^63); a lane that holds lesser ones, or NaN, which would go from one
// to the other, takes the functions one by one.  (Each lane for itself: a row's bits depend on no other row, and on nothing that lies where there is none.)
template <int ACT, int C>
__device__ __forceinline__ void lin_logistic(float (&y)[C])
{
    static_assert(C % 2 == 0, "pairs");
    float least = 0.0f;
#pragma unroll
    for (int j = 0; j < C; j += 2) asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(least) : "f"(least), "f"(y[j]), "f"(y[j + 1]));
    // (gelu's argument is above -43 down to -7.5; both rise with y)
    if (!(least >= (ACT == SPARQ_ACT_SILU ? -43.0f : -7.5f))) {
#pragma unroll
        for (int j = 0; j < C; ++j) y[j] = act_value<true, ACT>(y[j]);
    } else {
#pragma unroll
        for (int j = 0; j < C; j += 2) {
            float a[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float e;
                asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(__fmul_rn(act_argument<ACT>(y[j + q]), -1.4426950408889634f)));
                a[q] = __fadd_rn(1.0f, e);
            }
            const float r = reciprocal(__fmul_rn(a[0], a[1]));
            y[j] = __fmul_rn(y[j], __fmul_rn(a[1], r));
            y[j + 1] = __fmul_rn(y[j + 1], __fmul_rn(a[0], r));
        }
    }
    __syncwarp();
}

// A warp's lanes call it together.  ROW: the values are columns of one row (else rows of one column, and each is taken by itself).
template <bool FAST, bool ROW, int C>
__device__ __forceinline__ void lin_act(float (&y)[C], int act)
{
    if (act == SPARQ_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < C; ++j) y[j] = act_value<FAST, SPARQ_ACT_RELU>(y[j]);
    } else if (act == SPARQ_ACT_SILU) {
        if (FAST && ROW) {
            lin_logistic<SPARQ_ACT_SILU>(y);
        } else {
#pragma unroll
            for (int j = 0; j < C; ++j) y[j] = act_value<FAST, SPARQ_ACT_SILU>(y[j]);
        }
    } else if (act == SPARQ_ACT_GELU) {
        if (FAST && ROW) {
            lin_logistic<SPARQ_ACT_GELU>(y);
        } else {
#pragma unroll
            for (int j = 0; j < C; ++j) y[j] = FAST ? act_value<FAST, SPARQ_ACT_GELU>(y[j]) : gelu_exact(y[j]);
        }
    }
}

// 32 columns from n on of a row as one block of MXINT8: its codes go out, its scale comes back.  Columns past N hold zeros.
__device__ __forceinline__ uint32_t lin_keep(const LinArgs &g, const float (&z)[32], int64_t row, int64_t n)
{
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < 32; j += 2) asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(top) : "f"(top), "f"(z[j]), "f"(z[j + 1]));
    const uint32_t mb = __float_as_uint(top) & 0x7FFFFFFFu, code = e8m0_code(mb, 0u);
    uint32_t w[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float f[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) f[j] = z[16 * h + j];
        const uint4 c = int8_codes(f, code, mb);
        w[4 * h] = c.x;
        w[4 * h + 1] = c.y;
        w[4 * h + 2] = c.z;
        w[4 * h + 3] = c.w;
    }
    if (mb >= kInfBits) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 0u;
    }
    int8_t *const to = g.z_codes + row * g.z_pitch + n;
    if (reinterpret_cast<uintptr_t>(to) & 16u) {        // (32 bytes at once: half the lines that a store of 32 rows goes to)
        st_v4(to, w);
        st_v4(to + 16, w + 4);
    } else {
        st_v8(to, w);
    }
    return code;
}

// Scales of BLOCKS neighbouring blocks of a row, the first of columns n on (a multiple of 32 BLOCKS): at once, those of blocks past N as the zeros of the
// padding, and all of the padding behind the row's last one.
template <int BLOCKS>
__device__ __forceinline__ void lin_keep_scales(const LinArgs &g, uint32_t codes, int64_t row, int64_t n)
{
    uint8_t *const at = g.z_scales + row * g.z_spitch + n / 32;
    if (BLOCKS == 4) *reinterpret_cast<uint32_t *>(at) = codes;
    else if (BLOCKS == 2) *reinterpret_cast<uint16_t *>(at) = (uint16_t)codes;
    else *at = (uint8_t)codes;
    if (n + 32 * BLOCKS >= g.N)
        for (int64_t c = n / 32 + BLOCKS; c < g.z_spitch; ++c) at[c - n / 32] = 0;
}

// A lane's column of a block of 32 biases.
__device__ __forceinline__ float lin_bias(const LinArgs &g, int e, int64_t n)
{
    const int64_t at = n + (threadIdx.x & 31);
    return g.bias && at < g.N ? __ldg(g.bias + e * g.N + at) : 0.0f;
}

// z and act(z) of 32 columns from n on; a warp's lanes call it together, each with the bias of a column.  (Every lane's own loads of all of them came from L2, nothing of it being
// left to L1: 1100 cycles a block.)
template <bool F32, bool KEEP>
__device__ __forceinline__ void lin_value(const LinArgs &g, float (&y)[32], const uint32_t (&v)[32], float bias, int64_t row, bool live, int64_t n, uint32_t &scale)
{
#pragma unroll
    for (int j = 0; j < 32; ++j) y[j] = __uint_as_float(v[j]);
    if (g.bias) {
#pragma unroll
        for (int j = 0; j < 32; ++j) y[j] = __fadd_rn(y[j], __shfl_sync(0xFFFFFFFFu, bias, j));
    }
    if (KEEP && live && n < g.N) scale = lin_keep(g, y, row, n);
    lin_act<!F32, true>(y, g.act);
}

// The residual of 32 rows x 128 bytes: read in whole vectors (of rows that start anywhere shifted into place), handed to each lane its row
// through the warp's staging memory.  Columns from `last` on are not looked at.
template <bool F32>
struct LinFetch {
    static constexpr int width = F32 ? 4 : 2, per = 16 / width;
    uint32_t v[8][4];
    __device__ void issue(const LinArgs &g, int64_t m, int rows, int64_t n, int64_t last)
    {
        const int lane = threadIdx.x & 31;
        const uint8_t *const begin = reinterpret_cast<const uint8_t *>(g.residual), *const behind = begin + ((g.M - 1) * g.ldr + g.N) * width;
        const bool vec = ((reinterpret_cast<uintptr_t>(begin) | (uintptr_t)(g.ldr * width)) & 15u) == 0;
        const int64_t col = n + (lane & 7) * per, left = last - col;
        const uint8_t *p = begin + ((m + lane / 8) * g.ldr + col) * width;
#pragma unroll
        for (int i = 0; i < 8; ++i, p += 4 * g.ldr * width) {
            v[i][0] = v[i][1] = v[i][2] = v[i][3] = 0u;
            if (i * 4 + lane / 8 >= rows || left <= 0) continue;
            const uint32_t s = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15u;
            if (vec && left >= per) {
                ld_v4(v[i], p);
            } else if (left >= per && p - s >= begin && p - s + 32 <= behind) {
                uint32_t w[8];
                ld_v4(w, p - s);
                ld_v4(w + 4, p - s + 16);
                shift_words<!F32, 4>(w, s);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][j] = w[j];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (F32) {
                        if (j < left) v[i][j] = reinterpret_cast<const uint32_t *>(p)[j];
                    } else {
                        if (2 * j < left) v[i][j] = reinterpret_cast<const uint16_t *>(p)[2 * j];
                        if (2 * j + 1 < left) v[i][j] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[2 * j + 1] << 16;
                    }
                }
            }
        }
    }
    // Into the staging memory, which is free.
    __device__ void land(uint32_t stage) const
    {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = i * 4 + lane / 8;
            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" :: "r"(stage + (uint32_t)(r * 128 + (((lane & 7) ^ (r & 7)) << 4))), "r"(v[i][0]), "r"(v[i][1]),
                         "r"(v[i][2]), "r"(v[i][3]) : "memory");
        }
        __syncwarp();
    }
};

// Words 4 c .. 4 c + 3 of a lane's row of 128 bytes in the staging memory.
__device__ __forceinline__ uint32_t lin_chunk(uint32_t stage, int c)
{
    const uint32_t lane = threadIdx.x & 31;
    return stage + lane * 128u + (((uint32_t)c ^ (lane & 7u)) << 4);
}
__device__ __forceinline__ void lin_stage_free()
{
    if ((threadIdx.x & 31) == 0) tma_store_wait_read<0>();        // the box before has left
    __syncwarp();
}

// `rows` rows of `bytes` bytes (128 at the most) from the staging memory to `out`: whole vectors that start on 16-byte boundaries, shifted into
// place, eight lanes to a row; what is left in front of them and behind them in pieces of 8, 4 and 2 bytes, a row to each lane.  (Element by element, one load and
// store after the other: 3500 cycles.)
template <bool F32>
__device__ __forceinline__ void lin_flush_rows(uint8_t *out, int64_t pitch, uint32_t stage, int rows, int bytes)
{
    constexpr int width = F32 ? 4 : 2;
    const int lane = threadIdx.x & 31, c = lane & 7;
    auto chunk = [&](int r, int at) { return stage + (uint32_t)(r * 128 + ((at ^ (r & 7)) << 4)); };
    auto load = [&](uint32_t *w, uint32_t from) { asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from)); };
    __syncwarp();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t w[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (4 * h + i) * 4 + lane / 8;
            load(w[i], chunk(r, c));
            load(w[i] + 4, chunk(r, c < 7 ? c + 1 : 7));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (4 * h + i) * 4 + lane / 8;
            uint8_t *const a = out + r * pitch;
            const int s = (int)(reinterpret_cast<uintptr_t>(a) & 15u);
            if (s) shift_words<!F32, 4>(w[i], 16u - (uint32_t)s);
            if (r < rows && 16 * (c + (s ? 2 : 1)) - s <= bytes) st_v4(a + 16 * (c + (s ? 1 : 0)) - s, w[i]);
        }
    }
    uint8_t *const a = out + lane * pitch;
    const uint32_t s = (uint32_t)reinterpret_cast<uintptr_t>(a) & 15u;
    if (bytes == 128) {
        // a vector's bytes s .. 15 in front, bytes 0 .. s - 1 behind
        uint32_t head[8], tail[8];
        load(head + 4, chunk(lane, 0));
        load(tail, chunk(lane, 7));
#pragma unroll
        for (int j = 0; j < 4; ++j) head[j] = tail[4 + j] = 0u;
        shift_words<!F32, 4>(head, (16u - s) & 15u);
        shift_words<!F32, 4>(tail, (16u - s) & 15u);
        if (lane < rows && s) {
            uint8_t *const f = a - s, *const b = a + 128 - s;
            auto put2 = [](uint8_t *to, uint32_t v) { *reinterpret_cast<uint16_t *>(to) = (uint16_t)v; };
            auto put4 = [](uint8_t *to, uint32_t v) { *reinterpret_cast<uint32_t *>(to) = v; };
            auto put8 = [](uint8_t *to, uint32_t v, uint32_t w) { *reinterpret_cast<uint2 *>(to) = make_uint2(v, w); };
            if (s <= 8) put8(f + 8, head[2], head[3]);
            if (s <= 4) put4(f + 4, head[1]);
            else if (s > 8 && s <= 12) put4(f + 12, head[3]);
            if (!F32 && (s & 2u)) put2(a, (s < 4 ? head[0] : s < 8 ? head[1] : s < 12 ? head[2] : head[3]) >> 16);
            if (s >= 8) put8(b, tail[0], tail[1]);
            if (s & 4u) put4(b + (s & 8u), s & 8u ? tail[2] : tail[0]);
            if (!F32 && (s & 2u)) put2(b + (s & 12u), s < 4 ? tail[0] : s < 8 ? tail[1] : s < 12 ? tail[2] : tail[3]);
        }
    } else if (lane < rows) {           // the last columns of a row
        const int at = (int)s, head = at == 0 ? 0 : 16 - at < bytes ? 16 - at : bytes, whole = (bytes + at) / 16 * 16 - at, tail = whole > head ? whole : head;
        auto element = [&](int b) {
            const uint32_t from = chunk(lane, b >> 4) + (uint32_t)(b & 15);
            if (F32) {
                uint32_t v;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(from));
                *reinterpret_cast<uint32_t *>(a + b) = v;
            } else {
                uint16_t v;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(from));
                *reinterpret_cast<uint16_t *>(a + b) = v;
            }
        };
#pragma unroll 1
        for (int b = 0; b < head; b += width) element(b);
#pragma unroll 1
        for (int b = tail; b < bytes; b += width) element(b);
    }
    __syncwarp();
}

// 32 rows x 128 bytes of the output leave the staging memory: as a box, or where rows of the box are another expert's, or rows start
// anywhere, row by row.
template <bool F32>
__device__ __forceinline__ void lin_flush(const CUtensorMap &map, const LinArgs &g, uint32_t stage, int64_t m, int rows, bool clipped, int64_t n)
{
    if (g.staged && (rows >= 32 || clipped)) {
        fence_proxy_async_smem();
        __syncwarp();
        if ((threadIdx.x & 31) == 0 && rows > 0 && n < g.N) {
            tma_store_2d(&map, stage, (int)n, (int)m);
            tma_store_commit();
        }
        return;
    }
    constexpr int width = F32 ? 4 : 2;
    const int bytes = g.N - n < 128 / width ? (int)(g.N - n) * width : 128;
    lin_flush_rows<F32>(reinterpret_cast<uint8_t *>(g.out) + (m * g.ldo + n) * width, g.ldo * width, stage, rows, bytes);
}

// 32 columns of a lane's row, and the residual that lies there, rounded into its pieces c0 .. c0 + 3.
template <bool BF16>
__device__ __forceinline__ void lin_stage_row(const LinArgs &g, float (&y)[32], uint32_t stage, int c0)
{
    if (g.residual) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            uint32_t w[4];
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(lin_chunk(stage, c0 + c)) : "memory");
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float lo = __uint_as_float(w[j] << 16), hi = __uint_as_float(w[j] & 0xFFFF0000u);
                if (!BF16) floats_of_f16x2(w[j], lo, hi);
                y[8 * c + 2 * j] = __fadd_rn(y[8 * c + 2 * j], lo);
                y[8 * c + 2 * j + 1] = __fadd_rn(y[8 * c + 2 * j + 1], hi);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = BF16 ? bf16x2_of(y[8 * c + 2 * j], y[8 * c + 2 * j + 1]) : f16x2_of(y[8 * c + 2 * j], y[8 * c + 2 * j + 1]);
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" :: "r"(lin_chunk(stage, c0 + c)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
}

__device__ __forceinline__ void lin_stage_f32(const LinArgs &g, float (&y)[32], uint32_t stage)
{
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        if (g.residual) {
            float r[4];
            asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]) : "r"(lin_chunk(stage, c)) : "memory");
#pragma unroll
            for (int j = 0; j < 4; ++j) y[4 * c + j] = __fadd_rn(y[4 * c + j], r[j]);
        }
        asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" :: "r"(lin_chunk(stage, c)), "f"(y[4 * c]), "f"(y[4 * c + 1]), "f"(y[4 * c + 2]), "f"(y[4 * c + 3]) : "memory");
    }
}

// 64 columns from n on of a warp's 32 rows from m on, `rows` of them the expert's; `clipped`: those behind them are no
// rows of the output.  `scales`: those of z's two blocks.  `columns(q, v)`: sums of each half, q = 0 and then 1.  (Half a box at a time, one copy of the code: with both halves in registers
// and all of it unrolled, a launch spent microseconds on instruction fetches.)
template <bool F32, bool KEEP, class Columns>
__device__ __forceinline__ void lin_put_span(const CUtensorMap &map, const LinArgs &g, uint32_t stage, int64_t m, int rows, bool clipped, int64_t n,
                                             float bias0, float bias1, LinFetch<F32> &fetch, uint32_t &scales, const Columns &columns)
{
    const int lane = threadIdx.x & 31;
    if (!F32) {
        lin_stage_free();
        if (g.residual) fetch.land(stage);
    }
#pragma unroll 1
    for (int q = 0; q < 2; ++q) {
        uint32_t v[32];
        columns(q, v);
        if (n + 32 * q >= g.N) continue;
        float y[32];
        uint32_t scale = 0u;
        lin_value<F32, KEEP>(g, y, v, q ? bias1 : bias0, m + lane, lane < rows, n + 32 * q, scale);
        if (KEEP) scales |= scale << (8 * q);
        if (F32) {
            lin_stage_free();
            if (g.residual) {
                fetch.issue(g, m, rows, n + 32 * q, g.N);
                fetch.land(stage);
            }
            lin_stage_f32(g, y, stage);
            lin_flush<F32>(map, g, stage, m, rows, clipped, n + 32 * q);
        } else if (g.bf16) {
            lin_stage_row<true>(g, y, stage, 4 * q);
        } else {
            lin_stage_row<false>(g, y, stage, 4 * q);
        }
    }
    if (!F32) lin_flush<F32>(map, g, stage, m, rows, clipped, n);
}

// ---- pairs of CTAs -----------------------------------------------------------------------------------------
// Warps: 0 producer of x, 10 of w, 1 tensor memory and (leader) MMA issue, 2..9 epilogue (lane quarter warp % 4, two spans of 64 columns).
//
// PIECES: the epilogue's warps (4..11; 2 is w's producer, 3 has nothing to do) add the pieces up in registers and go on from there, so that both accumulators are free for the next tile's
// first pieces.  8192 x 4096 x 1024 with z kept 73 us (in one piece 63), fp32 out 75 (62): the third piece runs when the epilogue is over; 16384 x 4096 x 4096 371 (354) and 360 (356).  (The sum back
// in tensor memory: one piece runs beside the epilogue, 96 us in place of 73.  Tiles of 256 x 128, two sums and two pieces in tensor memory, warps of their own for the adding: 91, and a sum of 16384 432 us in
// place of 373.)

constexpr int kLinTile = 256;
constexpr int kLinEpiWarps = 8;
__host__ __device__ constexpr int lin_first_epi(bool pieces) { return pieces ? 4 : 2; }        // (whole groups of four warps, for setmaxnreg)
__host__ __device__ constexpr int lin_weight_warp(bool pieces) { return pieces ? 2 : 2 + kLinEpiWarps; }
__host__ __device__ constexpr int lin_threads(bool pieces) { return 32 * (pieces ? 4 + kLinEpiWarps : 3 + kLinEpiWarps); }
constexpr int kLinHalf = 128 * kLinBK * 2;      // one operand's bytes of a step in one CTA
constexpr int kLinStage = 2 * kLinHalf, kLinStages = 6;
constexpr int kLinSmem = 1024 + kLinStages * kLinStage + kLinEpiWarps * kMxStaging;

// W_KN: w is K x N; its boxes are 64 reduction rows x 64 columns, two for a CTA's 128 columns.
template <bool W_KN, bool F32, bool KEEP, bool PIECES>
struct LinPair : MxCta {
    int pair;

    template <bool X>
    __device__ void produce(const CUtensorMap &map, const LinArgs &g) const
    {
        if (X && lane == 0) dep_launch();
        const uint32_t leader_full = map_to_rank(full_bar(0), 0);
        int s = 0;
        uint32_t ph = 1, n = 0;
        bool live = true;
        LinWalk<kLinTile> walk(g, lane);
        LinTile tile;
        for (uint32_t t = (uint32_t)pair; live && walk.find(t, tile); t += (uint32_t)g.units) {
            if (lane == 0) {
                const int row = (int)(tile.m0 + rank * 128), col = tile.nt * kLinTile + rank * 128;
                for (int kb = 0; kb < g.k_blocks; ++kb) {
                    if (n >= kLinStages && !mbar_wait(empty_bar(s), ph, abort_flag, g.status, g.wait_limit)) { live = false; break; }
                    const uint32_t at = smem + (uint32_t)(s * kLinStage) + (X ? 0u : (uint32_t)kLinHalf), bar = leader_full + 8u * (uint32_t)s;
                    if (X) {
                        if (rank == 0) mbar_expect_tx(full_bar(s), 2 * kLinStage);
                        tma_load_pair_2d(at, &map, bar, kb * kLinBK, row);
                    } else if (W_KN) {
                        tma_load_pair_3d(at, &map, bar, col, kb * kLinBK, tile.e);
                        tma_load_pair_3d(at + kLinHalf / 2, &map, bar, col + 64, kb * kLinBK, tile.e);
                    } else {
                        tma_load_pair_3d(at, &map, bar, kb * kLinBK, col, tile.e);
                    }
                    ++n;
                    if (++s == kLinStages) { s = 0; ph ^= 1u; }
                }
            }
            live = __shfl_sync(0xFFFFFFFFu, live, 0);
        }
        if (lane == 0) store_remote(map_to_rank(smem_u32((const void *)(issued + 2 * rank + (X ? 0 : 1))), 0), n);
        __syncwarp();
    }

    __device__ void issue(const LinArgs &g) const
    {
        if (rank == 0) {
            const uint32_t elected = elect_one(), id = make_idesc_16(kLinTile, 256, (uint32_t)g.bf16, false, W_KN);
            int s = 0, i = 0;           // tiles, or pieces counted through all tiles: the i-th adds up in accumulator i & 1
            uint32_t ph = 0;
            bool live = true;
            LinWalk<kLinTile> walk(g, lane);
            LinTile tile;
            for (uint32_t t = (uint32_t)pair; live && walk.find(t, tile); t += (uint32_t)g.units, ++i) {
                uint32_t d = tmem + (uint32_t)((i & 1) * kLinTile);
                int in = 0;             // steps of the piece
                if (i > 1) live = mbar_wait_warp(elected, freed_bar(i & 1), (uint32_t)((i >> 1) - 1) & 1u, abort_flag, g.status, g.wait_limit);
                if (!live) break;
                for (int kb = 0; kb < g.k_blocks; ++kb, ++in) {
                    if (PIECES && in == g.piece) {
                        tc_commit_pair(acc_bar(i & 1), elected);
                        ++i;
                        in = 0;
                        d = tmem + (uint32_t)((i & 1) * kLinTile);
                        if (i > 1) live = mbar_wait_warp(elected, freed_bar(i & 1), (uint32_t)((i >> 1) - 1) & 1u, abort_flag, g.status, g.wait_limit);
                    }
                    if (live) live = mbar_wait_warp(elected, full_bar(s), ph, abort_flag, g.status, g.wait_limit);
                    if (!live) {
                        tc_commit_pair(acc_bar(i & 1), elected);        // what there is of the tile
                        break;
                    }
                    tc_fence_after();
                    const uint32_t at = smem + (uint32_t)(s * kLinStage);
                    const uint64_t adesc = make_smem_desc<128>(at);
                    const uint64_t bdesc = W_KN ? mn_major_desc(at + kLinHalf, kLinHalf / 2) : make_smem_desc<128>(at + kLinHalf);
                    const int mmas = g.k_mmas - kb * kLinSteps;
#pragma unroll
                    for (int k = 0; k < kLinSteps; ++k) {
                        if (k >= mmas) continue;
                        tc_mma_bf16_pair(d, adesc + (uint64_t)(k * 2), bdesc + (uint64_t)(k * (W_KN ? 128 : 2)), id, (in > 0 || k > 0) ? 1u : 0u, elected);
                    }
                    tc_commit_pair(empty_bar(s), elected);
                    if (kb == g.k_blocks - 1) tc_commit_pair(acc_bar(i & 1), elected);
                    if (++s == kLinStages) { s = 0; ph ^= 1u; }
                }
                if (!live) ++i;
                if (!live) break;
            }
            // every MMA has retired before the warp goes on
            if (i > 0) mbar_wait(acc_bar((i - 1) & 1), (uint32_t)((i - 1) >> 1) & 1u, abort_flag, g.status, g.wait_limit, true);
            if (!live && lane == 0) {
                store_remote(map_to_rank(smem_u32((const void *)abort_flag), 1), 1u);        // the other CTA's producers stop, too
                drain_pair(full_bar(0), kLinStages, issued, kLinHalf, kLinHalf, abort_flag, g.status, g.wait_limit);
            }
        }
        __syncwarp();
    }

    __device__ void finish(const CUtensorMap &map, const LinArgs &g) const
    {
        constexpr int kFirst = lin_first_epi(PIECES);
        const int quarter = warp & 3, half = (warp - kFirst) >> 2, pieces = PIECES ? (g.k_blocks + g.piece - 1) / g.piece : 1;
        const uint32_t freed = map_to_rank(freed_bar(0), 0), stage = smem + (uint32_t)(kLinStages * kLinStage + (warp - kFirst) * kMxStaging);
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 128);
        const auto free_one = [&](int b) { mbar_arrive_remote(freed + 8u * (uint32_t)b); };
        const bool ahead = !F32 && g.residual;
        LinWalk<kLinTile> walk(g, lane);
        LinTile tile;
        int i = 0;
        for (uint32_t t = (uint32_t)pair; walk.find(t, tile); t += (uint32_t)g.units, ++i) {
            const int64_t m = tile.m0 + rank * 128 + quarter * 32, n0 = (int64_t)tile.nt * kLinTile + half * 128;
            const int rows = tile.end - m < 0 ? 0 : tile.end - m < 32 ? (int)(tile.end - m) : 32;
            float sum[PIECES ? 128 : 1];
            if constexpr (PIECES) {
                lin_add_pieces(*this, g, pieces, i, sum, [&](int b, int h) { return lanes + (uint32_t)(b * kLinTile + h); }, free_one);
                --i;
                if (rows == 0 || n0 >= g.N) continue;        // nothing of the warp's is an expert's
            }
            float bias[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) bias[q] = lin_bias(g, tile.e, n0 + 32 * q);
            LinFetch<F32> fetch;
            if (ahead) fetch.issue(g, m, rows, n0, g.N);
            if (!PIECES) mbar_wait(acc_bar(i & 1), (uint32_t)(i >> 1) & 1u, abort_flag, g.status, g.wait_limit);
            tc_fence_after();
            if (!PIECES && (rows == 0 || n0 >= g.N)) {       // nothing of the warp's is an expert's
                tc_fence_before();
                __syncwarp();
                if (lane == 0) free_one(i & 1);
                continue;
            }
            const uint32_t taddr = lanes + (uint32_t)((i & 1) * kLinTile);
            uint32_t scales = 0u;
#pragma unroll (PIECES ? 2 : 1)
            for (int q = 0; q < 2; ++q) {
                const int64_t n = n0 + q * 64;
                uint32_t two = 0u;
                lin_put_span<F32, KEEP>(map, g, stage, m, rows, tile.end == g.M, n, bias[0], bias[1], fetch, two, [&](int h, uint32_t(&v)[32]) {
                    if constexpr (PIECES) {         // (the columns behind move up: registers have no index)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(sum[64 * q + j]);
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum[64 * q + j] = sum[64 * q + j + 32];
                    } else {
                        tmem_ld_32x32_issue(taddr + q * 64 + h * 32, v);
                        tmem_ld_wait();
                        if (q == 0 || h == 0) return;
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) free_one(i & 1);
                    }
                });
                if (KEEP) scales |= two << (16 * q);
                bias[0] = bias[2];
                bias[1] = bias[3];
                if (q == 0 && ahead) fetch.issue(g, m, rows, n + 64, g.N);
            }
            if (KEEP && lane < rows && n0 < g.N) lin_keep_scales<4>(g, scales, m + lane, n0);
        }
        if (lane == 0) tma_store_wait_all();
        __syncwarp();
        tc_fence_before();
    }
};

template <bool W_KN, bool F32, bool KEEP, bool PIECES>
__global__ void __launch_bounds__(lin_threads(PIECES), 1)
sparq_linear_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_out, const LinArgs g)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) MxBars bars;
    __shared__ uint32_t tmem_base_slot;
    __shared__ uint32_t abort_word;
    __shared__ volatile uint32_t issued[4];

    LinPair<W_KN, F32, KEEP, PIECES> c;
    const int warp = c.warp = threadIdx.x >> 5, lane = c.lane = threadIdx.x & 31;
    c.abort_flag = &abort_word;
    c.issued = issued;
    c.smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    c.bars = smem_u32(&bars);
    c.rank = (int)(blockIdx.x & 1u);
    c.pair = (int)(blockIdx.x >> 1);

    if (warp == 0) {
        if (lane == 0) {
            prefetch_tensormap(&map_x);
            prefetch_tensormap(&map_w);
            prefetch_tensormap(&map_out);
            for (int s = 0; s < kLinStages; ++s) {
                mbar_init(c.full_bar(s), 1);
                mbar_init(c.empty_bar(s), 1);
            }
            for (int b = 0; b < 2; ++b) {
                mbar_init(c.acc_bar(b), 1);
                mbar_init(c.freed_bar(b), 2 * kLinEpiWarps);
            }
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
    // Registers: with PIECES 384 threads were launched with 168 each; of the same 64512, the epilogue's take 224 and the first four warps 56.
    if (PIECES && warp >= lin_first_epi(true)) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        c.finish(map_out, g);
    } else {
        if (PIECES) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        switch (warp) {
        case 0: c.template produce<true>(map_x, g); break;
        case 1: c.issue(g); break;
        case lin_weight_warp(PIECES): c.template produce<false>(map_w, g); break;
        default:
            if (!PIECES) c.finish(map_out, g);
        }
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
