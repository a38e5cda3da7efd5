// Microscaled formats (sparq_quantize_mx and the calls that read its output): the layouts of codes and scales,
// and the conversions of one run of 16 elements.
//
//   format   block  element          scale                               tensor
//   MXFP4    32     e2m1             2^(floor(log2 max|x|) - 2), e8m0     -
//   NVFP4    16     e2m1             e4m3(max|x| * (448 / m))            m, fp32
//   MXINT8   32     q * 2^-6, s8     2^floor(log2 max|x|), e8m0           -
//
// A row's codes take round_up(cols, 32) elements, the missing ones are zeros.  The scales of the 4-bit formats lie
// as the tensor cores take them: tiles of 128 rows x 4 scales, 512 bytes each, row r and scale c at byte
// (r % 32) * 16 + (r % 128) / 32 * 4 + c % 4 of tile (r / 128) * ceil(C / 4) + c / 4, so that a tile goes into tensor memory
// with one copy (32 lanes x 16 bytes).  Those of MXINT8 lie row by row, each row padded to 16 bytes for TMA.
#pragma once

#include "sparq_common.cuh"

namespace sparq {

SPARQ_HD int64_t round_up64(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
SPARQ_HD int mx_block(int format) { return format == SPARQ_NVFP4 ? 16 : 32; }
SPARQ_HD int64_t mx_padded(int64_t cols) { return round_up64(cols, 32); }
// Bytes of a row of codes.
SPARQ_HD int64_t mx_code_pitch(int format, int64_t cols) { return format == SPARQ_MXINT8 ? mx_padded(cols) : mx_padded(cols) / 2; }
// Scales of a row, padding included: tiles of 4, or whole 16-byte pieces.
SPARQ_HD int64_t mx_scale_cols(int format, int64_t cols)
{
    return round_up64(mx_padded(cols) / mx_block(format), format == SPARQ_MXINT8 ? 16 : 4);
}
SPARQ_HD int64_t mx_scale_rows(int format, int64_t rows) { return format == SPARQ_MXINT8 ? rows : round_up64(rows, 128); }

// Scale c of row r; `pitch` = mx_scale_cols.
template <bool TILED>
__host__ __device__ __forceinline__ int64_t mx_scale_at(int64_t row, int64_t c, int64_t pitch)
{
    if (!TILED) return row * pitch + c;
    return ((row >> 7) * (pitch >> 2) + (c >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (c & 3);
}
// Runs of 16 elements that a row's walk takes: its coded ones, and those of a tile's padding.
SPARQ_HD int64_t mx_runs(int format, int64_t cols)
{
    return format == SPARQ_MXINT8 ? mx_padded(cols) / 16 : mx_scale_cols(format, cols) * (mx_block(format) / 16);
}

// Checks shared by the entry points (sparq_mx.cu).
constexpr int64_t kMxMost = INT64_C(2147483647) - 255;      // no extent reaches it, so that padded ones stay within 32 bits
int check_mx_extent(int64_t rows, int64_t cols, int64_t ld);
int check_mx_format(int format, bool four_bits);
int check_mx_max(int format, const float *max_dev, const char *name);

#ifdef __CUDACC__

// ---- 16 elements of a row -------------------------------------------------------------------------
// A run is 8 words of bf16 pairs or 16 of fp32.  ALIGN: bytes that every run's address is a multiple of.  32 and 16 are read and
// written whole; 0 (rows of odd length) goes through 16-byte vectors too, shifted to where the run starts: element by
// element such a tensor took up to seven times as long (8000 x 4100 bf16, gated silu and its gradient, 190 and 376 us).

__device__ __forceinline__ void ld_v8(uint32_t *v, const void *p)
{
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(p));
}
__device__ __forceinline__ void st_v8(void *p, const uint32_t *v)
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void ld_v4(uint32_t *v, const void *p)
{
    asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "l"(p));
}
__device__ __forceinline__ void st_v4(void *p, const uint32_t *v)
{
    asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" :: "l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}

// Two fp32 values as bf16, to nearest even (NaN stays NaN); lo in the low half.
__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

template <bool BF16>
constexpr int kRunWords = BF16 ? 8 : 16;

// A tensor's own bytes: vectors that a shifted run takes beyond its row stay within them.
struct Span {
    const uint8_t *first, *end;
};
template <bool BF16>
__device__ __forceinline__ Span span_of(const void *p, int64_t rows, int64_t cols, int64_t ld)
{
    const uint8_t *b = reinterpret_cast<const uint8_t *>(p);
    return {b, b + ((rows - 1) * ld + cols) * (BF16 ? 2 : 4)};
}

// W words from s bytes on (s < 16, a multiple of the element's width) of the W + 4 words w, in place.
template <bool BF16, int W>
__device__ __forceinline__ void shift_words(uint32_t (&w)[W + 4], uint32_t s)
{
#pragma unroll
    for (int i = 0; i < W + 2; ++i) w[i] = s & 8u ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < W + 1; ++i) w[i] = s & 4u ? w[i + 1] : w[i];
    if (BF16) {
        const uint32_t bits = (s & 2u) * 8u;
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], bits);
    }
}

// `p` points at the run's first element, `left` elements of the row remain from there (any number, negative too); what
// the row does not have is zero.
template <bool BF16, int ALIGN>
__device__ __forceinline__ void load_words(uint32_t (&v)[kRunWords<BF16>], const void *p, int64_t left, const Span &span)
{
    constexpr int W = kRunWords<BF16>;
    const uint8_t *b = reinterpret_cast<const uint8_t *>(p);
    if (ALIGN >= 16 && left >= 16) {
#pragma unroll
        for (int i = 0; i < W; i += ALIGN / 4) {
            if (ALIGN == 32) ld_v8(v + i, b + 4 * i);
            else ld_v4(v + i, b + 4 * i);
        }
        return;
    }
    if (ALIGN == 0 && left >= 16) {
        const uint32_t s = (uint32_t)reinterpret_cast<uintptr_t>(b) & 15u;
        const uint8_t *f = b - s;
        if (f >= span.first && f + 4 * W + 16 <= span.end) {
            uint32_t w[W + 4];
#pragma unroll
            for (int i = 0; i < W + 4; i += 4) ld_v4(w + i, f + 4 * i);
            shift_words<BF16, W>(w, s);
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = w[i];
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (BF16) {
            const uint16_t *e = reinterpret_cast<const uint16_t *>(p);
            v[i] = (2 * i < left ? (uint32_t)e[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)e[2 * i + 1] << 16 : 0u);
        } else {
            v[i] = i < left ? reinterpret_cast<const uint32_t *>(p)[i] : 0u;
        }
    }
}

template <bool BF16>
__device__ __forceinline__ void floats_of_words(float (&f)[16], const uint32_t (&v)[kRunWords<BF16>])
{
#pragma unroll
    for (int i = 0; i < 16; ++i)
        f[i] = __uint_as_float(!BF16 ? v[i] : i & 1 ? v[i / 2] & 0xFFFF0000u : v[i / 2] << 16);
}

// Elements first .. last - 1 of a run.
template <bool BF16>
__device__ __forceinline__ void store_elements(uint8_t *b, const uint32_t (&v)[kRunWords<BF16>], int first, int last)
{
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if (i < first || i >= last) continue;
        if (BF16) reinterpret_cast<uint16_t *>(b)[i] = (uint16_t)(i & 1 ? v[i / 2] >> 16 : v[i / 2]);
        else reinterpret_cast<uint32_t *>(b)[i] = v[i];
    }
}

// A warp's runs: neighbouring lanes hold neighbouring runs of a row (run 0 starts a row), and all lanes call this, `left` <= 0
// where there is nothing to store.  ALIGN 0: each lane stores the aligned vectors that begin in front of its run and so takes the end
// of its left neighbour's; what has no neighbour to take it goes element by element.
template <bool BF16, int ALIGN>
__device__ __forceinline__ void store_run(void *p, const float (&f)[16], int64_t left, int64_t run)
{
    constexpr int W = kRunWords<BF16>;
    uint8_t *b = reinterpret_cast<uint8_t *>(p);
    uint32_t v[W];
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = BF16 ? bf16x2_of(f[2 * i % 16], f[(2 * i + 1) % 16]) : __float_as_uint(f[i]);
    if (ALIGN >= 16) {
        if (left >= 16) {
#pragma unroll
            for (int i = 0; i < W; i += ALIGN / 4) {
                if (ALIGN == 32) st_v8(b + 4 * i, v + i);
                else st_v4(b + 4 * i, v + i);
            }
        } else {
            store_elements<BF16>(b, v, 0, (int)left);
        }
        return;
    }
    const int lane = threadIdx.x & 31;
    uint32_t w[W + 4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __shfl_up_sync(0xFFFFFFFFu, v[W - 4 + i], 1);
#pragma unroll
    for (int i = 0; i < W; ++i) w[4 + i] = v[i];
    const bool whole = left >= 16, next_whole = __shfl_down_sync(0xFFFFFFFFu, whole, 1), taken = lane < 31 && left > 16 && next_whole;
    if (!whole) {
        store_elements<BF16>(b, v, 0, (int)left);
        return;
    }
    const uint32_t s = (uint32_t)reinterpret_cast<uintptr_t>(b) & 15u;
    const int per = BF16 ? 2 : 4;
    if (s == 0) {
#pragma unroll
        for (int i = 0; i < W; i += 4) st_v4(b + 4 * i, v + i);
        return;
    }
    shift_words<BF16, W>(w, 16u - s);
    if (lane > 0 && run > 0) st_v4(b - s, w);
    else store_elements<BF16>(b, v, 0, (int)(16u - s) / per);
#pragma unroll
    for (int i = 4; i < W; i += 4) st_v4(b - s + 4 * i, w + i);
    if (!taken) store_elements<BF16>(b, v, 16 - (int)s / per, 16);
}

// ---- blocks ------------------------------------------------------------------------------------

// Largest magnitude of a run, as the bits of a non-negative fp32: NaN above infinity above every number.
template <bool BF16>
__device__ __forceinline__ uint32_t run_max_bits(const uint32_t (&v)[kRunWords<BF16>])
{
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < kRunWords<BF16>; ++i) m = BF16 ? __vmaxu2(m, v[i] & 0x7FFF7FFFu) : max(m, v[i] & 0x7FFFFFFFu);
    return BF16 ? max(m & 0xFFFF0000u, m << 16) : m;
}

constexpr uint32_t kInfBits = 0x7F800000u;
constexpr uint32_t kNanE8M0 = 0xFFu, kNanE4M3 = 0x7Fu;

// e8m0 code of a block: exponent of its largest magnitude less emax, at least 2^-127 (also for zeros and
// subnormals).  A block with an infinity or a NaN takes the scale's NaN.
__device__ __forceinline__ uint32_t e8m0_code(uint32_t max_bits, uint32_t emax)
{
    if (max_bits >= kInfBits) return kNanE8M0;
    const uint32_t e = max_bits >> 23;
    return e > emax ? e - emax : 0u;
}
// 2^(code - 127) and its reciprocal, both exact (code <= 254; subnormal at the ends).
__device__ __forceinline__ float pow2_of_code(uint32_t code) { return __uint_as_float(code ? code << 23 : 0x00400000u); }
__device__ __forceinline__ float inv_pow2_of_code(uint32_t code) { return __uint_as_float(code < 254u ? (254u - code) << 23 : 0x00400000u); }

// Eight values as e2m1, to nearest even, saturating; element 0 in the lowest four bits.
__device__ __forceinline__ uint32_t e2m1x8_of(const float *f)
{
    uint32_t d;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(d) : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
    return d;
}
// Two floats of a packed pair of halves (exact).
__device__ __forceinline__ void halves_to_floats(uint32_t h, float &lo, float &hi)
{
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
}
__device__ __forceinline__ void floats_of_e2m1x8(float *f, uint32_t v)
{
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(v));
#pragma unroll
    for (int i = 0; i < 4; ++i) halves_to_floats(h[i], f[2 * i], f[2 * i + 1]);
}
// One value as e4m3, to nearest even, saturating at 448 (NaN stays NaN), and back.
__device__ __forceinline__ uint32_t e4m3_of(float f)
{
    uint16_t d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(0.0f), "f"(f));
    return d & 0xFFu;
}
__device__ __forceinline__ float float_of_e4m3(uint32_t code)
{
    uint32_t h;
    float lo, hi;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)code));
    halves_to_floats(h, lo, hi);
    return lo;
}

// NVFP4's tensor scale.  A largest magnitude below 2^-100 counts as that, so that nothing overflows and a tensor of
// zeros needs no case of its own; NaN stays.
__device__ __forceinline__ float nvfp4_largest(float m) { return m < 0x1p-100f ? 0x1p-100f : m; }

// MXINT8 codes of a run: rint(x * 2^(6 - e)) clamped to +-127, as four words; code, max_bits: the block's e8m0 scale and its
// largest magnitude.  The product with a power of two is exact, so that one fused multiply-add with 1.5 * 2^23 leaves the
// rounded (to nearest even) value in the low byte; only a block whose largest magnitude rounds to 128 has to clamp.
__device__ __forceinline__ uint4 int8_codes(float (&f)[16], uint32_t code, uint32_t max_bits)
{
    float mul = __uint_as_float((260u - code) << 23);       // 2^(133 - code)
    if (code < 6u) {                                         // not a float; the elements are below 2^-120
        mul = 0x1p127f;
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = __fmul_rn(f[i], __uint_as_float((133u - code) << 23));
    }
    uint32_t b[16];
    if ((max_bits & 0x7FFFFFu) < 0x7F0000u) {                // below 127.5 / 64 of its power of two
#pragma unroll
        for (int i = 0; i < 16; ++i) b[i] = __float_as_uint(__fmaf_rn(f[i], mul, 12582912.0f));
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            b[i] = __float_as_uint(__fadd_rn(fminf(fmaxf(__fmul_rn(f[i], mul), -127.0f), 127.0f), 12582912.0f));
    }
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = prmt(prmt(b[4 * j], b[4 * j + 1], 0x0040u), prmt(b[4 * j + 2], b[4 * j + 3], 0x0040u), 0x5410u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// ... and back: q * 2^(e - 6), exact (2^-133 at the smallest).  Flipping its top bit makes a code q + 128, which in the low byte of 2^23 is
// the float 2^23 + 128 + q.
__device__ __forceinline__ void floats_of_int8(float (&f)[16], uint4 codes, uint32_t scale)
{
    float s = __uint_as_float((scale - 6u) << 23);
    if (scale - 7u > 247u) s = __uint_as_float(scale == kNanE8M0 ? 0x7FC00000u : 0x00400000u >> (6u - scale));
    const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t u = w[j] ^ 0x80808080u;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[4 * j + i] = __fmul_rn(__fadd_rn(__uint_as_float(prmt(u, 0x4B000000u, 0x7540u + i)), -8388736.0f), s);
    }
}

// MXINT8 scales of a warp's runs, each block's in two neighbouring lanes; the last run of a row clears the padding behind it.
__device__ __forceinline__ void put_int8_scale(uint8_t *scales, uint32_t row, uint32_t run, uint32_t per_row, int64_t pitch, uint32_t code)
{
    uint8_t *at = scales + (int64_t)row * pitch;
    if ((run & 1u) == 0) at[run >> 1] = (uint8_t)code;
    if (run == per_row - 1)
        for (int64_t c = per_row >> 1; c < pitch; ++c) at[c] = 0;
}

// A warp's four (eight) neighbouring lanes hold a scale each (each twice): the word of the four, valid in the
// first of the lanes.
template <int LANES>
__device__ __forceinline__ uint32_t gather_word(uint32_t code)
{
    constexpr int step = LANES / 4;
    uint32_t w = code | (__shfl_down_sync(0xFFFFFFFFu, code, step) << 8);
    return w | (__shfl_down_sync(0xFFFFFFFFu, w, 2 * step) << 16);
}

// ---- the walk over runs --------------------------------------------------------------------------
// Runs of 16 elements, row by row, `per_row` of them; a warp's 32 lanes take neighbouring ones.  Row and run of a
// thread are divided out once and then stepped.
struct RunWalk {
    uint32_t row, run;
    uint32_t per_row, d_row, d_run;
    __device__ RunWalk(int64_t first, int64_t stride, uint32_t per_row_) : per_row(per_row_)
    {
        if ((first >> 32) == 0) row = (uint32_t)first / per_row;       // a 64-bit division costs a small launch 0.2 us
        else row = (uint32_t)(first / per_row);
        d_row = (uint32_t)stride / per_row;
        run = (uint32_t)first - row * per_row;
        d_run = (uint32_t)stride - d_row * per_row;
    }
    __device__ void next()
    {
        row += d_row;
        run += d_run;
        if (run >= per_row) { run -= per_row; ++row; }
    }
};

constexpr int kRunThreads = 256;

#endif

// Blocks of kRunThreads for `runs` runs (sparq_mx.cu).
int run_grid(int64_t runs, int *blocks);

// Largest of 32, 16 and 0 that every run's address is a multiple of.
inline int run_align(const void *p, int64_t ld, int width)
{
    const uint64_t a = (uint64_t)(uintptr_t)p | (uint64_t)ld * (uint64_t)width;
    return (a & 31u) == 0 ? 32 : (a & 15u) == 0 ? 16 : 0;
}

}  // namespace sparq
