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

// Word w (scales 4w .. 4w + 3) of row r.
template <bool TILED>
__host__ __device__ __forceinline__ int64_t mx_scale_word(int64_t row, int64_t w, int64_t words)
{
    if (!TILED) return (row * words + w) * 4;
    return ((row >> 7) * words + w) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4;
}

// Checks shared by the entry points (sparq_mx.cu).
int check_mx_format(int format, bool four_bits);
int check_mx_max(int format, const float *max_dev, const char *name);

#ifdef __CUDACC__

// ---- 16 elements of a row as fp32 ---------------------------------------------------------------
// ALIGN: bytes that every run's address is a multiple of -- 32 and 16 are read whole, anything less element by element,
// as is a run that the row ends in.

__device__ __forceinline__ void ld_v8(uint32_t (&v)[8], const void *p)
{
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(p));
}
__device__ __forceinline__ void st_v8(void *p, const uint32_t (&v)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

template <int ALIGN>
__device__ __forceinline__ void ld_bytes32(uint32_t (&v)[8], const uint8_t *p)
{
    if (ALIGN == 32) {
        ld_v8(v, p);
    } else {
        const uint4 a = reinterpret_cast<const uint4 *>(p)[0], b = reinterpret_cast<const uint4 *>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}
template <int ALIGN>
__device__ __forceinline__ void st_bytes32(uint8_t *p, const uint32_t (&v)[8])
{
    if (ALIGN == 32) {
        st_v8(p, v);
    } else {
        reinterpret_cast<uint4 *>(p)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4 *>(p)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
}

// Two fp32 values as bf16, to nearest even (NaN stays NaN); lo in the low half.
__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

// `p` points at the run's first element, `left` elements of the row remain from there (any number, negative too).
template <bool BF16, int ALIGN>
__device__ __forceinline__ void load_run(float (&f)[16], const void *p, int64_t left)
{
    const uint8_t *b = reinterpret_cast<const uint8_t *>(p);
    if (ALIGN >= 16 && left >= 16) {
        uint32_t v[8];
        ld_bytes32<ALIGN>(v, b);
        if (BF16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[2 * i] = __uint_as_float(v[i] << 16);
                f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
            }
        } else {
            uint32_t w[8];
            ld_bytes32<ALIGN>(w, b + 32);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[i] = __uint_as_float(v[i]);
                f[8 + i] = __uint_as_float(w[i]);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        f[i] = 0.0f;
        if (i < left)
            f[i] = BF16 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << 16) : reinterpret_cast<const float *>(p)[i];
    }
}

template <bool BF16, int ALIGN>
__device__ __forceinline__ void store_run(void *p, const float (&f)[16], int64_t left)
{
    uint8_t *b = reinterpret_cast<uint8_t *>(p);
    uint32_t v[8];
    if (ALIGN >= 16 && left >= 16) {
        if (BF16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = bf16x2_of(f[2 * i], f[2 * i + 1]);
            st_bytes32<ALIGN>(b, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(f[i]);
            st_bytes32<ALIGN>(b, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(f[8 + i]);
            st_bytes32<ALIGN>(b + 32, v);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if (i >= left) continue;
        if (BF16) reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)bf16x2_of(f[i], 0.0f);
        else reinterpret_cast<float *>(p)[i] = f[i];
    }
}

// ---- blocks ------------------------------------------------------------------------------------

// Largest magnitude of a run, as the bits of a non-negative float: NaN above infinity above every number.
__device__ __forceinline__ uint32_t run_max_bits(const float (&f)[16])
{
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(f[i]) & 0x7FFFFFFFu);
    return m;
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

// MXINT8 codes of a run: rint(x * 2^(6 - e)) clamped to +-127, as four words.
__device__ __forceinline__ uint4 int8_codes(const float (&f)[16], float inv)
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float z = __fmul_rn(__fmul_rn(f[4 * j + i], inv), 64.0f);
            z = fminf(fmaxf(z, -127.0f), 127.0f);
            b[i] = __float_as_uint(__fadd_rn(z, 12582912.0f));      // 1.5 * 2^23: to nearest even in the low byte
        }
        w[j] = prmt(prmt(b[0], b[1], 0x0040u), prmt(b[2], b[3], 0x0040u), 0x5410u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// ... and back: q * 2^-6 * 2^e, exact (2^-133 at the smallest).
__device__ __forceinline__ void floats_of_int8(float (&f)[16], uint4 codes, uint32_t scale)
{
    const float s = pow2_of_code(scale);
    const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int q = (int)(int8_t)(w[j] >> (8 * i));
            f[4 * j + i] = __fmul_rn(__fmul_rn((float)q, 0.015625f), s);
        }
    if (scale == kNanE8M0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(0x7FC00000u);
    }
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
    int64_t row, run;
    int64_t per_row, d_row, d_run;
    __device__ RunWalk(int64_t first, int64_t stride, int64_t per_row_) : per_row(per_row_)
    {
        if (((first | stride | per_row) >> 31) == 0) {       // 64-bit divisions cost a small launch 0.2 us
            row = (uint32_t)first / (uint32_t)per_row;
            d_row = (uint32_t)stride / (uint32_t)per_row;
        } else {
            row = first / per_row;
            d_row = stride / per_row;
        }
        run = first - row * per_row;
        d_run = stride - d_row * per_row;
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
