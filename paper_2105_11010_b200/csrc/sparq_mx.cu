// Quantization to the microscaled formats and back (sparq_quantize_mx, sparq_dequantize_mx).
//
// A thread takes 16 elements of a row, 32 or 64 bytes of input; two neighbouring lanes share a block of 32.  Each
// element is read once and its code written once: HBM traffic is the bound.  16384 x 4096 bf16 to MXFP4 and back 62 us (5.5 TB/s;
// each way about half); the conversions keep the issue slots 60 to 75 % busy.  Rows of odd length 3 to 4.6 TB/s: their vectors are
// shifted into place, word by word.
#include "sparq_mx.cuh"

namespace sparq {

int check_mx_format(int format, bool four_bits)
{
    if (format == SPARQ_MXFP4 || format == SPARQ_NVFP4 || (!four_bits && format == SPARQ_MXINT8)) return SPARQ_OK;
    return set_error(SPARQ_ERR_INVALID_ARG, four_bits ? "format %d is neither SPARQ_MXFP4 nor SPARQ_NVFP4" : "format %d is not SPARQ_MXFP4, SPARQ_NVFP4 or SPARQ_MXINT8", format);
}

int check_mx_max(int format, const float *max_dev, const char *name)
{
    if (format == SPARQ_NVFP4 && !max_dev) return set_error(SPARQ_ERR_INVALID_ARG, "SPARQ_NVFP4 needs %s, the tensor's largest magnitude", name);
    if (format != SPARQ_NVFP4 && max_dev) return set_error(SPARQ_ERR_INVALID_ARG, "%s belongs to SPARQ_NVFP4 only", name);
    if ((uintptr_t)max_dev & 3u) return set_error(SPARQ_ERR_UNSUPPORTED, "%s must be 4-byte aligned", name);
    return SPARQ_OK;
}

int check_mx_extent(int64_t rows, int64_t cols, int64_t ld)
{
    if (rows >= kMxMost || cols >= kMxMost) return set_error(SPARQ_ERR_UNSUPPORTED, "rows and columns must be below 2^31 - 256");
    if ((__int128)(rows + 128) * (ld + 512) > INT64_C(1) << 60)
        return set_error(SPARQ_ERR_UNSUPPORTED, "%lld rows of %lld elements are more than any device holds", (long long)rows, (long long)ld);
    return SPARQ_OK;
}

int run_grid(int64_t runs, int *blocks)
{
    int sms = 0;
    const int rc = device_info(&sms);
    if (rc != SPARQ_OK) return rc;
    const int64_t want = (runs + kRunThreads - 1) / kRunThreads, cap = (int64_t)sms * 32;
    *blocks = (int)(want < cap ? want : cap);
    return SPARQ_OK;
}

namespace {

template <bool BF16, int ALIGN, int FORMAT>
__global__ void __launch_bounds__(kRunThreads)
quantize_mx_kernel(const void *x, int64_t rows, int64_t cols, int64_t ldx, uint32_t per_row, int64_t runs,
                   const float *max_dev, uint8_t *codes, uint8_t *scales)
{
    constexpr int kWidth = BF16 ? 2 : 4;
    const int64_t stride = (int64_t)gridDim.x * kRunThreads, first = (int64_t)blockIdx.x * kRunThreads + threadIdx.x;
    const int64_t pitch = mx_code_pitch(FORMAT, cols), spitch = mx_scale_cols(FORMAT, cols);
    const uint32_t coded = (uint32_t)(mx_padded(cols) / 16);
    const Span span = span_of<BF16>(x, rows, cols, ldx);
    RunWalk at(first, stride, per_row);
    dep_wait();
    dep_launch();
    float enc = 0.0f, enc_scale = 0.0f;
    if (FORMAT == SPARQ_NVFP4) {
        const float m = nvfp4_largest(*max_dev);
        enc = __fdiv_rn(2688.0f, m);
        enc_scale = __fdiv_rn(448.0f, m);
    }
    // a warp's lanes leave the loop together; those past the last run have nothing to read or write
    for (int64_t i = first; i < ((runs + 31) & ~INT64_C(31)); i += stride, at.next()) {
        const int64_t left = i < runs && at.row < rows ? cols - (int64_t)at.run * 16 : 0;
        uint32_t v[kRunWords<BF16>];
        load_words<BF16, ALIGN>(v, reinterpret_cast<const uint8_t *>(x) + (left > 0 ? (at.row * ldx + at.run * 16) * kWidth : 0), left, span);
        uint32_t mb = run_max_bits<BF16>(v);
        float f[16];
        floats_of_words<BF16>(f, v);
        uint32_t code;
        float mul = 1.0f;
        if (FORMAT == SPARQ_NVFP4) {
            code = mb >= kInfBits ? kNanE4M3 : e4m3_of(__fmul_rn(__uint_as_float(mb), enc_scale));
            const float s = float_of_e4m3(code);
            mul = s > 0.0f ? __fdiv_rn(enc, s) : 0.0f;
        } else {
            mb = max(mb, __shfl_xor_sync(0xFFFFFFFFu, mb, 1));
            code = e8m0_code(mb, FORMAT == SPARQ_MXFP4 ? 2u : 0u);
            if (FORMAT == SPARQ_MXFP4) mul = inv_pow2_of_code(code);
        }
        const bool none = mb >= kInfBits || mul == 0.0f;      // a scale that is zero or NaN: codes of zero
        const bool live = i < runs && at.row < rows && at.run < coded;
        if (live) {
            uint8_t *dst = codes + at.row * pitch;
            if (FORMAT == SPARQ_MXINT8) {
                const uint4 w = int8_codes(f, code, mb);
                reinterpret_cast<uint4 *>(dst)[at.run] = none ? make_uint4(0u, 0u, 0u, 0u) : w;
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) f[j] = __fmul_rn(f[j], mul);
                const uint32_t lo = e2m1x8_of(f), hi = e2m1x8_of(f + 8);
                reinterpret_cast<uint2 *>(dst)[at.run] = none ? make_uint2(0u, 0u) : make_uint2(lo, hi);
            }
        }
        if (FORMAT == SPARQ_MXINT8) {
            if (i < runs) put_int8_scale(scales, at.row, at.run, per_row, spitch, code);
        } else {
            // four scales at a time, the padding's too: zero, which is a number in either format.  (Whole words: runs are a multiple of 32.)
            constexpr int kLanes = FORMAT == SPARQ_NVFP4 ? 4 : 8;
            const uint32_t word = gather_word<kLanes>(live ? code : 0u);
            if ((threadIdx.x & (kLanes - 1)) == 0)
                *reinterpret_cast<uint32_t *>(scales + mx_scale_at<true>(at.row, at.run / kLanes * 4, spitch)) = word;
        }
    }
}

template <bool BF16, int ALIGN, int FORMAT>
__global__ void __launch_bounds__(kRunThreads)
dequantize_mx_kernel(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, uint32_t per_row, const float *max_dev,
                     void *out, int64_t ldo)
{
    constexpr int kWidth = BF16 ? 2 : 4;
    const int64_t stride = (int64_t)gridDim.x * kRunThreads, first = (int64_t)blockIdx.x * kRunThreads + threadIdx.x;
    const int64_t pitch = mx_code_pitch(FORMAT, cols), spitch = mx_scale_cols(FORMAT, cols), runs = rows * per_row;
    RunWalk at(first, stride, per_row);
    dep_wait();
    dep_launch();
    float dec = 1.0f;
    if (FORMAT == SPARQ_NVFP4) dec = __fdiv_rn(nvfp4_largest(*max_dev), 2688.0f);
    // a warp's lanes leave the loop together; those past the last run have nothing to store
    for (int64_t i = first; i < ((runs + 31) & ~INT64_C(31)); i += stride, at.next()) {
        float f[16];
        int64_t left = 0;
        if (i < runs) {
            const uint32_t c = FORMAT == SPARQ_NVFP4 ? at.run : at.run >> 1;
            const uint32_t code = scales[mx_scale_at<FORMAT != SPARQ_MXINT8>(at.row, c, spitch)];
            const uint8_t *src = codes + at.row * pitch;
            left = cols - (int64_t)at.run * 16;
            if (FORMAT == SPARQ_MXINT8) {
                floats_of_int8(f, reinterpret_cast<const uint4 *>(src)[at.run], code);
            } else {
                const uint2 w = reinterpret_cast<const uint2 *>(src)[at.run];
                floats_of_e2m1x8(f, w.x);
                floats_of_e2m1x8(f + 8, w.y);
                const float s = FORMAT == SPARQ_NVFP4 ? float_of_e4m3(code) : code == kNanE8M0 ? __uint_as_float(0x7FC00000u) : pow2_of_code(code);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    f[j] = __fmul_rn(f[j], s);
                    if (FORMAT == SPARQ_NVFP4) f[j] = __fmul_rn(f[j], dec);
                }
            }
        }
        store_run<BF16, ALIGN>(reinterpret_cast<uint8_t *>(out) + (at.row * ldo + at.run * 16) * kWidth, f, left, at.run);
    }
}

// What both directions refuse.
int check_tensor(int dtype, int64_t rows, int64_t cols, int64_t ld, const void *x, const void *codes, const void *scales, const char *name)
{
    const int rc = check_dtype(dtype);
    if (rc != SPARQ_OK) return rc;
    if (rows < 0 || cols < 0) return set_error(SPARQ_ERR_INVALID_ARG, "negative dimension");
    if (rows == 0 || cols == 0) return SPARQ_OK;
    if (!x || !codes || !scales) return set_error(SPARQ_ERR_INVALID_ARG, "%s/codes/scales pointer is NULL", name);
    if (ld < cols) return set_error(SPARQ_ERR_INVALID_ARG, "the leading dimension of %s (%lld) is less than its columns (%lld)", name, (long long)ld, (long long)cols);
    if ((uintptr_t)x & (dtype == SPARQ_DTYPE_BF16 ? 1u : 3u)) return set_error(SPARQ_ERR_UNSUPPORTED, "%s is not aligned to its elements", name);
    if (((uintptr_t)codes | (uintptr_t)scales) & 15u) return set_error(SPARQ_ERR_UNSUPPORTED, "codes and scales must be 16-byte aligned");
    return check_mx_extent(rows, cols, ld);
}

}  // namespace

}  // namespace sparq

using namespace sparq;

static int64_t mx_bytes(int format, int64_t rows, int64_t cols, bool codes)
{
    int rc = check_mx_format(format, false);
    if (rc != SPARQ_OK) return rc;
    if (rows < 0 || cols < 0) return set_error(SPARQ_ERR_INVALID_ARG, "negative dimension");
    if ((rc = check_mx_extent(rows, cols, cols)) != SPARQ_OK) return rc;
    return codes ? rows * mx_code_pitch(format, cols) : mx_scale_rows(format, rows) * mx_scale_cols(format, cols);
}

extern "C" int64_t sparq_mx_code_bytes(int format, int64_t rows, int64_t cols) { return mx_bytes(format, rows, cols, true); }
extern "C" int64_t sparq_mx_scale_bytes(int format, int64_t rows, int64_t cols) { return mx_bytes(format, rows, cols, false); }

// The instantiation for a tensor's type, alignment and format.
#define SPARQ_MX_PICK(KERNEL, bf16, align, format)                                                                      \
    ((format) == SPARQ_MXFP4 ? SPARQ_MX_PICK_A(KERNEL, bf16, align, SPARQ_MXFP4)                                        \
     : (format) == SPARQ_NVFP4 ? SPARQ_MX_PICK_A(KERNEL, bf16, align, SPARQ_NVFP4) : SPARQ_MX_PICK_A(KERNEL, bf16, align, SPARQ_MXINT8))
#define SPARQ_MX_PICK_A(KERNEL, bf16, align, F)                                                                         \
    ((bf16) ? ((align) == 32 ? KERNEL<true, 32, F> : (align) == 16 ? KERNEL<true, 16, F> : KERNEL<true, 0, F>)          \
            : ((align) == 32 ? KERNEL<false, 32, F> : (align) == 16 ? KERNEL<false, 16, F> : KERNEL<false, 0, F>))

extern "C" int sparq_quantize_mx(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int format, const float *max_dev,
                                 void *codes, uint8_t *scales, void *stream)
{
    int rc = check_mx_format(format, false);
    if (rc == SPARQ_OK) rc = check_mx_max(format, max_dev, "max_dev");
    if (rc == SPARQ_OK) rc = check_tensor(dtype, rows, cols, ldx, x, codes, scales, "x");
    if (rc != SPARQ_OK || rows == 0 || cols == 0) return rc;
    const bool bf16 = dtype == SPARQ_DTYPE_BF16;
    const uint32_t per_row = (uint32_t)mx_runs(format, cols);
    const int64_t runs = mx_scale_rows(format, rows) * per_row;
    int blocks = 0;
    if ((rc = run_grid(runs, &blocks)) != SPARQ_OK) return rc;
    const int align = run_align(x, ldx, bf16 ? 2 : 4);
    const auto kernel = SPARQ_MX_PICK(quantize_mx_kernel, bf16, align, format);
    const cudaError_t e = launch_overlapped(kernel, blocks, kRunThreads, 0, (cudaStream_t)stream, x, rows, cols, ldx, per_row, runs, max_dev,
                                            (uint8_t *)codes, scales);
    return e == cudaSuccess ? SPARQ_OK : cuda_error(e, "quantize_mx_kernel launch");
}

extern "C" int sparq_dequantize_mx(const void *codes, const uint8_t *scales, int64_t rows, int64_t cols, int format, const float *max_dev,
                                   void *out, int dtype, int64_t ldo, void *stream)
{
    int rc = check_mx_format(format, false);
    if (rc == SPARQ_OK) rc = check_mx_max(format, max_dev, "max_dev");
    if (rc == SPARQ_OK) rc = check_tensor(dtype, rows, cols, ldo, out, codes, scales, "out");
    if (rc != SPARQ_OK || rows == 0 || cols == 0) return rc;
    const bool bf16 = dtype == SPARQ_DTYPE_BF16;
    const uint32_t per_row = (uint32_t)((cols + 15) / 16);
    int blocks = 0;
    if ((rc = run_grid(rows * per_row, &blocks)) != SPARQ_OK) return rc;
    const int align = run_align(out, ldo, bf16 ? 2 : 4);
    const auto kernel = SPARQ_MX_PICK(dequantize_mx_kernel, bf16, align, format);
    const cudaError_t e = launch_overlapped(kernel, blocks, kRunThreads, 0, (cudaStream_t)stream, (const uint8_t *)codes, scales, rows, cols, per_row,
                                            max_dev, out, ldo);
    return e == cudaSuccess ? SPARQ_OK : cuda_error(e, "dequantize_mx_kernel launch");
}
