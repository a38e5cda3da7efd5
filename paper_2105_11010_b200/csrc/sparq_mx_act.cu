// Activation functions whose inputs are kept for the backward pass in 8 bits (MXINT8), and that backward pass.
//
//   forward    y = act(x)             or act(x) * up        from x and up as they are; both also go out as codes
//   backward   dx = dy * act'(x^)     or dy * up^ * act'(x^) and dup = dy * act(x^), x^ and up^ what the codes stand for
//
// silu(x) = x s(x) and gelu(x) = x s(2 sqrt(2/pi) (x + 0.044715 x^3)), the form with tanh, are both x s(z(x)) with
// s the logistic function: act' = s + x s (1 - s) z'.
//
// A thread takes 16 elements of a row as in sparq_mx.cu.  Every tensor is read and written once: HBM traffic is the bound,
// 8 bytes and a sixteenth forward and backward per element of a gated bf16 pair.  8192 x 8192, gated silu: forward 94.8 us (5.7 TB/s),
// backward 99.4 (5.5), where a copy reaches 6.55; at 64 registers half of an SM's warps fit, and the arithmetic (a power of two and
// a reciprocal an element, 2.8 instructions a cycle) takes most of the issue slots that the loads leave.  Both types with the arithmetic of
// fp32's (Logistic): 101.6 and 123, before it took its power of two as it does now; fp32 tensors themselves 141 and 143 with it, 140 and 142
// with that of bf16's, rows of odd length 2 to 7 % more.
#include "sparq_mx.cuh"

namespace sparq {

namespace {

constexpr float kGeluScale = 1.5957691216057308f;      // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;
constexpr float kHalfLog2e = 0.72134752044448170f, kHalfLog2eRest = 9.6298150e-9f;      // log2(e) / 2 in fp32, and what that leaves

// The reciprocal of a normal number whose reciprocal is one, off by 1 unit of 2^-23.
__device__ __forceinline__ float reciprocal(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// s(z) for bf16 tensors.  z log2(e) is rounded, so that the power of two is off by 2 + 1.16 |z| units of 2^-23: 2^-16 of s at the
// most, where bf16 keeps 2^-9.  s below 2^-126 counts as 0, and results below |x| 2^-126 with it.
__device__ __forceinline__ float logistic(float z)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(__fmul_rn(z, -1.4426950408889634f)));
    return reciprocal(__fadd_rn(1.0f, e));
}

// s(z) for fp32 tensors, to a few units of the last place: s = num * num * r and s (1 - s) = t r r, from h = exp(-|z| / 2), whose square
// t leaves the range of fp32 long before h does.
struct Logistic {
    float h, t, r, num;
    bool below;
    __device__ explicit Logistic(float z)
    {
        // h = 2^(-w log2(e) / 2): the product's rounding and the constant's come back as a factor 1 + lo ln 2
        const float w = fminf(fabsf(z), 256.0f), u = __fmul_rn(w, -kHalfLog2e);
        const float lo = __fmaf_rn(w, -kHalfLog2eRest, __fmaf_rn(w, -kHalfLog2e, -u));
        float p;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p) : "f"(u));
        h = __fmaf_rn(p, __fmul_rn(lo, 0.69314718055994531f), p);
        t = __fmul_rn(h, h);
        r = reciprocal(__fadd_rn(1.0f, t));
        below = z < 0.0f;
        num = below ? h : 1.0f;
    }
    __device__ float times(float x) const { return __fmul_rn(__fmul_rn(__fmul_rn(x, num), num), r); }
};

template <int ACT>
__device__ __forceinline__ float act_argument(float x) { return ACT == SPARQ_ACT_SILU ? x : kGeluScale * x * __fmaf_rn(kGeluCubic * x, x, 1.0f); }

template <bool BF16, int ACT>
__device__ __forceinline__ float act_value(float x)
{
    if (ACT == SPARQ_ACT_IDENTITY) return x;
    if (ACT == SPARQ_ACT_RELU) return x > 0.0f ? x : 0.0f;
    const float z = act_argument<ACT>(x);
    return BF16 ? x * logistic(z) : Logistic(z).times(x);
}

// act(x) and act'(x) of a number.
template <bool BF16, int ACT>
__device__ __forceinline__ void act_both(float x, float &y, float &d)
{
    if (ACT == SPARQ_ACT_IDENTITY) {
        y = x;
        d = 1.0f;
    } else if (ACT == SPARQ_ACT_RELU) {
        y = x > 0.0f ? x : 0.0f;
        d = x > 0.0f ? 1.0f : 0.0f;
    } else {
        // s is 0 or 1 to the last bit long before |x| = 64, and x^3 overflows far behind it
        const float c = ACT == SPARQ_ACT_SILU ? fminf(fmaxf(x, -128.0f), 128.0f) : fminf(fmaxf(x, -64.0f), 64.0f);
        const float z = act_argument<ACT>(c);
        const float dz = ACT == SPARQ_ACT_SILU ? 1.0f : __fmaf_rn(3.0f * kGeluCubic * kGeluScale * c, c, kGeluScale);
        if (BF16) {
            const float s = logistic(z);
            y = x * s;
            d = __fmaf_rn(c * s * (1.0f - s), dz, s);
        } else {
            const Logistic s(z);
            y = s.times(x);
            const float q = c * dz * s.r * s.r;           // the second term over t
            d = s.num * (s.num * __fmaf_rn(s.below ? 1.0f : s.t, q, s.r));
        }
    }
}

// Codes and scale of a run, its block's other half in the neighbouring lane.
template <bool BF16>
__device__ __forceinline__ void keep_run(const uint32_t (&v)[kRunWords<BF16>], const float (&x)[16], bool live, const RunWalk &at, int64_t pitch,
                                         int64_t spitch, int8_t *codes, uint8_t *scales)
{
    uint32_t mb = run_max_bits<BF16>(v);
    mb = max(mb, __shfl_xor_sync(0xFFFFFFFFu, mb, 1));
    if (!live) return;
    const uint32_t code = e8m0_code(mb, 0u);
    float f[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) f[j] = x[j];
    const uint4 w = int8_codes(f, code, mb);
    reinterpret_cast<uint4 *>(codes + at.row * pitch)[at.run] = mb >= kInfBits ? make_uint4(0u, 0u, 0u, 0u) : w;
    put_int8_scale(scales, at.row, at.run, at.per_row, spitch, code);
}

struct ActForward {
    const void *x, *up;
    int64_t rows, cols, ldx, ldy;
    uint32_t per_row;
    void *y;
    int8_t *codes, *up_codes;
    uint8_t *scales, *up_scales;
};

template <bool BF16, int ALIGN, int ACT, bool GATED>
__global__ void __launch_bounds__(kRunThreads)
act_forward_mx8_kernel(const ActForward g)
{
    constexpr int kWidth = BF16 ? 2 : 4;
    const int64_t stride = (int64_t)gridDim.x * kRunThreads, first = (int64_t)blockIdx.x * kRunThreads + threadIdx.x;
    const int64_t pitch = mx_padded(g.cols), spitch = mx_scale_cols(SPARQ_MXINT8, g.cols), runs = g.rows * g.per_row;
    RunWalk at(first, stride, g.per_row);
    dep_wait();
    dep_launch();
    const Span sx = span_of<BF16>(g.x, g.rows, g.cols, g.ldx), su = span_of<BF16>(g.up, g.rows, g.cols, g.ldx);
    // a warp's lanes leave the loop together; those past the last run have nothing to read or write
    for (int64_t i = first; i < ((runs + 31) & ~INT64_C(31)); i += stride, at.next()) {
        const bool live = i < runs;
        const int64_t left = live ? g.cols - (int64_t)at.run * 16 : 0, off = left > 0 ? (at.row * g.ldx + at.run * 16) * kWidth : 0;
        uint32_t vx[kRunWords<BF16>], vu[kRunWords<BF16>];
        load_words<BF16, ALIGN>(vx, reinterpret_cast<const uint8_t *>(g.x) + off, left, sx);
        if (GATED) load_words<BF16, ALIGN>(vu, reinterpret_cast<const uint8_t *>(g.up) + off, left, su);
        float f[16], u[16];
        floats_of_words<BF16>(f, vx);
        keep_run<BF16>(vx, f, live, at, pitch, spitch, g.codes, g.scales);
        if (GATED) {
            floats_of_words<BF16>(u, vu);
            keep_run<BF16>(vu, u, live, at, pitch, spitch, g.up_codes, g.up_scales);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            f[j] = act_value<BF16, ACT>(f[j]);
            if (GATED) f[j] = __fmul_rn(f[j], u[j]);
        }
        store_run<BF16, ALIGN>(reinterpret_cast<uint8_t *>(g.y) + (left > 0 ? (at.row * g.ldy + at.run * 16) * kWidth : 0), f, left, at.run);
    }
}

struct ActBackward {
    const void *dy;
    const int8_t *codes, *up_codes;
    const uint8_t *scales, *up_scales;
    int64_t rows, cols, lddy, lddx;
    uint32_t per_row;
    void *dx, *dup;
};

template <bool BF16, int ALIGN, int ACT, bool GATED>
__global__ void __launch_bounds__(kRunThreads)
act_backward_mx8_kernel(const ActBackward g)
{
    constexpr int kWidth = BF16 ? 2 : 4;
    const int64_t stride = (int64_t)gridDim.x * kRunThreads, first = (int64_t)blockIdx.x * kRunThreads + threadIdx.x;
    const int64_t pitch = mx_padded(g.cols), spitch = mx_scale_cols(SPARQ_MXINT8, g.cols), runs = g.rows * g.per_row;
    RunWalk at(first, stride, g.per_row);
    dep_wait();
    dep_launch();
    const Span sdy = span_of<BF16>(g.dy, g.rows, g.cols, g.lddy);
    // a warp's lanes leave the loop together; those past the last run have nothing to store
    for (int64_t i = first; i < ((runs + 31) & ~INT64_C(31)); i += stride, at.next()) {
        float dx[16], u[16];
        int64_t left = 0;
        if (i < runs) {
            left = g.cols - (int64_t)at.run * 16;
            const int64_t sc = mx_scale_at<false>(at.row, at.run >> 1, spitch);
            uint32_t v[kRunWords<BF16>];
            float x[16];
            load_words<BF16, ALIGN>(v, reinterpret_cast<const uint8_t *>(g.dy) + (at.row * g.lddy + at.run * 16) * kWidth, left, sdy);
            const uint32_t scale = g.scales[sc];
            floats_of_int8(x, reinterpret_cast<const uint4 *>(g.codes + at.row * pitch)[at.run], scale);
            if (GATED) floats_of_int8(u, reinterpret_cast<const uint4 *>(g.up_codes + at.row * pitch)[at.run], g.up_scales[sc]);
            floats_of_words<BF16>(dx, v);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                float y, d;
                act_both<BF16, ACT>(x[j], y, d);
                const float t = dx[j];
                dx[j] = __fmul_rn(GATED ? __fmul_rn(t, u[j]) : t, d);
                if (GATED) u[j] = __fmul_rn(t, y);
            }
            if (scale == kNanE8M0) {           // comparisons and minima lose it
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    dx[j] = x[j];
                    if (GATED) u[j] = x[j];
                }
            }
        }
        const int64_t off = (at.row * g.lddx + at.run * 16) * kWidth;
        store_run<BF16, ALIGN>(reinterpret_cast<uint8_t *>(g.dx) + off, dx, left, at.run);
        if (GATED) store_run<BF16, ALIGN>(reinterpret_cast<uint8_t *>(g.dup) + off, u, left, at.run);
    }
}

int check_act(int dtype, int act, int64_t rows, int64_t cols)
{
    const int rc = check_dtype(dtype);
    if (rc != SPARQ_OK) return rc;
    if (act < SPARQ_ACT_IDENTITY || act > SPARQ_ACT_GELU) return set_error(SPARQ_ERR_INVALID_ARG, "act %d is not one of SPARQ_ACT_*", act);
    if (rows < 0 || cols < 0) return set_error(SPARQ_ERR_INVALID_ARG, "negative dimension");
    return SPARQ_OK;
}

int check_pitches(int dtype, int64_t rows, int64_t cols, int64_t lda, int64_t ldb, uintptr_t values, uintptr_t kept)
{
    if (lda < cols || ldb < cols) return set_error(SPARQ_ERR_INVALID_ARG, "a leading dimension is less than the columns (%lld)", (long long)cols);
    if (values & (dtype == SPARQ_DTYPE_BF16 ? 1u : 3u)) return set_error(SPARQ_ERR_UNSUPPORTED, "a tensor is not aligned to its elements");
    if (kept & 15u) return set_error(SPARQ_ERR_UNSUPPORTED, "codes and scales must be 16-byte aligned");
    return check_mx_extent(rows, cols, lda > ldb ? lda : ldb);
}

int min_align(int a, int b) { return a < b ? a : b; }

}  // namespace

}  // namespace sparq

using namespace sparq;

#define SPARQ_ACT_PICK_A(KERNEL, B, align, ACT, GATED)                                                                  \
    ((align) == 32 ? KERNEL<B, 32, ACT, GATED> : (align) == 16 ? KERNEL<B, 16, ACT, GATED> : KERNEL<B, 0, ACT, GATED>)
#define SPARQ_ACT_PICK_G(KERNEL, bf16, align, ACT, gated)                                                               \
    ((bf16) ? ((gated) ? SPARQ_ACT_PICK_A(KERNEL, true, align, ACT, true) : SPARQ_ACT_PICK_A(KERNEL, true, align, ACT, false))   \
            : ((gated) ? SPARQ_ACT_PICK_A(KERNEL, false, align, ACT, true) : SPARQ_ACT_PICK_A(KERNEL, false, align, ACT, false)))
#define SPARQ_ACT_PICK(KERNEL, bf16, align, act, gated)                                                                 \
    ((act) == SPARQ_ACT_IDENTITY ? SPARQ_ACT_PICK_G(KERNEL, bf16, align, SPARQ_ACT_IDENTITY, gated)                     \
     : (act) == SPARQ_ACT_RELU ? SPARQ_ACT_PICK_G(KERNEL, bf16, align, SPARQ_ACT_RELU, gated)                           \
     : (act) == SPARQ_ACT_SILU ? SPARQ_ACT_PICK_G(KERNEL, bf16, align, SPARQ_ACT_SILU, gated)                           \
                               : SPARQ_ACT_PICK_G(KERNEL, bf16, align, SPARQ_ACT_GELU, gated))

extern "C" int sparq_act_forward_mx8(const void *x, const void *up, int dtype, int64_t rows, int64_t cols, int64_t ldx, int act,
                                     void *y, int64_t ldy, int8_t *codes, uint8_t *scales, int8_t *up_codes, uint8_t *up_scales, void *stream)
{
    int rc = check_act(dtype, act, rows, cols);
    if (rc != SPARQ_OK || rows == 0 || cols == 0) return rc;
    if (!x || !y || !codes || !scales) return set_error(SPARQ_ERR_INVALID_ARG, "x/y/codes/scales pointer is NULL");
    if (!up != !up_codes || !up != !up_scales) return set_error(SPARQ_ERR_INVALID_ARG, "up, up_codes and up_scales come together");
    rc = check_pitches(dtype, rows, cols, ldx, ldy, (uintptr_t)x | (uintptr_t)up | (uintptr_t)y,
                       (uintptr_t)codes | (uintptr_t)scales | (uintptr_t)up_codes | (uintptr_t)up_scales);
    if (rc != SPARQ_OK) return rc;
    if ((y == x || y == up) && ldy != ldx && rows > 1) return set_error(SPARQ_ERR_INVALID_ARG, "y in place of x or up has their leading dimension");
    const bool bf16 = dtype == SPARQ_DTYPE_BF16;
    const int width = bf16 ? 2 : 4;
    const int align = min_align(min_align(run_align(x, ldx, width), run_align(y, ldy, width)), up ? run_align(up, ldx, width) : 32);
    const ActForward g = {x, up, rows, cols, ldx, ldy, (uint32_t)mx_runs(SPARQ_MXINT8, cols), y, codes, up_codes, scales, up_scales};
    int blocks = 0;
    if ((rc = run_grid(rows * g.per_row, &blocks)) != SPARQ_OK) return rc;
    const auto kernel = SPARQ_ACT_PICK(act_forward_mx8_kernel, bf16, align, act, up != nullptr);
    const cudaError_t e = launch_overlapped(kernel, blocks, kRunThreads, 0, (cudaStream_t)stream, g);
    return e == cudaSuccess ? SPARQ_OK : cuda_error(e, "act_forward_mx8_kernel launch");
}

extern "C" int sparq_act_backward_mx8(const void *dy, int dtype, int64_t rows, int64_t cols, int64_t lddy, int act,
                                      const int8_t *codes, const uint8_t *scales, const int8_t *up_codes, const uint8_t *up_scales,
                                      void *dx, void *dup, int64_t lddx, void *stream)
{
    int rc = check_act(dtype, act, rows, cols);
    if (rc != SPARQ_OK || rows == 0 || cols == 0) return rc;
    if (!dy || !dx || !codes || !scales) return set_error(SPARQ_ERR_INVALID_ARG, "dy/dx/codes/scales pointer is NULL");
    if (!dup != !up_codes || !dup != !up_scales) return set_error(SPARQ_ERR_INVALID_ARG, "dup, up_codes and up_scales come together");
    rc = check_pitches(dtype, rows, cols, lddy, lddx, (uintptr_t)dy | (uintptr_t)dx | (uintptr_t)dup,
                       (uintptr_t)codes | (uintptr_t)scales | (uintptr_t)up_codes | (uintptr_t)up_scales);
    if (rc != SPARQ_OK) return rc;
    if ((dx == dy || dup == dy) && lddx != lddy && rows > 1) return set_error(SPARQ_ERR_INVALID_ARG, "dx or dup in place of dy has its leading dimension");
    if (dx == dup) return set_error(SPARQ_ERR_INVALID_ARG, "dx and dup are one matrix");
    const bool bf16 = dtype == SPARQ_DTYPE_BF16;
    const int width = bf16 ? 2 : 4;
    const int align = min_align(min_align(run_align(dy, lddy, width), run_align(dx, lddx, width)), dup ? run_align(dup, lddx, width) : 32);
    const ActBackward g = {dy, codes, up_codes, scales, up_scales, rows, cols, lddy, lddx, (uint32_t)((cols + 15) / 16), dx, dup};
    int blocks = 0;
    if ((rc = run_grid(rows * g.per_row, &blocks)) != SPARQ_OK) return rc;
    const auto kernel = SPARQ_ACT_PICK(act_backward_mx8_kernel, bf16, align, act, dup != nullptr);
    const cudaError_t e = launch_overlapped(kernel, blocks, kRunThreads, 0, (cudaStream_t)stream, g);
    return e == cudaSuccess ? SPARQ_OK : cuda_error(e, "act_backward_mx8_kernel launch");
}
