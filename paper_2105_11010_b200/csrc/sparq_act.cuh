// Activation functions and their derivatives on fp32 values: silu(x) = x s(x) and gelu(x) = x s(2 sqrt(2/pi) (x + 0.044715 x^3)), the
// form with tanh, are both x s(z(x)) with s the logistic function.
#pragma once

#include "sparq_mx.cuh"

namespace sparq {

#ifdef __CUDACC__

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
        take(z, u, __fmaf_rn(w, -kHalfLog2eRest, __fmaf_rn(w, -kHalfLog2e, -u)));
    }
    // s(z + rest), of |z| below 2^16: rest, a few units of z's last place, comes back in the same factor.
    __device__ Logistic(float z, float rest)
    {
        const float w = fminf(fabsf(z), 256.0f), u = __fmul_rn(w, -kHalfLog2e);
        const float lo = __fmaf_rn(w, -kHalfLog2eRest, __fmaf_rn(w, -kHalfLog2e, -u));
        take(z, u, __fmaf_rn(z < 0.0f ? rest : -rest, kHalfLog2e, lo));
    }
    __device__ __forceinline__ void take(float z, float u, float lo)
    {
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

// GELU to a few units of the last place.  An error of the argument is a relative one of the result, and what the argument's roundings in fp32 make of it is 72 units of 2^-23 near x = -9 (37 near -7, 16 near -5).  So
// the argument comes in two parts, its rounded value and what the roundings, the constants' among them, left of it.
constexpr float kGeluScaleRest = -4.5340680e-8f, kGeluCubicRest = 1.5461445e-9f;
__device__ __forceinline__ float gelu_exact(float x)
{
    const float c = fminf(fmaxf(x, -64.0f), 64.0f);        // s is 0 or 1 to the last bit long before
    const float t = __fmul_rn(c, c), t_rest = __fmaf_rn(c, c, -t);
    const float a = __fmul_rn(kGeluCubic, t), a_rest = __fadd_rn(__fmaf_rn(kGeluCubic, t, -a), __fmaf_rn(kGeluCubic, t_rest, __fmul_rn(kGeluCubicRest, t)));
    const float q = __fadd_rn(1.0f, a), back = __fsub_rn(q, 1.0f);
    const float q_rest = __fadd_rn(__fadd_rn(__fsub_rn(1.0f, __fsub_rn(q, back)), __fsub_rn(a, back)), a_rest);
    const float u = __fmul_rn(kGeluScale, c), u_rest = __fmaf_rn(kGeluScaleRest, c, __fmaf_rn(kGeluScale, c, -u));
    const float z = __fmul_rn(u, q), z_rest = __fadd_rn(__fmaf_rn(u, q, -z), __fmaf_rn(u, q_rest, __fmul_rn(u_rest, q)));
    return Logistic(z, z_rest).times(x);
}

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

#endif

}  // namespace sparq
