// Activation functions and their derivatives on one fp32 value.
#pragma once

#include <cuda_runtime.h>

#include "qfmt.h"

namespace qfmt {

// 2^x and 1/x of the special function unit (relative errors of about 2^-22; results below the smallest normal number are zero)
__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float fast_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// GELU needs Phi(-|x|) = exp(-x^2 / 2) R(|x|).  R falls smoothly from 1/2 like 1 / (|x| sqrt(2 pi)), so in t = 1 / (1 + 0.24 |x|) it
// is a short polynomial without a constant term: least squares of relative error on 0 <= |x| <= 40, reweighted until even, gave
// |error| < 4.4e-7 (2^-21), far below the half step of the codes it is rounded to (2^-9, 2^-12).  The same exponential gives the
// density that the derivative needs.
struct NormalTail {
    float q;  // Phi(-|x|)
    float e;  // exp(-x^2 / 2)
};
__device__ __forceinline__ NormalTail normal_tail(float x) {
    const float t = fast_rcp(__fmaf_rn(0.24f, fabsf(x), 1.0f));
    float r = -0.05299483f;
    r = __fmaf_rn(r, t, 0.15280514f);
    r = __fmaf_rn(r, t, -0.06571881f);
    r = __fmaf_rn(r, t, 0.1184004f);
    r = __fmaf_rn(r, t, 0.06339276f);
    r = __fmaf_rn(r, t, 0.09283971f);
    r = __fmaf_rn(r, t, 0.09552203f);
    r = __fmaf_rn(r, t, 0.0957538f);
    NormalTail n;
    n.e = fast_exp2(__fmul_rn(__fmul_rn(x, x), -0.72134752f));
    n.q = __fmul_rn(__fmul_rn(r, t), n.e);
    return n;
}

constexpr float kGeluTanhC = 1.5957691216f;  // 2 sqrt(2 / pi): 1/2 (1 + tanh u) = 1 / (1 + exp(-2 u))
constexpr float kLog2E = 1.4426950409f;

// kPrecise: for fp32 results, with the math library's functions; otherwise for results that are rounded to codes.
template <bool kPrecise>
__device__ __forceinline__ float logistic(float u) {
    if (kPrecise) return __frcp_rn(__fadd_rn(1.0f, expf(-u)));
    return fast_rcp(__fadd_rn(1.0f, fast_exp2(__fmul_rn(u, -kLog2E))));
}

// The same with p (1 - p), its derivative, from exp(-|u|): 1 - p would cancel where p is close to 1.
struct Logistic {
    float p, slope;
};
template <bool kPrecise>
__device__ __forceinline__ Logistic logistic_slope(float u) {
    const float a = kPrecise ? expf(-fabsf(u)) : fast_exp2(__fmul_rn(fabsf(u), -kLog2E));
    const float r = kPrecise ? __frcp_rn(__fadd_rn(1.0f, a)) : fast_rcp(__fadd_rn(1.0f, a));
    const float q = __fmul_rn(a, r);
    Logistic l;
    l.p = u < 0.0f ? q : r;
    l.slope = __fmul_rn(q, r);
    return l;
}

template <int kAct, bool kPrecise>
__device__ __forceinline__ float activate(float x) {
    if (kAct == QFMT_ACT_RELU) return x > 0.0f ? x : (x != x ? x : 0.0f);
    if (kAct == QFMT_ACT_GELU) {
        if (kPrecise) return __fmul_rn(__fmul_rn(0.5f, x), erfcf(__fmul_rn(x, -0.70710678f)));
        const float q = normal_tail(x).q;
        return __fmul_rn(x, x < 0.0f ? q : __fsub_rn(1.0f, q));
    }
    if (kAct == QFMT_ACT_GELU_TANH) {
        const float u = __fmul_rn(__fmul_rn(kGeluTanhC, x), __fmaf_rn(__fmul_rn(0.044715f, x), x, 1.0f));
        return __fmul_rn(x, logistic<kPrecise>(u));
    }
    if (kAct == QFMT_ACT_SILU) return __fmul_rn(x, logistic<kPrecise>(x));
    return x;
}

// Beyond +-100 every slope is 0 or 1 to the last bit; the squares of larger values would overflow.
template <int kAct, bool kPrecise>
__device__ __forceinline__ float activation_slope(float x) {
    if (kAct != QFMT_ACT_RELU && kAct != QFMT_ACT_NONE) x = fabsf(x) > 100.0f ? copysignf(100.0f, x) : x;
    if (kAct == QFMT_ACT_RELU) return x > 0.0f ? 1.0f : (x != x ? x : 0.0f);
    if (kAct == QFMT_ACT_GELU) {
        if (kPrecise) return __fmaf_rn(__fmul_rn(x, 0.39894228f), expf(__fmul_rn(__fmul_rn(-0.5f, x), x)), __fmul_rn(0.5f, erfcf(__fmul_rn(x, -0.70710678f))));
        const NormalTail n = normal_tail(x);
        return __fmaf_rn(__fmul_rn(x, 0.39894228f), n.e, x < 0.0f ? n.q : __fsub_rn(1.0f, n.q));
    }
    if (kAct == QFMT_ACT_GELU_TANH) {
        const float xx = __fmul_rn(x, x);
        const Logistic l = logistic_slope<kPrecise>(__fmul_rn(__fmul_rn(kGeluTanhC, x), __fmaf_rn(0.044715f, xx, 1.0f)));
        const float du = __fmul_rn(kGeluTanhC, __fmaf_rn(3.0f * 0.044715f, xx, 1.0f));
        return __fmaf_rn(__fmul_rn(x, l.slope), du, l.p);
    }
    if (kAct == QFMT_ACT_SILU) {
        const Logistic l = logistic_slope<kPrecise>(x);
        return __fmaf_rn(x, l.slope, l.p);
    }
    return 1.0f;
}

}  // namespace qfmt
