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

// Two fp32 values in one register pair, and one instruction for two operations (each rounded to nearest even).
typedef unsigned long long pair_t;
__device__ __forceinline__ pair_t make_pair(float lo, float hi) {
    pair_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 split_pair(pair_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ pair_t both(float v) { return make_pair(v, v); }
__device__ __forceinline__ pair_t fma2(pair_t a, pair_t b, pair_t c) {
    pair_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ pair_t mul2(pair_t a, pair_t b) {
    pair_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ pair_t add2(pair_t a, pair_t b) {
    pair_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// min(|x|, most), NaN where x is
__device__ __forceinline__ float least_abs(float x, float most) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(x)), "f"(most));
    return r;
}

// GELU needs Phi(-|x|) = exp(-x^2 / 2) R(|x|).  R falls smoothly from 1/2 like 1 / (|x| sqrt(2 pi)), so in t = 1 / (1 + 0.24 |x|) it
// is a short polynomial without a constant term: least squares of relative error on 0 <= |x| <= 40, reweighted until even, gave
// |error| < 4.4e-7 (2^-21), far below the half step of the codes it is rounded to (2^-9, 2^-12).  The same exponential gives the
// density that the derivative needs.
struct NormalTail {
    pair_t ax;  // |x|, at most 100: beyond, nothing changes, and infinities would meet zeros
    pair_t r;   // R(|x|)
    pair_t e;   // exp(-x^2 / 2)
};
// (Operations with a constant are done one value at a time, where the constant is part of the instruction.  In pairs they took 26 instead of
// 29 instructions an element of the pass over a gradient, and no less time: the special function unit's two are 16 issue cycles of a warp.)
__device__ __forceinline__ float tail_polynomial(float t) {
    float r = __fmaf_rn(-0.05299483f, t, 0.15280514f);
    r = __fmaf_rn(r, t, -0.06571881f);
    r = __fmaf_rn(r, t, 0.1184004f);
    r = __fmaf_rn(r, t, 0.06339276f);
    r = __fmaf_rn(r, t, 0.09283971f);
    r = __fmaf_rn(r, t, 0.09552203f);
    return __fmaf_rn(r, t, 0.0957538f);
}
__device__ __forceinline__ NormalTail normal_tail(float x0, float x1) {
    const float a0 = least_abs(x0, 100.0f), a1 = least_abs(x1, 100.0f);
    const float t0 = fast_rcp(__fmaf_rn(0.24f, a0, 1.0f)), t1 = fast_rcp(__fmaf_rn(0.24f, a1, 1.0f));
    NormalTail n;
    n.ax = make_pair(a0, a1);
    n.r = mul2(make_pair(tail_polynomial(t0), tail_polynomial(t1)), make_pair(t0, t1));
    const float2 s = split_pair(mul2(make_pair(__fmul_rn(a0, -0.72134752f), __fmul_rn(a1, -0.72134752f)), n.ax));
    n.e = make_pair(fast_exp2(s.x), fast_exp2(s.y));
    return n;
}

constexpr float kGeluTanhC = 1.5957691216f;  // 2 sqrt(2 / pi): 1/2 (1 + tanh u) = 1 / (1 + exp(-2 u))
constexpr float kLog2E = 1.4426950409f;

// For results that are rounded to codes, two values at a time.  1 / (1 + exp(-u)) and its derivative from a = exp(-|u|): with
// r = 1 / (1 + a) they are r or a r, and a r r (1 - p would cancel where p is close to 1).
template <int kAct>
__device__ __forceinline__ pair_t activate2(pair_t x) {
    const float2 v = split_pair(x);
    if (kAct == QFMT_ACT_RELU) return make_pair(v.x > 0.0f ? v.x : (v.x != v.x ? v.x : 0.0f), v.y > 0.0f ? v.y : (v.y != v.y ? v.y : 0.0f));
    if (kAct == QFMT_ACT_GELU) {  // x Phi(x) = max(x, 0) - |x| Phi(-|x|), without cancellation on either side
        const NormalTail n = normal_tail(v.x, v.y);
        const float2 low = split_pair(mul2(mul2(n.ax, n.r), n.e));
        return make_pair(__fsub_rn(fmaxf(v.x, 0.0f), low.x), __fsub_rn(fmaxf(v.y, 0.0f), low.y));
    }
    if (kAct == QFMT_ACT_GELU_TANH || kAct == QFMT_ACT_SILU) {
        float2 u = make_float2(__fmul_rn(v.x, -kLog2E), __fmul_rn(v.y, -kLog2E));
        if (kAct == QFMT_ACT_GELU_TANH) {
            const float2 xx = split_pair(mul2(x, x));
            u = split_pair(mul2(x, make_pair(__fmaf_rn(-0.044715f * kGeluTanhC * kLog2E, xx.x, -kGeluTanhC * kLog2E),
                                             __fmaf_rn(-0.044715f * kGeluTanhC * kLog2E, xx.y, -kGeluTanhC * kLog2E))));
        }
        return mul2(x, make_pair(fast_rcp(__fadd_rn(1.0f, fast_exp2(u.x))), fast_rcp(__fadd_rn(1.0f, fast_exp2(u.y)))));
    }
    return x;
}

template <int kAct>
__device__ __forceinline__ pair_t slope2(float x0, float x1) {
    if (kAct == QFMT_ACT_RELU) return make_pair(x0 > 0.0f ? 1.0f : (x0 != x0 ? x0 : 0.0f), x1 > 0.0f ? 1.0f : (x1 != x1 ? x1 : 0.0f));
    if (kAct == QFMT_ACT_GELU) {  // h = Phi(-|x|) - |x| phi(x) is the slope at -|x|, 1 - h the one at |x|
        const NormalTail n = normal_tail(x0, x1);
        const float2 ax = split_pair(n.ax), r = split_pair(n.r);
        const float2 h = split_pair(mul2(make_pair(__fmaf_rn(ax.x, -0.39894228f, r.x), __fmaf_rn(ax.y, -0.39894228f, r.y)), n.e));
        return make_pair(x0 < 0.0f ? h.x : __fsub_rn(1.0f, h.x), x1 < 0.0f ? h.y : __fsub_rn(1.0f, h.y));
    }
    if (kAct == QFMT_ACT_GELU_TANH || kAct == QFMT_ACT_SILU) {
        // at -|x| the slope is a r - |x| u'(x) a r r, at |x| it is 1 minus that; |x| at most 100 as above
        const float a0 = least_abs(x0, 100.0f), a1 = least_abs(x1, 100.0f);
        const pair_t ax = make_pair(a0, a1);
        pair_t xdu = ax;
        float2 w = make_float2(__fmul_rn(a0, -kLog2E), __fmul_rn(a1, -kLog2E));
        if (kAct == QFMT_ACT_GELU_TANH) {
            const float2 xx = split_pair(mul2(ax, ax));
            w = split_pair(mul2(ax, make_pair(__fmaf_rn(-0.044715f * kGeluTanhC * kLog2E, xx.x, -kGeluTanhC * kLog2E),
                                              __fmaf_rn(-0.044715f * kGeluTanhC * kLog2E, xx.y, -kGeluTanhC * kLog2E))));
            xdu = mul2(ax, make_pair(__fmaf_rn(3.0f * 0.044715f * kGeluTanhC, xx.x, kGeluTanhC), __fmaf_rn(3.0f * 0.044715f * kGeluTanhC, xx.y, kGeluTanhC)));
        }
        const float e0 = fast_exp2(w.x), e1 = fast_exp2(w.y);
        const pair_t r = make_pair(fast_rcp(__fadd_rn(1.0f, e0)), fast_rcp(__fadd_rn(1.0f, e1)));
        const float2 xr = split_pair(mul2(xdu, r));
        const float2 h = split_pair(mul2(mul2(make_pair(e0, e1), r), make_pair(__fsub_rn(1.0f, xr.x), __fsub_rn(1.0f, xr.y))));
        return make_pair(x0 < 0.0f ? h.x : __fsub_rn(1.0f, h.x), x1 < 0.0f ? h.y : __fsub_rn(1.0f, h.y));
    }
    return both(1.0f);
}

// The derivative for fp32 results, with the math library's functions.
template <int kAct>
__device__ __forceinline__ float slope(float x) {
    if (kAct == QFMT_ACT_RELU) return x > 0.0f ? 1.0f : (x != x ? x : 0.0f);
    const float ax = least_abs(x, 100.0f);
    if (kAct == QFMT_ACT_GELU) {
        const float h = __fmaf_rn(__fmul_rn(ax, -0.39894228f), expf(__fmul_rn(__fmul_rn(-0.5f, ax), ax)), __fmul_rn(0.5f, erfcf(__fmul_rn(ax, 0.70710678f))));
        return x < 0.0f ? h : __fsub_rn(1.0f, h);
    }
    if (kAct == QFMT_ACT_GELU_TANH || kAct == QFMT_ACT_SILU) {
        float u = ax, xdu = ax;
        if (kAct == QFMT_ACT_GELU_TANH) {
            const float xx = __fmul_rn(ax, ax), cx = __fmul_rn(ax, kGeluTanhC);
            u = __fmul_rn(cx, __fmaf_rn(0.044715f, xx, 1.0f));
            xdu = __fmul_rn(cx, __fmaf_rn(3.0f * 0.044715f, xx, 1.0f));
        }
        const float a = expf(-u), r = __frcp_rn(__fadd_rn(1.0f, a));
        const float h = __fmul_rn(__fmul_rn(a, r), __fmaf_rn(-xdu, r, 1.0f));
        return x < 0.0f ? h : __fsub_rn(1.0f, h);
    }
    return 1.0f;
}

}  // namespace qfmt
