// Activations of the products' epilogues and their slopes, in fp32 (internal).  Numbers as in include/dssp_kernels.h.
//   relu x [x > 0];  gelu x Phi(x);  gelu_tanh x (1 + tanh u) / 2 = x sigmoid(2 u), u = sqrt(2 / pi) (x + 0.044715 x^3);  silu x sigmoid(x)
// A NaN stays one.  sigmoid(v) = 1 / (1 + e^-v): e^-v overflows to infinity for v < -88, which gives 0, as it should.
#pragma once
#include "common.hpp"
#include "../../include/dssp_kernels.h"

namespace act {

constexpr float SQRT_8_OVER_PI = 1.5957691216057308f, CUBIC = 0.044715f;

// Two forms of each: FINE for fp32 results, whose errors are those of a handful of fp32 roundings (2^-24 of the results' root mean square), and a shorter one for bf16 results, whose
// errors, 1.4e-6 at most where the value is about 1 (the slope of gelu's tanh form), are a thousandth of what rounding to bf16 leaves.  An epilogue over 64 million elements takes 2 us for
// every vector instruction of an element (the library's exponential and error function take 15 and 40).

// e^v and 1 / v by the hardware's own instructions, a unit in the last place or so each
__device__ __forceinline__ float exp_fast(float v) { return __builtin_amdgcn_exp2f(v * 1.4426950408889634f); }
struct Sigmoid { float p, q; };         // sigmoid(v) and 1 - sigmoid(v)
template <bool FINE> __device__ __forceinline__ Sigmoid sigmoid(float v) {
    if constexpr (FINE) {
        // of e = e^-|v| <= 1, its exponent in two parts (the product with log2 e, and what that lost); 1 / (1 + e) with a Newton step.  Neither p nor q cancels.
        const float a = fabsf(v) > 128.f ? 128.f : fabsf(v), hi = a * -1.4426950408889634f;
        const float lo = fmaf(a, -1.925963033500e-8f, fmaf(a, -1.4426950408889634f, -hi));
        float e = __builtin_amdgcn_exp2f(hi);
        e = fmaf(e, lo * 0.6931471805599453f, e);
        const float d = 1.f + e;
        float r = __builtin_amdgcn_rcpf(d);
        r = fmaf(fmaf(-d, r, 1.f), r, r);
        return v < 0.f ? Sigmoid{e * r, r} : Sigmoid{r, e * r};
    } else {
        const float p = __builtin_amdgcn_rcpf(1.f + exp_fast(-v));
        return {p, 1.f - p};
    }
}

// The error function's part of gelu by polynomials fitted to it (largest error made small by Lawson's iteration, in 64 bits) in a = |x|, up to where nothing is left.
template <int MOST> __device__ __forceinline__ float reach(float x) { const float a = fabsf(x); return a > MOST ? (float)MOST : a; }
// FINE: Phi(-a) e^(a^2 / 2), off by at most 2.2e-9 e^(a^2 / 2) / max(a, 1); e: e^(-a^2 / 2).  Root mean square errors 3.4e-8 of gelu and of its slope (the formula with
// correctly rounded functions: 3.8e-8 and 4.0e-8).
__device__ __forceinline__ float tail(float a, float& e) {
    e = __builtin_amdgcn_exp2f(a * -0.7213475204444817f * a);
    float r = fmaf(-7.982273337e-09f, a, 2.551311826e-07f);
    r = fmaf(fmaf(fmaf(fmaf(r, a, -3.709441065e-06f), a, 3.280095373e-05f), a, -1.999334465e-04f), a, 9.088241295e-04f);
    r = fmaf(fmaf(fmaf(fmaf(r, a, -3.279617335e-03f), a, 9.921597838e-03f), a, -2.627040076e-02f), a, 6.236002615e-02f);
    r = fmaf(fmaf(fmaf(fmaf(r, a, -1.329446636e-01f), a, 2.499951506e-01f), a, -3.989420245e-01f), a, 4.999999978e-01f);
    return r;
}
// short: log2 Phi(-a), so that a Phi(-a) is off by at most 1e-7, and (Phi(-a) - a phi(a)) e^(a^2 / 2), so that the slope is off by at most 3.5e-7.
template <bool FINE> __device__ __forceinline__ float gelu(float x) {
    if constexpr (FINE) {
        float e;
        const float a = reach<8>(x), r = tail(a, e);
        return fmaf(-a, e * r, x < 0.f ? 0.f : x);
    } else {
        const float a = reach<12>(x);
        const float l = fmaf(fmaf(fmaf(fmaf(fmaf(fmaf(3.177492482e-05f, a, -7.569161963e-04f), a, 8.036975367e-03f), a, -5.333740498e-02f), a, -4.588343286e-01f), a,
                                  -1.151177109e+00f), a, -9.999963286e-01f);
        return fmaf(-a, __builtin_amdgcn_exp2f(l), x < 0.f ? 0.f : x);
    }
}
template <bool FINE> __device__ __forceinline__ float gelu_slope(float x) {
    float r;
    if constexpr (FINE) {
        float e;
        const float a = reach<8>(x);
        r = fmaf(a, -0.3989422804014327f, tail(a, e));
        r *= e;
    } else {
        const float a = reach<12>(x);
        r = fmaf(-8.063049657e-06f, a, 1.519415503e-04f);
        r = fmaf(fmaf(fmaf(fmaf(r, a, -1.271160005e-03f), a, 6.382798388e-03f), a, -2.223086296e-02f), a, 5.949677970e-02f);
        r = fmaf(fmaf(fmaf(fmaf(r, a, -1.317728762e-01f), a, 2.497522908e-01f), a, -7.978648987e-01f), a, 4.999997430e-01f);
        r *= exp_fast(-0.5f * a * a);
    }
    return x > 0.f ? 1.f - r : r;
}

template <bool FINE> __device__ __forceinline__ float value(int which, float x) {
    switch (which) {
        case DSSPK_ACT_RELU: return x < 0.f ? 0.f : x;
        case DSSPK_ACT_GELU: return gelu<FINE>(x);
        case DSSPK_ACT_GELU_TANH: return x * sigmoid<FINE>(SQRT_8_OVER_PI * x * fmaf(CUBIC * x, x, 1.f)).p;
        case DSSPK_ACT_SILU: return x * sigmoid<FINE>(x).p;
        default: return x;
    }
}

template <bool FINE> __device__ __forceinline__ float slope(int which, float x) {
    switch (which) {
        case DSSPK_ACT_RELU: return x > 0.f ? 1.f : x == x ? 0.f : x;
        case DSSPK_ACT_GELU: return gelu_slope<FINE>(x);
        case DSSPK_ACT_GELU_TANH: {
            const Sigmoid s = sigmoid<FINE>(SQRT_8_OVER_PI * x * fmaf(CUBIC * x, x, 1.f));
            const float c = fabsf(x) > 32.f ? 32.f : x;         // there one of p and q is zero, and stays the whole term when x^2 overflows
            return fmaf(c * s.p * s.q * SQRT_8_OVER_PI, fmaf(3.f * CUBIC * c, c, 1.f), s.p);
        }
        case DSSPK_ACT_SILU: {
            const Sigmoid s = sigmoid<FINE>(x);
            return s.p * fmaf(x, s.q, 1.f);
        }
        default: return 1.f;
    }
}

// f(Which<A>) with the activation as a constant: the switch stands in front of a loop, not in it
template <int A> struct Which { static constexpr int value = A; };
template <class F> __device__ __forceinline__ void with(int which, F f) {
    switch (which) {
        case DSSPK_ACT_RELU: f(Which<DSSPK_ACT_RELU>{}); break;
        case DSSPK_ACT_GELU: f(Which<DSSPK_ACT_GELU>{}); break;
        case DSSPK_ACT_GELU_TANH: f(Which<DSSPK_ACT_GELU_TANH>{}); break;
        case DSSPK_ACT_SILU: f(Which<DSSPK_ACT_SILU>{}); break;
        default: f(Which<DSSPK_ACT_NONE>{});
    }
}

}  // namespace act
