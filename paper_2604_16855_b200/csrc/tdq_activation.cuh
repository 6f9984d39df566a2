// The activations of the 8-bit layer's epilogue and their slopes, two elements at a time (packed binary32 multiply-adds).
#pragma once
#include "tdq_common.cuh"

#ifdef __CUDACC__
namespace tdq {
namespace {

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float min_nan(float a, float b) {   // NaN where either is
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// Gaussian tail: with a = |z|, e = exp(-a^2 / 2) and q = Phi(-a) = p e, p = 1/2 erfcx(a / sqrt 2).  The smooth factor p is a polynomial of degree 10 on [0, 5], fitted by
// least squares with weights moved to the largest errors of max(a, 1) q: 1.5e-7 at most, roundings of its evaluation among them (behind 5 the factor stays what it is there,
// b = min(a, 5), and b q is within 8e-8 of a q).  An element costs
// fourteen multiply-adds in all and one turn of the special functions' unit, which takes eight times as long as one.
__device__ __forceinline__ void gauss_tail(float2 z, float2& b, float2& e, float2& p) {
    const float2 g = __fmul2_rn(__fmul2_rn(z, z), both(-0.72134752f));          // -log2(e) / 2
    e = make_float2(ex2(g.x), ex2(g.y));
    b = make_float2(min_nan(fabsf(z.x), 5.f), min_nan(fabsf(z.y), 5.f));
    p = both(1.23802897e-06f);
    p = __ffma2_rn(p, b, both(-2.84340113e-05f));
    p = __ffma2_rn(p, b, both(0.00029121447f));
    p = __ffma2_rn(p, b, both(-0.00178629335f));
    p = __ffma2_rn(p, b, both(0.00750757195f));
    p = __ffma2_rn(p, b, both(-0.0237156842f));
    p = __ffma2_rn(p, b, both(0.060663037f));
    p = __ffma2_rn(p, b, both(-0.132287741f));
    p = __ffma2_rn(p, b, both(0.249865487f));
    p = __ffma2_rn(p, b, both(-0.398932129f));
    p = __ffma2_rn(p, b, both(0.499999881f));
}
// 1 / (1 + exp(-z))
__device__ __forceinline__ float2 sigmoid(float2 z) {
    const float2 g = __fmul2_rn(z, both(-1.44269504f));
    const float2 d = __fadd2_rn(make_float2(ex2(g.x), ex2(g.y)), both(1.f));
    return make_float2(rcp(d.x), rcp(d.y));
}
constexpr float kTanhA = 1.59576912f, kTanhB = 0.0713548163f;   // 2 sqrt(2 / pi) (1, 0.044715):  (1 + tanh u) / 2 = sigmoid(2 u)

template <int ACT>
__device__ __forceinline__ float2 activate(float2 z) {
    if constexpr (ACT == TDQ_ACT_RELU) {
        return make_float2(max_nan(z.x, 0.f), max_nan(z.y, 0.f));
    } else if constexpr (ACT == TDQ_ACT_GELU) {              // z Phi(z) = max(z, 0) - |z| Phi(-|z|)
        float2 b, e, p;
        gauss_tail(z, b, e, p);
        return __ffma2_rn(make_float2(-b.x, -b.y), __fmul2_rn(p, e), make_float2(max_nan(z.x, 0.f), max_nan(z.y, 0.f)));
    } else if constexpr (ACT == TDQ_ACT_GELU_TANH) {
        return __fmul2_rn(z, sigmoid(__fmul2_rn(z, __ffma2_rn(__fmul2_rn(z, z), both(kTanhB), both(kTanhA)))));
    } else if constexpr (ACT == TDQ_ACT_SILU) {
        return __fmul2_rn(z, sigmoid(z));
    } else {
        return z;
    }
}
// For |z| < 10^13: products of larger ones leave binary32's range in the tanh form, SiLU's at an infinity, and inf 0 is no slope.
template <int ACT>
__device__ __forceinline__ float2 slope(float2 z) {
    if constexpr (ACT == TDQ_ACT_RELU) {
        return make_float2(z.x > 0.f ? 1.f : 0.f, z.y > 0.f ? 1.f : 0.f);
    } else if constexpr (ACT == TDQ_ACT_GELU) {              // Phi(z) + z phi(z); the odd part is 1/2 - q + a phi = 1/2 + e (a / sqrt(2 pi) - p)
        float2 b, e, p;
        gauss_tail(z, b, e, p);
        const float2 a = make_float2(min_nan(fabsf(z.x), 20.f), min_nan(fabsf(z.y), 20.f));   // exp(-200) is 0 in binary32
        const float2 h = __ffma2_rn(e, __ffma2_rn(a, both(0.398942280f), make_float2(-p.x, -p.y)), both(0.5f));
        return make_float2(0.5f + copysignf(h.x, z.x), 0.5f + copysignf(h.y, z.y));
    } else if constexpr (ACT == TDQ_ACT_GELU_TANH) {         // s + z s (1 - s) (2 u)'
        const float2 z2 = __fmul2_rn(z, z);
        const float2 s = sigmoid(__fmul2_rn(z, __ffma2_rn(z2, both(kTanhB), both(kTanhA))));
        const float2 d = __fmul2_rn(z, __ffma2_rn(z2, both(3.f * kTanhB), both(kTanhA)));
        return __fmul2_rn(s, __ffma2_rn(d, __ffma2_rn(s, both(-1.f), both(1.f)), both(1.f)));
    } else if constexpr (ACT == TDQ_ACT_SILU) {              // s (1 + z (1 - s))
        const float2 s = sigmoid(z);
        return __fmul2_rn(s, __ffma2_rn(z, __ffma2_rn(s, both(-1.f), both(1.f)), both(1.f)));
    } else {
        return both(1.f);
    }
}

__device__ __forceinline__ float activate_by(int act, float z) {
    switch (act) {
        case TDQ_ACT_RELU: return activate<TDQ_ACT_RELU>(both(z)).x;
        case TDQ_ACT_GELU: return activate<TDQ_ACT_GELU>(both(z)).x;
        case TDQ_ACT_GELU_TANH: return activate<TDQ_ACT_GELU_TANH>(both(z)).x;
        case TDQ_ACT_SILU: return activate<TDQ_ACT_SILU>(both(z)).x;
        default: return z;
    }
}
// All of a thread's sums.  Bound by the multiply-adds' unit (GELU fifteen an element: 2.3 us a 256 x 256 tile).  Not kept: GELU by Abramowitz and Stegun's 7.1.26, four
// multiply-adds fewer and a quotient more, in every element's place or every other's (16384 x 1024 -> 4096 bf16 109 -> 115 us); the quotient of the
// others by Newton's iteration (103 both ways).
template <int ACT, int N>
__device__ __forceinline__ void activate_all(float2 (&v)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = activate<ACT>(v[j]);
}

}  // namespace
}  // namespace tdq
#endif
