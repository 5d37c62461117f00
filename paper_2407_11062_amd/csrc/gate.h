// The activations of the gated feed-forward.
#pragma once
#include "common.h"

namespace eqat {

// silu(x) = x / (1 + exp(-x)), and x (1 + tanh(k (x + 0.044715 x^3))) / 2 = x / (1 + exp(-2 k (x + 0.044715 x^3))) with k = sqrt(2 / pi): both x p, p = 1 / (1 + exp(-t)),
// t = x or t = 2 k (x + 0.044715 x^3), and the derivative is p + x p (1 - p) t'.  Where exp(-t) passes binary32, p is 0, and x p = 0 for every finite x.
// exp(-t) = 2^(-t log2 e): the product's error, |t| 2^-24 of it, is put right by what a multiply-add leaves of it, so p is good to eight roundings (2^-21: the power's and the reciprocal's approximations,
// the products and sums between them) for every t that leaves it a normal number.  Where 1 + exp(-t) is 2^126 or more, t below -87.3, it may be 0: x p is off by |x| 2^-126 there (silu(-88) 0 for -5e-37).
struct GateP { float p, q; };                                         // q = 1 - p, as good as p
__device__ __forceinline__ GateP gate_p(float t)
{
    constexpr float kLog2e = 1.44269504088896340736f, kLog2eRest = 1.925963033500011e-8f;
    t = __builtin_amdgcn_fmed3f(t, -1000.0f, 1000.0f);                // (an infinite t leaves no NaN)
    const float a = -t * kLog2e, rest = __builtin_fmaf(-t, kLog2e, -a) - t * kLog2eRest;
    const float e = __builtin_amdgcn_exp2f(a), c = __builtin_fmaf(rest, 0.693147182464599609375f, 1.0f);        // (denormal results are 0: p = 1)
    GateP r;
    r.p = __builtin_amdgcn_rcpf(__builtin_fmaf(e, c, 1.0f));
    r.q = t > 0.0f ? e * c * r.p : 1.0f - r.p;                        // right of 0 the difference would leave p's rounding
    return r;
}
template <int KIND> __device__ __forceinline__ float gate_t(float x)
{
    constexpr float k2 = 1.5957691216057307f;                         // 2 sqrt(2 / pi)
    return KIND == EQAT_GATE_SILU ? x : k2 * x * __builtin_fmaf(0.044715f * x, x, 1.0f);
}
// gelu's t'; where x^2 passes binary32, p or q has long been 0, and has to stay it in the product
__device__ __forceinline__ float slope_of_t(float x) { return fminf(1.5957691216057307f * __builtin_fmaf(0.134145f * x, x, 1.0f), 0x1p100f); }
template <int KIND> __device__ __forceinline__ float gate_act(float x) { return x * gate_p(gate_t<KIND>(x)).p; }
// value and derivative
template <int KIND> __device__ __forceinline__ void gate_both(float x, float &a, float &slope)
{
    const GateP r = gate_p(gate_t<KIND>(x));
    const float t1 = KIND == EQAT_GATE_SILU ? 1.0f : slope_of_t(x);
    a = x * r.p;
    slope = __builtin_fmaf(a * r.q, t1, r.p);
}


// What the kernels with bf16 results take, whose epilogue is arithmetic and little else: exp(-t) without the rest of its product (off by |t| 2^-23 of itself, where a result keeps 2^-9), q = 1 - p, no
// clamp (exp(-t) = inf leaves p = 0).
__device__ __forceinline__ float gate_p_near(float t) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t * -1.44269504088896340736f)); }
template <int KIND> __device__ __forceinline__ float gated_near(float g, float u) { return g * gate_p_near(gate_t<KIND>(g)) * u; }
struct Gated { float h, dg, du; };
template <int KIND> __device__ __forceinline__ Gated gated_both_near(float g, float u, float d)
{
    const float p = gate_p_near(gate_t<KIND>(g)), act = g * p, du = d * act;
    float slope;
    if constexpr (KIND == EQAT_GATE_SILU) slope = __builtin_fmaf(act, 1.0f - p, p);
    else slope = __builtin_fmaf(act * (1.0f - p), slope_of_t(g), p);
    return Gated{act * u, d * u * slope, du};
}
// of one element: act(g) u, and with the gradient d of it d u act'(g), d act(g)
__device__ __forceinline__ float gated_by(int kind, float g, float u) { return kind == EQAT_GATE_SILU ? gated_near<EQAT_GATE_SILU>(g, u) : gated_near<EQAT_GATE_GELU>(g, u); }
__device__ __forceinline__ Gated gated_both(int kind, float g, float u, float d)
{
    return kind == EQAT_GATE_SILU ? gated_both_near<EQAT_GATE_SILU>(g, u, d) : gated_both_near<EQAT_GATE_GELU>(g, u, d);
}

}  // namespace eqat
