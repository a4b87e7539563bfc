// The activations of the product's epilogue and their slopes, in fp32.
#pragma once
#include "device_helpers.h"
#include "operators_internal.h"

namespace lf {
namespace ops {

// e^x for the functions below: one multiplication and the exponential instruction.  log2(e) as it is held and the rounding of x
// log2(e) make it off by 1.25 |x| 2^-24 of itself, which none of them feels: where |x| is large e^x is small beside what it is
// added to, or the whole result is.  (The library's expf takes three times the instructions; the slopes of 4096 x 8192 values were bound by them.)
__device__ __forceinline__ float exponential(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// 1 / (1 + e^-z).  The reciprocal instruction is good to an ulp and gives 0 where e^-z is inf.
__device__ __forceinline__ float sigma(float z) { return __builtin_amdgcn_rcpf(1.0f + exponential(-z)); }

// Phi(-a) for a >= 0, from e = exp(-a^2 / 2):  e t Q(t) with t = 1 / (1 + 0.35 a).  Phi(-a) / e falls like 1 / a, so Phi(-a) / (e t) is
// smooth up to t = 0; Q is its least-squares fit of degree 8 over a <= 14.6 (beyond, e is 0), reweighted towards the
// least largest relative error: 3.2e-8, 1.8e-7 as evaluated.  One exponential serves the value and the slope, and the
// left tail keeps its digits, where 1 + erf would cancel.
__device__ __forceinline__ float normal_tail(float a, float e) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.35f, a, 1.0f));
    float q = -0.02915963903069496f;
    q = fmaf(q, t, 0.1440395712852478f);
    q = fmaf(q, t, -0.2558571696281433f);
    q = fmaf(q, t, 0.15934079885482788f);
    q = fmaf(q, t, -0.023227158933877945f);
    q = fmaf(q, t, 0.10555889457464218f);
    q = fmaf(q, t, 0.11981963366270065f);
    q = fmaf(q, t, 0.1398637443780899f);
    q = fmaf(q, t, 0.1396212875843048f);
    return e * t * q;
}
__device__ __forceinline__ float normal(float z, float e) {          // Phi(z)
    const float c = normal_tail(fabsf(z), e);
    return z > 0.0f ? 1.0f - c : c;
}

__device__ __forceinline__ float activate(int act, float z) {
    if (act == RELU) return z < 0.0f ? 0.0f : z;
    if (act == GELU) return z * normal(z, exponential(-0.5f * z * z));
    const float a = sigma(z);
    return act == SILU ? z * a : a;
}
__device__ __forceinline__ float slope(int act, float z) {
    if (act == RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (act == GELU) {
        const float e = exponential(-0.5f * z * z);
        return fmaf(z * e, 0.39894228040143268f, normal(z, e));      // z phi(z) + Phi(z)
    }
    // sigma and 1 - sigma from e^-|z|, both without a difference: 1 - sigma(z) as such loses its digits where z > 0 is large (6 % of the
    // slope at z = 16, all of it from 17.4 on).
    const float e = exponential(-fabsf(z)), r = __builtin_amdgcn_rcpf(1.0f + e), small = e * r;
    if (act == SIGMOID) return r * small;
    const float a = z >= 0.0f ? r : small, rest = z >= 0.0f ? small : r;
    return a * fmaf(z, rest, 1.0f);
}

}  // namespace ops
}  // namespace lf
