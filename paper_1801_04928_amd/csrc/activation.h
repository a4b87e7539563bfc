// The activations of the product's epilogue and their slopes, in fp32.
#pragma once
#include "device_helpers.h"
#include "operators_internal.h"

namespace lf {
namespace ops {

constexpr float kSqrtHalf = 0.70710678118654752f, kInvSqrt2Pi = 0.39894228040143268f;

// (1 + e^-z and its reciprocal: e^-z = inf gives 0, as it should; the products below then are 0 or -0, never NaN)
__device__ __forceinline__ float activate(int act, float z) {
    switch (act) {
        case SIGMOID: return sigmoidf(z);
        case RELU: return z < 0.0f ? 0.0f : z;
        case SILU: return z / (1.0f + expf(-z));
        case GELU: return 0.5f * z * erfcf(-z * kSqrtHalf);      // erfc keeps the relative accuracy of the left tail
        default: return z;
    }
}
__device__ __forceinline__ float slope(int act, float z) {
    switch (act) {
        case SIGMOID: { const float a = sigmoidf(z); return a * (1.0f - a); }
        case RELU: return z > 0.0f ? 1.0f : 0.0f;
        case SILU: { const float a = sigmoidf(z); return a * (1.0f + z * (1.0f - a)); }
        case GELU: return 0.5f * erfcf(-z * kSqrtHalf) + z * expf(-0.5f * z * z) * kInvSqrt2Pi;
        default: return 1.0f;
    }
}

}  // namespace ops
}  // namespace lf
