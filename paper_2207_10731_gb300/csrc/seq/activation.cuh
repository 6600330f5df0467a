// The activations of pss_linear_*, and their slopes.
#pragma once

#include "linear.h"

namespace pss {
namespace seq {

constexpr float kRootHalf = 0.70710678118654752f;
constexpr float kInvRoot2Pi = 0.39894228040143268f;

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if (ACT == ACT_RELU) return z < 0.f ? 0.f : z;   // NaN stays
    if (ACT == ACT_GELU) return 0.5f * z * erfcf(-kRootHalf * z);
    if (ACT == ACT_SILU) {
        const float e = __expf(-fabsf(z)), inv = __fdividef(z, 1.f + e);
        return z < 0.f ? e * inv : inv;
    }
    return z;
}

template <int ACT>
__device__ __forceinline__ float slope_of(float z) {
    if (ACT == ACT_RELU) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    if (ACT == ACT_GELU)
        return 0.5f * erfcf(-kRootHalf * z) + z * kInvRoot2Pi * __expf(-0.5f * z * z);
    if (ACT == ACT_SILU) {
        const float e = __expf(-fabsf(z)), inv = __fdividef(1.f, 1.f + e);
        const float s = z < 0.f ? e * inv : inv;
        return s + z * e * inv * inv;
    }
    return 1.f;
}

// f(Int<ACT>()) for the activation `act`.
template <typename F>
__device__ __forceinline__ void with_activation(int act, F f) {
    switch (act) {
        case ACT_RELU: return f(Int<ACT_RELU>());
        case ACT_GELU: return f(Int<ACT_GELU>());
        case ACT_SILU: return f(Int<ACT_SILU>());
        default: return f(Int<ACT_NONE>());
    }
}

}  // namespace seq
}  // namespace pss
