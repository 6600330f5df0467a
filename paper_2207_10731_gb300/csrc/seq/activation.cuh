// The activations of pss_linear_*, and their slopes.
#pragma once

#include "linear.h"

namespace pss {
namespace seq {

constexpr float kInvRoot2Pi = 0.39894228040143268f;

// 1 / x of a normal number with a normal reciprocal, to a unit in the last place.
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Phi(-a) = exp(-a^2 / 2) P(t) for a >= 0, t = 1 / (1 + 0.23 a): P is the polynomial of degree 8
// nearest to erfcx(a / sqrt 2) / 2 in relative error on 0 <= a <= 15 (a least-squares fit
// with weights raised where it is worst; 8.3e-8 with these coefficients, and 4.6e-7 evaluated in
// fp32).  gelu and its slope share the exponential, and both ends keep their relative accuracy.
// With CUDA's erfcf, which is exact to a few units, the pass over the gradient of 16384 x 4096
// took 144 us when it took 85 with this; it has become 69 since (linear.cu).
__device__ __forceinline__ float normal_below(float a, float e) {
    const float t = reciprocal(fmaf(0.23f, a, 1.f));
    float p = -0.07848794013261795f;
    p = fmaf(p, t, 0.2905181646347046f);
    p = fmaf(p, t, -0.2783527970314026f);
    p = fmaf(p, t, 0.30174607038497925f);
    p = fmaf(p, t, -0.033121444284915924f);
    p = fmaf(p, t, 0.11960627138614655f);
    p = fmaf(p, t, 0.08573728799819946f);
    p = fmaf(p, t, 0.09238240122795105f);
    p = fmaf(p, t, -2.8019605451845564e-05f);
    return e * p;
}

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if (ACT == ACT_RELU) return z < 0.f ? 0.f : z;   // NaN stays
    if (ACT == ACT_GELU) {
        // q is zero from 15 on: from there z itself, also where it is infinite and z q is not a number
        const float q = normal_below(fabsf(z), __expf(-0.5f * z * z));
        return z < 0.f ? z * q : z - fminf(z, 128.f) * q;
    }
    if (ACT == ACT_SILU) {
        const float e = __expf(-fabsf(z)), inv = z * reciprocal(1.f + e);
        return z < 0.f ? e * inv : inv;
    }
    return z;
}

template <int ACT>
__device__ __forceinline__ float slope_of(float z) {
    if (ACT == ACT_RELU) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    if (ACT == ACT_GELU) {
        // e is zero below 2^-126, and so is the slope's part from there on (three instructions
        // in about thirty)
        float e;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-0.72134752044448170f * z * z));
        const float q = normal_below(fabsf(z), e);
        return (z < 0.f ? q : 1.f - q) + z * kInvRoot2Pi * e;
    }
    if (ACT == ACT_SILU) {
        const float e = __expf(-fabsf(z)), inv = reciprocal(1.f + e);
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
