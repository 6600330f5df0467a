// The norms after and before a block, with its gate and the residual stream between
// them (pss_residual_norm_* of pss.h): what both directions share.
//
// Forward, one row of n values, r(v) = 1 / sqrt(sum v^2 / n + eps):
//   u = x r(x) w_post  (u = x without the first norm),
//   t = residual + scale sigmoid(gate) u,      y = t r(t) w_pre.
// Backward, with that = t r(t), xhat = x r(x), s = sigmoid(gate):
//   g = dy w_pre,   d = dt + r(t) (g - that sum(g that) / n)        (= dresidual),
//   dgate = scale d u s (1 - s)        (summed over the row where it has one gate),
//   e = scale d s,  h = e w_post,  dx = r(x) (h - xhat sum(h xhat) / n),
//   dw_pre = sum over rows of dy that,  dw_post = sum over rows of e xhat.
#pragma once

#include "rows.cuh"

namespace pss {
namespace seq {

constexpr int kNormMaxCols = 16384;

// CTAs an SM, at most, that the backward's partial sums have room for: 1024 threads' worth
// (40001 x 333 with four of 64 threads: 182 us).
inline int norm_per_sm(int64_t cols) {
    const int64_t threads = cols <= 256 ? 256 : cols <= 4096 ? (cols + 255) / 256 * 32 : 512;
    return (int)(1024 / threads);
}

// Rows up to 32 lanes' vectors: several to a CTA of 256 threads, within shuffles.  Up to
// 512 threads': a CTA to a row, the next row's loads ahead.  Above: two vectors to a
// thread, 1024 threads at most, whose 64 registers leave no room for a second row.
enum { NARROW, WIDE, WIDEST };
template <int VEC, int KIND>
struct Fit {
    static constexpr int kVectors = (VEC == 8 ? 1 : 8) * (KIND == WIDEST ? 2 : 1);
    static constexpr int kMost = KIND == NARROW ? 256 : KIND == WIDE ? 512 : 1024;
    static constexpr bool kAhead = KIND != WIDEST;
};

// extra: elements that a ragged row's first vector may hold in front of it.
inline Split norm_split(int cols, int extra, int* kind) {
    Split s;
    const int units = (cols + extra + 7) / 8;   // of 8 elements, VEC = 8 or 1
    s.ch = 0;
    s.log2_lanes = 0;
    if (units <= 32) {
        *kind = NARROW;
        s.lanes = 1;
        while (s.lanes < units) s.lanes *= 2, ++s.log2_lanes;
        s.threads = 256;
        s.groups = 256 / s.lanes;
        return s;
    }
    *kind = units <= 512 ? WIDE : WIDEST;
    s.lanes = ((*kind == WIDE ? units : (units + 1) / 2) + 31) / 32 * 32;
    s.threads = s.lanes;
    s.groups = 1;
    return s;
}

// Sums over the row's threads, both at once.  A call's slots are not written again
// before the next but one call, so that one barrier a call is enough: `turn` counts.
__device__ __forceinline__ float2 row_sums(float2 v, int lanes, float2 (*slots)[32], int& turn) {
    const int w = lanes < 32 ? lanes : 32;
    for (int m = w >> 1; m > 0; m >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, m);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, m);
    }
    if (lanes <= 32) return v;
    float2* slot = slots[turn & 1];
    ++turn;
    const int lane = threadIdx.x & 31, nw = blockDim.x >> 5;
    if (lane == 0) slot[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < nw ? slot[lane] : make_float2(0.f, 0.f);
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, m);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, m);
    }
    return v;
}

// sigmoid and its slope, both to a few units in the last place at either end (1 - sigmoid
// would cancel): through exp(-|v|), whose error is about 1.2 |v| units.
__device__ __forceinline__ float sigmoid(float v, float* slope = nullptr) {
    const float e = __expf(-fabsf(v)), inv = __fdividef(1.f, 1.f + e);
    if (slope) *slope = e * inv * inv;
    return v < 0.f ? e * inv : inv;
}

// 8 weights of a thread's vector, zeros outside the row.
template <int VEC, int MODE>
__device__ __forceinline__ void load_weight(const float* w, int at, int n, bool in,
                                            float (&to)[VEC]) {
    if (VEC == 8 && MODE == ALIGNED && ((uintptr_t)w & 15) == 0) {
        const float4 a = in ? reinterpret_cast<const float4*>(w + at)[0] : float4{};
        const float4 b = in ? reinterpret_cast<const float4*>(w + at)[1] : float4{};
        to[0] = a.x, to[1 % VEC] = a.y, to[2 % VEC] = a.z, to[3 % VEC] = a.w;
        to[4 % VEC] = b.x, to[5 % VEC] = b.y, to[6 % VEC] = b.z, to[7 % VEC] = b.w;
        return;
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i)
        to[i] = in && inside<MODE>(at + i, n, true) ? w[at + i] : 0.f;
}

enum { NO_GATE, ROW_GATE, VALUE_GATE };   // none, one to a row, one to a value

}  // namespace seq
}  // namespace pss
