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

#include <algorithm>

#include "rows.cuh"
#include "tc.cuh"

namespace pss {
namespace seq {

constexpr int kNormMaxCols = 16384;

// CTAs an SM, at most, that the backward's partial sums have room for: 1536 threads' worth.
inline int norm_per_sm(int64_t cols) {
    const int64_t threads = cols <= 256 ? 256 : cols <= 4096 ? (cols + 255) / 256 * 32 : 512;
    return (int)(1536 / threads);
}

// Rows up to 32 lanes' vectors, several to a CTA of 256 threads, or with two to a lane twice that, four
// to a CTA of 128: within shuffles.  (40001 x 333 bf16 backward 96 us; by CTAs of two warps to a row
// 146, by eight rows to a CTA 97, on an fp32 stream 119 for want of shared memory.)  Up to 256
// threads' (three CTAs an SM) or 512: a CTA to a row.  These with the next row's loads ahead.  Up to
// 1024 threads', and above with two vectors to a thread: without, for want of room.  (Forward in
// vectors the latter is faster from 512 on, half the warps to a barrier: 8000 x 8192 bf16 on an
// fp32 stream 135 instead of 190 us; backward 370 instead of 322.)
// (Two vectors to a thread for shorter rows too: 495 instead of 434 us for the gradients of
// 65536 x 2048, half the warps.)
enum { NARROW, DOUBLE, MIDDLE, WIDE, WIDER, WIDEST };
template <int VEC, int KIND>
struct Fit {
    static constexpr int kVectors = (VEC == 8 ? 1 : 8) * (KIND == WIDEST || KIND == DOUBLE ? 2 : 1);
    static constexpr bool kWarp = KIND <= DOUBLE;   // a row is a warp's
    static constexpr int kMost = KIND <= MIDDLE ? 256 : KIND == WIDE ? 512 : 1024;
    static constexpr int kLeast = KIND == MIDDLE && VEC == 8 ? 3 : KIND == DOUBLE ? 2 : 1;   // CTAs an SM
    static constexpr bool kAhead = VEC == 8 && KIND <= WIDE;
};
// What is there of norms and gates is known to the kernel where both norms are and rows go in
// vectors (up to 512 threads' aligned ones, 256 threads' others): FULL is the kind of gate then.  ANY
// asks at every turn.
enum { ANY = -1 };

// extra: elements that a ragged row's first vector may hold in front of it; wider: see above.
inline Split norm_split(int cols, int extra, bool wider, int* kind) {
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
    if (units <= 64) {
        *kind = DOUBLE;
        s.lanes = 32;
        s.log2_lanes = 5;
        s.threads = 128;
        s.groups = 4;
        return s;
    }
    *kind = units <= 256 ? MIDDLE : units <= 512 ? WIDE : units <= 1024 && wider ? WIDER : WIDEST;
    s.lanes = ((*kind == WIDEST ? (units + 1) / 2 : units) + 31) / 32 * 32;
    s.threads = s.lanes;
    s.groups = 1;
    return s;
}

__device__ __forceinline__ float2 add_pair(float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }
__device__ __forceinline__ float add_pair(float a, float b) { return a + b; }
__device__ __forceinline__ float2 shuffled(float2 a, int m) {
    return make_float2(__shfl_xor_sync(0xffffffffu, a.x, m), __shfl_xor_sync(0xffffffffu, a.y, m));
}
__device__ __forceinline__ float shuffled(float a, int m) { return __shfl_xor_sync(0xffffffffu, a, m); }

// Sums of one or two values over the row's threads.  A call's slots are not written again before
// the next but one call, so that one barrier a call is enough: `turn` counts.
template <int KIND, typename V>
__device__ __forceinline__ V row_sums(V v, int lanes, float2 (*slots)[32], int& turn) {
    if constexpr (KIND <= DOUBLE) {
        for (int m = lanes >> 1; m > 0; m >>= 1) v = add_pair(v, shuffled(v, m));
        return v;
    } else {
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) v = add_pair(v, shuffled(v, m));
        V* slot = reinterpret_cast<V*>(slots[turn & 1]);
        ++turn;
        const int lane = threadIdx.x & 31, nw = blockDim.x >> 5;
        if (lane == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = V{};
        if (lane < nw) v = slot[lane];
        // no more than 8 or 16 warps
        constexpr int kFirst = KIND == MIDDLE ? 4 : KIND == WIDE ? 8 : 16;
#pragma unroll
        for (int m = kFirst; m > 0; m >>= 1) v = add_pair(v, shuffled(v, m));
        if (KIND <= WIDE) {
            // the lanes behind these hold the sum of nothing: take the first one's
            if constexpr (sizeof(V) == 4) {
                v = __shfl_sync(0xffffffffu, v, 0);
            } else {
                v.x = __shfl_sync(0xffffffffu, v.x, 0);
                v.y = __shfl_sync(0xffffffffu, v.y, 0);
            }
        }
        return v;
    }
}

// sigmoid and its slope, both to a few units in the last place at either end (1 - sigmoid
// would cancel), through exp(-|v|), whose error is about 1.2 |v| units and which is zero below
// 2^-126.  (__expf and __fdividef, which keep numbers below that, are some ten instructions more.)
__device__ __forceinline__ float sigmoid(float v, float* slope = nullptr) {
    const float e = exp2_fast(-1.4426950408889634f * fabsf(v));
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(1.f + e));
    const float low = e * inv;
    if (slope) *slope = low * inv;
    return v < 0.f ? low : inv;
}

// 8 weights of a thread's vector, zeros outside the row.
template <int VEC, int MODE>
__device__ __forceinline__ void load_weight(const float* w, int at, int n, bool in,
                                            float (&to)[VEC]) {
    if constexpr (VEC == 8 && MODE == ALIGNED) {
        if (((uintptr_t)w & 15) == 0) {
            const float4 a = in ? reinterpret_cast<const float4*>(w + at)[0] : float4{};
            const float4 b = in ? reinterpret_cast<const float4*>(w + at)[1] : float4{};
            to[0] = a.x, to[1] = a.y, to[2] = a.z, to[3] = a.w;
            to[4] = b.x, to[5] = b.y, to[6] = b.z, to[7] = b.w;
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i)
        to[i] = in && inside<MODE>(at + i, n, true) ? w[at + i] : 0.f;
}

// A ragged row's first and last vectors hold values of its neighbours: zeros for them, so
// that no sum has to ask whose a value is.  (Other vectors without a row are zeros as they
// come.)
template <int VEC, int MODE>
__device__ __forceinline__ void own_only(float (&v)[VEC], int at, int n) {
    if constexpr (MODE == RAGGED) {
        if (at >= 0 && at + VEC <= n) return;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if ((unsigned)(at + i) >= (unsigned)n) v[i] = 0.f;
    }
}

template <int VEC>
__device__ __forceinline__ void mul(float (&o)[VEC], const float (&a)[VEC], const float (&b)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) o[i] = a[i] * b[i];
}
template <int VEC>
__device__ __forceinline__ void mul(float (&o)[VEC], const float (&a)[VEC], float b) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) o[i] = a[i] * b;
}
// o += a b
template <int VEC>
__device__ __forceinline__ void fma(float (&o)[VEC], const float (&a)[VEC], float b) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) o[i] = fmaf(a[i], b, o[i]);
}
// sum of a b, the even and the odd ones side by side
template <int VEC>
__device__ __forceinline__ float dot(const float (&a)[VEC], const float (&b)[VEC]) {
    float s[2] = {};
#pragma unroll
    for (int i = 0; i < VEC; ++i) s[i & 1] = fmaf(a[i], b[i], s[i & 1]);
    return s[0] + s[1];
}

// A thread's part of a tensor's rows.  AHEAD: of two rows, the one that is worked on and the
// next one, in shared memory, where each thread copies (asynchronously) and reads its own 16-byte
// pieces only, so that no barrier is needed.  In registers the next row's loads took 40 of them,
// and left two CTAs an SM instead of three.
template <typename T, int VEC, int CH, bool AHEAD>
struct Held {
    Part<T, VEC, CH> part;
    __device__ __forceinline__ uint32_t place_at(uint32_t at) { return at; }
    template <int MODE>
    __device__ __forceinline__ void fetch(int, const T* row, bool live, bool whole,
                                          const bool (&in)[CH], const Place<VEC, MODE>& place,
                                          const Shape& sh) {
        part.load(row, live, whole, in, place, sh);
    }
    __device__ __forceinline__ void get(int, int c, float (&to)[VEC]) const { part.get(c, to); }
    __device__ __forceinline__ void own(int, int) const {}
};
template <typename T, int CH>
constexpr int held_bytes() {   // a thread's
    return 2 * CH * 8 * (int)sizeof(T);
}
template <typename T, int CH>
struct Held<T, 8, CH, true> {
    static constexpr int kPieces = sizeof(T) / 2;   // of 16 bytes, to a vector
    uint32_t base, step;
    // the tensor's place from `at` on; returns what follows it
    __device__ __forceinline__ uint32_t place_at(uint32_t at) {
        base = at + threadIdx.x * 16;
        step = blockDim.x * 16;
        return at + blockDim.x * held_bytes<T, CH>();
    }
    __device__ __forceinline__ uint32_t slot(int stage, int c, int h) const {
        return base + ((stage * CH + c) * kPieces + h) * step;
    }
    // A vector that begins before its row is copied as it lies in memory (with what is in front
    // of the row, if `whole` says that there is memory) and cleaned by own() when it has arrived;
    // what lies behind the row's end arrives as zeros.
    template <int MODE>
    __device__ __forceinline__ void fetch(int stage, const T* row, bool live, bool whole,
                                          const bool (&in)[CH], const Place<8, MODE>& place,
                                          const Shape& sh) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = place.at(sh, c);
            if (live && in[c] && (MODE == ALIGNED || whole || at >= 0)) {
#pragma unroll
                for (int h = 0; h < kPieces; ++h) {
                    const T* from = row + at + h * (8 / kPieces);
                    if (MODE == ALIGNED) {
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                                     :: "r"(slot(stage, c, h)), "l"(from) : "memory");
                    } else {
                        // no bytes at all are copied from the vector's own start: the row's may
                        // lie off the 16-byte grid, which no copy's source may
                        const int left = (sh.cols - at) * (int)sizeof(T) - 16 * h;
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                                     :: "r"(slot(stage, c, h)), "l"(left > 0 ? from : row + at),
                                        "r"(min(max(left, 0), 16)) : "memory");
                    }
                }
            } else {
                const Raw8<T> r = live && in[c] ? load_raw_part(row, at, sh.cols, false) : Raw8<T>{};
#pragma unroll
                for (int h = 0; h < kPieces; ++h)
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};"
                                 :: "r"(slot(stage, c, h)), "r"(r.w[4 * h]), "r"(r.w[4 * h + 1]),
                                    "r"(r.w[4 * h + 2]), "r"(r.w[4 * h + 3]) : "memory");
            }
        }
    }
    // Zeros for the values in front of the row: the first thread's, once a row has arrived.
    __device__ __forceinline__ void own(int stage, int before) const {
        for (int i = 0; i < before; ++i) {
            if (sizeof(T) == 4)
                asm volatile("st.shared.u32 [%0], %1;" :: "r"(slot(stage, 0, i / 4) + 4 * (i & 3)), "r"(0)
                             : "memory");
            else
                asm volatile("st.shared.u16 [%0], %1;" :: "r"(slot(stage, 0, 0) + 2 * i), "h"((short)0)
                             : "memory");
        }
    }
    __device__ __forceinline__ void get(int stage, int c, float (&to)[8]) const {
        Raw8<T> r;
#pragma unroll
        for (int h = 0; h < kPieces; ++h)
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(r.w[4 * h]), "=r"(r.w[4 * h + 1]), "=r"(r.w[4 * h + 2]),
                           "=r"(r.w[4 * h + 3]) : "r"(slot(stage, c, h)) : "memory");
        unpack(r, to);
    }
};
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the newest group have arrived.
__device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

enum { NO_GATE, ROW_GATE, VALUE_GATE };   // none, one to a row, one to a value

}  // namespace seq
}  // namespace pss
