// The attention of one row at a time, by one warp: the definition written out,
// lane l holding the values 4l .. 4l+3 of every row.  A masked key is never
// read, so nothing it holds can reach the result.
#pragma once

#include "attention.h"

namespace pss {
namespace seq {

__device__ __forceinline__ float4 row4(const bf16* p, int dim) {
    const int c = 4 * (threadIdx.x & 31);
    if (c >= dim) return make_float4(0.f, 0.f, 0.f, 0.f);
    const uint2 w = *reinterpret_cast<const uint2*>(p + c);
    const float2 a = unpack2(w.x, bf16()), b = unpack2(w.y, bf16());
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ void put4(bf16* p, float4 v, int dim) {
    const int c = 4 * (threadIdx.x & 31);
    if (c >= dim) return;
    uint2 w;
    w.x = pack2(v.x, v.y, bf16());
    w.y = pack2(v.z, v.w, bf16());
    *reinterpret_cast<uint2*>(p + c) = w;
}
__device__ __forceinline__ float dot4(float4 a, float4 b) {
    float s = a.x * b.x + a.y * b.y + a.z * b.z + a.w * b.w;
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
    return s;
}
__device__ __forceinline__ void add4(float4& a, float s, float4 b) {
    a.x += s * b.x;
    a.y += s * b.y;
    a.z += s * b.z;
    a.w += s * b.w;
}

// out and lse of query token t, head h, which sees the keys first .. end.
static __device__ void forward_row(const Attn& a, int first, int end, int t, int h) {
    const int hk = h / a.group;
    const float4 q = row4(a.q.at(t, h), a.dim);
    float top = -INFINITY, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int j = first; j < end; ++j) {
        const float s = dot4(q, row4(a.k.at(j, hk), a.dim)) * a.scale;
        const float next = fmaxf(top, s);
        const float keep = next == -INFINITY ? 1.f : expf(top - next);
        // no weight for a score of -infinity; a NaN, which fmaxf passes over, goes on
        const float p = s == -INFINITY ? 0.f : expf(s - next);
        sum = sum * keep + p;
        o.x *= keep;
        o.y *= keep;
        o.z *= keep;
        o.w *= keep;
        add4(o, p, row4(a.v.at(j, hk), a.dim));
        top = next;
    }
    const float inv = end > first ? 1.f / sum : 0.f;
    put4(a.out.at(t, h), make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv), a.dim);
    if ((threadIdx.x & 31) == 0)
        a.lse[(int64_t)t * a.heads + h] = end > first ? top + logf(sum) : -INFINITY;
}

// dq of query token t, head h.
static __device__ void dq_row(const Attn& a, int first, int end, int t, int h) {
    const int hk = h / a.group;
    const float4 q = row4(a.q.at(t, h), a.dim), g = row4(a.grad.at(t, h), a.dim);
    float4 d = make_float4(0.f, 0.f, 0.f, 0.f);
    if (end > first) {
        const float lse = a.lse[(int64_t)t * a.heads + h];
        const float delta = dot4(g, row4(a.out.at(t, h), a.dim));
        for (int j = first; j < end; ++j) {
            const float4 k = row4(a.k.at(j, hk), a.dim);
            const float p = expf(dot4(q, k) * a.scale - lse);
            add4(d, p * (dot4(g, row4(a.v.at(j, hk), a.dim)) - delta) * a.scale, k);
        }
    }
    put4(a.dq.at(t, h), d, a.dim);
}

// dk and dv of key j, key head hk, which the query tokens first .. end see.
static __device__ void dkv_row(const Attn& a, int first, int end, int j, int hk) {
    const float4 k = row4(a.k.at(j, hk), a.dim), v = row4(a.v.at(j, hk), a.dim);
    float4 dk = make_float4(0.f, 0.f, 0.f, 0.f), dv = dk;
    for (int t = first; t < end; ++t)
        for (int h = hk * a.group; h < (hk + 1) * a.group; ++h) {
            const float4 q = row4(a.q.at(t, h), a.dim), g = row4(a.grad.at(t, h), a.dim);
            const float p = expf(dot4(q, k) * a.scale - a.lse[(int64_t)t * a.heads + h]);
            const float delta = dot4(g, row4(a.out.at(t, h), a.dim));
            add4(dv, p, g);
            add4(dk, p * (dot4(g, v) - delta) * a.scale, q);
        }
    put4(a.dk.at(j, hk), dk, a.dim);
    put4(a.dv.at(j, hk), dv, a.dim);
}

}  // namespace seq
}  // namespace pss
