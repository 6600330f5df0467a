// Rows that the tiles cannot answer, computed again by a warp: those whose result
// is not finite (a product with a zero probability takes up an infinite or NaN
// value behind the mask) and those whose tile did not come to its end.
//
// A warp takes 16 rows against 16 rows of the other side at a time, operands from
// global memory (L1 holds them) straight into the fragments of the warp-level
// product 16 x 8 x 16, fp32 sums in registers.  Where all rows see all 16, nothing
// is behind a mask and the products stand.  Elsewhere what is not finite on the
// other side is taken out of the second product and added, element by element, to
// the rows that see it; a block whose sums are all NaN stops.  So one bad value costs
// its tile a second pass at a fraction of the tensor core's speed, not a walk over single
// keys: a NaN in a training step must not hold the GPU for seconds.  Measured: training
// pass of 4 x 2-7.8 k tokens, 16/4 heads of 128, 1.57 ms clean, 5.8 ms with a NaN in the
// last gradient, 6.1 in the last value, 3.7 where everything is NaN; the dearest is a
// forward pass in which every value is NaN and no score (8192 tokens, 16/4 heads of 128:
// 4.5 ms instead of 0.27).
//
// Lane 4 g + t holds of a row (g) the values 32 q + 8 t .. + 8 for each q, as words
// of two: the contraction does not mind the order of its columns, and a word's
// 8 x 8 block transposed is the second product's operand, whose result then has
// the same columns in the same lane.
#pragma once

#include <climits>

#include "attention.h"

namespace pss {
namespace seq {

constexpr unsigned kLanes = 0xffffffffu;

// acc (16 x 8) += A (16 x 16) B (16 x 8): rows g and g + 8 of A are x0, x2 and x1, x3.
__device__ __forceinline__ void warp_mma(float (&acc)[4], uint32_t x0, uint32_t x1, uint32_t x2,
                                         uint32_t x3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7},"
        " {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(acc[0]), "+f"(acc[1]), "+f"(acc[2]), "+f"(acc[3])
        : "r"(x0), "r"(x1), "r"(x2), "r"(x3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t w) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(w));
    return r;
}

// 8 values from column c of a row; zeros past its end and where there is no row.
__device__ __forceinline__ uint4 row8(const bf16* row, int c, int dim) {
    return row && c < dim ? *reinterpret_cast<const uint4*>(row + c) : make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ void put8(bf16* p, const float (&v)[8]) {
    uint4 w;
    w.x = pack2(v[0], v[1], bf16());
    w.y = pack2(v[2], v[3], bf16());
    w.z = pack2(v[4], v[5], bf16());
    w.w = pack2(v[6], v[7], bf16());
    *reinterpret_cast<uint4*>(p) = w;
}

// s[b][2 i + e]: row 8 i + g of x with row 8 b + 2 t + e of y.  y stays in `kept`.
template <int HD>
__device__ __forceinline__ void row_products(float (&s)[2][4], const bf16* const (&x)[2],
                                             const bf16* const (&y)[2], int dim,
                                             uint32_t (&kept)[2][HD / 8]) {
    const int t = threadIdx.x & 3;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[b][e] = 0.f;
#pragma unroll
    for (int q = 0; q < HD / 32; ++q) {
        const int c = 32 * q + 8 * t;
        const uint4 x0 = row8(x[0], c, dim), x1 = row8(x[1], c, dim);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const uint4 w = row8(y[b], c, dim);
            kept[b][4 * q] = w.x;
            kept[b][4 * q + 1] = w.y;
            kept[b][4 * q + 2] = w.z;
            kept[b][4 * q + 3] = w.w;
            warp_mma(s[b], x0.x, x1.x, x0.y, x1.y, w.x, w.y);
            warp_mma(s[b], x0.z, x1.z, x0.w, x1.w, w.z, w.w);
        }
    }
}

// Whether either half of a word of two bf16 is not finite.
__device__ __forceinline__ bool low_odd(uint32_t w) { return (w & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ bool high_odd(uint32_t w) {
    return (w & 0x7f800000u) == 0x7f800000u;
}

// acc[n] += P y, P (16 x 16, as row_products leaves it) rounded to bf16, with TWO its
// rest in a second product.  acc[4 q + i][2 r + e]: row 8 r + g, column 32 q + 8 t +
// 2 i + e.  whole: every row sees all 16 rows of y; else seen(r, k) says whether
// the lane's row 8 r + g sees row k.
template <int HD, bool TWO, typename F>
__device__ __forceinline__ void add_rows(float (&acc)[HD / 8][4], const float (&p)[2][4],
                                         const uint32_t (&y)[2][HD / 8], bool whole, F seen) {
    const int lane = threadIdx.x & 31, t = lane & 3;
    uint32_t a[2][2], rest[2][2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            a[b][r] = pack2(p[b][2 * r], p[b][2 * r + 1], bf16());
            const float2 kept = unpack2(a[b][r], bf16());
            rest[b][r] = pack2(p[b][2 * r] - kept.x, p[b][2 * r + 1] - kept.y, bf16());
        }
#pragma unroll
    for (int n = 0; n < HD / 8; ++n) {
        uint32_t w[2] = {y[0][n], y[1][n]};
        const bool odd = low_odd(w[0]) || high_odd(w[0]) || low_odd(w[1]) || high_odd(w[1]);
        if (!whole && __any_sync(kLanes, odd)) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll 1
                for (int k = 0; k < 8; ++k) {
                    const uint32_t word = __shfl_sync(kLanes, w[b], 4 * k + t);
                    const float2 v = unpack2(word, bf16());
                    const int from = (lane & 28) + k / 2;   // who holds P of row k
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float even = __shfl_sync(kLanes, p[b][2 * r], from);
                        const float uneven = __shfl_sync(kLanes, p[b][2 * r + 1], from);
                        const float weight = k & 1 ? uneven : even;
                        if (!seen(r, 8 * b + k)) continue;
                        if (low_odd(word)) acc[n][2 * r] += weight * v.x;
                        if (high_odd(word)) acc[n][2 * r + 1] += weight * v.y;
                    }
                }
                if (low_odd(w[b])) w[b] &= 0xffff0000u;
                if (high_odd(w[b])) w[b] &= 0xffffu;
            }
        }
        const uint32_t b0 = transposed(w[0]), b1 = transposed(w[1]);
        warp_mma(acc[n], a[0][0], a[0][1], a[1][0], a[1][1], b0, b1);
        if (TWO) warp_mma(acc[n], rest[0][0], rest[0][1], rest[1][0], rest[1][1], b0, b1);
    }
}

// The lane's two of 16 rows: rows 8 r + g of block `blk` of the warp's 32, each brought
// by its own lane.  A row that is not wanted sees nothing.
struct Pair {
    bool want[2];
    int lo[2], hi[2];   // what they see
    int from, to;       // what any of the 16 sees
    __device__ __forceinline__ Pair(unsigned wanted, int blk, int own_lo, int own_hi) {
        const int g = (threadIdx.x & 31) >> 2;
        int first = INT_MAX, last = 0;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int src = 16 * blk + 8 * r + g;
            want[r] = (wanted >> src) & 1;
            lo[r] = __shfl_sync(kLanes, own_lo, src);
            hi[r] = __shfl_sync(kLanes, own_hi, src);
            if (!want[r] || hi[r] <= lo[r]) {
                lo[r] = hi[r] = 0;
            } else {
                first = min(first, lo[r]);
                last = max(last, hi[r]);
            }
        }
        from = __reduce_min_sync(kLanes, first);
        to = __reduce_max_sync(kLanes, last);
    }
    __device__ __forceinline__ bool none(int r) const { return hi[r] <= lo[r]; }
};

// Takes the rows of one sequence out of those left in a block: the ones that agree
// with the first on where the other side begins (query rows) or ends (key rows).
// One sequence at a time, since where two share a block no step would be whole.
__device__ __forceinline__ unsigned one_sequence(unsigned& left, int blk, int at) {
    const int first = __shfl_sync(kLanes, at, __ffs(left) - 1);
    const unsigned same = __ballot_sync(kLanes, at == first) & left & (0xffffu << (16 * blk));
    left &= ~same;
    return same;
}

// Whether every value of every row's sum is NaN: nothing added changes that.
template <int HD>
__device__ __forceinline__ bool all_nan(const float (&d)[HD / 8][4], const Pair& see, int dim) {
    bool all = true;
#pragma unroll
    for (int q = 0; q < HD / 32; ++q) {
        if (32 * q + 8 * (int)(threadIdx.x & 3) >= dim) break;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) all = all && (see.none(e / 2) || isnan(d[4 * q + i][e]));
    }
    return __all_sync(kLanes, all);
}
constexpr int kAsk = 128;   // rows of the other side between two looks

// out and lse of the rows wanted among a warp's 32, lane l's being query token `token`,
// head h, which sees the keys lo .. hi.  partial: null, or where the warp's first row
// goes as a piece of a split range ([row][dim] fp32 sums / denominators, and its lse).
template <int HD>
static __device__ __noinline__ void forward_rows(const Attn& a, int hk, int token, int h, int lo,
                                                 int hi, bool want, float* partial,
                                                 float* partial_lse) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const unsigned wanted = __ballot_sync(kLanes, want);
#pragma unroll 1
    for (unsigned left = wanted; left;) {
        const int blk = (__ffs(left) - 1) / 16;
        const Pair see(one_sequence(left, blk, lo), blk, lo, hi);
        const bf16* x[2];
        int tok[2], head[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            tok[r] = __shfl_sync(kLanes, token, 16 * blk + 8 * r + g);
            head[r] = __shfl_sync(kLanes, h, 16 * blk + 8 * r + g);
            x[r] = see.want[r] ? a.q.at(tok[r], head[r]) : nullptr;
        }
        float o[HD / 8][4], top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
        for (int n = 0; n < HD / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
#pragma unroll 1
        for (int j = see.from; j < see.to; j += 16) {
            const bf16* y[2];
            const bf16* z[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int key = j + 8 * b + g;
                y[b] = key < see.to ? a.k.at(key, hk) : nullptr;
                z[b] = key < see.to ? a.v.at(key, hk) : nullptr;
            }
            uint32_t kept[2][HD / 8];
            float s[2][4];
            row_products<HD>(s, x, y, a.dim, kept);
            bool whole = true;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                whole = whole && (see.none(r) || (see.lo[r] <= j && see.hi[r] >= j + 16));
                float next = top[r];
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int key = j + 8 * b + 2 * t + e;
                        float& v = s[b][2 * r + e];
                        v = key >= see.lo[r] && key < see.hi[r] ? v * a.scale : -INFINITY;
                        next = fmaxf(next, v);
                    }
                next = fmaxf(next, __shfl_xor_sync(kLanes, next, 1));
                next = fmaxf(next, __shfl_xor_sync(kLanes, next, 2));
                const float keep = next == -INFINITY ? 1.f : expf(top[r] - next);
                top[r] = next;
                sum[r] *= keep;
#pragma unroll
                for (int n = 0; n < HD / 8; ++n) {
                    o[n][2 * r] *= keep;
                    o[n][2 * r + 1] *= keep;
                }
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        // no weight for a score of -infinity; a NaN, which fmaxf passes
                        // over, goes on
                        float& v = s[b][2 * r + e];
                        v = v == -INFINITY ? 0.f : expf(v - next);
                        sum[r] += v;
                    }
            }
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int q = 0; q < HD / 32; ++q) {
                    const uint4 w = row8(z[b], 32 * q + 8 * t, a.dim);
                    kept[b][4 * q] = w.x;
                    kept[b][4 * q + 1] = w.y;
                    kept[b][4 * q + 2] = w.z;
                    kept[b][4 * q + 3] = w.w;
                }
            add_rows<HD, false>(o, s, kept, __all_sync(kLanes, whole), [&](int r, int k) {
                return j + k >= see.lo[r] && j + k < see.hi[r];
            });
            // a NaN sum makes the row and its lse NaN
            if ((j - see.from) % kAsk == kAsk - 16) {
                bool all = true;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const unsigned odd = __ballot_sync(kLanes, isnan(sum[r]));
                    all = all && (see.none(r) || ((odd >> (lane & 28)) & 15u));
                }
                if (__all_sync(kLanes, all)) break;
            }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float total = sum[r] + __shfl_xor_sync(kLanes, sum[r], 1);
            total += __shfl_xor_sync(kLanes, total, 2);
            if (!see.want[r]) continue;
            const bool none = see.none(r);
            const float inv = 1.f / total, lse = none ? -INFINITY : top[r] + logf(total);
            const int row = 16 * blk + 8 * r + g;
#pragma unroll
            for (int q = 0; q < HD / 32; ++q) {
                const int c = 32 * q + 8 * t;
                if (c >= a.dim) break;
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = none ? 0.f : o[4 * q + i / 2][2 * r + (i & 1)] * inv;
                if (!partial)
                    put8(a.out.at(tok[r], head[r]) + c, v);
                else if (lse != -INFINITY)
                    store8(partial + (int64_t)row * a.dim + c, v);
            }
            if (t == 0) {
                if (!partial)
                    a.lse[(int64_t)tok[r] * a.heads + head[r]] = lse;
                else
                    partial_lse[row] = lse;
            }
        }
    }
}

// dq of the rows wanted in block `blk` of a warp's 32; stats: lane l's (lse * log2 e, or
// +infinity where that is -infinity; delta).
template <int HD>
static __device__ __noinline__ void dq_rows(const Attn& a, int hk, int token, int h, int lo, int hi,
                                            bool want, float2 stats, int blk) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const unsigned wanted = __ballot_sync(kLanes, want);
    const float c2 = a.scale * 1.4426950408889634f;
#pragma unroll 1
    for (unsigned left = wanted & (0xffffu << (16 * blk)); left;) {
        const Pair see(one_sequence(left, blk, lo), blk, lo, hi);
        const bf16 *x[2], *u[2];
        int tok[2], head[2];
        float l[2], delta[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int src = 16 * blk + 8 * r + g;
            tok[r] = __shfl_sync(kLanes, token, src);
            head[r] = __shfl_sync(kLanes, h, src);
            l[r] = __shfl_sync(kLanes, stats.x, src);
            delta[r] = __shfl_sync(kLanes, stats.y, src);
            x[r] = see.want[r] ? a.q.at(tok[r], head[r]) : nullptr;
            u[r] = see.want[r] ? a.grad.at(tok[r], head[r]) : nullptr;
        }
        float d[HD / 8][4];
#pragma unroll
        for (int n = 0; n < HD / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[n][e] = 0.f;
#pragma unroll 1
        for (int j = see.from; j < see.to; j += 16) {
            const bf16 *y[2], *z[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int key = j + 8 * b + g;
                y[b] = key < see.to ? a.k.at(key, hk) : nullptr;
                z[b] = key < see.to ? a.v.at(key, hk) : nullptr;
            }
            uint32_t kept[2][HD / 8];
            float s[2][4], dp[2][4];
            row_products<HD>(dp, u, z, a.dim, kept);
            row_products<HD>(s, x, y, a.dim, kept);
            bool whole = true;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                whole = whole && (see.none(r) || (see.lo[r] <= j && see.hi[r] >= j + 16));
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int key = j + 8 * b + 2 * t + e;
                        float& v = s[b][2 * r + e];
                        v = key >= see.lo[r] && key < see.hi[r]
                                ? exp2f(v * c2 - l[r]) * (dp[b][2 * r + e] - delta[r])
                                : 0.f;
                    }
            }
            add_rows<HD, true>(d, s, kept, __all_sync(kLanes, whole), [&](int r, int k) {
                return j + k >= see.lo[r] && j + k < see.hi[r];
            });
            if ((j - see.from) % kAsk == kAsk - 16 && all_nan<HD>(d, see, a.dim)) break;
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (!see.want[r]) continue;
#pragma unroll
            for (int q = 0; q < HD / 32; ++q) {
                const int c = 32 * q + 8 * t;
                if (c >= a.dim) break;
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = see.none(r) ? 0.f : d[4 * q + i / 2][2 * r + (i & 1)] * a.scale;
                put8(a.dq.at(tok[r], head[r]) + c, v);
            }
        }
    }
}

// dk (DK) or dv of the rows wanted among a warp's 32, lane l's being key `key`, which
// the query tokens lo .. hi see.  Without the tiles' factor on P, which a large dO may
// not bear: exp2f keeps what is below the normal numbers, and so does bf16.
template <int HD, bool DK>
static __device__ __noinline__ void dkv_rows(const Attn& a, const float2* all_stats, int hk, int key,
                                             int lo, int hi, bool want) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const unsigned wanted = __ballot_sync(kLanes, want);
    const float c2 = a.scale * 1.4426950408889634f;
    const float2* stats = all_stats + (int64_t)hk * a.q_tokens * a.group;
    const Rows& to_rows = DK ? a.dk : a.dv;
#pragma unroll 1
    for (unsigned left = wanted; left;) {
        const int blk = (__ffs(left) - 1) / 16;
        const Pair see(one_sequence(left, blk, hi), blk, lo, hi);
        const bf16 *x[2], *u[2];
        int own[2];
        int64_t first[2], last[2];   // rows of the query side, group to a token
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            own[r] = __shfl_sync(kLanes, key, 16 * blk + 8 * r + g);
            x[r] = see.want[r] ? a.k.at(own[r], hk) : nullptr;
            u[r] = see.want[r] ? a.v.at(own[r], hk) : nullptr;
            first[r] = (int64_t)see.lo[r] * a.group;
            last[r] = (int64_t)see.hi[r] * a.group;
        }
        float d[HD / 8][4];
#pragma unroll
        for (int n = 0; n < HD / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[n][e] = 0.f;
        const int64_t from = see.to > 0 ? (int64_t)see.from * a.group : 0;
        const int64_t to = (int64_t)see.to * a.group;
        // the lane's two rows of the query side, 16 further on at every step
        int tok[2], h[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            tok[b] = (see.to > 0 ? see.from : 0) + (8 * b + g) / a.group;
            h[b] = (8 * b + g) % a.group;
        }
        const int more_tokens = 16 / a.group, more_heads = 16 % a.group;
#pragma unroll 1
        for (int64_t j = from; j < to; j += 16) {
            const bf16 *y[2], *z[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const bool there = j + 8 * b + g < to;
                y[b] = there ? a.q.at(tok[b], hk * a.group + h[b]) : nullptr;
                z[b] = there ? a.grad.at(tok[b], hk * a.group + h[b]) : nullptr;
                tok[b] += more_tokens;
                h[b] += more_heads;
                if (h[b] >= a.group) {
                    h[b] -= a.group;
                    ++tok[b];
                }
            }
            uint32_t kept[2][HD / 8];
            float s[2][4], dp[2][4];
            if (DK) row_products<HD>(dp, u, z, a.dim, kept);
            row_products<HD>(s, x, y, a.dim, kept);
            bool whole = true;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int64_t row = j + 8 * b + 2 * t + e;
                    const float2 st = row < to ? stats[row] : make_float2(INFINITY, 0.f);
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float& v = s[b][2 * r + e];
                        const float p = exp2f(v * c2 - st.x);
                        v = row < first[r] || row >= last[r] ? 0.f
                            : DK ? p * (dp[b][2 * r + e] - st.y)
                                 : p;
                    }
                }
#pragma unroll
            for (int r = 0; r < 2; ++r)
                whole = whole && (see.none(r) || (first[r] <= j && last[r] >= j + 16));
            if (!DK) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int q = 0; q < HD / 32; ++q) {
                        const uint4 w = row8(z[b], 32 * q + 8 * t, a.dim);
                        kept[b][4 * q] = w.x;
                        kept[b][4 * q + 1] = w.y;
                        kept[b][4 * q + 2] = w.z;
                        kept[b][4 * q + 3] = w.w;
                    }
            }
            add_rows<HD, false>(d, s, kept, __all_sync(kLanes, whole), [&](int r, int k) {
                return j + k >= first[r] && j + k < last[r];
            });
            if ((j - from) % kAsk == kAsk - 16 && all_nan<HD>(d, see, a.dim)) break;
        }
        const float scale = DK ? a.scale : 1.f;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (!see.want[r]) continue;
#pragma unroll
            for (int q = 0; q < HD / 32; ++q) {
                const int c = 32 * q + 8 * t;
                if (c >= a.dim) break;
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = see.none(r) ? 0.f : d[4 * q + i / 2][2 * r + (i & 1)] * scale;
                put8(to_rows.at(own[r], hk) + c, v);
            }
        }
    }
}

}  // namespace seq
}  // namespace pss
