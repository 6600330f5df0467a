// The work list of an attention call: what each token sees, which tiles that
// makes, the longest first.
//
// The sequence lengths live on the device, so the list is made there, in two
// steps: a thread per token finds its sequence in the offsets and writes the
// range that it sees (coalesced later for whoever needs it); one CTA then turns
// the ranges at the ends of each tile into work items, sorted by cost so that
// the last tiles to start are short ones.  Where a tile stands among those of
// equal cost follows the scheduling; no result depends on it.  A
// forward call of up to kSmallTokens tokens leaves both steps to the one CTA: one
// launch less.
#include "attention.h"

namespace pss {
namespace seq {
namespace {

constexpr int kBuckets = 128;
constexpr int kPlanThreads = 1024;
constexpr int kSmallTokens = 4096;
constexpr int kSmallSequences = 1024, kSmallItems = 1024;
constexpr float kLog2e = 1.4426950408889634f;

// Exact up to 15, four steps to a doubling above.
__device__ __forceinline__ int bucket(int cost) {
    if (cost < 16) return cost;
    const int e = 31 - __clz(cost);
    return min(kBuckets - 1, 16 + (e - 4) * 4 + ((cost >> (e - 2)) & 3));
}

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) {
    return x < lo ? lo : x > hi ? hi : x;
}

// The last sequence that starts at or before t, or -1.
__device__ __forceinline__ int64_t find(const int64_t* off, int64_t n, int64_t t) {
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (off[mid] <= t)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo - 1;
}

// What token t of one side sees on the other side; the offsets may be copies.
template <bool KEYS>
__device__ __forceinline__ Range range_of(const Attn& a, int64_t t, const int64_t* q_off,
                                          const int64_t* k_off) {
    const int64_t* own = KEYS ? k_off : q_off;
    const int64_t* other = KEYS ? q_off : k_off;
    const int64_t own_n = KEYS ? a.k_tokens : a.q_tokens;
    const int64_t other_n = KEYS ? a.q_tokens : a.k_tokens;
    const int64_t s = find(own, a.sequences, t);
    if (s < 0) {
        const int at = (int)clamp64(other[0], 0, other_n);
        return Range{at, -1 - at};
    }
    const int64_t begin = own[s], end = own[s + 1], lo = other[s], hi = other[s + 1];
    if (begin < 0 || t >= end || end > own_n || lo < 0 || lo > hi || hi > other_n) {
        const int at = (int)clamp64(hi, 0, other_n);
        return Range{at, -1 - at};
    }
    if (!a.causal) return Range{(int)lo, (int)hi};
    // query i stands at key i + (end of the keys - end of the queries)
    if (KEYS) return Range{(int)clamp64(t - (end - hi), lo, hi), (int)hi};
    return Range{(int)lo, (int)clamp64(t + 1 + (hi - end), lo, hi)};
}

// (lse * log2 e, sum_c grad out) of consecutive rows of the query side, by a
// warp: LANES lanes to a row, four rows to a thread, all loads before the first
// use.  In the order of the tiles' rows:
// stats[key head][token * group + head of the group].
template <int LANES>
__device__ __forceinline__ void stats_of(const Attn& a, const Plan& p, int64_t first) {
    constexpr int kRows = 4, kSide = 32 / LANES;   // rows of a thread, rows side by side
    const int64_t rows = (int64_t)a.q_tokens * a.heads;
    const int lane = threadIdx.x & 31, c = (lane % LANES) * 8;
    const int64_t row0 = first + lane / LANES;
    const int64_t t0 = row0 / a.heads;
    const int h0 = (int)(row0 - t0 * a.heads);
    uint4 g[kRows], o[kRows];
    int64_t t = t0;
    int h = h0;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        g[i] = o[i] = make_uint4(0, 0, 0, 0);
        if (row0 + i * kSide < rows && c < a.dim) {
            g[i] = load16(a.grad.at(t, h) + c);
            o[i] = load16(a.out.at(t, h) + c);
        }
        for (h += kSide; h >= a.heads; h -= a.heads) ++t;
    }
    t = t0;
    h = h0;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        float s = dot2(g[i].x, o[i].x) + dot2(g[i].y, o[i].y) + dot2(g[i].z, o[i].z) +
                  dot2(g[i].w, o[i].w);
#pragma unroll
        for (int m = LANES / 2; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
        const int64_t row = row0 + i * kSide;
        if (c == 0 && row < rows) {
            const int hk = h / a.group;
            const float lse = a.lse[row];
            p.stats[((int64_t)hk * a.q_tokens + t) * a.group + h - hk * a.group] =
                make_float2(lse == -INFINITY ? INFINITY : lse * kLog2e, s);
        }
        for (h += kSide; h >= a.heads; h -= a.heads) ++t;
    }
}

// blockIdx.y 0: what the query tokens see, 1: who sees the keys, 2: stats.
__global__ void __launch_bounds__(kThreads) k_attention_ready(Attn a, Plan p) {
    pdl_prologue();
    const int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (blockIdx.y == 0) {
        if (t < a.q_tokens) p.q_range[t] = range_of<false>(a, t, a.q_off, a.k_off);
    } else if (blockIdx.y == 1) {
        if (t < a.k_tokens) p.k_range[t] = range_of<true>(a, t, a.q_off, a.k_off);
    } else {
        const int64_t rows = (int64_t)a.q_tokens * a.heads;
        const int each = a.dim <= 64 ? 16 : 8;   // rows of a warp
        const int64_t warp = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
        for (int64_t first = warp * each; first < rows;
             first += (int64_t)gridDim.x * kWarps * each) {
            if (a.dim <= 64)
                stats_of<8>(a, p, first);
            else
                stats_of<16>(a, p, first);
        }
    }
}

__global__ void __launch_bounds__(kPlanThreads)
k_attention_plan(Attn a, Plan p, int target_items, int small) {
    pdl_prologue();
    __shared__ unsigned count[kBuckets], next[kBuckets];
    __shared__ unsigned slots, joins, total;
    __shared__ unsigned long long work;
    __shared__ int64_t offsets[2][kSmallSequences];
    __shared__ int from_of[kSmallItems], tiles_of[kSmallItems];
    const bool keys = blockIdx.x == 1;
    const int tid = threadIdx.x;
    if (tid < kBuckets) count[tid] = 0;
    if (tid == 0) {
        slots = joins = 0;
        work = 0;
        if (!keys && a.status) *a.status = ~0ull;
    }
    if (small) {
        // the search's steps wait on one another: in shared memory where it fits
        const int64_t *q_off = a.q_off, *k_off = a.k_off;
        if (a.sequences < kSmallSequences) {
            for (int i = tid; i <= a.sequences; i += kPlanThreads) {
                offsets[0][i] = q_off[i];
                offsets[1][i] = k_off[i];
            }
            __syncthreads();
            q_off = offsets[0];
            k_off = offsets[1];
        }
        for (int t = tid; t < a.q_tokens; t += kPlanThreads)
            p.q_range[t] = range_of<false>(a, t, q_off, k_off);
    }
    __syncthreads();
    if (!keys && a.status)
        for (int64_t s = tid; s < a.sequences; s += kPlanThreads)
            if (a.q_off[s] < 0 || a.q_off[s] > a.q_off[s + 1] || a.q_off[s + 1] > a.q_tokens ||
                a.k_off[s] < 0 || a.k_off[s] > a.k_off[s + 1] || a.k_off[s + 1] > a.k_tokens)
                atomicMin(a.status, (unsigned long long)s);

    const int tiles = keys ? p.key_tiles : p.tiles;
    const int step = keys ? kTile : p.tokens * p.per_item;
    const int items = keys ? tiles : (p.tiles + p.per_item - 1) / p.per_item;
    const int cap = keys ? items : p.most_items;
    const int64_t own_n = keys ? a.k_tokens : a.q_tokens;
    const Range* ranges = keys ? p.k_range : p.q_range;
    const int other = keys ? p.key_tokens : p.keys;
    // the key range of item i: its first key and its tiles
    auto span = [&](int i, int* from) {
        const int64_t first = (int64_t)i * step, past = first + step;
        *from = ranges[first].lo;
        const int to = ranges[(past < own_n ? past : own_n) - 1].end();
        return to > *from ? (int)(((int64_t)to - *from + other - 1) / other) : 0;
    };
    const bool kept = items <= kSmallItems;   // asked for once instead of every sweep
    if (kept) {
        for (int i = tid; i < items; i += kPlanThreads) tiles_of[i] = span(i, &from_of[i]);
        __syncthreads();
    }
    // sweep 0: total work, where long ranges may be split; 1: count; 2: place
    const bool split = p.most_slots > 0 && !keys;
    int chunk = 1 << 30;
    for (int sweep = split ? 0 : 1; sweep < 3; ++sweep) {
        unsigned long long mine = 0;
        // a thread to an item; a warp where an item may have many pieces
        const int lane = tid & 31;
        const bool wide = split && sweep == 2;
        for (int i = wide ? tid >> 5 : tid; i < items; i += wide ? 32 : kPlanThreads) {
            int from;
            const int all = kept ? tiles_of[i] : span(i, &from);
            if (kept) from = from_of[i];
            if (sweep == 0) {
                mine += all;
                continue;
            }
            const int parts = all > chunk ? (all + chunk - 1) / chunk : 1;
            const int each = all / parts, rest = all - each * parts;
            const int cost = bucket(each + (rest > 0));
            if (sweep == 1) {
                atomicAdd(&count[cost], (unsigned)parts);
                continue;
            }
            int at = 0, slot = -1;
            if (!wide || lane == 0) {
                at = (int)atomicAdd(&next[cost], (unsigned)parts);
                if (parts > 1) {
                    slot = (int)atomicAdd(&slots, (unsigned)parts);
                    if (slot + parts <= p.most_slots)   // else: cannot be
                        p.joins[atomicAdd(&joins, 1u)] = Join{i * step, slot, parts, 0};
                }
            }
            if (wide) {
                at = __shfl_sync(0xffffffffu, at, 0);
                slot = __shfl_sync(0xffffffffu, slot, 0);
            }
            if (at + parts > cap || (slot >= 0 && slot + parts > p.most_slots)) continue;
            Item* list = (keys ? p.key_items : p.items) + at;
            for (int j = wide ? lane : 0; j < parts; j += wide ? 32 : 1) {
                Item it{};
                it.q0 = keys ? from : i * step;
                it.k0 = keys ? i * step : from;
                it.t0 = j * each + min(j, rest);
                it.t1 = it.t0 + each + (j < rest);
                it.slot = slot < 0 ? -1 : slot + j;
                list[j] = it;
            }
        }
        if (sweep == 0) {
            if (mine) atomicAdd(&work, mine);
            __syncthreads();
            // at most target_items pieces (every tile may end in a short one), and not
            // shorter than kLeastPiece: joining costs a pass over the partial sums
            const unsigned long long whole = max(1, target_items - items);
            const unsigned long long each = (work + whole - 1) / whole;
            chunk = (int)(each < kLeastPiece ? kLeastPiece : each > (1 << 30) ? (1 << 30) : each);
        }
        if (sweep == 1) {
            __syncthreads();
            if (tid < 32) {   // longest first: an exclusive sum from the last bucket down
                unsigned at = 0;
                for (int b = kBuckets - 32; b >= 0; b -= 32) {
                    const unsigned own = count[b + 31 - tid];
                    unsigned sum = own;
#pragma unroll
                    for (int m = 1; m < 32; m <<= 1) {
                        const unsigned up = __shfl_up_sync(0xffffffffu, sum, m);
                        if (tid >= m) sum += up;
                    }
                    next[b + 31 - tid] = at + sum - own;
                    at += __shfl_sync(0xffffffffu, sum, 31);
                }
                if (tid == 0) total = at;
            }
            __syncthreads();
        }
    }
    __syncthreads();
    if (tid == 0 && !keys) {
        p.head->items = min((int)total, cap);
        p.head->joins = (int)joins;
    }
}

}  // namespace

cudaError_t launch_plan(const Attn& a, const Plan& p, bool backward, int target_items,
                        cudaStream_t st) {
    const int64_t most = backward && a.k_tokens > a.q_tokens ? a.k_tokens : a.q_tokens;
    const bool small = !backward && most <= kSmallTokens;
    if (!small && most > 0) {
        int64_t blocks = (most + kThreads - 1) / kThreads;
        if (backward) {
            // the rows of stats, up to 32 CTAs an SM in all
            const int64_t rows = ((int64_t)a.q_tokens * a.heads + 8 * kWarps - 1) / (8 * kWarps);
            const int64_t enough = (int64_t)sm_count() * 32;
            const int64_t some = rows < enough ? rows : enough;
            if (blocks < some) blocks = some;
        }
        const cudaError_t e = launch_k(k_attention_ready, dim3((unsigned)blocks, backward ? 3 : 1),
                                       dim3(kThreads), 0, st, a, p);
        if (e != cudaSuccess) return e;
    }
    return launch_k(k_attention_plan, dim3(backward ? 2 : 1), dim3(kPlanThreads), 0, st, a, p,
                    target_items, (int)small);
}

}  // namespace seq
}  // namespace pss
