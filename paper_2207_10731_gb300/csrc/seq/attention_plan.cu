// What an attention call has to know before its products: the work list, what
// each token sees, and for the backward pass two numbers a query row.  One launch.
//
// The sequence lengths live on the device, so the list is made there, by one CTA
// (one more for the list of key tiles): it looks up the sequences at the ends of
// each tile, which gives the tile's range on the other side, and sorts the tiles
// by cost, so that the last ones to start are short.  Where a tile stands among
// those of equal cost follows the scheduling; no result depends on it.  The other
// CTAs meanwhile write every token's range, to be read where the rows are, and
// (lse * log2 e, sum_c grad out) of every row.
//
// The lookups are what takes time: a binary search's steps wait on one another,
// so the offsets of up to kSmallSequences sequences are searched in shared
// memory.
#include "attention.h"

namespace pss {
namespace seq {
namespace {

constexpr int kBuckets = 128;
constexpr int kPlanThreads = 1024;
constexpr int kSmallSequences = 2048, kSmallItems = 1024;
constexpr float kLog2e = 1.4426950408889634f;

// Exact up to 15, four steps to a doubling above.
__device__ __forceinline__ int bucket(int cost) {
    if (cost < 16) return cost;
    const int e = 31 - __clz(cost);
    return min(kBuckets - 1, 16 + (e - 4) * 4 + ((cost >> (e - 2)) & 3));
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

struct PlanShared {
    unsigned count[kBuckets], next[kBuckets];
    unsigned slots, joins, total;
    unsigned long long work;
    int64_t offsets[2][kSmallSequences];
    int from[kSmallItems], tiles[kSmallItems];
};

// The work list of query tiles, or of key tiles.
template <bool KEYS>
__device__ void make_list(const Attn& a, const Plan& p, int target_items, PlanShared& sh) {
    const int tid = threadIdx.x;
    if (tid < kBuckets) sh.count[tid] = 0;
    if (tid == 0) {
        sh.slots = sh.joins = 0;
        sh.work = 0;
        if (!KEYS && a.status) *a.status = ~0ull;
    }
    const int64_t *q_off = a.q_off, *k_off = a.k_off;
    if (a.sequences < kSmallSequences) {
        for (int i = tid; i <= a.sequences; i += kPlanThreads) {
            sh.offsets[0][i] = q_off[i];
            sh.offsets[1][i] = k_off[i];
        }
        q_off = sh.offsets[0];
        k_off = sh.offsets[1];
    }
    __syncthreads();
    if (!KEYS && a.status)
        for (int64_t s = tid; s < a.sequences; s += kPlanThreads)
            if (q_off[s] < 0 || q_off[s] > q_off[s + 1] || q_off[s + 1] > a.q_tokens ||
                k_off[s] < 0 || k_off[s] > k_off[s + 1] || k_off[s + 1] > a.k_tokens)
                atomicMin(a.status, (unsigned long long)s);

    const int step = KEYS ? kTile : p.tokens * p.per_item;
    const int items = KEYS ? p.key_tiles : (p.tiles + p.per_item - 1) / p.per_item;
    const int cap = KEYS ? items : p.most_items;
    const int64_t own_n = KEYS ? a.k_tokens : a.q_tokens;
    const int other = KEYS ? p.key_tokens : p.keys;
    // the other side's range of item i: where it starts, and its tiles
    auto span = [&](int i, int* from) {
        const int64_t first = (int64_t)i * step, past = first + step;
        *from = range_of<KEYS>(a, first, q_off, k_off).lo;
        const int to = range_of<KEYS>(a, (past < own_n ? past : own_n) - 1, q_off, k_off).end();
        return to > *from ? (int)(((int64_t)to - *from + other - 1) / other) : 0;
    };
    const bool kept = items <= kSmallItems;   // asked for once instead of every sweep
    if (kept) {
        for (int i = tid; i < items; i += kPlanThreads) sh.tiles[i] = span(i, &sh.from[i]);
        __syncthreads();
    }
    // sweep 0: total work, where long ranges may be split; 1: count; 2: place
    const bool split = p.most_slots > 0 && !KEYS;
    int chunk = 1 << 30;
    for (int sweep = split ? 0 : 1; sweep < 3; ++sweep) {
        unsigned long long mine = 0;
        // a thread to an item; a warp where an item may have many pieces
        const int lane = tid & 31;
        const bool wide = split && sweep == 2;
        for (int i = wide ? tid >> 5 : tid; i < items; i += wide ? 32 : kPlanThreads) {
            int from;
            const int all = kept ? sh.tiles[i] : span(i, &from);
            if (kept) from = sh.from[i];
            if (sweep == 0) {
                mine += all;
                continue;
            }
            const int parts = all > chunk ? (all + chunk - 1) / chunk : 1;
            const int each = all / parts, rest = all - each * parts;
            const int cost = bucket(each + (rest > 0));
            if (sweep == 1) {
                atomicAdd(&sh.count[cost], (unsigned)parts);
                continue;
            }
            int at = 0, slot = -1;
            if (!wide || lane == 0) {
                at = (int)atomicAdd(&sh.next[cost], (unsigned)parts);
                if (parts > 1) {
                    slot = (int)atomicAdd(&sh.slots, (unsigned)parts);
                    if (slot + parts <= p.most_slots)   // else: cannot be
                        p.joins[atomicAdd(&sh.joins, 1u)] = Join{i * step, slot, parts, 0};
                }
            }
            if (wide) {
                at = __shfl_sync(0xffffffffu, at, 0);
                slot = __shfl_sync(0xffffffffu, slot, 0);
            }
            if (at + parts > cap || (slot >= 0 && slot + parts > p.most_slots)) continue;
            Item* list = (KEYS ? p.key_items : p.items) + at;
            for (int j = wide ? lane : 0; j < parts; j += wide ? 32 : 1) {
                Item it{};
                it.q0 = KEYS ? from : i * step;
                it.k0 = KEYS ? i * step : from;
                it.t0 = j * each + min(j, rest);
                it.t1 = it.t0 + each + (j < rest);
                it.slot = slot < 0 ? -1 : slot + j;
                list[j] = it;
            }
        }
        if (sweep == 0) {
            if (mine) atomicAdd(&sh.work, mine);
            __syncthreads();
            // at most target_items pieces (every tile may end in a short one), and not
            // shorter than kLeastPiece: joining costs a pass over the partial sums
            const unsigned long long whole = max(1, target_items - items);
            const unsigned long long each = (sh.work + whole - 1) / whole;
            chunk = (int)(each < kLeastPiece ? kLeastPiece : each > (1 << 30) ? (1 << 30) : each);
        }
        if (sweep == 1) {
            __syncthreads();
            if (tid < 32) {   // longest first: an exclusive sum from the last bucket down
                unsigned at = 0;
                for (int b = kBuckets - 32; b >= 0; b -= 32) {
                    const unsigned own = sh.count[b + 31 - tid];
                    unsigned sum = own;
#pragma unroll
                    for (int m = 1; m < 32; m <<= 1) {
                        const unsigned up = __shfl_up_sync(0xffffffffu, sum, m);
                        if (tid >= m) sum += up;
                    }
                    sh.next[b + 31 - tid] = at + sum - own;
                    at += __shfl_sync(0xffffffffu, sum, 31);
                }
                if (tid == 0) sh.total = at;
            }
            __syncthreads();
        }
    }
    __syncthreads();
    if (tid == 0 && !KEYS) {
        p.head->items = min((int)sh.total, cap);
        p.head->joins = (int)sh.joins;
    }
}

// How the CTAs of the launch are shared out: the lists, then row statistics,
// then what the query tokens see, then who sees the keys.
struct Roles {
    int lists, stats, queries;
};

__global__ void __launch_bounds__(kPlanThreads)
k_attention_ready(Attn a, Plan p, int target_items, Roles roles) {
    pdl_prologue();
    __shared__ PlanShared sh;
    int block = blockIdx.x;
    if (block < roles.lists) {
        if (block == 0)
            make_list<false>(a, p, target_items, sh);
        else
            make_list<true>(a, p, target_items, sh);
        return;
    }
    block -= roles.lists;
    if (block < roles.stats) {
        const int64_t rows = (int64_t)a.q_tokens * a.heads;
        const int each = a.dim <= 64 ? 16 : 8;   // rows of a warp
        const int64_t warp = (int64_t)block * (kPlanThreads / 32) + (threadIdx.x >> 5);
        for (int64_t first = warp * each; first < rows;
             first += (int64_t)roles.stats * (kPlanThreads / 32) * each) {
            if (a.dim <= 64)
                stats_of<8>(a, p, first);
            else
                stats_of<16>(a, p, first);
        }
        return;
    }
    block -= roles.stats;
    if (block < roles.queries) {
        const int64_t t = (int64_t)block * kPlanThreads + threadIdx.x;
        if (t < a.q_tokens) p.q_range[t] = range_of<false>(a, t, a.q_off, a.k_off);
    } else {
        const int64_t t = (int64_t)(block - roles.queries) * kPlanThreads + threadIdx.x;
        if (t < a.k_tokens) p.k_range[t] = range_of<true>(a, t, a.q_off, a.k_off);
    }
}

}  // namespace

cudaError_t launch_plan(const Attn& a, const Plan& p, bool backward, int target_items,
                        cudaStream_t st) {
    auto blocks = [](int64_t n, int64_t each) { return (int)((n + each - 1) / each); };
    Roles r{backward ? 2 : 1, 0, blocks(a.q_tokens, kPlanThreads)};
    if (backward) {
        // one CTA an SM fits, which then loops over its rows: new CTAs would each wait for
        // their first loads
        const int rows = blocks((int64_t)a.q_tokens * a.heads, 8 * (kPlanThreads / 32));
        const int most = sm_count();
        r.stats = rows < most ? rows : most;
    }
    const int keys = backward ? blocks(a.k_tokens, kPlanThreads) : 0;
    return launch_k(k_attention_ready, dim3(r.lists + r.stats + r.queries + keys),
                    dim3(kPlanThreads), 0, st, a, p, target_items, r);
}

}  // namespace seq
}  // namespace pss
