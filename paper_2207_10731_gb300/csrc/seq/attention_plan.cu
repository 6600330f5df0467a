// The work list of an attention call: which tiles of query rows (and of key
// rows, for the backward pass) the packed sequences make, the longest first.
//
// The sequence lengths live on the device, so the list is made there: one CTA,
// a warp per sequence and a lane per tile, two sweeps (count by cost, place).
// Sorted by cost so that the last tiles to start are short ones.  Where a tile
// stands among those of equal cost follows the scheduling; no result depends
// on it.
#include "attention.h"

namespace pss {
namespace seq {
namespace {

constexpr int kBuckets = 128;

// Exact up to 15, four steps to a doubling above.
__device__ __forceinline__ int bucket(int cost) {
    if (cost < 16) return cost;
    const int e = 31 - __clz(cost);
    return min(kBuckets - 1, 16 + (e - 4) * 4 + ((cost >> (e - 2)) & 3));
}

__device__ bool range_of(const int64_t* off, int64_t s, int64_t tokens, int* lo, int* hi) {
    const int64_t a = off[s], b = off[s + 1];
    const bool ok = a >= 0 && a <= b && b <= tokens;
    *lo = ok ? (int)a : 0;
    *hi = ok ? (int)b : 0;
    return ok;
}

__global__ void __launch_bounds__(1024) k_attention_plan(Attn a, Plan p, int target_items) {
    pdl_prologue();
    __shared__ unsigned count[kBuckets], next[kBuckets];
    __shared__ unsigned slots, joins, total;
    __shared__ long long work;
    const bool keys = blockIdx.x == 1;
    const unsigned cap = keys ? p.most_key_items : p.most_items;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x < kBuckets) count[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        slots = joins = 0;
        work = 0;
        if (!keys && a.status) *a.status = ~0ull;
    }
    __syncthreads();

    // sweep 0: total work, where long ranges may be split; sweep 1: count; 2: place
    int chunk = 1 << 30;
    for (int sweep = p.most_slots > 0 && !keys ? 0 : 1; sweep < 3; ++sweep) {
        long long mine = 0;
        for (int64_t s = warp; s < a.sequences; s += 32) {
            int q_lo, q_hi, k_lo, k_hi;
            const bool ok_q = range_of(a.q_off, s, a.q_tokens, &q_lo, &q_hi);
            const bool ok_k = range_of(a.k_off, s, a.k_tokens, &k_lo, &k_hi);
            if (!ok_q || !ok_k) {
                if (sweep == 1 && !keys && lane == 0 && a.status)
                    atomicMin(a.status, (unsigned long long)s);
                continue;
            }
            const int shift = k_hi - q_hi;   // the last key that token t sees is t + shift
            const int step = keys ? kTile : p.tokens * p.per_item;
            const int lo = keys ? k_lo : q_lo, hi = keys ? k_hi : q_hi;
            for (int i = lane; i < (hi - lo + step - 1) / step; i += 32) {
                Item it;
                it.q0 = q_lo;
                it.q_end = q_hi;
                it.k0 = k_lo;
                it.k_end = k_hi;
                it.t0 = 0;
                it.slot = -1;
                it.pad = 0;
                if (keys) {
                    it.k0 = lo + i * step;
                    if (a.causal) it.q0 = max(q_lo, it.k0 - shift);
                    it.t1 = it.q0 < q_hi ? (q_hi - it.q0 + p.tokens - 1) / p.tokens : 0;
                } else {
                    it.q0 = lo + i * step;
                    const int last = min(q_hi - it.q0, step) + it.q0 - 1;
                    const int end = a.causal ? min(k_hi, last + 1 + shift) : k_hi;
                    it.t1 = end > k_lo ? (end - k_lo + kTile - 1) / kTile : 0;
                }
                if (sweep == 0) {
                    mine += it.t1;
                    continue;
                }
                const int parts = it.t1 > chunk ? (it.t1 + chunk - 1) / chunk : 1;
                const int all = it.t1;
                const int cost = bucket((all + parts - 1) / parts);
                if (sweep == 1) {
                    atomicAdd(&count[cost], (unsigned)parts);
                    continue;
                }
                const unsigned at = atomicAdd(&next[cost], (unsigned)parts);
                int slot = -1;
                bool fits = at < cap && cap - at >= (unsigned)parts;
                if (parts > 1 && fits) {
                    slot = (int)atomicAdd(&slots, (unsigned)parts);
                    fits = slot + parts <= p.most_slots;
                    if (fits)
                        p.joins[atomicAdd(&joins, 1u)] =
                            Join{it.q0, it.q_end, it.k0, it.k_end, slot, parts, {0, 0}};
                }
                Item* to = (keys ? p.key_items : p.items) + at;
                if (!fits) {
                    // offsets that go back make more tiles than the tokens can:
                    // what does not fit the list becomes empty pieces
                    for (int j = 0; j < parts && at + j < cap; ++j)
                        to[j] = Item{0, 0, 0, 0, 0, 0, -1, 0};
                    continue;
                }
                for (int j = 0; j < parts; ++j) {
                    it.t0 = (int)((long long)all * j / parts);
                    it.t1 = (int)((long long)all * (j + 1) / parts);
                    if (slot >= 0) it.slot = slot + j;
                    to[j] = it;
                }
            }
        }
        if (sweep == 0) {
            for (int m = 16; m > 0; m >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, m);
            if (lane == 0) atomicAdd((unsigned long long*)&work, (unsigned long long)mine);
            __syncthreads();
            // at least 4 key tiles a piece: joining costs a pass over the partial sums
            const long long each = (work + target_items - 1) / target_items;
            chunk = (int)(each < 4 ? 4 : each > (1 << 30) ? (1 << 30) : each);
        }
        if (sweep == 1) {
            __syncthreads();
            if (threadIdx.x == 0) {   // longest first
                unsigned at = 0;
                for (int b = kBuckets - 1; b >= 0; --b) {
                    next[b] = at;
                    at += count[b];
                }
                total = at;
            }
            __syncthreads();
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        if (keys) {
            p.head->key_items = (int)min(total, cap);
        } else {
            p.head->items = (int)min(total, cap);
            p.head->joins = (int)joins;
        }
    }
}

}  // namespace

cudaError_t launch_plan(const Attn& a, const Plan& p, bool keys, int target_items,
                        cudaStream_t st) {
    return launch_k(k_attention_plan, dim3(keys ? 2 : 1), dim3(1024), 0, st, a, p, target_items);
}

}  // namespace seq
}  // namespace pss
