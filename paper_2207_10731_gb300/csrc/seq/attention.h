// Shared by the translation units of the packed-sequence attention.
#pragma once

#include "seq_common.cuh"

namespace pss {
namespace seq {

// A bf16 tensor [tokens][heads][dim] as the kernels see it.
struct Rows {
    bf16* data;
    int64_t token, head;   // strides in elements
    __device__ __forceinline__ bf16* at(int64_t t, int h) const {
        return data + t * token + h * head;
    }
};

// One attention call.
struct Attn {
    int64_t sequences;
    const int64_t* q_off;
    const int64_t* k_off;
    int q_tokens, k_tokens;
    int heads, kv_heads, group, dim, causal;
    float scale;
    Rows q, k, v, out, grad, dq, dk, dv;
    float* lse;                    // [q_tokens][heads]
    unsigned long long* status;    // see pss.h, or null
};

// The keys lo .. hi that a query token sees, or the query tokens that see a key;
// hi < 0: the token is in no sequence (and -1 - hi stands for hi).  lo and hi
// never fall along the tokens.
struct Range {
    int lo, hi;
    __device__ __forceinline__ bool live() const { return hi >= 0; }
    __device__ __forceinline__ int end() const { return hi < 0 ? -1 - hi : hi; }
};

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

// A piece of work: a tile of consecutive query tokens (or keys), whichever
// sequences they belong to, and the tiles of the other side that hold all that
// they see.  Short neighbouring sequences so share a tile; what a row does not
// see is masked.
//   queries: tokens from q0, key tiles t0 <= t < t1, `keys` each from k0;
//   keys: keys from k0, query tiles t0 = 0 <= t < t1, `key_tokens` each from q0.
// slot: where the partial result of a split piece goes, else -1.
struct Item {
    int q0, k0, t0, t1, slot, pad[3];
};
// A query tile whose keys are split: slots slot .. slot + n are to be joined.
struct Join {
    int q0, slot, n, pad;
};
// Written by the planner at the head of the workspace.
struct PlanHead {
    int items, joins, pad[2];
};

constexpr int kTile = 128;               // rows of one tensor-core tile
constexpr int kLeastPiece = 4;           // key tiles of a piece of a split range, at least

// Sizes of a call's work list and scratch, from what the host knows.
struct Plan {
    int tokens;                          // tokens of a query tile: 128 / group
    int per_item;                        // query tiles of an item (1 or 2)
    int keys;                            // keys of a key tile that a query item runs over
    int key_tokens;                      // tokens of a query tile that a key item runs over
    int tiles, key_tiles;                // query and key tiles of the call
    int most_items;                      // query items: tiles / per_item, and splits
    int most_slots;                      // > 0: long key ranges may be split
    bool direct;                         // no list: each CTA works its item out itself
    PlanHead* head;
    Item* items;
    Item* key_items;
    Join* joins;
    Range* q_range;                      // [q_tokens]
    Range* k_range;                      // [k_tokens], backward only
    float* partial;                      // [slot][kv head][128][dim] sums / denominators
    float* partial_lse;                  // [slot][kv head][128]
    float2* stats;                       // [kv head][q_tokens * group] (lse * log2 e, delta)
};

// Rows of the tiles that a backward item runs over: 64 where a head fits one
// 128-byte row and a group 64 rows (see attention_backward.cu), else 128.
inline int backward_columns(const pss_attention_shape& s) {
    return s.dim <= 64 && s.heads / s.kv_heads <= 64 ? 64 : kTile;
}

cudaError_t launch_plan(const Attn& a, const Plan& p, bool keys, int target_items,
                        cudaStream_t st);
cudaError_t launch_tiles_forward(const Attn& a, const Plan& p, cudaStream_t st);
cudaError_t launch_tiles_backward(const Attn& a, const Plan& p, cudaStream_t st);

}  // namespace seq
}  // namespace pss
