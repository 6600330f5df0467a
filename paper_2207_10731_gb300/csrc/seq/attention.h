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

// A piece of work: a tile of query rows (or of key rows) of one sequence and
// the tiles of the other side that it runs over.
//   queries: tokens q0 .. q_end (the sequence's end; the tile's own end follows
//     from its size), key tiles t0 <= t < t1, 128 keys each from k0;
//   keys: keys k0 .. k_end, query tiles 0 <= t < t1, each `tile tokens` from q0.
// slot: where the partial result of a split piece goes, else -1.
struct Item {
    int q0, q_end, k0, k_end;
    int t0, t1, slot, pad;
};
// A query tile whose keys are split: slots slot .. slot + n are to be joined.
struct Join {
    int q0, q_end, k0, k_end;
    int slot, n, pad[2];
};
// Written by the planner at the head of the workspace.
struct PlanHead {
    int items, joins, key_items, pad;
};

constexpr int kTile = 128;               // rows of one tensor-core tile

// Sizes of a call's work list and scratch, from what the host knows.
struct Plan {
    int tokens;                          // tokens of a query tile: 128 / group
    int per_item;                        // query tiles of an item (1 or 2)
    int most_items, most_key_items;      // upper bounds
    int most_slots;                      // > 0: long key ranges may be split
    PlanHead* head;
    Item* items;
    Item* key_items;
    Join* joins;
    float* partial;                      // [slot][kv head][128][dim] sums / denominators
    float* partial_lse;                  // [slot][kv head][128]
    float2* stats;                       // [kv head][q_tokens * group] (lse * log2 e, delta)
};

cudaError_t launch_plan(const Attn& a, const Plan& p, bool keys, int target_items,
                        cudaStream_t st);
cudaError_t launch_tiles_forward(const Attn& a, const Plan& p, cudaStream_t st);
cudaError_t launch_tiles_backward(const Attn& a, const Plan& p, cudaStream_t st);

}  // namespace seq
}  // namespace pss
