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

}  // namespace seq
}  // namespace pss
