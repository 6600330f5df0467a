// Attention over packed sequences (pss_attention_* of pss.h): the C entry
// points and the row-by-row kernels.
#include <cmath>

#include "attention_tma.h"
#include <cudaTypedefs.h>

using namespace pss;
using namespace pss::seq;

namespace {

// Work items times heads are one launch's CTAs.
bool grids_ok(const pss_attention_shape& s) {
    const int64_t tokens = kTile / (s.heads / s.kv_heads);
    const int64_t most = int64_t(1) << 30;
    return s.q_tokens / tokens + 1 < most / s.kv_heads &&
           s.k_tokens / kTile + 1 < most / s.kv_heads &&
           s.q_tokens < (int64_t(1) << 34) / s.heads;
}

bool shape_ok(const pss_attention_shape* s) {
    return s && s->sequences >= 0 && s->q_tokens >= 0 && s->k_tokens >= 0 &&
           s->q_tokens < (int64_t(1) << 31) - 1024 && s->k_tokens < (int64_t(1) << 31) - 1024 &&
           s->sequences < (int64_t(1) << 31) - 1024 && s->kv_heads >= 1 && s->heads >= 1 &&
           s->heads % s->kv_heads == 0 && s->heads / s->kv_heads <= 128 && s->dim >= 8 &&
           s->dim <= 128 && s->dim % 8 == 0 && (s->causal == 0 || s->causal == 1) &&
           s->scale > 0.f && std::isfinite(s->scale) && grids_ok(*s);
}

// Checks one tensor; an empty one needs no memory.
bool rows_ok(const pss_rows* r, int64_t tokens, int64_t heads, int64_t dim, Rows* out) {
    if (!r) return false;
    *out = Rows{static_cast<bf16*>(r->data), r->token_stride, r->head_stride};
    if (tokens == 0) return true;
    if (!device_ptr(r->data) || !aligned_to(r->data, 16)) return false;
    const int64_t ts = r->token_stride, hs = r->head_stride;
    const int64_t most = int64_t(1) << 39;   // strides of a tensor map: below 2^40 bytes
    if (ts < 0 || hs < 0 || ts % 8 || hs % 8 || ts >= most || hs >= most) return false;
    // rows must not overlap: the smaller stride holds a row, the larger all the others
    if (heads == 1) return tokens == 1 || ts >= dim;
    if (tokens == 1) return hs >= dim;
    return hs >= dim && ts >= dim && (ts >= (heads - 1) * hs + dim || hs >= (tokens - 1) * ts + dim);
}

pss_status fill(const pss_attention_shape* s, const pss_rows* q, const pss_rows* k,
                const pss_rows* v, const pss_rows* out, const float* lse, void* workspace,
                int64_t workspace_bytes, int64_t* status, int backward, Attn* a) {
    if (!shape_ok(s)) return PSS_ERR_INVALID_ARG;
    *a = Attn{};
    a->sequences = s->sequences;
    a->q_off = s->q_offsets;
    a->k_off = s->k_offsets;
    a->q_tokens = (int)s->q_tokens;
    a->k_tokens = (int)s->k_tokens;
    a->heads = s->heads;
    a->kv_heads = s->kv_heads;
    a->group = s->heads / s->kv_heads;
    a->dim = s->dim;
    a->causal = s->causal;
    a->scale = s->scale;
    a->lse = const_cast<float*>(lse);
    a->status = reinterpret_cast<unsigned long long*>(status);
    if (status && !(device_ptr(status) && aligned_to(status, 8))) return PSS_ERR_INVALID_ARG;
    if (s->sequences > 0 && (!device_ptr(s->q_offsets) || !device_ptr(s->k_offsets) ||
                             !aligned_to(s->q_offsets, 8) || !aligned_to(s->k_offsets, 8)))
        return PSS_ERR_INVALID_ARG;
    if (!rows_ok(q, s->q_tokens, s->heads, s->dim, &a->q) ||
        !rows_ok(k, s->k_tokens, s->kv_heads, s->dim, &a->k) ||
        !rows_ok(v, s->k_tokens, s->kv_heads, s->dim, &a->v) ||
        !rows_ok(out, s->q_tokens, s->heads, s->dim, &a->out))
        return PSS_ERR_INVALID_ARG;
    if (s->q_tokens > 0 && !(device_ptr(lse) && aligned_to(lse, 4))) return PSS_ERR_INVALID_ARG;
    const int64_t need = pss_attention_workspace(s, backward);
    if (need > 0 && (!device_ptr(workspace) || !aligned_to(workspace, 16) ||
                     workspace_bytes < need))
        return PSS_ERR_INVALID_ARG;
    return PSS_OK;
}

// The sizes of a call's tiles and scratch, and where each part of the workspace
// lies: a pure function of the shape, so that the size asked for beforehand is
// the size used.  Returns the bytes.
int64_t lay_out(const pss_attention_shape& s, bool backward, void* base, Plan* p, int* target) {
    *p = Plan{};
    const int group = s.heads / s.kv_heads;
    p->tokens = kTile / group;
    p->tiles = (int)((s.q_tokens + p->tokens - 1) / p->tokens);
    p->key_tiles = (int)((s.k_tokens + kTile - 1) / kTile);
    const int64_t ctas = (int64_t)p->tiles * s.kv_heads;
    const int sms = sm_count() > 0 ? sm_count() : 1;
    // With fewer tiles than CTAs fit the GPU, long key ranges are split into as
    // many pieces as do (two CTAs an SM; twice as many: 94 instead of 88 us for 48
    // users' steps over 0.5-16k keys), of four key tiles at least.
    const bool split = !backward && ctas < 2 * sms && s.k_tokens > kLeastPiece * kTile;
    *target = split ? (2 * sms + s.kv_heads - 1) / s.kv_heads : 1;
    const int64_t slots = split ? p->tiles + (int64_t)*target : 0;
    // Two query tiles to a CTA share its K and V tiles and hide each other's
    // softmax; one to a CTA puts two CTAs on an SM, which hides the start and the
    // end of short ones.
    p->per_item = !backward && ctas >= 8 * sms && s.q_tokens >= 512 * s.sequences ? 2 : 1;
    p->keys = backward ? backward_columns(s) : kTile;
    p->key_tokens = backward_columns(s) / group;
    Take take(base);
    p->most_items = (int)((p->tiles + p->per_item - 1) / p->per_item + slots);
    p->most_slots = (int)slots;
    p->head = static_cast<PlanHead*>(take(sizeof(PlanHead)));
    p->items = static_cast<Item*>(take(p->most_items * sizeof(Item)));
    p->q_range = static_cast<Range*>(take(s.q_tokens * sizeof(Range)));
    if (backward) {
        p->key_items = static_cast<Item*>(take(p->key_tiles * sizeof(Item)));
        p->k_range = static_cast<Range*>(take(s.k_tokens * sizeof(Range)));
        p->stats = static_cast<float2*>(take(s.q_tokens * s.heads * 8));
    }
    p->joins = static_cast<Join*>(take(slots / 2 * sizeof(Join)));
    p->partial = static_cast<float*>(take(slots * s.kv_heads * kTile * s.dim * 4));
    p->partial_lse = static_cast<float*>(take(slots * s.kv_heads * kTile * 4));
    return take.bytes();
}

// Nothing to do but to say so.
pss_status no_sequences(const Attn& a, cudaStream_t st) {
    return a.status ? status_of(cudaMemsetAsync(a.status, 0xff, 8, st)) : PSS_OK;
}

}  // namespace

extern "C" int64_t pss_attention_workspace(const pss_attention_shape* s, int32_t backward) {
    if (!shape_ok(s)) return 0;
    Plan p;
    int target;
    return lay_out(*s, backward != 0, nullptr, &p, &target);
}

extern "C" pss_status pss_attention_forward(const pss_attention_shape* shape, const pss_rows* q,
                                            const pss_rows* k, const pss_rows* v,
                                            const pss_rows* out, float* lse, void* workspace,
                                            int64_t workspace_bytes, int64_t* status,
                                            pss_stream stream) {
    Attn a;
    const pss_status rc =
        fill(shape, q, k, v, out, lse, workspace, workspace_bytes, status, 0, &a);
    if (rc != PSS_OK) return rc;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    Plan p;
    int target;
    lay_out(*shape, false, workspace, &p, &target);
    if (a.sequences == 0) return no_sequences(a, st);
    // A few tiles of a few sequences need no list: their order does not matter, and
    // a CTA's two short searches cost less than a launch (1 user x 200 keys: 27 us a
    // call with the list, 22 without).  The status word is the list's business.
    p.direct = !status && p.most_slots == 0 && p.per_item == 1 && a.sequences <= 64 &&
               p.tiles * a.kv_heads <= sm_count();
    cudaError_t e = p.direct ? cudaSuccess : launch_plan(a, p, false, target, st);
    if (e == cudaSuccess && a.q_tokens > 0) e = launch_tiles_forward(a, p, st);
    return status_of(e);
}

extern "C" pss_status pss_attention_backward(const pss_attention_shape* shape, const pss_rows* grad,
                                             const pss_rows* q, const pss_rows* k,
                                             const pss_rows* v, const pss_rows* out,
                                             const float* lse, const pss_rows* dq,
                                             const pss_rows* dk, const pss_rows* dv,
                                             void* workspace, int64_t workspace_bytes,
                                             int64_t* status, pss_stream stream) {
    Attn a;
    const pss_status rc =
        fill(shape, q, k, v, out, lse, workspace, workspace_bytes, status, 1, &a);
    if (rc != PSS_OK) return rc;
    if (!rows_ok(grad, shape->q_tokens, a.heads, a.dim, &a.grad) ||
        !rows_ok(dq, shape->q_tokens, a.heads, a.dim, &a.dq) ||
        !rows_ok(dk, shape->k_tokens, a.kv_heads, a.dim, &a.dk) ||
        !rows_ok(dv, shape->k_tokens, a.kv_heads, a.dim, &a.dv))
        return PSS_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    Plan p;
    int target;
    lay_out(*shape, true, workspace, &p, &target);
    if (a.sequences == 0) return no_sequences(a, st);
    cudaError_t e = launch_plan(a, p, true, target, st);
    if (e == cudaSuccess) e = launch_tiles_backward(a, p, st);
    return status_of(e);
}

namespace pss {
namespace seq {

void* driver_call(const char* name, std::atomic<void*>* found) {
    void* fn = found->load(std::memory_order_acquire);
    if (fn) return fn;
    cudaDriverEntryPointQueryResult how;
    if (cudaGetDriverEntryPointByVersion(name, &fn, 12000, cudaEnableDefault, &how) !=
            cudaSuccess ||
        how != cudaDriverEntryPointSuccess) {
        cudaGetLastError();
        return nullptr;
    }
    found->store(fn, std::memory_order_release);
    return fn;
}

cudaError_t bind_context() {
    static thread_local int bound = -1;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || dev == bound) return e;
    e = cudaSetDevice(dev);
    if (e == cudaSuccess) bound = dev;
    return e;
}

bool device_ptr(const void* p) {
    static std::atomic<void*> found{nullptr};
    void* fn = driver_call("cuPointerGetAttribute", &found);
    CUmemorytype type;
    return p && fn &&
           reinterpret_cast<PFN_cuPointerGetAttribute_v4000>(fn)(
               &type, CU_POINTER_ATTRIBUTE_MEMORY_TYPE, (CUdeviceptr)p) == CUDA_SUCCESS &&
           type == CU_MEMORYTYPE_DEVICE;
}

cudaError_t tile_map(CUtensorMap* map, const Rows& r, int tokens, int heads, int dim,
                     int heads_box, int tokens_box, const void* spare) {
    static std::atomic<void*> found{nullptr};
    void* fn = driver_call("cuTensorMapEncodeTiled", &found);
    if (!fn) return cudaErrorNotSupported;
    const cudaError_t bound = bind_context();
    if (bound != cudaSuccess) return bound;
    const bool empty = tokens == 0;   // nothing is loaded; the map only has to be valid
    // a stride over a size of one is free, but the encoder checks it
    const int64_t row = heads == 1 ? dim : r.head, token = tokens <= 1 ? dim : r.token;
    const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)(empty ? 1 : tokens)};
    const cuuint64_t strides[2] = {(cuuint64_t)row * 2, (cuuint64_t)token * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)heads_box, (cuuint32_t)tokens_box};
    const cuuint32_t one[3] = {1, 1, 1};
    const CUresult rc = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn)(
        map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, empty ? const_cast<void*>(spare) : r.data, dims,
        strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace seq
}  // namespace pss
