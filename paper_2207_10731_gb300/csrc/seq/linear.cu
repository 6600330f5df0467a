// Products with bias, activation and residual, and their gradients (pss_linear_* of pss.h):
// the C entry points, and the pass over the upstream gradient.
//
// Forward:  z = x W + b,  y = act(z) + residual.
// Backward: dz = grad act'(z),  dx = dz W^T,  dW = x^T dz,  db = sum over tokens of dz.
#include <cmath>

#include "activation.cuh"
#include "rows.cuh"

namespace pss {
namespace seq {
namespace {

constexpr int kSlopeCols = 256;   // columns of a CTA: 32 lanes x 8

// dz, rounded as an operand of both products (which are of 16-bit operands; the products' error
// against 64 bits is 1.4 times one rounding's with it, and dz in two parts of 16 bits would
// double them), and the sums of the unrounded ones over the rows of a part: a warp to every
// eighth row, three rows' loads in flight (16384 x 4096 through gelu: four 72 us, of fewer warps
// an SM, three 69, two 81), the warps' sums added in a fixed order.  Bound by memory, but for
// gelu's slope, whose instructions take about as long.
template <typename T, typename TG, bool VECTOR>
__global__ void __launch_bounds__(kThreads)
k_linear_slope(const __grid_constant__ Slope s, int parts) {
    pdl_prologue();
    __shared__ float sums[kWarps][kSlopeCols + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * kSlopeCols + 8 * lane, part = blockIdx.y;
    const int64_t r0 = s.tokens * part / parts, r1 = s.tokens * (part + 1) / parts;
    const TG* grad = static_cast<const TG*>(s.grad);
    const T* z = static_cast<const T*>(s.z);
    float sum[8] = {};
    constexpr int U = 3;
    if (c < s.cols) {
        with_activation(s.activation, [&](auto act) {
            constexpr int kAct = decltype(act)::value;
            for (int64_t r = r0 + warp; r < r1; r += U * kWarps) {
                Raw8<TG> rg[U];
                Raw8<T> rz[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t row = r + u * kWarps;
                    if (row >= r1) continue;
                    if constexpr (VECTOR) {
                        rg[u] = load_raw_part(grad + row * s.grad_stride, c, s.cols, false);
                        if (kAct != ACT_NONE)
                            rz[u] = load_raw_part(z + row * s.z_stride, c, s.cols, false);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const bool in = c + i < s.cols;
                            set_raw(rg[u], i, in ? grad[row * s.grad_stride + c + i] : round_to<TG>(0.f));
                            if (kAct != ACT_NONE)
                                set_raw(rz[u], i, in ? z[row * s.z_stride + c + i] : round_to<T>(0.f));
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t row = r + u * kWarps;
                    if (row >= r1) continue;
                    float g[8], v[8];
                    unpack(rg[u], g);
                    if (kAct != ACT_NONE) {
                        unpack(rz[u], v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) g[i] *= slope_of<kAct>(v[i]);
                    }
                    if (s.dz) store8(static_cast<T*>(s.dz) + row * s.dz_stride + c, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] += g[i];
                }
            }
        });
    }
    if (!s.dbias) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[warp][8 * lane + i] = sum[i];
    __syncthreads();
    const int col = blockIdx.x * kSlopeCols + threadIdx.x;
    if (col >= s.cols) return;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += sums[w][threadIdx.x];
    (parts == 1 ? s.dbias : s.partial)[(int64_t)part * s.cols + col] = v;
}

// Parts of the rows: the GPU filled four CTAs an SM, of 32 rows each at least.
int slope_parts(int64_t tokens, int64_t cols) {
    const int64_t blocks = (cols + kSlopeCols - 1) / kSlopeCols;
    const int64_t most = std::max<int64_t>(1, 4 * (int64_t)sm_count() / blocks);
    return (int)std::max<int64_t>(1, std::min(most, (tokens + 31) / 32));
}

}  // namespace

int64_t slope_values(int64_t tokens, int64_t cols) { return slope_parts(tokens, cols) * cols; }

cudaError_t launch_slope(const Slope& s, int type, cudaStream_t st) {
    const int parts = slope_parts(s.tokens, s.cols);
    const bool vector = aligned8(s.grad, s.grad_stride, s.grad_f32 ? 4 : 2) &&
                        (s.activation == ACT_NONE || aligned8(s.z, s.z_stride, 2));
    auto go = [&](auto* k) {
        const dim3 grid((unsigned)((s.cols + kSlopeCols - 1) / kSlopeCols), (unsigned)parts);
        return launch_k(k, grid, dim3(kThreads), 0, st, s, parts);
    };
    auto typed = [&](auto t) {
        using T = decltype(t);
        return s.grad_f32 ? vector ? go(k_linear_slope<T, float, true>) : go(k_linear_slope<T, float, false>)
               : vector   ? go(k_linear_slope<T, T, true>)
                          : go(k_linear_slope<T, T, false>);
    };
    const cudaError_t e = type == PSS_BF16 ? typed(bf16()) : typed(f16());
    if (e != cudaSuccess || !s.dbias || parts == 1) return e;
    return launch_k(k_row_columns, dim3((unsigned)((s.cols + 31) / 32)), dim3(1024), 0, st,
                    static_cast<const float*>(s.partial), parts, s.cols, s.cols, 0, s.cols, s.dbias,
                    static_cast<float*>(nullptr));
}

namespace {

constexpr int64_t kMost = (int64_t(1) << 31) - 1024;
constexpr int kFewTokens = 64;   // up to here the tokens are the product's columns

bool types_ok(int32_t type, int32_t wide) {
    return (type == PSS_BF16 || type == PSS_F16) && (wide == type || wide == PSS_F32);
}
bool sizes_ok(int64_t tokens, int64_t in, int64_t out) {
    return tokens >= 0 && in >= 1 && out >= 1 && tokens < kMost && in < kMost && out < kMost;
}
bool ok(const void* p, size_t size) { return device_ptr(p) && aligned_to(p, size); }

// A matrix [in][out] with one dense dimension; the stride over a single row or column is
// free.  A dense column is one row of `in` values, not `in` rows of one value (which would
// lie off the 16-byte grid and be copied).
bool weight_matrix(const void* data, int64_t in, int64_t out, int64_t in_stride,
                   int64_t out_stride, Matrix* m, bool* along_out) {
    const bool column = out == 1 && in > 1 && in_stride == 1;
    if (!column && (out == 1 || out_stride == 1) && (in == 1 || in_stride >= out)) {
        *m = Matrix{data, in, out, in_stride};
        *along_out = true;
        return true;
    }
    if ((in == 1 || in_stride == 1) && (out == 1 || out_stride >= in)) {
        *m = Matrix{data, out, in, out_stride};
        *along_out = false;
        return true;
    }
    return false;
}

bool rows16(const void* p, int64_t stride, int size) {
    return !p || (aligned_to(p, 16) && stride * size % 16 == 0);
}

// Tiles and parts fit a launch.
bool product_fits(const Product& p) {
    return (int64_t)p.m_tiles * p.n_tiles * p.splits < (int64_t(1) << 31) - 1024;
}

// A product whose one side are the tokens: few of them are its columns.
void orient(Product* p, const Operand& tokens, const Operand& others) {
    p->f.swapped = tokens.rows() <= kFewTokens;
    p->a = p->f.swapped ? others : tokens;
    p->b = p->f.swapped ? tokens : others;
    plan_product(p);
}

struct ForwardCall {
    Matrix x, w;
    bool w_along_out;
    void *x_copy, *w_copy;
    Product p;
};
// What a forward call does and where its workspace lies; returns the bytes, -1: refused.
int64_t lay_out(const pss_linear_forward_args* a, void* base, ForwardCall* c) {
    if (!a || !types_ok(a->type, a->y_type) || !sizes_ok(a->tokens, a->in, a->out) ||
        a->activation < 0 || a->activation > ACT_SILU || (a->tokens > 1 && a->x_stride < a->in))
        return -1;
    *c = ForwardCall{};
    if (!weight_matrix(a->weight, a->in, a->out, a->weight_in_stride, a->weight_out_stride, &c->w,
                       &c->w_along_out))
        return -1;
    c->x = Matrix{a->x, a->tokens, a->in, a->x_stride};
    if (a->tokens == 0) return 0;
    Take take(base);
    if (!on_grid(c->x)) c->x_copy = take(copy_bytes(c->x));
    if (!on_grid(c->w)) c->w_copy = take(copy_bytes(c->w));
    c->p.f = Finish{a->bias, a->residual, a->z, a->y, a->residual_stride, a->z_stride, a->y_stride,
                    a->activation, a->y_type == PSS_F32, false, false, aligned_to(a->bias, 16)};
    const int size = a->y_type == PSS_F32 ? 4 : 2;
    c->p.f.tiles = rows16(a->y, a->y_stride, size) && rows16(a->z, a->z_stride, 2) &&
                     rows16(a->residual, a->residual_stride, size);
    orient(&c->p, Operand{c->x, false}, Operand{c->w, c->w_along_out});
    c->p.partial = static_cast<float*>(take(partial_values(c->p) * 4));
    return take.bytes();
}

struct BackwardCall {
    Matrix x, w, dz;
    bool w_along_out, dw_along_out, needs_dz;
    void *x_copy, *w_copy, *dz_made;
    float* sums;
    Product dx, dw;
};
int64_t lay_out(const pss_linear_backward_args* a, void* base, BackwardCall* c) {
    if (!a || !types_ok(a->type, a->grad_type) || !types_ok(a->type, a->dweight_type) ||
        !sizes_ok(a->tokens, a->in, a->out) || a->activation < 0 || a->activation > ACT_SILU ||
        (a->tokens > 1 && (a->grad_stride < a->out || (a->dweight && a->x_stride < a->in) ||
                           (a->activation && a->z_stride < a->out) ||
                           (a->dx && a->dx_stride < a->in))))
        return -1;
    *c = BackwardCall{};
    Matrix dw;
    if (a->dx && !weight_matrix(a->weight, a->in, a->out, a->weight_in_stride,
                                a->weight_out_stride, &c->w, &c->w_along_out))
        return -1;
    if (a->dweight && !weight_matrix(a->dweight, a->in, a->out, a->dweight_in_stride,
                                     a->dweight_out_stride, &dw, &c->dw_along_out))
        return -1;
    if (a->tokens == 0) return 0;
    Take take(base);
    c->x = Matrix{a->x, a->tokens, a->in, a->x_stride};
    c->dz = Matrix{a->grad, a->tokens, a->out, a->grad_stride};
    c->needs_dz = (a->dx || a->dweight) &&
                  (a->activation || a->grad_type == PSS_F32 || !on_grid(c->dz));
    if (c->needs_dz) {
        c->dz_made = take(copy_bytes(c->dz));
        c->dz = Matrix{c->dz_made, a->tokens, a->out, (a->out + 7) / 8 * 8};
    }
    if (a->dbias) c->sums = static_cast<float*>(take(slope_values(a->tokens, a->out) * 4));
    int64_t shared = 0;   // the two products' parts, one after the other in the same place
    if (a->dx) {
        if (!on_grid(c->w)) c->w_copy = take(copy_bytes(c->w));
        c->dx.f = Finish{nullptr, nullptr, nullptr, a->dx, 0, 0, a->dx_stride, ACT_NONE, false, false,
                         rows16(a->dx, a->dx_stride, 2)};
        orient(&c->dx, Operand{c->dz, false}, Operand{c->w, !c->w_along_out});
        shared = partial_values(c->dx);
    }
    if (a->dweight) {
        if (!on_grid(c->x)) c->x_copy = take(copy_bytes(c->x));
        const bool wide = a->dweight_type == PSS_F32;
        c->dw.f = Finish{nullptr, nullptr, nullptr, a->dweight, 0, 0, dw.stride, ACT_NONE, wide, false,
                         rows16(a->dweight, dw.stride, wide ? 4 : 2)};
        const Operand x{c->x, true}, dz{c->dz, true};
        c->dw.a = c->dw_along_out ? x : dz;
        c->dw.b = c->dw_along_out ? dz : x;
        plan_product(&c->dw);
        shared = std::max(shared, partial_values(c->dw));
    }
    c->dx.partial = c->dw.partial = static_cast<float*>(take(shared * 4));
    return take.bytes();
}

pss_status clear_status(int64_t* status, cudaStream_t st) {
    return status ? status_of(cudaMemsetAsync(status, 0xff, 8, st)) : PSS_OK;
}

cudaError_t zero_matrix(void* p, int64_t outer, int64_t inner, int64_t stride, size_t size,
                        cudaStream_t st) {
    return outer == 1 ? cudaMemsetAsync(p, 0, inner * size, st)
                      : cudaMemset2DAsync(p, stride * size, 0, inner * size, outer, st);
}

}  // namespace
}  // namespace seq
}  // namespace pss

using namespace pss;
using namespace pss::seq;

extern "C" int64_t pss_linear_forward_workspace(const pss_linear_forward_args* a) {
    ForwardCall c;
    return std::max<int64_t>(0, lay_out(a, nullptr, &c));
}

extern "C" pss_status pss_linear_forward(const pss_linear_forward_args* a, void* workspace,
                                         int64_t workspace_bytes, int64_t* status,
                                         pss_stream stream) {
    ForwardCall c;
    const int64_t need = lay_out(a, workspace, &c);
    if (need < 0 || (status && !ok(status, 8))) return PSS_ERR_INVALID_ARG;
    const int size = a->y_type == PSS_F32 ? 4 : 2;
    if (a->tokens > 0) {
        if (!ok(a->x, 2) || !ok(a->weight, 2) || !ok(a->y, size) || (a->bias && !ok(a->bias, 4)) ||
            (a->residual && !ok(a->residual, size)) || (a->z && !ok(a->z, 2)) ||
            (a->tokens > 1 && (a->y_stride < a->out || (a->residual && a->residual_stride < a->out) ||
                               (a->z && a->z_stride < a->out))) ||
            (need > 0 && (!ok(workspace, 16) || workspace_bytes < need)))
            return PSS_ERR_INVALID_ARG;
        if (!product_fits(c.p)) return PSS_ERR_UNSUPPORTED;
    }
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const pss_status rc = clear_status(status, st);
    if (rc != PSS_OK || a->tokens == 0) return rc;
    cudaError_t e = cudaSuccess;
    Operand *x = c.p.f.swapped ? &c.p.b : &c.p.a, *w = c.p.f.swapped ? &c.p.a : &c.p.b;
    if (c.x_copy || c.w_copy) e = copy_matrices(&x->matrix, c.x_copy, &w->matrix, c.w_copy, st);
    if (e == cudaSuccess)
        e = launch_product(c.p, a->type, reinterpret_cast<unsigned long long*>(status), st);
    return status_of(e);
}

extern "C" int64_t pss_linear_backward_workspace(const pss_linear_backward_args* a) {
    BackwardCall c;
    return std::max<int64_t>(0, lay_out(a, nullptr, &c));
}

extern "C" pss_status pss_linear_backward(const pss_linear_backward_args* a, void* workspace,
                                          int64_t workspace_bytes, int64_t* status,
                                          pss_stream stream) {
    BackwardCall c;
    const int64_t need = lay_out(a, workspace, &c);
    if (need < 0 || (status && !ok(status, 8))) return PSS_ERR_INVALID_ARG;
    const int gsize = a->grad_type == PSS_F32 ? 4 : 2, wsize = a->dweight_type == PSS_F32 ? 4 : 2;
    if ((a->dbias && !ok(a->dbias, 4)) || (a->dweight && !ok(a->dweight, wsize)))
        return PSS_ERR_INVALID_ARG;
    if (a->tokens > 0) {
        if (!ok(a->grad, gsize) || (a->activation && !ok(a->z, 2)) || (a->dx && !ok(a->dx, 2)) ||
            (a->dx && !ok(a->weight, 2)) || (a->dweight && !ok(a->x, 2)) ||
            (need > 0 && (!ok(workspace, 16) || workspace_bytes < need)))
            return PSS_ERR_INVALID_ARG;
        if ((a->dx && !product_fits(c.dx)) || (a->dweight && !product_fits(c.dw)))
            return PSS_ERR_UNSUPPORTED;
    }
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const pss_status rc = clear_status(status, st);
    if (rc != PSS_OK) return rc;
    cudaError_t e = cudaSuccess;
    if (a->tokens == 0) {
        if (a->dbias) e = cudaMemsetAsync(a->dbias, 0, 4 * a->out, st);
        if (a->dweight && e == cudaSuccess)
            e = c.dw_along_out
                    ? zero_matrix(a->dweight, a->in, a->out, a->dweight_in_stride, wsize, st)
                    : zero_matrix(a->dweight, a->out, a->in, a->dweight_out_stride, wsize, st);
        return status_of(e);
    }
    if (c.needs_dz || a->dbias) {
        const Slope s{a->grad, a->z, c.dz_made, a->dbias, c.sums, a->grad_stride, a->z_stride,
                      (a->out + 7) / 8 * 8, a->tokens, (int)a->out, a->activation,
                      a->grad_type == PSS_F32};
        e = launch_slope(s, a->type, st);
    }
    unsigned long long* word = reinterpret_cast<unsigned long long*>(status);
    Matrix* w = &(c.dx.f.swapped ? c.dx.a : c.dx.b).matrix;
    Matrix* x = &(c.dw_along_out ? c.dw.a : c.dw.b).matrix;
    if (e == cudaSuccess && (c.w_copy || c.x_copy)) e = copy_matrices(w, c.w_copy, x, c.x_copy, st);
    if (e == cudaSuccess && a->dx) e = launch_product(c.dx, a->type, word, st);
    if (e == cudaSuccess && a->dweight) e = launch_product(c.dw, a->type, word, st);
    return status_of(e);
}
