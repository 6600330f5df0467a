// The norms after and before a block, backward (residual_norm.cuh).  Bound by memory:
// every tensor's row is read once, the next row's loads under way meanwhile, and
// written once.  The weights' gradients: a thread meets the same columns in every row,
// so their sums are its own, in registers (rows of a warp) or in shared memory (rows of
// a CTA, where two sums a value would take the registers of the next row's loads); a
// CTA leaves one partial row, and a second kernel adds these in a fixed order.
#include <algorithm>
#include <cmath>

#include "residual_norm.cuh"

using namespace pss;
using namespace pss::seq;

namespace {

template <typename T, typename R>
struct Backward {
    const R* grad_total;   // or null
    const T* grad_y;
    const T* x;
    const R* total;
    const T* gate;
    T* dx;
    R* dresidual;
    T* dgate;
    int64_t gts, gys, xs, ts, gs, dxs, drs, dgs;   // strides
    const float *post, *pre, *post_rstd, *pre_rstd;
    float scale;
    int gates;
    bool reads_x;
    float* partial;
    Shape sh;
};

template <typename T, typename R, int VEC, int KIND, int MODE, int FULL>
__global__ void __launch_bounds__(Fit<VEC, KIND>::kMost, Fit<VEC, KIND>::kLeast)
k_residual_norm_backward(const __grid_constant__ Backward<T, R> a) {
    pdl_prologue();
    // constants where FULL
    const int gates = FULL == ANY ? a.gates : FULL;
    const bool post = FULL != ANY || a.post, pre = FULL != ANY || a.pre;
    const bool grad_total = FULL != ANY || a.grad_total, reads_x = FULL != ANY || a.reads_x;
    using F = Fit<VEC, KIND>;
    constexpr int CH = F::kVectors;
    constexpr bool kShared = !F::kWarp;
    constexpr int kDirty = F::kAhead ? ALIGNED : MODE;   // whether a vector may hold a neighbour's values
    extern __shared__ __align__(16) float sums[];
    __shared__ float2 slots[2][32];
    const Shape& sh = a.sh;
    const Place<VEC, MODE> place(sh);
    const float inv_n = 1.f / (float)sh.cols;
    bool in[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) in[c] = place.at(sh, c) < sh.cols;
    // The thread's sums k (0: post, 1: pre) of vector c.  In shared memory the threads'
    // pieces of 4 lie side by side (those of a thread would meet in the same banks).
    float own[kShared ? 1 : 2][kShared ? 1 : CH][VEC] = {};
    constexpr int kPiece = VEC == 8 ? 4 : 1;
    auto slot = [&](int k, int c, int i) -> float* {
        return sums + (((k * CH + c) * (VEC / kPiece) + i / kPiece) * blockDim.x + threadIdx.x) * kPiece +
               i % kPiece;
    };
    auto add = [&](int k, int c, const float (&v)[VEC]) {
        if constexpr (!kShared) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) own[k][c][i] += v[i];
        } else if constexpr (VEC == 8) {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) {
                float4* p = reinterpret_cast<float4*>(slot(k, c, i));
                float4 w = *p;
                w.x += v[i], w.y += v[i + 1], w.z += v[i + 2], w.w += v[i + 3];
                *p = w;
            }
        } else {
            *slot(k, c, 0) += v[0];
        }
    };
    if (kShared)
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) *slot(k, c, i) = 0.f;

    const int64_t step = (int64_t)gridDim.x * sh.groups;
    Held<R, VEC, CH, F::kAhead> held_gt, held_t;
    Held<T, VEC, CH, F::kAhead> held_gy, held_x, held_g;
    uint32_t at = smem_addr(sums) + (kShared ? 8 * CH * VEC * blockDim.x : 0);
    if (grad_total) at = held_gt.place_at(at);
    if (pre) at = held_gy.place_at(held_t.place_at(at));
    if (reads_x) at = held_x.place_at(at);
    if (gates == VALUE_GATE) at = held_g.place_at(at);
    // A ragged row's weights are no vectors: they are laid out once, since a thread's columns are
    // the same in all of its rows.
    constexpr bool kLaid = MODE == RAGGED && F::kAhead;
    uint32_t laid = 0;
    if constexpr (kLaid) {
        laid = at + threadIdx.x * 16;
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float w[8] = {};
                const float* from = k == 0 ? a.post : a.pre;
                if (from) load_weight<VEC, MODE>(from, place.at(sh, c), sh.cols, in[c], w);
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};"
                                 :: "r"(laid + (2 * (k * CH + c) + h) * blockDim.x * 16), "f"(w[4 * h]),
                                    "f"(w[4 * h + 1]), "f"(w[4 * h + 2]), "f"(w[4 * h + 3]) : "memory");
            }
    }
    auto weights = [&](int k, int c, float (&w)[VEC]) {
        if constexpr (kLaid) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];"
                             : "=f"(w[4 * h]), "=f"(w[4 * h + 1]), "=f"(w[4 * h + 2]), "=f"(w[4 * h + 3])
                             : "r"(laid + (2 * (k * CH + c) + h) * blockDim.x * 16) : "memory");
        } else {
            load_weight<VEC, MODE>(k == 0 ? a.post : a.pre, place.at(sh, c), sh.cols, in[c], w);
        }
    };
    float next_gate = 0.f, next_post = 0.f, next_pre = 0.f;
    auto fetch = [&](int stage, int64_t r) {
        const bool live = !F::kWarp || r < sh.rows;
        auto whole = [&](int64_t stride) { return MODE == ALIGNED || inner(sh, r, stride); };
        if (pre) {
            held_t.fetch(stage, a.total + r * a.ts, live, whole(a.ts), in, place, sh);
            held_gy.fetch(stage, a.grad_y + r * a.gys, live, whole(a.gys), in, place, sh);
            next_pre = live ? a.pre_rstd[r] : 0.f;
        }
        if (grad_total)
            held_gt.fetch(stage, a.grad_total + r * a.gts, live, whole(a.gts), in, place, sh);
        if (reads_x) held_x.fetch(stage, a.x + r * a.xs, live, whole(a.xs), in, place, sh);
        if (post) next_post = live ? a.post_rstd[r] : 0.f;
        if (gates == VALUE_GATE)
            held_g.fetch(stage, a.gate + r * a.gs, live, whole(a.gs), in, place, sh);
        if (gates == ROW_GATE) next_gate = live ? load_f32(a.gate[r * a.gs]) : 0.f;
    };
    if (F::kAhead) fetch(0, (int64_t)blockIdx.x * sh.groups + place.group);
    copies_issued();
    int turn = 0, stage = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * sh.groups; r0 < sh.rows; r0 += step, stage ^= 1) {
        const int64_t r = r0 + place.group;
        const bool live = !F::kWarp || r < sh.rows;
        if (!F::kAhead) fetch(0, r);
        const float row_gate = next_gate, post_rstd = next_post, pre_rstd = next_pre;
        if (F::kAhead) {
            if (r0 + step < sh.rows) fetch(stage ^ 1, r + step);
            copies_issued();
            copies_arrived();
            if (MODE == RAGGED && place.t == 0 && place.shift > 0) {
                if (pre) held_t.own(stage, place.shift), held_gy.own(stage, place.shift);
                if (grad_total) held_gt.own(stage, place.shift);
                if (reads_x) held_x.own(stage, place.shift);
                if (gates == VALUE_GATE) held_g.own(stage, place.shift);
            }
        }

        // the second norm: d = dt + r g - that (r / n sum g that)
        float d[CH][VEC];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (grad_total) {
                held_gt.get(stage, c, d[c]);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) d[c][i] = 0.f;
            }
        }
        if (pre) {
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float g[VEC], t[VEC], w[VEC];
                held_gy.get(stage, c, g);
                held_t.get(stage, c, t);
                own_only<VEC, kDirty>(g, place.at(sh, c), sh.cols);
                own_only<VEC, kDirty>(t, place.at(sh, c), sh.cols);
                weights(1, c, w);
                mul(t, t, pre_rstd);
                mul(t, t, g);   // g that, before the weight
                add(1, c, t);
                sum += dot(t, w);
                mul(g, g, w);
                fma(d[c], g, pre_rstd);
            }
            const float s = row_sums<KIND>(sum, sh.lanes, slots, turn) * inv_n;
            const float k = -s * pre_rstd * pre_rstd;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float t[VEC];
                held_t.get(stage, c, t);
                fma(d[c], t, k);
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (live && in[c]) store_part(a.dresidual + r * a.drs, place.at(sh, c), sh.cols, d[c]);
            own_only<VEC, kDirty>(d[c], place.at(sh, c), sh.cols);
        }

        // the gate and the first norm
        float row_slope = 0.f;
        const float row_open = gates == ROW_GATE ? sigmoid(row_gate, &row_slope) : 1.f;
        float2 sum = make_float2(0.f, 0.f);   // of h xhat; of the row's gate gradient
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float hat[VEC], u[VEC], w[VEC];
            if (reads_x) {
                held_x.get(stage, c, hat);
                own_only<VEC, kDirty>(hat, place.at(sh, c), sh.cols);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) hat[i] = 0.f;
            }
            mul(d[c], d[c], a.scale);
            if (post) {
                weights(0, c, w);
                mul(hat, hat, post_rstd);
                mul(u, hat, w);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) u[i] = hat[i];
            }
            if (gates == VALUE_GATE) {
                float g[VEC], slope[VEC];
                held_g.get(stage, c, g);
                own_only<VEC, kDirty>(g, place.at(sh, c), sh.cols);
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] = sigmoid(g[i], &slope[i]);
                mul(slope, slope, u);
                mul(slope, slope, d[c]);
                if (live && in[c])
                    store_part(a.dgate + r * a.dgs, place.at(sh, c), sh.cols, slope);
                mul(d[c], d[c], g);
            } else if (gates == ROW_GATE) {
                sum.y += dot(d[c], u);
                mul(d[c], d[c], row_open);
            }
            if (post) {
                mul(hat, hat, d[c]);   // e xhat
                add(0, c, hat);
                sum.x += dot(hat, w);
                mul(d[c], d[c], w);
            }
        }
        if (post || gates == ROW_GATE) {
            const float2 s = gates == ROW_GATE
                                 ? row_sums<KIND>(sum, sh.lanes, slots, turn)
                                 : make_float2(row_sums<KIND>(sum.x, sh.lanes, slots, turn), 0.f);
            if (gates == ROW_GATE && live && place.t == 0)
                a.dgate[r * a.dgs] = round_to<T>(s.y * row_slope);
            sum.x = s.x * inv_n;
        }
        const float k = -sum.x * post_rstd * post_rstd;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (post) {
                float x[VEC];
                held_x.get(stage, c, x);
                mul(d[c], d[c], post_rstd);
                fma(d[c], x, k);
            }
            if (live && in[c]) store_part(a.dx + r * a.dxs, place.at(sh, c), sh.cols, d[c]);
        }
    }
    if (!post && !pre) return;   // no weights, and no workspace
    // the CTA's partial row: [post, pre][cols] at blockIdx.x
    float* out = a.partial + (int64_t)blockIdx.x * 2 * sh.cols;
    if constexpr (kShared) {
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const int at = place.at(sh, c) + i;
                    if (inside<MODE>(at, sh.cols, in[c])) out[k * sh.cols + at] = *slot(k, c, i);
                }
    } else {
        // add the groups of the CTA: shared memory holds [groups][2][cols], over the rows
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const int at = place.at(sh, c) + i;
                    if (inside<MODE>(at, sh.cols, in[c]))
                        sums[(place.group * 2 + k) * sh.cols + at] = own[k][c][i];
                }
        __syncthreads();
        for (int k = threadIdx.x; k < 2 * sh.cols; k += blockDim.x) {
            float s = 0.f;
            for (int q = 0; q < sh.groups; ++q) s += sums[q * 2 * sh.cols + k];
            out[k] = s;
        }
    }
}

}  // namespace

extern "C" int64_t pss_residual_norm_workspace(int64_t rows, int64_t cols) {
    if (rows < 1 || cols < 1 || cols > kNormMaxCols) return 0;
    const int64_t most = (int64_t)norm_per_sm(cols) * sm_count();
    return (rows < most ? rows : most) * 8 * cols;
}

extern "C" pss_status pss_residual_norm_backward(
    const void* grad_total, int64_t grad_total_stride, const void* grad_y, int64_t grad_y_stride,
    const void* x, pss_dtype type, int64_t x_stride, const void* total, pss_dtype stream_type,
    int64_t total_stride, const void* gate, int32_t gates, int64_t gate_stride,
    const float* post_weight, const float* pre_weight, const float* post_rstd,
    const float* pre_rstd, int64_t rows, int64_t cols, float scale, void* dx, int64_t dx_stride,
    void* dresidual, int64_t dresidual_stride, void* dgate, int64_t dgate_stride,
    float* dpost_weight, float* dpre_weight, void* workspace, int64_t workspace_bytes,
    pss_stream stream) {
    if (!dtype_ok(type) || (stream_type != type && stream_type != PSS_F32) || rows < 0 ||
        cols < 1 || !std::isfinite(scale) || (grad_total && grad_total_stride < cols) ||
        (pre_weight && (grad_y_stride < cols || total_stride < cols)) || dx_stride < cols ||
        dresidual_stride < cols || gates < 0 || gates > 2 ||
        (gates == 1 && (gate_stride < 1 || dgate_stride < 1)) ||
        (gates == 2 && (gate_stride < cols || dgate_stride < cols)))
        return PSS_ERR_INVALID_ARG;
    const bool reads_x = post_weight || gates, sums = post_weight || pre_weight;
    if (reads_x && x_stride < cols) return PSS_ERR_INVALID_ARG;
    if (cols > kNormMaxCols) return PSS_ERR_UNSUPPORTED;
    auto ok = [](const void* p, size_t size) { return device_ptr(p) && aligned_to(p, size); };
    if ((post_weight && !ok(dpost_weight, 4)) || (pre_weight && !ok(dpre_weight, 4)))
        return PSS_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (rows == 0) {
        cudaError_t e = cudaSuccess;
        if (post_weight) e = cudaMemsetAsync(dpost_weight, 0, 4 * cols, st);
        if (pre_weight && e == cudaSuccess) e = cudaMemsetAsync(dpre_weight, 0, 4 * cols, st);
        return status_of(e);
    }
    const size_t a = dtype_size(type), b = dtype_size(stream_type);
    if ((grad_total && !ok(grad_total, b)) || !ok(dx, a) || !ok(dresidual, b) ||
        (reads_x && !ok(x, a)) || (gates && (!ok(gate, a) || !ok(dgate, a))) ||
        (post_weight && (!ok(post_weight, 4) || !ok(post_rstd, 4))) ||
        (pre_weight && (!ok(pre_weight, 4) || !ok(pre_rstd, 4) || !ok(grad_y, a) || !ok(total, b))) ||
        (sums && (!ok(workspace, 16) || workspace_bytes < pss_residual_norm_workspace(rows, cols))))
        return PSS_ERR_INVALID_ARG;
    const bool values = gates == VALUE_GATE;
    const Lie lie = rows_lie<8>(
        cols,
        {dx, dresidual, grad_total ? grad_total : dresidual, pre_weight ? grad_y : dx,
         pre_weight ? total : dresidual, reads_x ? x : dx, values ? gate : dx, values ? dgate : dx},
        {dx_stride, dresidual_stride, grad_total ? grad_total_stride : dresidual_stride,
         pre_weight ? grad_y_stride : dx_stride, pre_weight ? total_stride : dresidual_stride,
         reads_x ? x_stride : dx_stride, values ? gate_stride : dx_stride,
         values ? dgate_stride : dx_stride},
        {type, stream_type, stream_type, type, stream_type, type, type, type});
    auto go = [&](auto t, auto r) {
        using T = decltype(t);
        using R = decltype(r);
        Backward<T, R> f{static_cast<const R*>(grad_total), static_cast<const T*>(grad_y),
                         static_cast<const T*>(x), static_cast<const R*>(total),
                         static_cast<const T*>(gate), static_cast<T*>(dx),
                         static_cast<R*>(dresidual), static_cast<T*>(dgate),
                         grad_total_stride, grad_y_stride, x_stride, total_stride, gate_stride,
                         dx_stride, dresidual_stride, dgate_stride, post_weight, pre_weight,
                         post_rstd, pre_rstd, scale, gates, reads_x, nullptr, Shape{}};
        const bool ragged = lie.how == SHIFTED && cols <= kNormMaxCols - 8;
        int kind;
        const Split s = norm_split((int)cols, ragged ? 7 : 0, true, &kind);
        f.sh = Shape{rows, (int)cols, s.lanes, s.log2_lanes, s.groups, lie.shift0, lie.step};
        f.partial = static_cast<float*>(workspace);
        auto launch = [&](auto vec, auto k, auto mode, auto full) -> cudaError_t {
            auto* kernel = k_residual_norm_backward<T, R, decltype(vec)::value, decltype(k)::value,
                                                    decltype(mode)::value, decltype(full)::value>;
            using F = Fit<decltype(vec)::value, decltype(k)::value>;
            constexpr int kT = held_bytes<T, F::kVectors>(), kR = held_bytes<R, F::kVectors>();
            const size_t ahead =
                F::kAhead ? s.threads * (size_t)((decltype(mode)::value == RAGGED ? 64 * F::kVectors : 0) +
                                                 (grad_total ? kR : 0) + (pre_weight ? kR + kT : 0) +
                                                 (reads_x ? kT : 0) + (values ? kT : 0))
                          : 0;
            // rows of a warp: at the end, the groups' sums instead
            const size_t smem =
                kind <= DOUBLE ? std::max(ahead, (size_t)s.groups * 8 * cols)
                              : ahead + (size_t)8 * F::kVectors * decltype(vec)::value * s.threads;
            cudaError_t e = cudaSuccess;
            static std::atomic<uint64_t> ready{0};
            if (smem + 1024 > 48 * 1024) e = allow_most_smem(kernel, &ready);   // 48 KB with the kernel's own
            if (e != cudaSuccess) return e;
            const int n = ctas_of(
                rows, s, [&] { return resident(kernel, s.threads, smem, norm_per_sm(cols)); },
                decltype(mode)::value);
            e = launch_k(kernel, dim3(n), dim3(s.threads), smem, st, f);
            if (e != cudaSuccess || !sums) return e;
            // a norm that is not there has no sums: its columns are left out
            const int first = post_weight ? 0 : (int)cols, last = pre_weight ? 2 * (int)cols : (int)cols;
            return launch_k(k_row_columns, dim3((unsigned)((last - first + 31) / 32)), dim3(1024), 0,
                            st, static_cast<const float*>(workspace), n, 2 * (int)cols, (int)cols, first, last,
                            dpost_weight, dpre_weight);
        };
        auto with = [&](auto vec, auto k, auto mode) -> cudaError_t {
            if constexpr (decltype(vec)::value == 8 &&
                          decltype(k)::value <= (decltype(mode)::value == ALIGNED ? WIDE : MIDDLE)) {
                if (post_weight && pre_weight && grad_total)
                    return gates == NO_GATE    ? launch(vec, k, mode, Int<NO_GATE>())
                           : gates == ROW_GATE ? launch(vec, k, mode, Int<ROW_GATE>())
                                               : launch(vec, k, mode, Int<VALUE_GATE>());
            }
            return launch(vec, k, mode, Int<ANY>());
        };
        auto wide = [&](auto vec, auto mode) {
            return kind == NARROW   ? with(vec, Int<NARROW>(), mode)
                   : kind == DOUBLE ? with(vec, Int<DOUBLE>(), mode)
                   : kind == MIDDLE ? with(vec, Int<MIDDLE>(), mode)
                   : kind == WIDE   ? with(vec, Int<WIDE>(), mode)
                   : kind == WIDER  ? with(vec, Int<WIDER>(), mode)
                                    : with(vec, Int<WIDEST>(), mode);
        };
        return lie.how == VECTORS ? wide(Int<8>(), Int<ALIGNED>())
               : ragged           ? wide(Int<8>(), Int<RAGGED>())
                                  : wide(Int<1>(), Int<ALIGNED>());
    };
    return status_of(stream_type != type ? type == PSS_BF16 ? go(bf16(), float()) : go(f16(), float())
                     : type == PSS_F32   ? go(float(), float())
                     : type == PSS_BF16  ? go(bf16(), bf16())
                                         : go(f16(), f16()));
}
