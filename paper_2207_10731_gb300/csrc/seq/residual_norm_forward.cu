// The norms after and before a block, forward.  Bound by memory: a row of the block's
// output, its gate and the stream is read once, kept in registers through both
// reductions and written once; the next row's loads are under way meanwhile.
#include <cmath>

#include "residual_norm.cuh"

using namespace pss;
using namespace pss::seq;

namespace {

template <typename T, typename R>
struct Forward {
    const T* x;
    const R* residual;
    const T* gate;
    R* total;
    T* y;
    int64_t xs, rs, gs, ts, ys;   // strides
    const float *post, *pre;
    float *post_rstd, *pre_rstd;
    float scale, eps;
    int gates;
    Shape sh;
};

template <typename T, typename R, int VEC, int KIND, int MODE, int FULL>
__global__ void __launch_bounds__(Fit<VEC, KIND>::kMost)
k_residual_norm_forward(const __grid_constant__ Forward<T, R> a) {
    pdl_prologue();
    // constants where FULL
    const int gates = FULL == ANY ? a.gates : FULL;
    const bool post = FULL != ANY || a.post, pre = FULL != ANY || a.pre;
    using F = Fit<VEC, KIND>;
    constexpr int CH = F::kVectors;
    __shared__ float2 slots[2][32];
    const Shape& sh = a.sh;
    const Place<VEC, MODE> place(sh);
    const float inv_n = 1.f / (float)sh.cols;
    bool in[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) in[c] = place.at(sh, c) < sh.cols;
    const int64_t step = (int64_t)gridDim.x * sh.groups;
    // A ragged row's weights are no vectors: they are laid out once in shared memory, 16-byte
    // pieces of a thread, since its columns are the same in all of its rows.
    constexpr bool kLaid = MODE == RAGGED && F::kAhead;
    extern __shared__ __align__(16) float4 laid[];
    if constexpr (kLaid) {
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float w[8] = {};
                const float* from = k == 0 ? a.post : a.pre;
                if (from) load_weight<VEC, MODE>(from, place.at(sh, c), sh.cols, in[c], w);
                float4* to = laid + 2 * (k * CH + c) * blockDim.x + threadIdx.x;
                to[0] = make_float4(w[0], w[1], w[2], w[3]);
                to[blockDim.x] = make_float4(w[4], w[5], w[6], w[7]);
            }
    }
    auto weights = [&](int k, int c, float (&w)[VEC]) {
        if constexpr (kLaid) {
            const float4* from = laid + 2 * (k * CH + c) * blockDim.x + threadIdx.x;
            const float4 x = from[0], y = from[blockDim.x];
            w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
            w[4] = y.x, w[5] = y.y, w[6] = y.z, w[7] = y.w;
        } else {
            load_weight<VEC, MODE>(k == 0 ? a.post : a.pre, place.at(sh, c), sh.cols, in[c], w);
        }
    };
    // The next row's loads are under way in registers, which reach here (in shared memory, as
    // backward: 350 instead of 300 us for 131072 x 1024 with an fp32 stream).
    Part<T, VEC, CH> next_x, next_g;
    Part<R, VEC, CH> next_r;
    float next_gate = 0.f;
    auto fetch = [&](int64_t r) {
        const bool live = !F::kWarp || r < sh.rows;
        auto whole = [&](int64_t stride) { return MODE == ALIGNED || inner(sh, r, stride); };
        next_x.load(a.x + r * a.xs, live, whole(a.xs), in, place, sh);
        next_r.load(a.residual + r * a.rs, live, whole(a.rs), in, place, sh);
        if (gates == VALUE_GATE)
            next_g.load(a.gate + r * a.gs, live, whole(a.gs), in, place, sh);
        if (gates == ROW_GATE) next_gate = live ? load_f32(a.gate[r * a.gs]) : 0.f;
    };
    if (F::kAhead) fetch((int64_t)blockIdx.x * sh.groups + place.group);
    int turn = 0;
    // the same trip count for every thread of the CTA (shuffles and barriers inside);
    // rows past the end are computed from zeros and dropped
    for (int64_t r0 = (int64_t)blockIdx.x * sh.groups; r0 < sh.rows; r0 += step) {
        const int64_t r = r0 + place.group;
        const bool live = !F::kWarp || r < sh.rows;
        if (!F::kAhead) fetch(r);
        const Part<T, VEC, CH> part_x = next_x, part_g = next_g;
        const Part<R, VEC, CH> part_r = next_r;
        const float row_gate = next_gate;
        if (F::kAhead && r0 + step < sh.rows) fetch(r + step);
        float v[CH][VEC], sum = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            part_x.get(c, v[c]);
            own_only<VEC, MODE>(v[c], place.at(sh, c), sh.cols);
            sum += dot(v[c], v[c]);
        }
        if (post) {
            const float s = row_sums<KIND>(sum, sh.lanes, slots, turn) * inv_n;
            const float rstd = 1.f / sqrtf(s + a.eps);
            if (live && place.t == 0) a.post_rstd[r] = rstd;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float w[VEC];
                weights(0, c, w);
                mul(v[c], v[c], rstd);
                mul(v[c], v[c], w);
            }
        }
        sum = 0.f;
        const float row_scale = gates == ROW_GATE ? a.scale * sigmoid(row_gate) : a.scale;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float t[VEC];
            part_r.get(c, t);
            own_only<VEC, MODE>(t, place.at(sh, c), sh.cols);
            if (gates == VALUE_GATE) {
                float g[VEC];
                part_g.get(c, g);
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] = sigmoid(g[i]);
                mul(v[c], v[c], g);
            }
            fma(t, v[c], row_scale);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[c][i] = t[i];
            // what a gate makes of a neighbour's NaN times zero
            if (gates == VALUE_GATE) own_only<VEC, MODE>(v[c], place.at(sh, c), sh.cols);
            sum += dot(v[c], v[c]);
            if (live && in[c]) store_part(a.total + r * a.ts, place.at(sh, c), sh.cols, v[c]);
        }
        if (pre) {
            // of the unrounded sum: total's rounding is not in y
            const float s = row_sums<KIND>(sum, sh.lanes, slots, turn) * inv_n;
            const float rstd = 1.f / sqrtf(s + a.eps);
            if (live && place.t == 0) a.pre_rstd[r] = rstd;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float w[VEC];
                weights(1, c, w);
                mul(v[c], v[c], rstd);
                mul(v[c], v[c], w);
                if (live && in[c]) store_part(a.y + r * a.ys, place.at(sh, c), sh.cols, v[c]);
            }
        }
    }
}

}  // namespace

extern "C" pss_status pss_residual_norm_forward(
    const void* x, pss_dtype type, int64_t x_stride, const void* residual, pss_dtype stream_type,
    int64_t residual_stride, const void* gate, int32_t gates, int64_t gate_stride,
    const float* post_weight, const float* pre_weight, int64_t rows, int64_t cols, float scale,
    float eps, void* total, int64_t total_stride, void* y, int64_t y_stride, float* post_rstd,
    float* pre_rstd, pss_stream stream) {
    if (!dtype_ok(type) || (stream_type != type && stream_type != PSS_F32) || rows < 0 ||
        cols < 1 || !(eps >= 0.f) || std::isinf(eps) || !std::isfinite(scale) || x_stride < cols ||
        residual_stride < cols || total_stride < cols || (pre_weight && y_stride < cols) ||
        gates < 0 || gates > 2 || (gates == 1 && gate_stride < 1) ||
        (gates == 2 && gate_stride < cols))
        return PSS_ERR_INVALID_ARG;
    if (cols > kNormMaxCols) return PSS_ERR_UNSUPPORTED;
    if (rows == 0) return PSS_OK;
    const size_t a = dtype_size(type), b = dtype_size(stream_type);
    auto ok = [](const void* p, size_t size) { return device_ptr(p) && aligned_to(p, size); };
    if (!ok(x, a) || !ok(residual, b) || !ok(total, b) || (gates && !ok(gate, a)) ||
        (post_weight && (!ok(post_weight, 4) || !ok(post_rstd, 4))) ||
        (pre_weight && (!ok(pre_weight, 4) || !ok(pre_rstd, 4) || !ok(y, a))))
        return PSS_ERR_INVALID_ARG;
    const bool values = gates == VALUE_GATE;
    const Lie lie = rows_lie<5>(
        cols, {x, residual, total, pre_weight ? y : x, values ? gate : x},
        {x_stride, residual_stride, total_stride, pre_weight ? y_stride : x_stride,
         values ? gate_stride : x_stride},
        {type, stream_type, stream_type, type, type});
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    auto go = [&](auto t, auto r) {
        using T = decltype(t);
        using R = decltype(r);
        Forward<T, R> f{static_cast<const T*>(x), static_cast<const R*>(residual),
                        static_cast<const T*>(gate), static_cast<R*>(total), static_cast<T*>(y),
                        x_stride, residual_stride, gate_stride, total_stride, y_stride,
                        post_weight, pre_weight, post_rstd, pre_rstd, scale, eps, gates, Shape{}};
        const bool ragged = lie.how == SHIFTED && cols <= kNormMaxCols - 8;
        int kind;
        const Split s = norm_split((int)cols, ragged ? 7 : 0, lie.how != VECTORS && !ragged, &kind);
        f.sh = Shape{rows, (int)cols, s.lanes, s.log2_lanes, s.groups, lie.shift0, lie.step};
        auto launch = [&](auto vec, auto k, auto mode, auto full) -> cudaError_t {
            auto* kernel = k_residual_norm_forward<T, R, decltype(vec)::value, decltype(k)::value,
                                                   decltype(mode)::value, decltype(full)::value>;
            using F = Fit<decltype(vec)::value, decltype(k)::value>;
            constexpr bool kLaid = decltype(mode)::value == RAGGED && F::kAhead;
            const size_t smem = kLaid ? 64 * F::kVectors * s.threads : 0;   // at most 32 KB
            const int n = ctas_of(rows, s, [&] { return resident(kernel, s.threads, smem, 32); },
                                  decltype(mode)::value);
            return launch_k(kernel, dim3(n), dim3(s.threads), smem, st, f);
        };
        auto with = [&](auto vec, auto k, auto mode) -> cudaError_t {
            if constexpr (decltype(vec)::value == 8 &&
                          decltype(k)::value <= (decltype(mode)::value == ALIGNED ? WIDE : MIDDLE)) {
                if (post_weight && pre_weight)
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
                   : kind == WIDER  ? with(vec, Int<decltype(vec)::value == 1 ? WIDER : WIDEST>(), mode)
                                    : with(vec, Int<WIDEST>(), mode);
        };
        return lie.how == VECTORS ? wide(Int<8>(), Int<ALIGNED>())
               : ragged           ? wide(Int<8>(), Int<RAGGED>())
                                  : wide(Int<1>(), Int<ALIGNED>());
    };
    return status_of(stream_type != type  ? type == PSS_BF16 ? go(bf16(), float()) : go(f16(), float())
                     : type == PSS_F32    ? go(float(), float())
                     : type == PSS_BF16   ? go(bf16(), bf16())
                                          : go(f16(), f16()));
}
