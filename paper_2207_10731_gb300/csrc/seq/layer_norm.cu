// Layer norm of rows, forward and backward (pss_layer_norm_* of pss.h).
//
// Forward, one row x of n values:
//   mean = sum x / n,  rstd = 1 / sqrt(sum (x - mean)^2 / n + eps),
//   y = (x - mean) * rstd * w + b.
// Backward, with h = (x - mean) * rstd and g = grad * w:
//   dx = rstd * (g - sum g / n - h * sum(g h) / n),
//   dw = sum over rows of grad * h,  db = sum over rows of grad.
//
// Both are bound by memory: a row is read once, kept in registers through its
// two reductions and written once.  A row is shared by `lanes` threads: a
// power of two up to 32 (several rows to a warp for the embedding's short
// rows, all within shuffles), or a whole CTA for rows above one warp's
// registers (a barrier a reduction, hidden by the SM's other CTAs).  The
// variance is taken from the differences in registers: the textbook
// sum(x^2) - mean^2 would cancel for rows far from zero.
//
// The weight's gradient: each thread keeps the same columns for every row it
// meets, so their sums stay in registers; a CTA then adds its groups in a
// fixed order into one partial row, and a second kernel adds the partial rows
// of all CTAs, again in a fixed order.  No atomics: equal inputs, equal bits.
#include <cmath>

#include "rows.cuh"

using namespace pss;
using namespace pss::seq;

namespace {

constexpr int kMaxCols = 16384;

// Only the largest CH of a vector width ever runs with more than 256 threads
// (split_row).
template <int VEC, int CH>
constexpr int max_threads(int wide) {
    return (VEC == 8 && CH == 2) || (VEC == 1 && CH == 16) ? wide : 256;
}

// Weight and bias stay in registers, and the next row's loads ahead, where the
// instantiation's threads are at most 256: the one with the largest CH is bounded at
// 1024 threads, 64 registers each, and so does without also for rows of 257 columns
// and more that take fewer threads (262144 x 512 bf16: 258 us, 31 % of the copy
// bandwidth, where 262144 x 256 takes 65).
template <typename TX, typename TY, int VEC, int CH, int MODE>
__global__ void __launch_bounds__(max_threads<VEC, CH>(1024))
k_layer_norm_forward(const TX* x, int64_t xs, const float* __restrict__ weight,
                     const float* __restrict__ bias, TY* y, int64_t ys,
                     float* __restrict__ mean_out, float* __restrict__ rstd_out, Shape sh,
                     float eps) {
    pdl_prologue();
    __shared__ float slots[2][32];
    const Place<VEC, MODE> place(sh);
    const float inv_n = 1.f / (float)sh.cols;
    constexpr bool kKeep = max_threads<VEC, CH>(1024) == 256;
    float w[kKeep ? CH : 1][VEC], b[kKeep ? CH : 1][VEC];
    bool in[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = place.at(sh, c);
        in[c] = at < sh.cols;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            if (!kKeep) continue;
            const bool use = inside<MODE>(at + i, sh.cols, in[c]);
            w[kKeep ? c : 0][i] = use ? weight[at + i] : 0.f;
            b[kKeep ? c : 0][i] = use ? bias[at + i] : 0.f;
        }
    }
    // The next row's loads are issued before this row is worked on, where the
    // registers reach.  The trip count is the same for every thread of the CTA
    // (shuffles and barriers inside); rows past the end are computed from zeros
    // and dropped.
    const int64_t step = (int64_t)gridDim.x * sh.groups;
    Part<TX, VEC, CH> next;
    auto fetch = [&](int64_t r) {
        next.load(x + r * xs, r < sh.rows, MODE == ALIGNED || inner(sh, r, xs), in, place, sh);
    };
    if (kKeep) fetch((int64_t)blockIdx.x * sh.groups + place.group);
    for (int64_t r0 = (int64_t)blockIdx.x * sh.groups; r0 < sh.rows; r0 += step) {
        const int64_t r = r0 + place.group;
        const bool live = r < sh.rows;
        if (!kKeep) fetch(r);
        const Part<TX, VEC, CH> part = next;
        if (kKeep && r0 + step < sh.rows) fetch(r + step);
        float v[CH][VEC];
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) part.get(c, v[c]);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (inside<MODE>(place.at(sh, c) + i, sh.cols, true)) s += v[c][i];
        const float mean = row_sum(s, sh.lanes, slots[0]) * inv_n;
        s = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[c][i] -= mean;
                if (inside<MODE>(place.at(sh, c) + i, sh.cols, in[c])) s += v[c][i] * v[c][i];
            }
        const float rstd = 1.f / sqrtf(row_sum(s, sh.lanes, slots[1]) * inv_n + eps);
        if (live) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!in[c]) continue;
                const int at = place.at(sh, c);
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const bool use = kKeep || inside<MODE>(at + i, sh.cols, true);
                    const float wi = kKeep ? w[kKeep ? c : 0][i] : use ? weight[at + i] : 0.f;
                    const float bi = kKeep ? b[kKeep ? c : 0][i] : use ? bias[at + i] : 0.f;
                    o[i] = v[c][i] * rstd * wi + bi;
                }
                store_part(y + r * ys, at, sh.cols, o);
            }
            if (place.t == 0) {
                mean_out[r] = mean;
                rstd_out[r] = rstd;
            }
        }
    }
}

// A row's loads are issued before the row in front of it is worked on: between
// its loads and its store a row waits for two reductions, and the rows of the
// two or three CTAs that the column sums leave room for do not cover that.
// SUMS: where the columns' sums are kept: in registers, or in shared memory (2 *
// cols floats, each touched by its one thread) for rows of more than 8192
// columns, where 1024 threads leave 64 registers each.  (Shared memory for
// shorter rows: 302 instead of 138 us at 16384 x 3328, for bank conflicts.)
enum { REGISTERS, SHARED };
template <typename TG, typename TX, int VEC, int CH, int MODE, int SUMS>
__global__ void __launch_bounds__(max_threads<VEC, CH>(SUMS == SHARED ? 1024 : 512))
k_layer_norm_backward(const TG* grad, int64_t gs, const TX* x, int64_t xs,
                      const float* __restrict__ weight, const float* __restrict__ mean_in,
                      const float* __restrict__ rstd_in, TX* dx, int64_t ds,
                      float* __restrict__ partial, Shape sh) {
    pdl_prologue();
    extern __shared__ float sums[];
    __shared__ float slots[2][32];
    constexpr bool kShared = SUMS == SHARED;
    const Place<VEC, MODE> place(sh);
    const float inv_n = 1.f / (float)sh.cols;
    // the weights stay in registers where these reach
    constexpr bool kKeep = !kShared && VEC * CH < 16;
    float w[kKeep ? CH : 1][VEC], dw[kShared ? 1 : CH][VEC], db[kShared ? 1 : CH][VEC];
    bool in[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = place.at(sh, c);
        in[c] = at < sh.cols;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const bool use = inside<MODE>(at + i, sh.cols, in[c]);
            if (kShared) {
                if (use) sums[at + i] = sums[sh.cols + at + i] = 0.f;
            } else {
                if (kKeep) w[kKeep ? c : 0][i] = use ? weight[at + i] : 0.f;
                dw[kShared ? 0 : c][i] = db[kShared ? 0 : c][i] = 0.f;
            }
        }
    }
    const int64_t step = (int64_t)gridDim.x * sh.groups;
    const int64_t first = (int64_t)blockIdx.x * sh.groups + place.group;
    Part<TX, VEC, CH> next_x;
    Part<TG, VEC, CH> next_g;
    float next_mean = 0.f, next_rstd = 0.f;
    auto fetch = [&](int64_t r) {
        const bool live = r < sh.rows;
        const bool whole = MODE == ALIGNED || (inner(sh, r, xs) && inner(sh, r, gs));
        next_x.load(x + r * xs, live, whole, in, place, sh);
        next_g.load(grad + r * gs, live, whole, in, place, sh);
        next_mean = live ? mean_in[r] : 0.f;
        next_rstd = live ? rstd_in[r] : 0.f;
    };
    if (!kShared) fetch(first);
    for (int64_t r0 = (int64_t)blockIdx.x * sh.groups; r0 < sh.rows; r0 += step) {
        const int64_t r = r0 + place.group;
        const bool live = r < sh.rows;
        if (kShared) fetch(r);   // no registers for two rows
        const Part<TX, VEC, CH> part_x = next_x;
        const Part<TG, VEC, CH> part_g = next_g;
        const float mean = next_mean, rstd = next_rstd;
        if (!kShared && r0 + step < sh.rows) fetch(r + step);
        float h[CH][VEC], g[CH][VEC];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            part_x.get(c, h[c]);
            part_g.get(c, g[c]);
        }
        float s = 0.f, sh_ = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int at = place.at(sh, c) + i;
                const bool use = live && inside<MODE>(at, sh.cols, in[c]);
                h[c][i] = use ? (h[c][i] - mean) * rstd : 0.f;
                if (MODE == RAGGED && !use) g[c][i] = 0.f;   // another row's
                if (kShared) {
                    if (use) {
                        sums[at] += g[c][i] * h[c][i];
                        sums[sh.cols + at] += g[c][i];
                        g[c][i] *= weight[at];
                    }
                } else {
                    dw[kShared ? 0 : c][i] += g[c][i] * h[c][i];
                    db[kShared ? 0 : c][i] += g[c][i];
                    if (kKeep)
                        g[c][i] *= w[kKeep ? c : 0][i];
                    else if (use)
                        g[c][i] *= weight[at];
                }
                s += g[c][i];
                sh_ += g[c][i] * h[c][i];
            }
        s = row_sum(s, sh.lanes, slots[0]) * inv_n;
        sh_ = row_sum(sh_, sh.lanes, slots[1]) * inv_n;
        if (live) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!in[c]) continue;
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) o[i] = (g[c][i] - s - h[c][i] * sh_) * rstd;
                store_part(dx + r * ds, place.at(sh, c), sh.cols, o);
            }
        }
    }
    // the CTA's partial row: [2][cols] at blockIdx.x
    float* out = partial + (int64_t)blockIdx.x * 2 * sh.cols;
    if (sh.lanes > 32) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int at = place.at(sh, c) + i;
                if (inside<MODE>(at, sh.cols, in[c])) {
                    out[at] = kShared ? sums[at] : dw[kShared ? 0 : c][i];
                    out[sh.cols + at] = kShared ? sums[sh.cols + at] : db[kShared ? 0 : c][i];
                }
            }
        return;
    }
    // add the groups of the CTA: shared memory holds [groups][2][cols]
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int at = place.at(sh, c) + i;
            if (inside<MODE>(at, sh.cols, in[c])) {
                sums[(place.group * 2) * sh.cols + at] = dw[kShared ? 0 : c][i];
                sums[(place.group * 2 + 1) * sh.cols + at] = db[kShared ? 0 : c][i];
            }
        }
    __syncthreads();
    for (int k = threadIdx.x; k < 2 * sh.cols; k += blockDim.x) {
        float s = 0.f;
        for (int q = 0; q < sh.groups; ++q) s += sums[q * 2 * sh.cols + k];
        out[k] = s;
    }
}

constexpr int kBackwardPerSm = 4;

template <typename TX, typename TY, int VEC, int CH, int MODE>
cudaError_t launch_forward(const TX* x, int64_t xs, const float* w, const float* b, TY* y,
                           int64_t ys, float* mean, float* rstd, int64_t rows, int cols,
                           const Split& s, const Lie& lie, float eps, cudaStream_t st) {
    auto* k = k_layer_norm_forward<TX, TY, VEC, CH, MODE>;
    const Shape sh{rows, cols, s.lanes, s.log2_lanes, s.groups, lie.shift0, lie.step};
    const int ctas = ctas_of(rows, s, [&] { return resident(k, s.threads, 0, 32); }, MODE);
    return launch_k(k, dim3(ctas), dim3(s.threads), 0, st, x, xs, w, b, y, ys, mean, rstd, sh,
                    eps);
}

template <typename TG, typename TX, int VEC, int CH, int MODE, int SUMS>
cudaError_t launch_backward(const TG* g, int64_t gs, const TX* x, int64_t xs, const float* w,
                            const float* mean, const float* rstd, TX* dx, int64_t ds,
                            float* dw, float* db, float* partial, int64_t rows, int cols,
                            const Split& s, const Lie& lie, cudaStream_t st) {
    auto* k = k_layer_norm_backward<TG, TX, VEC, CH, MODE, SUMS>;
    const size_t smem =
        SUMS == SHARED ? (size_t)8 * cols : s.lanes <= 32 ? (size_t)s.groups * 8 * cols : 0;
    if (smem > 48 * 1024) {
        static std::atomic<uint64_t> ready{0};
        const cudaError_t e = allow_most_smem(k, &ready);
        if (e != cudaSuccess) return e;
    }
    const Shape sh{rows, cols, s.lanes, s.log2_lanes, s.groups, lie.shift0, lie.step};
    const int ctas = ctas_of(
        rows, s, [&] { return resident(k, s.threads, smem, kBackwardPerSm); }, MODE);
    cudaError_t e = launch_k(k, dim3(ctas), dim3(s.threads), smem, st, g, gs, x, xs, w, mean, rstd,
                             dx, ds, partial, sh);
    if (e != cudaSuccess) return e;
    return launch_k(k_row_columns, dim3((2 * cols + 31) / 32), dim3(1024), 0, st,
                    static_cast<const float*>(partial), ctas, 2 * cols, cols, 0, 2 * cols, dw, db);
}

}  // namespace

extern "C" pss_status pss_layer_norm_forward(const void* x, pss_dtype x_type, int64_t x_stride,
                                             const float* weight, const float* bias, int64_t rows,
                                             int64_t cols, float eps, void* y, pss_dtype y_type,
                                             int64_t y_stride, float* mean, float* rstd,
                                             pss_stream stream) {
    if (!dtype_ok(x_type) || !dtype_ok(y_type) || rows < 0 || cols < 1 || !(eps >= 0.f) ||
        std::isinf(eps) || x_stride < cols || y_stride < cols)
        return PSS_ERR_INVALID_ARG;
    if (cols > kMaxCols) return PSS_ERR_UNSUPPORTED;
    if (rows == 0) return PSS_OK;
    for (const void* p : {x, (const void*)weight, (const void*)bias, (const void*)y,
                          (const void*)mean, (const void*)rstd})
        if (!device_ptr(p)) return PSS_ERR_INVALID_ARG;
    if (!aligned_to(x, dtype_size(x_type)) || !aligned_to(y, dtype_size(y_type)) ||
        !aligned_to(weight, 4) || !aligned_to(bias, 4) || !aligned_to(mean, 4) ||
        !aligned_to(rstd, 4))
        return PSS_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const Lie lie = rows_lie<2>(cols, {x, y}, {x_stride, y_stride}, {x_type, y_type});
    return status_of(with_type(x_type, [&](auto tx) {
        return with_type(y_type, [&](auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            auto go = [&](auto vec, auto ch, auto mode, const Split& s) {
                return launch_forward<TX, TY, decltype(vec)::value, decltype(ch)::value,
                                      decltype(mode)::value>(
                    static_cast<const TX*>(x), x_stride, weight, bias, static_cast<TY*>(y),
                    y_stride, mean, rstd, rows, (int)cols, s, lie, eps, st);
            };
            if (lie.how == VECTORS) {
                const Split s = split_row((int)cols, 8, 2, 0);
                return s.ch <= 1 ? go(Int<8>(), Int<1>(), Int<ALIGNED>(), s)
                                 : go(Int<8>(), Int<2>(), Int<ALIGNED>(), s);
            }
            if (lie.how == SHIFTED && cols <= kMaxCols - 8) {
                const Split s = split_row((int)cols, 8, 2, 7);
                return s.ch <= 1 ? go(Int<8>(), Int<1>(), Int<RAGGED>(), s)
                                 : go(Int<8>(), Int<2>(), Int<RAGGED>(), s);
            }
            const Split s = split_row((int)cols, 1, 16, 0);
            return s.ch <= 4 ? go(Int<1>(), Int<4>(), Int<ALIGNED>(), s)
                             : go(Int<1>(), Int<16>(), Int<ALIGNED>(), s);
        });
    }));
}

extern "C" int64_t pss_layer_norm_workspace(int64_t rows, int64_t cols) {
    if (rows < 1 || cols < 1 || cols > kMaxCols) return 0;
    const int64_t most = (int64_t)kBackwardPerSm * sm_count();
    return (rows < most ? rows : most) * 8 * cols;
}

extern "C" pss_status pss_layer_norm_backward(
    const void* grad, pss_dtype grad_type, int64_t grad_stride, const void* x, pss_dtype x_type,
    int64_t x_stride, const float* weight, const float* mean, const float* rstd, int64_t rows,
    int64_t cols, void* dx, int64_t dx_stride, float* dweight, float* dbias, void* workspace,
    int64_t workspace_bytes, pss_stream stream) {
    if (!dtype_ok(grad_type) || !dtype_ok(x_type) || rows < 0 || cols < 1 || grad_stride < cols ||
        x_stride < cols || dx_stride < cols)
        return PSS_ERR_INVALID_ARG;
    if (cols > kMaxCols) return PSS_ERR_UNSUPPORTED;
    if (!device_ptr(dweight) || !device_ptr(dbias) || !aligned_to(dweight, 4) ||
        !aligned_to(dbias, 4))
        return PSS_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (rows == 0) {
        const cudaError_t e = cudaMemsetAsync(dweight, 0, 4 * cols, st);
        return status_of(e != cudaSuccess ? e : cudaMemsetAsync(dbias, 0, 4 * cols, st));
    }
    for (const void* p : {grad, x, (const void*)weight, (const void*)mean, (const void*)rstd,
                          (const void*)dx, (const void*)workspace})
        if (!device_ptr(p)) return PSS_ERR_INVALID_ARG;
    if (!aligned_to(grad, dtype_size(grad_type)) || !aligned_to(x, dtype_size(x_type)) ||
        !aligned_to(dx, dtype_size(x_type)) || !aligned_to(weight, 4) || !aligned_to(mean, 4) ||
        !aligned_to(rstd, 4) || !aligned_to(workspace, 16) ||
        workspace_bytes < pss_layer_norm_workspace(rows, cols))
        return PSS_ERR_INVALID_ARG;
    const Lie lie = rows_lie<3>(cols, {x, grad, dx}, {x_stride, grad_stride, dx_stride},
                                {x_type, grad_type, x_type});
    return status_of(with_type(grad_type, [&](auto tg) {
        return with_type(x_type, [&](auto tx) {
            using TG = decltype(tg);
            using TX = decltype(tx);
            auto go = [&](auto vec, auto ch, auto mode, auto sums, const Split& s) {
                return launch_backward<TG, TX, decltype(vec)::value, decltype(ch)::value,
                                       decltype(mode)::value, decltype(sums)::value>(
                    static_cast<const TG*>(grad), grad_stride, static_cast<const TX*>(x), x_stride,
                    weight, mean, rstd, static_cast<TX*>(dx), dx_stride, dweight, dbias,
                    static_cast<float*>(workspace), rows, (int)cols, s, lie, st);
            };
            if (lie.how == VECTORS) {
                const Split s = split_row((int)cols, 8, 2, 0);
                return s.ch <= 1 ? go(Int<8>(), Int<1>(), Int<ALIGNED>(), Int<REGISTERS>(), s)
                       : s.threads > 512
                           ? go(Int<8>(), Int<2>(), Int<ALIGNED>(), Int<SHARED>(), s)
                           : go(Int<8>(), Int<2>(), Int<ALIGNED>(), Int<REGISTERS>(), s);
            }
            if (lie.how == SHIFTED && cols <= kMaxCols - 8) {
                const Split s = split_row((int)cols, 8, 2, 7);
                return s.ch <= 1 ? go(Int<8>(), Int<1>(), Int<RAGGED>(), Int<REGISTERS>(), s)
                       : s.threads > 512
                           ? go(Int<8>(), Int<2>(), Int<RAGGED>(), Int<SHARED>(), s)
                           : go(Int<8>(), Int<2>(), Int<RAGGED>(), Int<REGISTERS>(), s);
            }
            const Split s = split_row((int)cols, 1, 16, 0);
            return s.ch <= 4 ? go(Int<1>(), Int<4>(), Int<ALIGNED>(), Int<REGISTERS>(), s)
                   : s.threads > 512
                       ? go(Int<1>(), Int<16>(), Int<ALIGNED>(), Int<SHARED>(), s)
                       : go(Int<1>(), Int<16>(), Int<ALIGNED>(), Int<REGISTERS>(), s);
        });
    }));
}
