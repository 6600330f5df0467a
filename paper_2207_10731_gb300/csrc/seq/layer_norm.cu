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
// registers (two barriers a reduction, hidden by the SM's other CTAs).  The
// variance is taken from the differences in registers: the textbook
// sum(x^2) - mean^2 would cancel for rows far from zero.
//
// The weight's gradient: each thread keeps the same columns for every row it
// meets, so their sums stay in registers; a CTA then adds its groups in a
// fixed order into one partial row, and a second kernel adds the partial rows
// of all CTAs, again in a fixed order.  No atomics: equal inputs, equal bits.
#include <cmath>

#include "seq_common.cuh"

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

// Sum over the row's threads: `lanes` <= 32 lanes of a warp, or the whole CTA
// (lanes == blockDim.x) through `slot`, one float per warp.  Slots alternate
// between calls, so one barrier separates the reads of a call from the
// writes two calls later.
__device__ __forceinline__ float row_sum(float v, int lanes, float* slot) {
    const int w = lanes < 32 ? lanes : 32;
    for (int m = w >> 1; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    if (lanes <= 32) return v;
    const int lane = threadIdx.x & 31, nw = blockDim.x >> 5;
    if (lane == 0) slot[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < nw ? slot[lane] : 0.f;
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
}

// How the rows are spread over threads: `lanes` threads to a row, each with
// CH vectors of VEC elements, vector c of thread t at (c*lanes + t)*VEC.
struct Shape {
    int64_t rows;
    int cols, lanes, log2_lanes;   // log2_lanes: for lanes <= 32
    int groups;                    // rows of a CTA at a time
};

template <typename TX, typename TY, int VEC, int CH>
__global__ void __launch_bounds__(max_threads<VEC, CH>(1024))
k_layer_norm_forward(const TX* x, int64_t xs, const float* __restrict__ weight,
                     const float* __restrict__ bias, TY* y, int64_t ys,
                     float* __restrict__ mean_out, float* __restrict__ rstd_out, Shape sh,
                     float eps) {
    pdl_prologue();
    __shared__ float slots[2][32];
    const bool wide = sh.lanes > 32;
    const int t = wide ? threadIdx.x : threadIdx.x & (sh.lanes - 1);
    const int group = wide ? 0 : threadIdx.x >> sh.log2_lanes;
    const float inv_n = 1.f / (float)sh.cols;
    // weight and bias stay in registers where these reach (64 with 1024 threads)
    constexpr bool kKeep = max_threads<VEC, CH>(1024) == 256;
    float w[kKeep ? CH : 1][VEC], b[kKeep ? CH : 1][VEC];
    bool in[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = (c * sh.lanes + t) * VEC;
        in[c] = at < sh.cols;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            if (!kKeep) continue;
            w[kKeep ? c : 0][i] = in[c] ? weight[at + i] : 0.f;
            b[kKeep ? c : 0][i] = in[c] ? bias[at + i] : 0.f;
        }
    }
    // the trip count is the same for every thread of the CTA (shuffles and
    // barriers inside); rows past the end are computed from zeros and dropped
    for (int64_t r0 = (int64_t)blockIdx.x * sh.groups; r0 < sh.rows;
         r0 += (int64_t)gridDim.x * sh.groups) {
        const int64_t r = r0 + group;
        const bool live = r < sh.rows;
        float v[CH][VEC];
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (live && in[c]) {
                load_vec(x + r * xs + (c * sh.lanes + t) * VEC, v[c]);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[c][i] = 0.f;
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += v[c][i];
        const float mean = row_sum(s, sh.lanes, slots[0]) * inv_n;
        s = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[c][i] -= mean;
                s += in[c] ? v[c][i] * v[c][i] : 0.f;
            }
        const float rstd = 1.f / sqrtf(row_sum(s, sh.lanes, slots[1]) * inv_n + eps);
        if (live) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!in[c]) continue;
                const int at = (c * sh.lanes + t) * VEC;
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    o[i] = v[c][i] * rstd * (kKeep ? w[kKeep ? c : 0][i] : weight[at + i]) +
                           (kKeep ? b[kKeep ? c : 0][i] : bias[at + i]);
                store_vec(y + r * ys + at, o);
            }
            if (t == 0) {
                mean_out[r] = mean;
                rstd_out[r] = rstd;
            }
        }
    }
}

// SMEM: the column sums live in shared memory (2 * cols floats, each touched
// by its one thread) instead of registers, for rows of more than 8192 columns:
// 1024 threads leave 64 registers each.
template <typename TG, typename TX, int VEC, int CH, bool SMEM>
__global__ void __launch_bounds__(max_threads<VEC, CH>(SMEM ? 1024 : 512))
k_layer_norm_backward(const TG* grad, int64_t gs, const TX* x,
                      int64_t xs, const float* __restrict__ weight,
                      const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
                      TX* dx, int64_t ds, float* __restrict__ partial, Shape sh) {
    pdl_prologue();
    extern __shared__ float sums[];
    __shared__ float slots[2][32];
    const bool wide = sh.lanes > 32;
    const int t = wide ? threadIdx.x : threadIdx.x & (sh.lanes - 1);
    const int group = wide ? 0 : threadIdx.x >> sh.log2_lanes;
    const float inv_n = 1.f / (float)sh.cols;
    // the weights stay in registers where these reach
    constexpr bool kKeep = !SMEM && (VEC > 1 || CH < 16);
    float w[kKeep ? CH : 1][VEC], dw[SMEM ? 1 : CH][VEC], db[SMEM ? 1 : CH][VEC];
    bool in[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = (c * sh.lanes + t) * VEC;
        in[c] = at < sh.cols;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            if (SMEM) {
                if (in[c]) sums[at + i] = sums[sh.cols + at + i] = 0.f;
            } else {
                if (kKeep) w[kKeep ? c : 0][i] = in[c] ? weight[at + i] : 0.f;
                dw[SMEM ? 0 : c][i] = db[SMEM ? 0 : c][i] = 0.f;
            }
        }
    }
    for (int64_t r0 = (int64_t)blockIdx.x * sh.groups; r0 < sh.rows;
         r0 += (int64_t)gridDim.x * sh.groups) {
        const int64_t r = r0 + group;
        const bool live = r < sh.rows;
        float h[CH][VEC], g[CH][VEC];
        float mean = 0.f, rstd = 0.f;
        if (live) {
            mean = mean_in[r];
            rstd = rstd_in[r];
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = (c * sh.lanes + t) * VEC;
            if (live && in[c]) {
                load_vec(x + r * xs + at, h[c]);
                load_vec(grad + r * gs + at, g[c]);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) h[c][i] = g[c][i] = 0.f;
            }
        }
        float s = 0.f, sh_ = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int at = (c * sh.lanes + t) * VEC + i;
                const bool use = live && in[c];
                h[c][i] = use ? (h[c][i] - mean) * rstd : 0.f;
                if (SMEM) {
                    if (use) {
                        sums[at] += g[c][i] * h[c][i];
                        sums[sh.cols + at] += g[c][i];
                        g[c][i] *= weight[at];
                    }
                } else {
                    dw[SMEM ? 0 : c][i] += g[c][i] * h[c][i];
                    db[SMEM ? 0 : c][i] += g[c][i];
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
                store_vec(dx + r * ds + (c * sh.lanes + t) * VEC, o);
            }
        }
    }
    // the CTA's partial row: [2][cols] at blockIdx.x
    float* out = partial + (int64_t)blockIdx.x * 2 * sh.cols;
    if (SMEM) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int at = (c * sh.lanes + t) * VEC + i;
                if (in[c]) {
                    out[at] = sums[at];
                    out[sh.cols + at] = sums[sh.cols + at];
                }
            }
        return;
    }
    if (wide) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int at = (c * sh.lanes + t) * VEC + i;
                if (in[c]) {
                    out[at] = dw[SMEM ? 0 : c][i];
                    out[sh.cols + at] = db[SMEM ? 0 : c][i];
                }
            }
        return;
    }
    // add the groups of the CTA: shared memory holds [groups][2][cols]
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int at = (c * sh.lanes + t) * VEC + i;
            if (in[c]) {
                sums[(group * 2) * sh.cols + at] = dw[SMEM ? 0 : c][i];
                sums[(group * 2 + 1) * sh.cols + at] = db[SMEM ? 0 : c][i];
            }
        }
    __syncthreads();
    for (int k = threadIdx.x; k < 2 * sh.cols; k += blockDim.x) {
        float s = 0.f;
        for (int q = 0; q < sh.groups; ++q) s += sums[q * 2 * sh.cols + k];
        out[k] = s;
    }
}

// dweight / dbias: column sums of the partial rows [parts][2*cols].  A CTA
// takes 32 columns, its 32 warps every 32nd partial row.
__global__ void __launch_bounds__(1024)
k_layer_norm_columns(const float* __restrict__ partial, int parts, int cols,
                     float* __restrict__ dweight, float* __restrict__ dbias) {
    pdl_prologue();
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int k = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (k < 2 * cols)
        for (int p = warp; p < parts; p += 32) s += partial[(int64_t)p * 2 * cols + k];
    part[warp][lane] = s;
    __syncthreads();
    s = part[lane][warp];
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
    const int c = blockIdx.x * 32 + warp;
    if (lane == 0 && c < 2 * cols) (c < cols ? dweight[c] : dbias[c - cols]) = s;
}

// Threads to a row and vectors to a thread.
//   most: the largest CH of this vector width.  A row within one warp's reach
//   (32 * most vectors) takes the fewest lanes that hold it with one vector
//   each, up to 32; a longer row takes a CTA.
struct Split {
    int lanes, log2_lanes, ch, threads, groups;
};
Split split_row(int cols, int vec, int most, int cta) {
    Split s;
    const int vecs = (cols + vec - 1) / vec;
    if (vecs <= 32 * most) {
        s.lanes = 1;
        s.log2_lanes = 0;
        while (s.lanes < 32 && s.lanes < vecs) s.lanes *= 2, ++s.log2_lanes;
        s.ch = (vecs + s.lanes - 1) / s.lanes;
        s.threads = cta;
        s.groups = cta / s.lanes;
    } else {
        s.ch = most;
        s.lanes = ((vecs + most - 1) / most + 31) / 32 * 32;
        s.log2_lanes = 0;
        s.threads = s.lanes;
        s.groups = 1;
    }
    return s;
}

// CTAs of the backward pass: as many partial rows as `per_sm` CTAs on every SM
// write.  Two for long rows: their partial rows (8 bytes a column) are then a
// few percent of the traffic.
int backward_ctas(int64_t rows, int groups, int per_sm, int sms) {
    const int64_t need = (rows + groups - 1) / groups;
    const int64_t most = (int64_t)per_sm * sms;
    return (int)(need < most ? (need > 0 ? need : 1) : most);
}

constexpr int kBackwardPerSm = 4;

template <typename K>
int resident(K kernel, int threads, size_t smem, int most) {
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess)
        n = 1;
    return n < 1 ? 1 : n < most ? n : most;
}

template <typename TX, typename TY, int VEC, int CH>
cudaError_t launch_forward(const TX* x, int64_t xs, const float* w, const float* b, TY* y,
                           int64_t ys, float* mean, float* rstd, int64_t rows, int cols,
                           const Split& s, float eps, cudaStream_t st) {
    auto* k = k_layer_norm_forward<TX, TY, VEC, CH>;
    const Shape sh{rows, cols, s.lanes, s.log2_lanes, s.groups};
    const int64_t need = (rows + s.groups - 1) / s.groups;
    const int64_t most = (int64_t)sm_count() * resident(k, s.threads, 0, 32);
    return launch_k(k, dim3((unsigned)(need < most ? need : most)), dim3(s.threads), 0, st, x, xs,
                    w, b, y, ys, mean, rstd, sh, eps);
}

template <typename TG, typename TX, int VEC, int CH, bool SMEM>
cudaError_t launch_backward(const TG* g, int64_t gs, const TX* x, int64_t xs, const float* w,
                            const float* mean, const float* rstd, TX* dx, int64_t ds,
                            float* dw, float* db, float* partial, int64_t rows, int cols,
                            const Split& s, cudaStream_t st) {
    auto* k = k_layer_norm_backward<TG, TX, VEC, CH, SMEM>;
    const size_t smem = SMEM ? (size_t)8 * cols : s.lanes <= 32 ? (size_t)s.groups * 8 * cols : 0;
    if (smem > 48 * 1024) {
        const cudaError_t e =
            cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    const Shape sh{rows, cols, s.lanes, s.log2_lanes, s.groups};
    const int ctas =
        backward_ctas(rows, s.groups, resident(k, s.threads, smem, kBackwardPerSm), sm_count());
    cudaError_t e = launch_k(k, dim3(ctas), dim3(s.threads), smem, st, g, gs, x, xs, w, mean, rstd,
                             dx, ds, partial, sh);
    if (e != cudaSuccess) return e;
    return launch_k(k_layer_norm_columns, dim3((2 * cols + 31) / 32), dim3(1024), 0, st,
                    static_cast<const float*>(partial), ctas, cols, dw, db);
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
    const bool wide = cols % 8 == 0 && aligned8(x, x_stride, dtype_size(x_type)) &&
                      aligned8(y, y_stride, dtype_size(y_type));
    return status_of(with_type(x_type, [&](auto tx) {
        return with_type(y_type, [&](auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            auto go = [&](auto vec, auto ch, const Split& s) {
                return launch_forward<TX, TY, decltype(vec)::value, decltype(ch)::value>(
                    static_cast<const TX*>(x), x_stride, weight, bias, static_cast<TY*>(y),
                    y_stride, mean, rstd, rows, (int)cols, s, eps, st);
            };
            if (wide) {
                const Split s = split_row((int)cols, 8, 2, 256);
                return s.ch <= 1 ? go(Int<8>(), Int<1>(), s) : go(Int<8>(), Int<2>(), s);
            }
            const Split s = split_row((int)cols, 1, 16, 256);
            return s.ch <= 2   ? go(Int<1>(), Int<2>(), s)
                   : s.ch <= 4 ? go(Int<1>(), Int<4>(), s)
                   : s.ch <= 8 ? go(Int<1>(), Int<8>(), s)
                   : s.ch <= 12 ? go(Int<1>(), Int<12>(), s)
                                : go(Int<1>(), Int<16>(), s);
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
    const bool wide = cols % 8 == 0 && aligned8(x, x_stride, dtype_size(x_type)) &&
                      aligned8(dx, dx_stride, dtype_size(x_type)) &&
                      aligned8(grad, grad_stride, dtype_size(grad_type));
    return status_of(with_type(grad_type, [&](auto tg) {
        return with_type(x_type, [&](auto tx) {
            using TG = decltype(tg);
            using TX = decltype(tx);
            auto go = [&](auto vec, auto ch, auto smem, const Split& s) {
                return launch_backward<TG, TX, decltype(vec)::value, decltype(ch)::value,
                                       decltype(smem)::value != 0>(
                    static_cast<const TG*>(grad), grad_stride, static_cast<const TX*>(x), x_stride,
                    weight, mean, rstd, static_cast<TX*>(dx), dx_stride, dweight, dbias,
                    static_cast<float*>(workspace), rows, (int)cols, s, st);
            };
            const bool smem = cols > 8192;
            if (wide) {
                const Split s = split_row((int)cols, 8, 2, 256);
                return s.ch <= 1 ? go(Int<8>(), Int<1>(), Int<0>(), s)
                       : smem    ? go(Int<8>(), Int<2>(), Int<1>(), s)
                                 : go(Int<8>(), Int<2>(), Int<0>(), s);
            }
            const Split s = split_row((int)cols, 1, 16, 256);
            return s.ch <= 4   ? go(Int<1>(), Int<4>(), Int<0>(), s)
                   : s.ch <= 8 ? go(Int<1>(), Int<8>(), Int<0>(), s)
                   : s.ch <= 12 ? go(Int<1>(), Int<12>(), Int<0>(), s)
                   : smem      ? go(Int<1>(), Int<16>(), Int<1>(), s)
                               : go(Int<1>(), Int<16>(), Int<0>(), s);
        });
    }));
}
