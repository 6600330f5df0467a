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
// CH vectors of VEC elements, vector c of thread t at (c*lanes + t)*VEC - shift.
// shift > 0: rows do not start at a multiple of 8 elements.  Row r starts
// (shift0 + r*step) % 8 past one, and a thread only meets rows a multiple of 8
// apart (RAGGED), so its vectors stay aligned and its columns the same; a row's
// ends are moved one by one.
struct Shape {
    int64_t rows;
    int cols, lanes, log2_lanes;   // log2_lanes: for lanes <= 32
    int groups;                    // rows of a CTA at a time
    int shift0, step;              // RAGGED
};
enum { ALIGNED, RAGGED };          // 8 elements at a time, or VEC = 1 (ALIGNED)

// The thread's place in its row: VEC-element vector c at at(c).
template <int VEC, int MODE>
struct Place {
    int t, group, shift;
    __device__ __forceinline__ Place(const Shape& sh) {
        const bool wide = sh.lanes > 32;
        t = wide ? threadIdx.x : threadIdx.x & (sh.lanes - 1);
        group = wide ? 0 : threadIdx.x >> sh.log2_lanes;
        const int first = (blockIdx.x * sh.groups + group) & 7;
        shift = MODE == RAGGED ? (sh.shift0 + first * sh.step) & 7 : 0;
    }
    __device__ __forceinline__ int at(const Shape& sh, int c) const {
        return (c * sh.lanes + t) * VEC - shift;
    }
};
// Whether the 7 elements before and after row r are between the tensor's first
// and last; otherwise (the first and last rows) they must not be touched.
__device__ __forceinline__ bool inner(const Shape& sh, int64_t r, int64_t stride) {
    return r * stride >= 7 && (sh.rows - 1 - r) * stride >= 7;
}
// Whether element e of n exists; a vector that exists at all holds only such
// elements unless the rows are ragged.
template <int MODE>
__device__ __forceinline__ bool inside(int e, int n, bool vector) {
    return MODE == RAGGED ? (unsigned)e < (unsigned)n : vector;
}

// A thread's part of one row of a tensor, as it comes from memory.
template <typename T, int VEC, int CH>
struct Part;
template <typename T, int CH>
struct Part<T, 8, CH> {
    Raw8<T> v[CH];
    template <int MODE>
    __device__ __forceinline__ void load(const T* row, bool live, bool whole, const bool (&in)[CH],
                                         const Place<8, MODE>& place, const Shape& sh) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            v[c] = live && in[c] ? load_raw_part(row, place.at(sh, c), sh.cols, whole) : Raw8<T>{};
    }
    __device__ __forceinline__ void get(int c, float (&to)[8]) const { unpack(v[c], to); }
};
template <typename T, int CH>
struct Part<T, 1, CH> {
    float v[CH];
    template <int MODE>
    __device__ __forceinline__ void load(const T* row, bool live, bool, const bool (&in)[CH],
                                         const Place<1, MODE>& place, const Shape& sh) {
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = live && in[c] ? load_f32(row[place.at(sh, c)]) : 0.f;
    }
    __device__ __forceinline__ void get(int c, float (&to)[1]) const { to[0] = v[c]; }
};

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
//   most: the largest CH of this vector width; extra: elements that a ragged
//   row's first vector may hold in front of it.  A row within one warp's reach
//   (32 * most vectors) takes the fewest lanes that hold it with one vector
//   each, up to 32; a longer row takes a CTA.
struct Split {
    int lanes, log2_lanes, ch, threads, groups;
};
Split split_row(int cols, int vec, int most, int extra) {
    constexpr int kCta = 256;
    Split s;
    const int vecs = (cols + extra + vec - 1) / vec;
    if (vecs <= 32 * most) {
        s.lanes = 1;
        s.log2_lanes = 0;
        while (s.lanes < 32 && s.lanes < vecs) s.lanes *= 2, ++s.log2_lanes;
        s.ch = (vecs + s.lanes - 1) / s.lanes;
        s.threads = kCta;
        s.groups = kCta / s.lanes;
    } else {
        s.ch = most;
        s.lanes = ((vecs + most - 1) / most + 31) / 32 * 32;
        s.log2_lanes = 0;
        s.threads = s.lanes;
        s.groups = 1;
    }
    return s;
}

// How a call's rows lie: 8 elements at a time where every row starts at a
// multiple of 8, or where all tensors' rows start equally far past one.
enum { VECTORS, SHIFTED, SINGLE };
struct Lie {
    int how, shift0, step;
};
template <int N>
Lie rows_lie(int64_t cols, const void* const (&p)[N], const int64_t (&stride)[N],
             const int (&type)[N]) {
    bool aligned = cols % 8 == 0, same = true;
    for (int i = 0; i < N; ++i) {
        const size_t size = dtype_size(type[i]);
        aligned = aligned && aligned8(p[i], stride[i], size);
        same = same && past8(p[i], size) == past8(p[0], dtype_size(type[0])) &&
               stride[i] % 8 == stride[0] % 8;
    }
    return Lie{aligned ? VECTORS : same ? SHIFTED : SINGLE,
               past8(p[0], dtype_size(type[0])), (int)(stride[0] % 8)};
}

constexpr int kBackwardPerSm = 4;

template <typename K>
int resident(K kernel, int threads, size_t smem, int most) {
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess)
        n = 1;
    return n < 1 ? 1 : n < most ? n : most;
}

// CTAs of a launch; with RAGGED a CTA's rows have to be a multiple of 8 apart.
template <typename F>
int ctas_of(int64_t rows, const Split& s, F per_sm, int mode) {
    const int64_t need = (rows + s.groups - 1) / s.groups;
    if (need <= sm_count()) return (int)need;   // a small call does not ask how many fit
    int64_t most = (int64_t)per_sm() * sm_count();
    if (need <= most) return (int)need;
    if (mode == RAGGED) most -= most % 8;
    return (int)(most > 0 ? most : need < 8 ? need : 8);
}

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
        const cudaError_t e =
            cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    const Shape sh{rows, cols, s.lanes, s.log2_lanes, s.groups, lie.shift0, lie.step};
    const int ctas = ctas_of(
        rows, s, [&] { return resident(k, s.threads, smem, kBackwardPerSm); }, MODE);
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
