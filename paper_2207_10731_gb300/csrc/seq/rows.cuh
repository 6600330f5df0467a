// Shared by the norms of rows: how a row is spread over threads and moved, its
// reductions, and the sums over rows.
#pragma once

#include "seq_common.cuh"

namespace pss {
namespace seq {

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

// Column sums of the partial rows [parts][width]: columns first .. last, the first `cols`
// to `one`, the others to `two`.  A CTA takes 32 columns, its 32 warps every
// 32nd partial row.
static __global__ void __launch_bounds__(1024)
k_row_columns(const float* __restrict__ partial, int parts, int width, int cols, int first,
              int last, float* __restrict__ one, float* __restrict__ two) {
    pdl_prologue();
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int k = first + blockIdx.x * 32 + lane;
    float s = 0.f;
    if (k < last)
        for (int p = warp; p < parts; p += 32) s += partial[(int64_t)p * width + k];
    part[warp][lane] = s;
    __syncthreads();
    s = part[lane][warp];
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
    const int c = first + blockIdx.x * 32 + warp;
    if (lane == 0 && c < last) (c < cols ? one[c] : two[c - cols]) = s;
}

// Threads to a row and vectors to a thread.
//   most: the largest CH of this vector width; extra: elements that a ragged
//   row's first vector may hold in front of it.  A row within one warp's reach
//   (32 * most vectors) takes the fewest lanes that hold it with one vector
//   each, up to 32; a longer row takes a CTA.
struct Split {
    int lanes, log2_lanes, ch, threads, groups;
};
inline Split split_row(int cols, int vec, int most, int extra) {
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

}  // namespace seq
}  // namespace pss
