// Dropout with a mask that is never stored (pss_dropout of pss.h).
//
// Element e of the row-major [rows][cols] tensor is kept when 16 bits of
// Philox4x32-10 at counter (e / 8, offset) are at least t = round(65536 p);
// kept values are multiplied by 65536 / (65536 - t).  A thread takes one
// counter, i.e. 8 consecutive elements: one 16- or 32-byte access each way and
// ten rounds of two 32x32->64 bit products.
//
// Bound by memory.  16 random bits an element: a generator call is about 80
// integer instructions, so with 32 bits an element (four elements a call) the
// 16-bit types would need more issue slots than their four bytes of traffic
// leave.
#include <cmath>

#include "seq_common.cuh"

using namespace pss;
using namespace pss::seq;

namespace {

struct Params {
    int64_t n, cols;               // n = rows * cols elements
    uint64_t inv;                  // floor((2^64 - 1) / d), d of the division below
    int64_t xs, rs, ys;            // row strides
    uint32_t off0, off1;
    uint32_t key[10][2];           // of each round
    uint32_t below;                // (threshold << 16) - 1
    bool all;                      // the threshold is 0
    float scale;
};

// The generator of Salmon, Moraes, Dror & Shaw, "Parallel random numbers: as
// easy as 1, 2, 3" (SC 2011), 4x32 bits, 10 rounds;
// the rounds' keys come with the launch, as constants.
__device__ __forceinline__ void philox(uint64_t counter, const Params& p, uint32_t (&c)[4]) {
    c[0] = (uint32_t)counter;
    c[1] = (uint32_t)(counter >> 32);
    c[2] = p.off0;
    c[3] = p.off1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c[0] * 0xD2511F53u;
        const uint64_t b = (uint64_t)c[2] * 0xCD9E8D57u;
        c[0] = (uint32_t)(b >> 32) ^ c[1] ^ p.key[r][0];
        c[1] = (uint32_t)b;
        c[2] = (uint32_t)(a >> 32) ^ c[3] ^ p.key[r][1];
        c[3] = (uint32_t)a;
    }
}
// Whether 16-bit value i is at least the threshold: the value in the upper half
// of a word against the last word below the threshold's.
__device__ __forceinline__ bool kept(const uint32_t (&c)[4], int i, const Params& p) {
    const uint32_t w = c[i >> 1];
    return ((i & 1) ? w : w << 16) > p.below || p.all;
}
// A dropped element is left out before the product, which would keep a NaN.
template <bool RES>
__device__ __forceinline__ float dropped(bool keep, float v, float scale, float add) {
    const float t = keep ? v : 0.f;
    return RES ? fmaf(t, scale, add) : t * scale;
}

// s / d for s < 2^63, inv = floor((2^64 - 1) / d): umulhi gives the quotient or
// one less (Barrett, CRYPTO '86).
__device__ __forceinline__ int64_t divide(int64_t s, int64_t d, uint64_t inv, int64_t* rest) {
    uint64_t q = __umul64hi((uint64_t)s, inv);
    int64_t r = s - (int64_t)q * d;
    if (r >= d) {
        r -= d;
        ++q;
    }
    *rest = r;
    return (int64_t)q;
}

// FLAT: one run of n elements, aligned for vectors; the last n % 8 one by one.
// ROWS: strided rows of cols % 8 == 0 elements, aligned (d = cols / 8).
// SINGLE: any strides and alignment, element by element (d = cols).
enum { FLAT, ROWS, SINGLE };

template <typename T, int MODE, bool RES>
__global__ void __launch_bounds__(kThreads, 4)
k_dropout(const T* x, const T* res, T* y, Params p) {
    pdl_prologue();
    const int64_t whole = MODE == SINGLE ? 0 : p.n / 8;
    const int64_t groups = (p.n + 7) / 8;
    const int64_t step = (int64_t)gridDim.x * kThreads;
    // several groups a turn, their loads first and kept as they came: 64 bytes a
    // thread and tensor in flight
    constexpr int kGroups = sizeof(T) == 4 ? 2 : 4;
    for (int64_t g0 = (int64_t)blockIdx.x * kThreads + threadIdx.x; g0 < groups;
         g0 += kGroups * step) {
        Raw8<T> in[kGroups], add[RES ? kGroups : 1];
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int64_t g = g0 + u * step;
            if (g >= whole) continue;
            int64_t row = 0, at = 8 * g;
            if (MODE == ROWS) {
                row = divide(g, p.cols / 8, p.inv, &at);
                at *= 8;
            }
            in[u] = load_raw(x + row * p.xs + at);
            if (RES) add[RES ? u : 0] = load_raw(res + row * p.rs + at);
        }
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int64_t g = g0 + u * step;
            if (g >= groups) continue;
            uint32_t c[4];
            philox((uint64_t)g, p, c);
            if (g < whole) {
                int64_t row = 0, at = 8 * g;
                if (MODE == ROWS) {
                    row = divide(g, p.cols / 8, p.inv, &at);
                    at *= 8;
                }
                float v[8], w[8];
                unpack(in[u], v);
                if (RES) unpack(add[RES ? u : 0], w);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = dropped<RES>(kept(c, i, p), v[i], p.scale, RES ? w[i] : 0.f);
                store8(y + row * p.ys + at, v);
                continue;
            }
            int64_t r = 0, k = 8 * g;
            if (MODE == SINGLE) r = divide(k, p.cols, p.inv, &k);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (8 * g + i >= p.n) break;
                y[r * p.ys + k] = round_to<T>(
                    dropped<RES>(kept(c, i, p), load_f32(x[r * p.xs + k]), p.scale,
                                 RES ? load_f32(res[r * p.rs + k]) : 0.f));
                if (++k == p.cols && MODE == SINGLE) {
                    k = 0;
                    ++r;
                }
            }
        }
    }
}

template <typename T, int MODE, bool RES>
cudaError_t launch(const void* x, const void* res, void* y, const Params& p, cudaStream_t st) {
    auto* k = k_dropout<T, MODE, RES>;
    const int64_t blocks = ((p.n + 7) / 8 + kThreads - 1) / kThreads;
    const int64_t most = (int64_t)sm_count() * 16;
    return launch_k(k, dim3((unsigned)(blocks < most ? blocks : most)), dim3(kThreads), 0, st,
                    static_cast<const T*>(x), static_cast<const T*>(res), static_cast<T*>(y), p);
}

}  // namespace

extern "C" pss_status pss_dropout(const void* x, int64_t x_stride, const void* residual,
                                  int64_t residual_stride, int64_t rows, int64_t cols, double p,
                                  uint64_t seed, uint64_t offset, pss_dtype type, void* y,
                                  int64_t y_stride, pss_stream stream) {
    if (!dtype_ok(type) || rows < 0 || cols < 0 || !(p >= 0.0 && p <= 1.0) || x_stride < cols ||
        y_stride < cols || (residual && residual_stride < cols))
        return PSS_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return PSS_OK;
    if (rows > (INT64_MAX / 2) / cols) return PSS_ERR_INVALID_ARG;
    const size_t size = dtype_size(type);
    if (!device_ptr(x) || !device_ptr(y) || (residual && !device_ptr(residual)) ||
        !aligned_to(x, size) || !aligned_to(y, size) || (residual && !aligned_to(residual, size)))
        return PSS_ERR_INVALID_ARG;
    Params q{};
    q.n = rows * cols;
    q.cols = cols;
    q.xs = x_stride;
    q.rs = residual_stride;
    q.ys = y_stride;
    for (uint32_t r = 0; r < 10; ++r) {
        q.key[r][0] = (uint32_t)seed + r * 0x9E3779B9u;
        q.key[r][1] = (uint32_t)(seed >> 32) + r * 0xBB67AE85u;
    }
    q.off0 = (uint32_t)offset;
    q.off1 = (uint32_t)(offset >> 32);
    const uint32_t threshold = (uint32_t)std::nearbyint(p * 65536.0);
    q.below = (uint32_t)(((uint64_t)threshold << 16) - 1);
    q.all = threshold == 0;
    q.scale = threshold < 65536u ? (float)(65536.0 / (65536.0 - threshold)) : 0.f;
    const bool packed = rows == 1 || (x_stride == cols && y_stride == cols &&
                                      (!residual || residual_stride == cols));
    const bool bases = aligned_to(x, 8 * size) && aligned_to(y, 8 * size) &&
                       (!residual || aligned_to(residual, 8 * size));
    const bool strides = cols % 8 == 0 && x_stride % 8 == 0 && y_stride % 8 == 0 &&
                         (!residual || residual_stride % 8 == 0);
    const int mode = bases && packed ? FLAT : bases && strides ? ROWS : SINGLE;
    const uint64_t d = mode == ROWS ? (uint64_t)cols / 8 : (uint64_t)cols;
    q.inv = UINT64_MAX / d;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return status_of(with_type(type, [&](auto t) {
        using T = decltype(t);
        if (residual)
            return mode == FLAT   ? launch<T, FLAT, true>(x, residual, y, q, st)
                   : mode == ROWS ? launch<T, ROWS, true>(x, residual, y, q, st)
                                  : launch<T, SINGLE, true>(x, residual, y, q, st);
        return mode == FLAT   ? launch<T, FLAT, false>(x, residual, y, q, st)
               : mode == ROWS ? launch<T, ROWS, false>(x, residual, y, q, st)
                              : launch<T, SINGLE, false>(x, residual, y, q, st);
    }));
}
