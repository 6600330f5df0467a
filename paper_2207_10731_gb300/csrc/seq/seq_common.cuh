// Shared by the sequence operators (layer norm, dropout, attention): element
// types, vector loads and stores, and the checks of their C entry points.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "pss.h"
#include "pss_device.cuh"

namespace pss {
namespace seq {

using bf16 = __nv_bfloat16;
using f16 = __half;

__device__ __forceinline__ float load_f32(float v) { return v; }
__device__ __forceinline__ float load_f32(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float load_f32(f16 v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T round_to(float v);
template <>
__device__ __forceinline__ float round_to<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 round_to<bf16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ f16 round_to<f16>(float v) { return __float2half_rn(v); }

// Two values of a 16-bit type in one 32-bit word, low half first.
__device__ __forceinline__ float2 unpack2(uint32_t w, bf16) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t w, f16) {
    const __half2 h = *reinterpret_cast<const __half2*>(&w);
    return __half22float2(h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, bf16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, f16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// The product of two pairs of bf16.
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b) {
    const float2 x = unpack2(a, bf16()), y = unpack2(b, bf16());
    return x.x * y.x + x.y * y.y;
}

// Streaming access to global memory: the operators read and write each element
// once, so nothing is gained by keeping it in L1.  A thread moves 8 elements:
// 32 bytes in one instruction (sm_100 and later) or 16.
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]),
                    "f"(v[6]), "f"(v[7]) : "memory");
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1], T());
    asm volatile("st.global.v4.u32 [%0], {%1,%2,%3,%4};"
                 :: "l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}

// 8 elements as they are in memory, to be unpacked when they are needed.
template <typename T>
struct Raw8 {
    uint32_t w[2 * sizeof(T)];
};
__device__ __forceinline__ Raw8<float> load_raw(const float* p) {
    Raw8<float> r;
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]),
                   "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
                 : "l"(p) : "memory");
    return r;
}
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw(const T* p) {
    Raw8<T> r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(p) : "memory");
    return r;
}
__device__ __forceinline__ void unpack(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
}
template <typename T>
__device__ __forceinline__ void unpack(const Raw8<T>& r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2(r.w[i], T());
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void set_raw(Raw8<float>& r, int i, float v) {
    r.w[i] = __float_as_uint(v);
}
template <typename T>
__device__ __forceinline__ void set_raw(Raw8<T>& r, int i, T v) {
    reinterpret_cast<T*>(r.w)[i] = v;
}

// 16 bytes, issued here: the compiler does not move the load to its use.
__device__ __forceinline__ uint4 load16(const void* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// Elements at .. at + 8 of a row of n, at < 0 and at + 8 > n allowed.  Where
// `whole` says that memory on both sides of the row may be read (it is another
// row's, or lies between rows), the vector is read as it is, and the caller
// leaves out what is not the row's; else its elements one by one, zeros outside.
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw_part(const T* row, int at, int n, bool whole) {
    if (whole || (at >= 0 && at + 8 <= n)) return load_raw(row + at);
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        set_raw(r, i, (unsigned)(at + i) < (unsigned)n ? row[at + i] : round_to<T>(0.f));
    return r;
}
template <typename T>
__device__ __forceinline__ void store_part(T* row, int at, int n, const float (&v)[8]) {
    if (at >= 0 && at + 8 <= n) {
        store8(row + at, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((unsigned)(at + i) < (unsigned)n) row[at + i] = round_to<T>(v[i]);
    }
}
template <typename T>
__device__ __forceinline__ void store_part(T* row, int at, int n, const float (&v)[1]) {
    row[at] = round_to<T>(v[0]);
}

// ---- host side -----------------------------------------------------------

inline size_t dtype_size(int t) { return t == PSS_F32 ? 4 : 2; }
inline bool dtype_ok(int t) { return t == PSS_F32 || t == PSS_BF16 || t == PSS_F16; }

// Whether p is memory that the kernels of the current device may use.  Asked of
// the driver: a call checks up to ten pointers, and the runtime's
// cudaPointerGetAttributes collects all attributes of each.
bool device_ptr(const void* p);

// Whether rows of `size`-byte elements may be moved 8 elements at a time.
inline bool aligned8(const void* p, int64_t stride, size_t size) {
    return ((uintptr_t)p % (8 * size)) == 0 && stride % 8 == 0;
}
// How many elements p stands past a multiple of 8 elements.
inline int past8(const void* p, size_t size) { return (int)((uintptr_t)p / size % 8); }
inline bool aligned_to(const void* p, size_t n) { return ((uintptr_t)p % n) == 0; }

// Hands out the parts of a workspace, each a multiple of 256 bytes behind the first.  A workspace
// need only be 16-byte aligned, but fp32 values are moved 32 bytes at a time, so the first
// part lies at the workspace's first multiple of 32, for which bytes() has room.
struct Take {
    char* base;
    int64_t at = 0;
    explicit Take(void* workspace)
        : base(reinterpret_cast<char*>(((uintptr_t)workspace + 31) / 32 * 32)) {}
    void* operator()(int64_t bytes) {
        char* p = base + at;
        at += (bytes + 255) / 256 * 256;
        return p;
    }
    int64_t bytes() const { return at > 0 ? at + 16 : 0; }
};

inline int sm_count() {
    static int cached[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64 && cached[dev]) return cached[dev];
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64) cached[dev] = n;
    return n;
}

inline pss_status status_of(cudaError_t e) {
    if (e == cudaSuccess) return PSS_OK;
    cudaGetLastError();
    return e == cudaErrorMemoryAllocation ? PSS_ERR_OOM : PSS_ERR_CUDA;
}

// A compile-time integer to pass to a generic lambda.
template <int N>
struct Int {
    static constexpr int value = N;
};

// f(T()) for the element type t.
template <typename F>
cudaError_t with_type(int t, F f) {
    switch (t) {
        case PSS_F32: return f(float());
        case PSS_BF16: return f(bf16());
        default: return f(f16());
    }
}

}  // namespace seq
}  // namespace pss
