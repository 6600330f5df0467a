// Blackwell building blocks of the attention kernels (sm_103a): mbarriers with
// bounded waits, TMA tile loads, tensor memory and the 5th-generation tensor
// core's instructions.
#pragma once

#include <cuda.h>

#include "seq_common.cuh"

namespace pss {
namespace seq {

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
    return (uint32_t)__cvta_generic_to_shared(p);
}

// ---- mbarriers -------------------------------------------------------------

__device__ __forceinline__ void bar_init(uint64_t* b, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_addr(b)), "r"(count)
                 : "memory");
}
__device__ __forceinline__ void bar_init_done() {
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(smem_addr(b)) : "memory");
}
// Arrive and announce `bytes` that TMA loads will deliver.
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;"
                 :: "r"(smem_addr(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n"
                 " mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
                 " selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(smem_addr(b)), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}

// Every wait ends: after kWaitNs, or as soon as another wait of the CTA has
// given up (*stop, in shared memory).  The caller then leaves its loop, the CTA
// lets its loads and products end, computes its rows another way, frees
// its tensor memory and reports through the call's status word.
constexpr uint64_t kWaitNs = 2000000000ull;
__device__ __forceinline__ bool bar_wait_slow(uint64_t* b, uint32_t parity,
                                                  volatile int* stop) {
    const uint64_t start = now_ns();
    while (!bar_try(b, parity)) {
        if (*stop) return false;
        if (now_ns() - start > kWaitNs) {
            *stop = 1;
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile int* stop) {
    if (bar_try(b, parity)) return true;
    return bar_wait_slow(b, parity, stop);
}

// Leaves the waits' verdict in the call's status word.
__device__ __forceinline__ void report_stop(unsigned long long* status) {
    if (status) atomicExch(status, ~1ull);   // -2
}

// Products are issued one by one as the tensor core takes them; it holds only one
// or two, and a thread's barrier operations queue behind its own products.  So a
// thread that looks for its next operands after its last product leaves the pipe
// empty for some 400 cycles.  Two threads therefore take turns: each waits for
// its operands while the other's products run, and hands over the turn kAhead
// products before its own end.  (Without turns their products alternate one by
// one, which costs the tensor core more than the waits did.)
constexpr int kAhead = 3;

// ---- TMA ---------------------------------------------------------------------

// Loads box (c0 .., c1 .., c2 ..) of a 3-D tensor map into shared memory.
__device__ __forceinline__ void tma_load3(void* dst, const CUtensorMap* map, int c0, int c1,
                                          int c2, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];"
        :: "r"(smem_addr(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(smem_addr(bar))
        : "memory");
}
// Fetches a tensor map ahead of its first use.
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" :: "l"(map) : "memory");
}
// Generic-proxy writes to shared memory become visible to TMA and the tensor core.
__device__ __forceinline__ void fence_async() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// ---- tensor memory and tcgen05 -------------------------------------------------

// One warp: allocate `cols` (a power of two, 32 .. 512) columns; the address
// appears at *at (shared memory).
__device__ __forceinline__ void tmem_alloc(uint32_t* at, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 :: "r"(smem_addr(at)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(addr), "r"(cols)
                 : "memory");
}
__device__ __forceinline__ void tc_before_sync() {
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_after_sync() {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
// The barrier receives one arrival when every tcgen05.mma issued so far by this
// thread has completed.
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];"
                 :: "r"(smem_addr(bar)) : "memory");
}

// Shared-memory operand: tiles of 128-byte rows in the 128-byte swizzle, as TMA
// writes them (8 rows = 1024 bytes repeat).
//   K-major (the contraction runs along the row): 8-row groups are 1024 bytes
//   apart; `lead` is unused.
//   MN-major (the contraction runs across the rows): the next 64 values of the
//   other dimension are `lead` bytes away, the next 8 rows 1024 bytes.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(lead >> 4) << 16) |
           ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: bf16 x bf16 -> fp32, M x N; b_mn: B is MN-major.
constexpr uint32_t mma_desc(int m, int n, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n / 8) << 17) |
           ((uint32_t)(m / 16) << 24);
}
// D (tensor memory) = A B (+ D): A from shared memory, K = 16.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc,
                                       bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 :: "r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory");
}
// A from tensor memory (two bf16 to a 32-bit column, 8 columns for K = 16).
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc,
                                       bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 :: "r"(d), "r"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory");
}

// 32 columns of the warp's 32 lanes (a warp reaches lanes 32 * (warp % 4) ..):
// thread l holds row l.
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32]) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32"
        " {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
          "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
          "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
          "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_store32(uint32_t addr, const float (&v)[32]) {
    const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0],"
        " {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        :: "r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]),
           "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
           "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
           "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
           "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0],"
        " {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        :: "r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]),
           "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
           "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_wait_load() {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// No use of v may be moved above the wait that makes it valid.
__device__ __forceinline__ void tmem_loaded(float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("" : "+f"(v[i]));
}
__device__ __forceinline__ void tmem_wait_store() {
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// Scores outside columns lo .. hi of a thread's 32 become -infinity.  Where the
// warp hides nothing it costs a vote.
__device__ __forceinline__ void hide(float (&s)[32], int lo, int hi) {
    if (!__any_sync(0xffffffffu, lo > 0 || hi < 32)) return;
    uint32_t see = hi >= 32 ? 0xffffffffu : hi <= 0 ? 0u : (1u << hi) - 1u;
    see &= lo <= 0 ? 0xffffffffu : lo >= 32 ? 0u : ~((1u << lo) - 1u);
#pragma unroll
    for (int e = 0; e < 32; ++e)
        if (!(see & (1u << e))) s[e] = -INFINITY;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    return fmaxf(fmaxf(a, b), c);
}

// All warps of a warpgroup: this many registers a thread from here on.  The
// block's warpgroups must stay within what it was launched with.
template <int N, bool MORE>
__device__ __forceinline__ void set_registers() {
    if (MORE)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(N));
    else
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(N));
}

// A barrier of `threads` threads of the CTA, number `id` (1 and up).
__device__ __forceinline__ void part_sync(int id, int threads) {
    asm volatile("bar.sync %0, %1;" :: "r"(id), "r"(threads) : "memory");
}

// The same, and whether any of the threads says yes.
__device__ __forceinline__ bool part_any(int id, int threads, bool yes) {
    uint32_t any;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %3, 0;\n"
                 " barrier.cta.red.or.pred p, %1, %2, q;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(any) : "r"(id), "r"(threads), "r"((uint32_t)yes) : "memory");
    return any != 0;
}

// 2^x, the hardware's approximation (relative error below 2^-22).
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<uint64_t&>(d))
        : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)),
          "l"(reinterpret_cast<uint64_t&>(c)));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<uint64_t&>(d))
        : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<uint64_t&>(d))
        : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
    return d;
}

// Result rows leave through shared memory, in the layout that the loads have: a
// thread holds a row (or half of one), and 32 rows' 16-byte pieces written at
// once would touch 32 lines.
// stage_row: N columns from tensor memory, times `scale`, as bf16 into row r of
// a tile, from its 16-byte piece `piece` on; zeros where there are no columns to
// read (`load`, the same for the warp).  Returns whether all are finite.
template <int N>
__device__ __forceinline__ bool stage_row(uint32_t at, uint8_t* tile, int r, int piece, float scale,
                                          bool load) {
    uint32_t most = 0;   // the largest exponent field of each half
    const float2 scale2 = make_float2(scale, scale);
#pragma unroll 1
    for (int i = 0; i < N; i += 32) {
        float v[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = 0.f;
        if (load) {
            tmem_load32(at + i, v);
            tmem_wait_load();
            tmem_loaded(v);
        }
        uint32_t w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float2 x = mul2(make_float2(v[2 * e], v[2 * e + 1]), scale2);
            w[e] = pack2(x.x, x.y, bf16());
            most = __vmaxu2(most, w[e] & 0x7f807f80u);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = piece + i / 8 + e;
            *reinterpret_cast<uint4*>(tile + (c / 8) * 16384 + r * 128 +
                                      (((c & 7) ^ (r & 7)) * 16)) =
                make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
        }
    }
    return (most & 0xffffu) < 0x7f80u && (most >> 16) < 0x7f80u;
}
// A staged tile to memory in one go, by one thread (after a fence_async of every
// thread that staged and a barrier): what lies outside the tensor is left out.
template <int HD>
__device__ __forceinline__ void store_tile(const CUtensorMap* map, const uint8_t* tile, int head,
                                           int token) {
#pragma unroll
    for (int h = 0; h < HD / 64; ++h)
        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group"
                     " [%0, {%1, %2, %3}], [%4];"
                     :: "l"(map), "r"(64 * h), "r"(head), "r"(token),
                        "r"(smem_addr(tile + h * 16384)) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}
// Or row by row: N rows from `first` on, HD / 8 lanes of a warp to a row; to(r):
// where row r goes, or null.
template <int HD, int N, typename F>
__device__ __forceinline__ void store_rows(const uint8_t* tile, int first, int dim, F to) {
    constexpr int kLanes = HD / 8, kRows = 32 / kLanes;
    const int lane = threadIdx.x & 31, c = lane % kLanes;
    for (int i = lane / kLanes; i < N; i += kRows) {
        const int r = first + i;
        bf16* p = to(r);
        if (p && c * 8 < dim)
            *reinterpret_cast<uint4*>(p + c * 8) = *reinterpret_cast<const uint4*>(
                tile + (c / 8) * 16384 + r * 128 + (((c & 7) ^ (r & 7)) * 16));
    }
}

}  // namespace seq
}  // namespace pss
