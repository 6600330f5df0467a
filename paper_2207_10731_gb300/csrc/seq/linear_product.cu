// Matrix products with an epilogue, on the tensor cores (linear.h).
//
// D = A B^T in tiles of 128 x BN: A and B arrive in blocks of 64 along the contraction by TMA,
// through a ring of shared-memory stages, as they lie in memory (rows dense along the
// contraction or across it: the product's descriptors say which), and D stays in tensor
// memory.  One CTA an SM takes tiles in turn.  Roles: one warp loads, one thread issues the
// products, eight warps finish a tile (bias, activation, residual, rounding) from one of
// two accumulators while the products run into the other.
//
// Few tokens (a serving step) are the columns of the product, and the weight's outputs its
// rows, so that a tile is 128 outputs wide and no more tokens than needed high; the
// contraction is split over CTAs until they fill the GPU, as it is for the weight's
// gradient, whose result is small and whose contraction runs over all tokens.  The parts
// are added in a fixed order by a second kernel: equal inputs give equal bits.
#include <atomic>

#include "activation.cuh"
#include "attention_tma.h"
#include "tc.cuh"
#include <cudaTypedefs.h>
#include <type_traits>

namespace pss {
namespace seq {
namespace {

constexpr int kBlock = 64;                   // of the contraction: 128 bytes
constexpr int kFinishers = 8;                // warps
constexpr int kProductThreads = 128 + 32 * kFinishers;
constexpr int kPad = 33;                     // a staged row of 32 values

// PAIR: two CTAs of a cluster, on neighbouring SMs, make a tile of 256 x BN: each loads its 128
// rows of A and half of B's, one thread of the first issues products that read both, and
// each CTA's tensor memory holds its rows of the result.  B so passes through each SM's shared
// memory half as often.
template <int BN, bool PAIR>
struct Ring {
    static constexpr int kA = 128 * kBlock * 2, kRows = PAIR ? BN / 2 : BN, kB = kRows * kBlock * 2;
    static constexpr int kStage = kA + kB;
    static constexpr int kStages = PAIR || BN == 128 ? 6 : BN == 256 ? 4 : 8;
    static constexpr int kStaging = kFinishers * 32 * kPad * 4;
    static constexpr int kSmem = kStages * kStage + kStaging;
    static constexpr int kCols = 2 * BN;     // tensor-memory columns: two accumulators
};

__device__ __forceinline__ void tma_load2(void* dst, const CUtensorMap* map, int c0, int c1,
                                          uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3}], [%4];"
        :: "r"(smem_addr(dst)), "l"(map), "r"(c0), "r"(c1), "r"(smem_addr(bar)) : "memory");
}

// ---- pairs of CTAs -------------------------------------------------------------

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address, in the cluster's shared memory, of p in its first CTA.
__device__ __forceinline__ uint32_t first_cta(const void* p) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_addr(p)));
    return r;
}
// A load into this CTA that reports to a barrier of the first one.
__device__ __forceinline__ void tma_load2_pair(void* dst, const CUtensorMap* map, int c0, int c1,
                                               uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3}], [%4];"
        :: "r"(smem_addr(dst)), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t* at, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                 :: "r"(smem_addr(at)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free_pair(uint32_t addr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(addr), "r"(cols)
                 : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t desc,
                                         bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                 :: "r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory");
}
// The barrier of both CTAs receives one arrival when this thread's products have completed.
__device__ __forceinline__ void tc_commit_pair(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster"
                 ".multicast::cluster.b64 [%0], %1;"
                 :: "r"(smem_addr(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void bar_arrive_first(uint64_t* bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(first_cta(bar))
                 : "memory");
}
// As bar_wait, for what a thread of the other CTA did before it arrived.
__device__ __forceinline__ bool bar_wait_cluster(uint64_t* b, uint32_t parity, volatile int* stop) {
    const uint64_t start = now_ns();
    for (;;) {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n"
                     " mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
                     " selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok) : "r"(smem_addr(b)), "r"(parity) : "memory");
        if (ok) return true;
        if (*stop) return false;
        if (now_ns() - start > kWaitNs) {
            *stop = 1;
            return false;
        }
    }
}

// 128 (or, of a pair, 256) x N, fp32 sums of f16 or bf16; which operands lie across the
// contraction.
__device__ __forceinline__ uint32_t product_desc(int m, int n, bool half, bool a_across,
                                                 bool b_across) {
    const uint32_t format = half ? 0u : 1u;
    return (1u << 4) | (format << 7) | (format << 10) | ((a_across ? 1u : 0u) << 15) |
           ((b_across ? 1u : 0u) << 16) | ((uint32_t)(n / 8) << 17) | ((uint32_t)(m / 16) << 24);
}

struct Args {
    Finish f;
    float* partial;
    int64_t ld;
    int m, n, blocks, m_tiles, n_tiles, splits, units;
    bool a_across, b_across;
    unsigned long long* status;
};

// A unit of work: a tile and a part of its contraction.  Tiles run down bands of 16 rows of
// tiles, so that those under way at a time read few different rows and columns.
struct Unit {
    int m, n, k0, k1, split;
};
__device__ __forceinline__ Unit unit_of(const Args& a, int u) {
    constexpr int kBand = 16;
    Unit w;
    w.split = u % a.splits;
    const int t = u / a.splits, per = kBand * a.n_tiles, band = t / per, in = t - band * per;
    const int high = min(kBand, a.m_tiles - band * kBand);
    w.n = in / high;
    w.m = band * kBand + in - w.n * high;
    w.k0 = (int)((int64_t)a.blocks * w.split / a.splits);
    w.k1 = (int)((int64_t)a.blocks * (w.split + 1) / a.splits);
    return w;
}

// 16 values of 16 bits, or 8 of 32: 32 bytes in one instruction.
__device__ __forceinline__ void load32b(const void* p, uint32_t (&r)[8]) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
                   "=r"(r[6]), "=r"(r[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store32b(void* p, const uint32_t (&r)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]),
                    "r"(r[6]), "r"(r[7]) : "memory");
}
// 32 values of T or fp32 at p.
template <typename T>
__device__ __forceinline__ void put32(T* p, const float (&v)[32]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack2(v[16 * h + 2 * i], v[16 * h + 2 * i + 1], T());
        store32b(p + 16 * h, w);
    }
}
__device__ __forceinline__ void put32(float* p, const float (&v)[32]) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[8 * h + i]);
        store32b(p + 8 * h, w);
    }
}
template <typename T>
__device__ __forceinline__ void add32(const T* p, float (&v)[32]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t w[8];
        load32b(p + 16 * h, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 x = unpack2(w[i], T());
            v[16 * h + 2 * i] += x.x;
            v[16 * h + 2 * i + 1] += x.y;
        }
    }
}
__device__ __forceinline__ void add32(const float* p, float (&v)[32]) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        uint32_t w[8];
        load32b(p + 8 * h, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[8 * h + i] += __uint_as_float(w[i]);
    }
}

template <typename T>
__device__ __forceinline__ float residual_at(const Finish& f, int64_t t, int64_t c) {
    const int64_t at = t * f.residual_stride + c;
    return f.y_f32 ? static_cast<const float*>(f.residual)[at]
                   : load_f32(static_cast<const T*>(f.residual)[at]);
}

// One value of the result; `more`: its residual.
template <typename T>
__device__ __forceinline__ void finish_one(const Finish& f, float v, int64_t t, int64_t c,
                                           float bias, float more) {
    v += bias;
    if (f.z) static_cast<T*>(f.z)[t * f.z_stride + c] = round_to<T>(v);
    with_activation(f.activation, [&](auto act) { v = activate<decltype(act)::value>(v); });
    const int64_t at = t * f.y_stride + c;
    if (f.residual) v += more;
    if (f.y_f32)
        static_cast<float*>(f.y)[at] = v;
    else
        static_cast<T*>(f.y)[at] = round_to<T>(v);
}

// 32 values of row t from column c on, all inside.
template <typename T>
__device__ __forceinline__ void finish_32(const Finish& f, float (&v)[32], int64_t t, int64_t c) {
    if (f.bias) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] += __ldg(f.bias + c + i);
    }
    if (f.z) put32(static_cast<T*>(f.z) + t * f.z_stride + c, v);
    with_activation(f.activation, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = activate<decltype(act)::value>(v[i]);
    });
    const int64_t at = t * f.y_stride + c, from = t * f.residual_stride + c;
    if (f.y_f32) {
        if (f.residual) add32(static_cast<const float*>(f.residual) + from, v);
        put32(static_cast<float*>(f.y) + at, v);
    } else {
        if (f.residual) add32(static_cast<const T*>(f.residual) + from, v);
        put32(static_cast<T*>(f.y) + at, v);
    }
}

template <int BN, bool PAIR, typename T>
__global__ void __launch_bounds__(kProductThreads, 1)
k_linear_product(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb,
                 const __grid_constant__ Args a) {
    pdl_prologue();
    using R = Ring<BN, PAIR>;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ uint64_t full[R::kStages], empty[R::kStages], done[2], free_[2], drained;
    __shared__ uint32_t tmem_at;
    __shared__ volatile int stop;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kCtas = PAIR ? 2 : 1;
    const int rank = PAIR ? (int)cluster_rank() : 0;
    const int first_unit = blockIdx.x / kCtas, step = gridDim.x / kCtas;
    if (threadIdx.x == 0) {
        prefetch_map(&ma);
        prefetch_map(&mb);
        stop = 0;
        for (int i = 0; i < R::kStages; ++i) {
            bar_init(&full[i], 1);
            bar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(&done[i], 1);
            bar_init(&free_[i], kCtas * kFinishers);
        }
        bar_init(&drained, 1);
        bar_init_done();
    }
    if (warp == 1) {
        if (PAIR)
            tmem_alloc_pair(&tmem_at, R::kCols);
        else
            tmem_alloc(&tmem_at, R::kCols);
    }
    tc_before_sync();
    __syncthreads();
    if (PAIR) cluster_sync();
    tc_after_sync();
    const uint32_t tmem = tmem_at;

    if (warp == 0) {
        // ---- loads ----
        if (lane == 0) {
            int s = 0;
            bool ok = true;
            for (int u = first_unit; ok && u < a.units; u += step) {
                const Unit w = unit_of(a, u);
                const int row = (w.m * kCtas + rank) * 128, col = w.n * BN + rank * R::kRows;
                for (int k = w.k0; k < w.k1; ++k, ++s) {
                    const int slot = s % R::kStages, turn = s / R::kStages;
                    if (turn > 0 && !bar_wait(&empty[slot], (turn - 1) & 1, &stop)) {
                        ok = false;
                        break;
                    }
                    uint8_t* at = smem + slot * R::kStage;
                    if (rank == 0) bar_expect(&full[slot], kCtas * R::kStage);
                    const uint32_t bar = PAIR ? first_cta(&full[slot]) : 0;
                    auto load = [&](uint8_t* to, const CUtensorMap* map, int c0, int c1) {
                        if (PAIR)
                            tma_load2_pair(to, map, c0, c1, bar);
                        else
                            tma_load2(to, map, c0, c1, &full[slot]);
                    };
                    if (a.a_across) {
                        for (int i = 0; i < 2; ++i)
                            load(at + i * 8192, &ma, row + i * 64, k * kBlock);
                    } else {
                        load(at, &ma, k * kBlock, row);
                    }
                    at += R::kA;
                    if (a.b_across) {
                        for (int i = 0; i < R::kRows / 64; ++i)
                            load(at + i * 8192, &mb, col + i * 64, k * kBlock);
                    } else {
                        load(at, &mb, k * kBlock, col);
                    }
                }
            }
            // The loads must land before the CTA ends, also where nobody waits for them.  A pair's
            // second CTA cannot see them land: the first one's wait ends after them, and both
            // CTAs end together.
            int never = 0;
            if (rank == 0)
                for (int w = max(0, s - R::kStages); w < s; ++w)
                    bar_wait(&full[w % R::kStages], (w / R::kStages) & 1, &never);
            else if (!ok)
                for (const uint64_t t = now_ns(); now_ns() - t < 10000000ull;) __nanosleep(1000);
        }
    } else if (warp == 1) {
        // ---- products ----
        if (lane == 0 && rank == 0) {
            const uint32_t desc =
                product_desc(128 * kCtas, BN, std::is_same<T, f16>::value, a.a_across, a.b_across);
            const uint32_t base = smem_addr(smem);
            const uint32_t a_lead = a.a_across ? 8192 : 16, b_lead = a.b_across ? 8192 : 16;
            const uint32_t a_step = a.a_across ? 2048 : 32, b_step = a.b_across ? 2048 : 32;
            auto commit = [&](uint64_t* bar) {
                if (PAIR)
                    tc_commit_pair(bar);
                else
                    tc_commit(bar);
            };
            int s = 0, i = 0;
            bool ok = true;
            for (int u = first_unit; ok && u < a.units; u += step, ++i) {
                const Unit w = unit_of(a, u);
                const uint32_t d = tmem + (i & 1) * BN;
                if (i > 1)
                    ok = PAIR ? bar_wait_cluster(&free_[i & 1], ((i >> 1) - 1) & 1, &stop)
                              : bar_wait(&free_[i & 1], ((i >> 1) - 1) & 1, &stop);
                for (int k = w.k0; ok && k < w.k1; ++k, ++s) {
                    const int slot = s % R::kStages;
                    ok = bar_wait(&full[slot], (s / R::kStages) & 1, &stop);
                    if (!ok) break;
                    tc_after_sync();
                    const uint32_t a_at = base + slot * R::kStage, b_at = a_at + R::kA;
#pragma unroll
                    for (int j = 0; j < kBlock / 16; ++j) {
                        const uint64_t x = smem_desc(a_at + j * a_step, a_lead);
                        const uint64_t y = smem_desc(b_at + j * b_step, b_lead);
                        if (PAIR)
                            mma_pair(d, x, y, desc, k > w.k0 || j > 0);
                        else
                            mma_ss(d, x, y, desc, k > w.k0 || j > 0);
                    }
                    commit(&empty[slot]);
                }
                if (ok) commit(&done[i & 1]);
            }
            // the products must end before their memory is freed, also after a wait gave up
            int never = 0;
            commit(&drained);
            bar_wait(&drained, 0, &never);
        }
    } else if (warp >= 4) {
        // ---- finishing: a thread to a row of the tile, every second 32 columns ----
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        float* staged = reinterpret_cast<float*>(smem + R::kStages * R::kStage) +
                        (warp - 4) * 32 * kPad;
        int i = 0;
        for (int u = first_unit; u < a.units; u += step, ++i) {
            const Unit w = unit_of(a, u);
            if (!__all_sync(0xffffffffu, bar_wait(&done[i & 1], (i >> 1) & 1, &stop))) break;
            tc_after_sync();
            const uint32_t d = tmem + (i & 1) * BN + ((uint32_t)quarter << 21);
            const int row0 = (w.m * kCtas + rank) * 128 + quarter * 32, row = row0 + lane;
            const Finish& f = a.f;
            float* partial = a.partial ? a.partial + (int64_t)w.split * (f.swapped ? a.n : a.m) * a.ld
                                       : nullptr;
            for (int c = half; c < BN / 32; c += 2) {
                const int col = w.n * BN + c * 32;
                if (col >= a.n) break;
                float v[32];
                tmem_load32(d + c * 32, v);
                tmem_wait_load();
                tmem_loaded(v);
                if (f.swapped) {
                    // lanes are neighbours in memory already
                    if (row < a.m) {
                        const float bias = !partial && f.bias ? f.bias[row] : 0.f;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            if (col + j >= a.n) break;
                            if (partial)
                                partial[(int64_t)(col + j) * a.ld + row] = v[j];
                            else
                                finish_one<T>(f, v[j], col + j, row, bias,
                                              f.residual ? residual_at<T>(f, col + j, row) : 0.f);
                        }
                    }
                } else if (partial) {
                    if (row < a.m) {
#pragma unroll
                        for (int j = 0; j < 32; j += 8) {
                            float x[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) x[e] = v[j + e];
                            if (col + j < a.n) store8(partial + (int64_t)row * a.ld + col + j, x);
                        }
                    }
                } else if (f.vectors && col + 32 <= a.n) {
                    if (row < a.m) finish_32<T>(f, v, row, col);
                } else {
                    // through shared memory: a row at a time, a lane to a column
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 32; ++j) staged[lane * kPad + j] = v[j];
                    __syncwarp();
                    if (col + lane < a.n) {
                        const float bias = f.bias ? f.bias[col + lane] : 0.f;
                        const int last = min(32, a.m - row0);
                        // eight rows' residuals are asked for before the first is waited for
                        for (int j = 0; j < last; j += 8) {
                            float more[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                more[e] = f.residual && j + e < last
                                              ? residual_at<T>(f, row0 + j + e, col + lane) : 0.f;
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (j + e < last)
                                    finish_one<T>(f, staged[(j + e) * kPad + lane], row0 + j + e,
                                                  col + lane, bias, more[e]);
                        }
                    }
                }
            }
            tc_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (PAIR)
                    bar_arrive_first(&free_[i & 1]);
                else
                    bar_arrive(&free_[i & 1]);
            }
        }
    }
    tc_before_sync();
    __syncthreads();
    if (PAIR) cluster_sync();   // neither CTA ends while the other may reach into it
    tc_after_sync();
    if (warp == 1) {
        if (PAIR)
            tmem_free_pair(tmem, R::kCols);
        else
            tmem_free(tmem, R::kCols);
    }
    if (threadIdx.x == 0 && stop) report_stop(a.status);
}

// Adds the parts of a split product in their order, and finishes: a thread to 8 values.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_linear_join(const float* __restrict__ partial, int splits, int64_t rows, int cols, int64_t ld,
              const __grid_constant__ Finish f) {
    pdl_prologue();
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, vecs = ld / 8;
    const int64_t t = i / vecs;
    const int c = (int)(i - t * vecs) * 8;
    if (t >= rows) return;
    float sum[8] = {};
    constexpr int U = 4;
    for (int s0 = 0; s0 < splits; s0 += U) {
        Raw8<float> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            raw[u] = s0 + u < splits ? load_raw(partial + ((s0 + u) * rows + t) * ld + c)
                                     : Raw8<float>{};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[8];
            unpack(raw[u], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + e < cols)
            finish_one<T>(f, sum[e], t, c + e, f.bias ? f.bias[c + e] : 0.f,
                          f.residual ? residual_at<T>(f, t, c + e) : 0.f);
}

// Boxes of 64 along the dense dimension and `box` (at most 256) along the other.
cudaError_t operand_map(CUtensorMap* map, const Operand& o, int box, int type) {
    static std::atomic<void*> found{nullptr};
    void* fn = driver_call("cuTensorMapEncodeTiled", &found);
    if (!fn) return cudaErrorNotSupported;
    const cudaError_t bound = bind_context();
    if (bound != cudaSuccess) return bound;
    const Matrix& x = o.matrix;
    // the stride over a single row is free, but the encoder checks it
    const int64_t stride = x.outer > 1 ? x.stride : (x.inner + 7) / 8 * 8;
    const cuuint64_t dims[2] = {(cuuint64_t)x.inner, (cuuint64_t)x.outer};
    const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t sizes[2] = {64, (cuuint32_t)(o.across ? kBlock : box)};
    const cuuint32_t one[2] = {1, 1};
    const CUresult rc = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn)(
        map, type == PSS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
        const_cast<void*>(x.data), dims, strides, sizes, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int BN, bool PAIR, typename T>
cudaError_t launch(const Product& p, int type, unsigned long long* status, cudaStream_t st) {
    using R = Ring<BN, PAIR>;
    CUtensorMap ma, mb;
    cudaError_t e = operand_map(&ma, p.a, 128, type);
    if (e == cudaSuccess) e = operand_map(&mb, p.b, R::kRows, type);
    if (e != cudaSuccess) return e;
    auto* k = k_linear_product<BN, PAIR, T>;
    static std::atomic<uint64_t> ready{0};
    e = allow_smem(k, R::kSmem, &ready);
    if (e != cudaSuccess) return e;
    const int units = p.m_tiles * p.n_tiles * p.splits, fit = sm_count() / (PAIR ? 2 : 1);
    const Args a{p.f, p.splits > 1 ? p.partial : nullptr, p.ld, p.m, p.n, p.blocks, p.m_tiles,
                 p.n_tiles, p.splits, units, p.a.across, p.b.across, status};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((units < fit ? units : fit) * (PAIR ? 2 : 1)));
    cfg.blockDim = dim3(kProductThreads);
    cfg.dynamicSmemBytes = R::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = PAIR ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, k, ma, mb, a);
    if (e != cudaSuccess || p.splits == 1) return e;
    const int64_t rows = p.f.swapped ? p.n : p.m, threads = rows * (p.ld / 8);
    return launch_k(k_linear_join<T>, dim3((unsigned)((threads + kThreads - 1) / kThreads)),
                    dim3(kThreads), 0, st, static_cast<const float*>(p.partial), p.splits, rows,
                    p.f.swapped ? p.m : p.n, p.ld, p.f);
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_linear_copy(const T* __restrict__ from, int64_t stride, int64_t rows, int64_t cols, T* to,
              int64_t ld) {
    pdl_prologue();
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, vecs = ld / 8;
    const int64_t r = i / vecs, c = (i - r * vecs) * 8;
    if (r >= rows) return;
    Raw8<T> v;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        set_raw(v, e, c + e < cols ? from[r * stride + c + e] : round_to<T>(0.f));
    *reinterpret_cast<uint4*>(to + r * ld + c) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
}

}  // namespace

bool on_grid(const Matrix& x) {
    return aligned_to(x.data, 16) && (x.outer <= 1 || x.stride % 8 == 0);
}

int64_t copy_bytes(const Matrix& x) { return x.outer * ((x.inner + 7) / 8 * 8) * 2; }

cudaError_t copy_matrix(Matrix* x, void* to, cudaStream_t st) {
    const int64_t ld = (x->inner + 7) / 8 * 8, threads = x->outer * (ld / 8);
    // the values are moved as they are, whichever 16-bit type they have
    const cudaError_t e = launch_k(
        k_linear_copy<f16>, dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), 0,
        st, static_cast<const f16*>(x->data), x->stride, x->outer, x->inner, static_cast<f16*>(to), ld);
    x->data = to;
    x->stride = ld;
    return e;
}

// The width of the tiles and the parts of the contraction: the pair that leaves the fullest SM
// the least time, by what was measured of a block (64 along the contraction) of each width, of a
// unit's start and end, and of the parts' way through memory; in SM cycles.
void plan_product(Product* p) {
    p->m = (int)p->a.rows();
    p->n = (int)p->b.rows();
    p->blocks = (int)((p->a.k() + kBlock - 1) / kBlock);
    p->ld = ((p->f.swapped ? p->m : p->n) + 7) / 8 * 8;
    const int sms = sm_count() > 1 ? sm_count() : 2;
    struct Kind {
        int bn, cycles;
        bool pair;
    };
    const Kind kinds[] = {{256, 530, true}, {256, 560, false}, {128, 330, false}, {64, 250, false},
                          {32, 220, false}};
    double best = 0;
    p->bn = 0;
    for (const Kind& kind : kinds) {
        const int bn = kind.bn, rows = kind.pair ? 256 : 128, fit = kind.pair ? sms / 2 : sms;
        if (bn == 32 && (p->b.across || p->n > 32)) continue;   // a box across is 64 wide
        if (bn > 64 && p->n <= bn / 2) continue;
        if (kind.pair && p->m <= 128) continue;
        const int m_tiles = (p->m + rows - 1) / rows, n_tiles = (p->n + bn - 1) / bn;
        const int64_t tiles = (int64_t)m_tiles * n_tiles;
        for (int s = 1; s <= 64 && s <= p->blocks; ++s) {
            const int64_t rounds = (tiles * s + fit - 1) / fit;
            double cost = 2000. + (double)rounds * ((p->blocks + s - 1) / s * kind.cycles + 300.);
            // written and read at some 1800 bytes a cycle each, and a launch
            if (s > 1) cost += 4000. + (double)p->m * p->n * s * 8 / 1800;
            if (p->bn == 0 || cost < best) {
                best = cost;
                p->bn = bn;
                p->pair = kind.pair;
                p->m_tiles = m_tiles;
                p->n_tiles = n_tiles;
                p->splits = s;
            }
            if (tiles * s >= 16 * fit) break;
        }
    }
}

int64_t partial_values(const Product& p) {
    return p.splits > 1 ? p.splits * (int64_t)(p.f.swapped ? p.n : p.m) * p.ld : 0;
}

cudaError_t launch_product(const Product& p, int type, unsigned long long* status,
                           cudaStream_t st) {
    auto go = [&](auto t) {
        using T = decltype(t);
        switch (p.bn) {
            case 256:
                return p.pair ? launch<256, true, T>(p, type, status, st)
                              : launch<256, false, T>(p, type, status, st);
            case 128: return launch<128, false, T>(p, type, status, st);
            case 64: return launch<64, false, T>(p, type, status, st);
            default: return launch<32, false, T>(p, type, status, st);
        }
    };
    return type == PSS_BF16 ? go(bf16()) : go(f16());
}

}  // namespace seq
}  // namespace pss
