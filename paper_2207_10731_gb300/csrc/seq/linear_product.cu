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
constexpr int kStaged = 4096;                // a finishing warp's tile: 32 rows of 128 bytes

// PAIR: two CTAs of a cluster, on neighbouring SMs, make a tile of 256 x BN: each loads its 128
// rows of A and half of B's, one thread of the first issues products that read both, and
// each CTA's tensor memory holds its rows of the result.  B so passes through each SM's shared
// memory half as often.
template <int BN, bool PAIR>
struct Ring {
    static constexpr int kA = 128 * kBlock * 2, kRows = PAIR ? BN / 2 : BN, kB = kRows * kBlock * 2;
    static constexpr int kStage = kA + kB;
    // (pairs, 16384 x 4096 x 4096: 3 stages 399 us, 4 335, 5 311, 6 310)
    static constexpr int kStages = PAIR || BN == 128 ? 6 : 8;
    static constexpr int kSmem = kStages * kStage + kFinishers * kStaged;
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
__device__ __forceinline__ void tma_load3_pair(void* dst, const CUtensorMap* map, int c0, int c1,
                                               int c2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];"
        :: "r"(smem_addr(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
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
    int m, n, bn, blocks, m_tiles, n_tiles, splits, units;
    bool a_across, b_across;
    bool a_boxes, b_boxes;   // across: in pairs of boxes of 64 (operand_map)
    unsigned long long* status;
};

// A unit of work: a tile and a part of its contraction.  Tiles run down bands of 16 rows of
// tiles, so that those under way at a time read few different rows and columns.
struct Unit {
    int m, n, k0, k1, split;
};
// blocks < 2^25, splits <= 64
__device__ __forceinline__ int part_start(const Args& a, int split) {
    return a.splits == 1 ? split * a.blocks : (int)((unsigned)a.blocks * (unsigned)split / (unsigned)a.splits);
}
__device__ __forceinline__ Unit unit_of(const Args& a, int u) {
    constexpr int kBand = 16;
    Unit w;
    w.split = u % a.splits;
    const int t = u / a.splits, per = kBand * a.n_tiles, band = t / per, in = t - band * per;
    const int high = min(kBand, a.m_tiles - band * kBand);
    w.n = in / high;
    w.m = band * kBand + in - w.n * high;
    w.k0 = part_start(a, w.split);
    w.k1 = part_start(a, w.split + 1);
    return w;
}
// The blocks of unit u.
__device__ __forceinline__ int blocks_of(const Args& a, int u) {
    if (a.splits == 1) return a.blocks;
    const int split = u % a.splits;
    return part_start(a, split + 1) - part_start(a, split);
}

// ---- finishing through shared memory -------------------------------------------
// A warp's tile: 32 rows of 128 bytes, the 16-byte piece p of row r in the 128-byte swizzle, as
// TMA stores it.  (32-byte stores of a row a lane, 32 lines an instruction: 55 instead of 42 us for
// 16384 x 64 x 4096, where finishing is nearly all there is to do.)

__device__ __forceinline__ uint32_t piece_at(uint32_t tile, int row, int p) {
    return tile + row * 128 + ((p ^ (row & 7)) << 4);
}
__device__ __forceinline__ void put_piece(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}
__device__ __forceinline__ uint4 get_piece(uint32_t at) {
    uint4 w;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(at) : "memory");
    return w;
}
// The word w as it is, or its half h.
__device__ __forceinline__ void put_raw(float* to, uint32_t w, int) { *to = __uint_as_float(w); }
template <typename T>
__device__ __forceinline__ void put_raw(T* to, uint32_t w, int h) {
    *reinterpret_cast<uint16_t*>(to) = (uint16_t)(w >> (16 * h));
}
// 32 values of row `row`, from its piece p on.
template <typename T>
__device__ __forceinline__ void put32(uint32_t tile, int row, int p, const float (&v)[32], T) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        put_piece(piece_at(tile, row, p + i), pack2(v[8 * i], v[8 * i + 1], T()),
                  pack2(v[8 * i + 2], v[8 * i + 3], T()), pack2(v[8 * i + 4], v[8 * i + 5], T()),
                  pack2(v[8 * i + 6], v[8 * i + 7], T()));
}
__device__ __forceinline__ void put32(uint32_t tile, int row, int p, const float (&v)[32], float) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        put_piece(piece_at(tile, row, p + i), __float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                  __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
}
template <typename T>
__device__ __forceinline__ void add32(uint32_t tile, int row, int p, float (&v)[32], T) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint4 w = get_piece(piece_at(tile, row, p + i));
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 y = unpack2(x[e], T());
            v[8 * i + 2 * e] += y.x;
            v[8 * i + 2 * e + 1] += y.y;
        }
    }
}
__device__ __forceinline__ void add32(uint32_t tile, int row, int p, float (&v)[32], float) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint4 w = get_piece(piece_at(tile, row, p + i));
        v[4 * i] += __uint_as_float(w.x);
        v[4 * i + 1] += __uint_as_float(w.y);
        v[4 * i + 2] += __uint_as_float(w.z);
        v[4 * i + 3] += __uint_as_float(w.w);
    }
}
// Copies a tile's rows of the residual in, 8 lanes to a row; zeros outside the tensor.
template <typename TY>
__device__ __forceinline__ void fetch_tile(uint32_t tile, const TY* from, int64_t stride, int rows,
                                           int cols) {
    constexpr int kValues = 16 / sizeof(TY);
    const int lane = threadIdx.x & 31, p = lane & 7;
    const int left = min(16, max(0, (cols - p * kValues) * (int)sizeof(TY)));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 3), size = r < rows ? left : 0;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                     :: "r"(piece_at(tile, r, p)),
                        "l"(size > 0 ? from + r * stride + p * kValues : from), "r"(size) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap* map, uint32_t tile, int c0, int c1,
                                          int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
                 :: "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(tile) : "memory");
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

__device__ __forceinline__ void add_bias(const Finish& f, float (&v)[32], int c, int n) {
    if (f.bias_vectors && c + 32 <= n) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 b = __ldg(reinterpret_cast<const float4*>(f.bias + c) + i);
            v[4 * i] += b.x;
            v[4 * i + 1] += b.y;
            v[4 * i + 2] += b.z;
            v[4 * i + 3] += b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] += c + i < n ? __ldg(f.bias + c + i) : 0.f;
    }
}

// 32 values of row t from column c of n on, with their bias, as they lie.
template <typename T, typename TY>
__device__ __forceinline__ void finish_row(const Finish& f, float (&v)[32], int64_t t, int c, int n) {
    auto put = [&](auto* row) {
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = v[i + e];
            if (c + i < n) store_part(row, c + i, n, x);
        }
    };
    if (f.z) put(static_cast<T*>(f.z) + t * f.z_stride);
    with_activation(f.activation, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = activate<decltype(act)::value>(v[i]);
    });
    if (f.residual) {
        const TY* row = static_cast<const TY*>(f.residual) + t * f.residual_stride;
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (c + i < n) v[i] += load_f32(row[c + i]);
    }
    put(static_cast<TY*>(f.y) + t * f.y_stride);
}

// A finishing warp's part of a tile, rows row0 .. +32 and columns col .. of the accumulator at d:
// tiles of 128 bytes' width (64 columns of 16 bits, 32 of fp32) are made in shared memory,
// over the residual's where there is one, and stored by TMA, which leaves out what lies outside, but
// writes whole 16-byte pieces: its maps end with the last whole one (launch), and what a row has
// behind that, its lane stores value by value.
// z goes first, and y from the accumulator again.  wait(): until the accumulator is there;
// asked for after the first residual.
template <int BN, typename T, typename TY, typename W>
__device__ __forceinline__ bool finish_tiles(const Args& a, const CUtensorMap* my,
                                             const CUtensorMap* mz, uint32_t tile, uint32_t d,
                                             int row0, int col0, int half, int split, W wait) {
    const Finish& f = a.f;
    constexpr int kWide = 128 / sizeof(TY) < BN ? 128 / sizeof(TY) : BN;   // columns of a tile
    const int lane = threadIdx.x & 31;
    const bool partial = a.partial != nullptr;
    bool waited = false;
    // the tile's last store has read it (two tiles in turns: no faster)
    auto tile_free = [&] {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    };
    constexpr int kValues = 16 / sizeof(TY);
    const int whole = partial ? a.n : a.n / kValues * kValues;
    auto store = [&](const CUtensorMap* map, TY* to, int64_t stride, int col, int part) {
        fence_async();
        __syncwarp();
        if (lane == 0 && col < whole) {
            tma_store(map, tile, col, row0, part);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        if (whole < a.n && whole < col + kWide && row0 + lane < a.m) {
            const uint4 w = get_piece(piece_at(tile, lane, (whole - col) / kValues));
            const uint32_t x[4] = {w.x, w.y, w.z, w.w};
            TY* row = to + (row0 + lane) * stride + whole;
#pragma unroll
            for (int i = 0; i < kValues - 1; ++i)
                if (whole + i < a.n) put_raw(row + i, x[i / (kValues / 4)], i % (kValues / 4));
        }
    };
    auto sums = [&](float (&v)[32], int c, int col) {
        tmem_load32(d + c, v);
        tmem_wait_load();
        tmem_loaded(v);
        if (f.bias && !partial) add_bias(f, v, col, a.n);
    };
    for (int c = half * kWide; c < a.bn; c += 2 * kWide) {
        const int col = col0 + c;
        if (col >= a.n || row0 >= a.m) break;
        if (c + kWide > a.bn) {
            // 32 columns are left of the tile, and the next 32 another's: a row to a lane
            if (!waited && !wait()) return false;
            waited = true;
            float v[32];
            sums(v, c, col);
            if (row0 + lane < a.m) finish_row<T, TY>(f, v, row0 + lane, col, a.n);
            break;
        }
        const bool more = f.residual && !partial, first_z = f.z && !partial;
        auto fetch = [&] {
            fetch_tile(tile, static_cast<const TY*>(f.residual) + (int64_t)row0 * f.residual_stride + col,
                       f.residual_stride, a.m - row0, a.n - col);
        };
        tile_free();
        if (more && !first_z) fetch();
        if (!waited) {
            if (!wait()) return false;
            waited = true;
        }
        if (first_z) {
#pragma unroll
            for (int h = 0; h < kWide; h += 32) {
                float v[32];
                sums(v, c + h, col + h);
                if (sizeof(TY) == 2) {
                    put32(tile, lane, h / 8, v, T());
                } else if (row0 + lane < a.m) {   // half a tile's width: as it is
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = v[i + e];
                        T* to = static_cast<T*>(f.z) + (int64_t)(row0 + lane) * f.z_stride;
                        if (col + i < a.n) store_part(to, col + i, a.n, x);
                    }
                }
            }
            if (sizeof(TY) == 2) {
                store(mz, static_cast<TY*>(f.z), f.z_stride, col, 0);
                tile_free();
            }
            if (more) fetch();
        }
        if (more) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
        }
#pragma unroll
        for (int h = 0; h < kWide; h += 32) {
            float v[32];
            sums(v, c + h, col + h);
            if (!partial) {
                with_activation(f.activation, [&](auto act) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = activate<decltype(act)::value>(v[i]);
                });
                if (more) add32(tile, lane, h / (16 / (int)sizeof(TY)), v, TY());
            }
            put32(tile, lane, h / (16 / (int)sizeof(TY)), v, TY());
        }
        store(my, static_cast<TY*>(f.y), f.y_stride, col, partial ? split : 0);
    }
    return waited || wait();
}

template <int BN, bool PAIR, typename T>
__global__ void __launch_bounds__(kProductThreads, 1)
k_linear_product(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb,
                 const __grid_constant__ CUtensorMap my, const __grid_constant__ CUtensorMap mz,
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
            // the CTA's rows of B; across the contraction they come in boxes of 64
            const int b_rows = a.bn / kCtas, b_boxes = (b_rows + 63) / 64;
            const uint32_t bytes =
                kCtas * (R::kA + (a.b_across ? b_boxes * 64 : b_rows) * kBlock * 2);
            const uint32_t first_full = PAIR ? first_cta(&full[0]) : 0;
            int s = 0, slot = 0;
            uint32_t turn = 1;   // a stage's first use waits for nobody
            bool ok = true;
            for (int u = first_unit; ok && u < a.units; u += step) {
                const Unit w = unit_of(a, u);
                const int row = (w.m * kCtas + rank) * 128, col = w.n * a.bn + rank * b_rows;
                for (int k = w.k0; k < w.k1; ++k, ++s) {
                    if (s >= R::kStages && !bar_wait(&empty[slot], turn, &stop)) {
                        ok = false;
                        break;
                    }
                    uint8_t* at = smem + slot * R::kStage;
                    if (rank == 0) bar_expect(&full[slot], bytes);
                    const uint32_t bar = first_full + 8 * slot;
                    auto load = [&](uint8_t* to, const CUtensorMap* map, int c0, int c1) {
                        if (PAIR)
                            tma_load2_pair(to, map, c0, c1, bar);
                        else
                            tma_load2(to, map, c0, c1, &full[slot]);
                    };
                    auto load_pair = [&](uint8_t* to, const CUtensorMap* map, int c0, int c1) {
                        if (PAIR)
                            tma_load3_pair(to, map, 0, c1, c0 / 64, bar);
                        else
                            tma_load3(to, map, 0, c1, c0 / 64, &full[slot]);
                    };
                    if (a.a_boxes) {
                        load_pair(at, &ma, row, k * kBlock);
                    } else if (a.a_across) {
                        for (int i = 0; i < 2; ++i)
                            load(at + i * 8192, &ma, row + i * 64, k * kBlock);
                    } else {
                        load(at, &ma, k * kBlock, row);
                    }
                    at += R::kA;
                    if (a.b_boxes) {
                        load_pair(at, &mb, col, k * kBlock);
                    } else if (a.b_across) {
                        for (int i = 0; i < b_boxes; ++i)
                            load(at + i * 8192, &mb, col + i * 64, k * kBlock);
                    } else {
                        load(at, &mb, k * kBlock, col);
                    }
                    if (++slot == R::kStages) slot = 0, turn ^= 1;
                }
            }
            // The loads must land before the CTA ends, also where nobody waits for them.  A pair's
            // second CTA cannot see them land, but its stages are free again only after they have
            // been multiplied.  The products' arrivals must be there too: one still on its way to
            // this CTA's barriers would reach the shared memory of whichever CTA comes next.
            int never = 0;
            if (rank == 0)
                for (int w = max(0, s - R::kStages); w < s; ++w)
                    bar_wait(&full[w % R::kStages], (w / R::kStages) & 1, &never);
            for (int w = max(0, s - R::kStages); ok && w < s; ++w)
                ok = bar_wait(&empty[w % R::kStages], (w / R::kStages) & 1, &stop);
            if (rank != 0 && !ok)
                for (const uint64_t t = now_ns(); now_ns() - t < 10000000ull;) __nanosleep(1000);
        }
    } else if (warp == 1) {
        // ---- products ----
        if (lane == 0 && rank == 0) {
            const uint32_t desc =
                product_desc(128 * kCtas, a.bn, std::is_same<T, f16>::value, a.a_across, a.b_across);
            // A product of 16 along the contraction takes the tensor core 128 cycles (256 columns), and
            // what this one thread does for it has to be less: descriptors differ in the low word's
            // address alone, stages and their turns are counted, not divided for.
            const uint32_t base = smem_addr(smem);
            const uint64_t a0 = smem_desc(base, a.a_across ? 8192 : 16);
            const uint64_t b0 = smem_desc(base + R::kA, a.b_across ? 8192 : 16);
            const uint32_t a_step = (a.a_across ? 2048 : 32) >> 4, b_step = (a.b_across ? 2048 : 32) >> 4;
            auto commit = [&](uint64_t* bar) {
                if (PAIR)
                    tc_commit_pair(bar);
                else
                    tc_commit(bar);
            };
            auto at = [](uint64_t desc, uint32_t offset) {
                return (desc & 0xffffffff00000000ull) | ((uint32_t)desc + offset);
            };
            int i = 0;
            uint32_t slot = 0, turn = 0, from = 0;   // from: the stage's place, in 16 bytes
            bool ok = true;
            // a unit's blocks are counted before the one in front of it is worked on: divisions
            // between two units' products leave the tensor core idle
            int blocks = first_unit < a.units ? blocks_of(a, first_unit) : 0, next = 0;
            for (int u = first_unit; ok && u < a.units; u += step, ++i, blocks = next) {
                next = blocks_of(a, u + step);
                const uint32_t d = tmem + (i & 1) * BN;
                if (i > 1)
                    ok = PAIR ? bar_wait_cluster(&free_[i & 1], ((i >> 1) - 1) & 1, &stop)
                              : bar_wait(&free_[i & 1], ((i >> 1) - 1) & 1, &stop);
                bool add = false;
                for (int k = 0; ok && k < blocks; ++k) {
                    ok = bar_wait(&full[slot], turn, &stop);
                    if (!ok) break;
                    tc_after_sync();
#pragma unroll
                    for (int j = 0; j < kBlock / 16; ++j) {
                        const uint64_t x = at(a0, from + j * a_step), y = at(b0, from + j * b_step);
                        if (PAIR)
                            mma_pair(d, x, y, desc, add || j > 0);
                        else
                            mma_ss(d, x, y, desc, add || j > 0);
                    }
                    commit(&empty[slot]);
                    add = true;
                    from += R::kStage >> 4;
                    if (++slot == R::kStages) slot = 0, from = 0, turn ^= 1;
                }
                if (ok) commit(&done[i & 1]);
            }
            // the products must end before their memory is freed, also after a wait gave up
            int never = 0;
            commit(&drained);
            bar_wait(&drained, 0, &never);
        } else if (lane == 0) {
            // the pair's last commit arrives here as well, and must not come after the CTA's end
            int never = 0;
            bar_wait_cluster(&drained, 0, &never);
        }
    } else if (warp >= 4) {
        // ---- finishing: a thread to a row of the tile, two warps to 32 rows ----
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        uint8_t* staged = smem + R::kStages * R::kStage + (warp - 4) * kStaged;
        const Finish& f = a.f;
        const uint32_t tile = smem_addr(staged);
        bool stopped = false;
        int i = 0;
        for (int u = first_unit; u < a.units; u += step, ++i) {
            const Unit w = unit_of(a, u);
            const uint32_t d = tmem + (i & 1) * BN + ((uint32_t)quarter << 21);
            const int row0 = (w.m * kCtas + rank) * 128 + quarter * 32, row = row0 + lane;
            auto wait = [&] {
                const bool ok = __all_sync(0xffffffffu, bar_wait(&done[i & 1], (i >> 1) & 1, &stop));
                tc_after_sync();
                return ok;
            };
            if (f.tiles) {
                const bool ok =
                    a.partial || f.y_f32
                        ? finish_tiles<BN, T, float>(a, &my, &mz, tile, d, row0, w.n * a.bn,
                                                     half, w.split, wait)
                        : finish_tiles<BN, T, T>(a, &my, &mz, tile, d, row0, w.n * a.bn,
                                                 half, w.split, wait);
                stopped = !ok;
            } else {
                float* partial = a.partial ? a.partial + (int64_t)w.split * a.n * a.ld : nullptr;
                bool waited = false;
                for (int c = half; c < a.bn / 32 && !stopped; c += 2) {
                    const int col = w.n * a.bn + c * 32;
                    if (col >= a.n) break;
                    // a column's residuals, asked for before the sums are waited for
                    float more[32], bias = 0.f;
#pragma unroll
                    for (int j = 0; j < 32; ++j) more[j] = 0.f;
                    if (!f.swapped && f.residual && col + lane < a.n)
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (row0 + j < a.m) more[j] = residual_at<T>(f, row0 + j, col + lane);
                    if (!waited && !wait()) {
                        stopped = true;
                        break;
                    }
                    waited = true;
                    float v[32];
                    tmem_load32(d + c * 32, v);
                    tmem_wait_load();
                    tmem_loaded(v);
                    if (f.swapped) {
                        // lanes are neighbours in memory already
                        if (row < a.m) {
                            if (!partial && f.bias) bias = f.bias[row];
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
                    } else {
                        // bias and activation a lane to a row, where bias and code are the warp's; then
                        // through shared memory, a row at a time and a lane to a column
                        float* values = reinterpret_cast<float*>(staged);
                        const bool mine = col + lane < a.n;
                        const int last = min(32, a.m - row0);
                        auto spread = [&](auto* to, int64_t stride, bool add) {
                            using TO = typename std::remove_pointer<decltype(to)>::type;
                            __syncwarp();
#pragma unroll
                            for (int j = 0; j < 32; ++j) values[lane * 32 + (j ^ lane)] = v[j];
                            __syncwarp();
                            if (!mine) return;
                            TO* at = to + (int64_t)row0 * stride + col + lane;
#pragma unroll
                            for (int j = 0; j < 32; ++j, at += stride)
                                if (j < last)
                                    *at = round_to<TO>(values[j * 32 + (lane ^ j)] +
                                                       (add ? more[j] : 0.f));
                        };
                        if (f.bias) add_bias(f, v, col, a.n);
                        if (f.z) spread(static_cast<T*>(f.z), f.z_stride, false);
                        with_activation(f.activation, [&](auto act) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = activate<decltype(act)::value>(v[j]);
                        });
                        if (f.y_f32)
                            spread(static_cast<float*>(f.y), f.y_stride, f.residual != nullptr);
                        else
                            spread(static_cast<T*>(f.y), f.y_stride, f.residual != nullptr);
                    }
                }
                if (!waited && !stopped) stopped = !wait();
            }
            if (stopped) break;
            tc_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (PAIR)
                    bar_arrive_first(&free_[i & 1]);
                else
                    bar_arrive(&free_[i & 1]);
            }
        }
        // the stores have read their tiles before the CTA's memory is another's
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
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

// Whether an operand across the contraction may be loaded two boxes of 64 at a time: its rows are
// seen as boxes beside each other then, all of them whole, and each CTA's begin with one.
bool in_boxes(const Operand& o, int rows) {
    return o.across && rows == 128 && o.matrix.inner % 64 == 0;
}

// Boxes of 64 along the dense dimension and `box` (at most 256) along the other; or, across and
// `boxes`, two boxes of 64 x 64 side by side.
cudaError_t operand_map(CUtensorMap* map, const Operand& o, int box, bool boxes, int type) {
    static std::atomic<void*> found{nullptr};
    void* fn = driver_call("cuTensorMapEncodeTiled", &found);
    if (!fn) return cudaErrorNotSupported;
    const cudaError_t bound = bind_context();
    if (bound != cudaSuccess) return bound;
    const Matrix& x = o.matrix;
    // the stride over a single row is free, but the encoder checks it
    const int64_t stride = x.outer > 1 ? x.stride : (x.inner + 7) / 8 * 8;
    const cuuint64_t dims[3] = {boxes ? 64 : (cuuint64_t)x.inner, (cuuint64_t)x.outer,
                                (cuuint64_t)(x.inner / 64)};
    const cuuint64_t strides[2] = {(cuuint64_t)stride * 2, 128};
    const cuuint32_t sizes[3] = {64, (cuuint32_t)(o.across ? kBlock : box), 2};
    const cuuint32_t one[3] = {1, 1, 1};
    const CUresult rc = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn)(
        map, type == PSS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
        boxes ? 3 : 2, const_cast<void*>(x.data), dims, strides, sizes, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// Results [parts][rows][cols], stored in boxes of `width` columns (at most 128 bytes) x 32 rows.
// TMA leaves out what lies outside the tensor by 16-byte pieces only: a store to 517 columns of
// 16 bits writes 520.  What is behind a row's last whole piece is not TMA's, then, unless the rows
// have room for it (`padded`).
cudaError_t result_map(CUtensorMap* map, void* data, int64_t cols, int64_t rows, int64_t parts,
                       int64_t stride, int64_t part_stride, int width, int type, bool padded) {
    static std::atomic<void*> found{nullptr};
    void* fn = driver_call("cuTensorMapEncodeTiled", &found);
    if (!fn) return cudaErrorNotSupported;
    const int64_t size = type == PSS_F32 ? 4 : 2, grid = 16 / size;
    if (!padded) cols = cols < grid ? grid : cols / grid * grid;   // (of less than a piece: never used)
    if (rows <= 1) stride = (cols + grid - 1) / grid * grid;       // free, but checked
    if (parts <= 1) part_stride = stride;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)parts};
    const cuuint64_t strides[2] = {(cuuint64_t)(stride * size), (cuuint64_t)(part_stride * size)};
    const cuuint32_t box[3] = {(cuuint32_t)width, 32, 1}, one[3] = {1, 1, 1};
    const CUresult rc = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn)(
        map,
        type == PSS_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
        : type == PSS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                           : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
        3, data, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int BN, bool PAIR, typename T>
cudaError_t launch(const Product& p, int type, unsigned long long* status, cudaStream_t st) {
    using R = Ring<BN, PAIR>;
    CUtensorMap ma, mb, my = {}, mz = {};
    const int b_rows = p.bn / (PAIR ? 2 : 1);
    const bool a_boxes = in_boxes(p.a, 128), b_boxes = in_boxes(p.b, b_rows);
    cudaError_t e = operand_map(&ma, p.a, 128, a_boxes, type);
    if (e == cudaSuccess) e = operand_map(&mb, p.b, b_rows, b_boxes, type);
    Finish f = p.f;
    const bool split = p.splits > 1;
    f.tiles = !f.swapped && (split || f.tiles);
    if (f.tiles && e == cudaSuccess) {
        const int width = 64;   // 128 bytes, also where BN = 32 is all there is
        if (split)
            e = result_map(&my, p.partial, p.n, p.m, p.splits, p.ld, (int64_t)p.m * p.ld, 32, PSS_F32,
                           true);
        else
            e = result_map(&my, f.y, p.n, p.m, 1, f.y_stride, (int64_t)p.m * f.y_stride,
                           f.y_f32 ? 32 : width, f.y_f32 ? PSS_F32 : type, false);
        if (!split && f.z && !f.y_f32 && e == cudaSuccess)
            e = result_map(&mz, f.z, p.n, p.m, 1, f.z_stride, (int64_t)p.m * f.z_stride, width, type,
                           false);
    }
    if (e != cudaSuccess) return e;
    auto* k = k_linear_product<BN, PAIR, T>;
    static std::atomic<uint64_t> ready{0};
    e = allow_smem(k, R::kSmem, &ready);
    if (e != cudaSuccess) return e;
    const int units = p.m_tiles * p.n_tiles * p.splits, fit = sm_count() / (PAIR ? 2 : 1);
    const Args a{f, split ? p.partial : nullptr, p.ld, p.m, p.n, p.bn, p.blocks, p.m_tiles,
                 p.n_tiles, p.splits, units, p.a.across, p.b.across, a_boxes, b_boxes, status};
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
    e = cudaLaunchKernelEx(&cfg, k, ma, mb, my, mz, a);
    if (e != cudaSuccess || p.splits == 1) return e;
    const int64_t rows = p.f.swapped ? p.n : p.m, threads = rows * (p.ld / 8);
    return launch_k(k_linear_join<T>, dim3((unsigned)((threads + kThreads - 1) / kThreads)),
                    dim3(kThreads), 0, st, static_cast<const float*>(p.partial), p.splits, rows,
                    p.f.swapped ? p.m : p.n, p.ld, p.f);
}

// Rows into rows of `ld` values, 8 to a thread, zeros behind a row's end.  The values are moved
// as they are, whichever 16-bit type they have.
struct Copy {
    const uint16_t* from;
    uint16_t* to;
    int64_t stride, rows, cols, ld;
};
__global__ void __launch_bounds__(kThreads)
k_linear_copy(const __grid_constant__ Copy x, const __grid_constant__ Copy y, unsigned x_ctas) {
    pdl_prologue();
    const Copy& c = blockIdx.x < x_ctas ? x : y;
    const int64_t cta = blockIdx.x < x_ctas ? blockIdx.x : blockIdx.x - x_ctas;
    const int64_t i = cta * kThreads + threadIdx.x, vecs = c.ld / 8;
    const int64_t r = i / vecs, col = (i - r * vecs) * 8;
    if (r >= c.rows) return;
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = col + e < c.cols ? c.from[r * c.stride + col + e] : 0;
    *reinterpret_cast<uint4*>(c.to + r * c.ld + col) =
        make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

}  // namespace

bool on_grid(const Matrix& x) {
    return aligned_to(x.data, 16) && (x.outer <= 1 || x.stride % 8 == 0);
}

int64_t copy_bytes(const Matrix& x) { return x.outer * ((x.inner + 7) / 8 * 8) * 2; }

cudaError_t copy_matrices(Matrix* x, void* to_x, Matrix* y, void* to_y, cudaStream_t st) {
    unsigned ctas[2];
    Copy copies[2];
    Matrix* const from[2] = {x, y};
    void* const to[2] = {to_x, to_y};
    for (int i = 0; i < 2; ++i) {
        Matrix& m = *from[i];
        const int64_t ld = (m.inner + 7) / 8 * 8;
        copies[i] = Copy{static_cast<const uint16_t*>(m.data), static_cast<uint16_t*>(to[i]), m.stride,
                         to[i] ? m.outer : 0, m.inner, ld};
        ctas[i] = to[i] ? (unsigned)((m.outer * (ld / 8) + kThreads - 1) / kThreads) : 0;
        if (to[i]) {
            m.data = to[i];
            m.stride = ld;
        }
    }
    return launch_k(k_linear_copy, dim3(ctas[0] + ctas[1]), dim3(kThreads), 0, st, copies[0],
                    copies[1], ctas[0]);
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
    const Kind kinds[] = {{256, 540, true},  {224, 480, true}, {192, 440, true},  {160, 400, true},
                          {128, 330, false}, {64, 250, false}, {32, 220, false}};
    double best = 0;
    p->bn = 0;
    for (const Kind& kind : kinds) {
        const int bn = kind.bn, rows = kind.pair ? 256 : 128, fit = kind.pair ? sms / 2 : sms;
        if (bn == 32 && (p->b.across || p->n > 32)) continue;   // a box across is 64 wide
        if (bn > 64 && p->n <= bn / 2) continue;
        if (kind.pair && p->m <= 128) continue;
        const int m_tiles = (p->m + rows - 1) / rows, n_tiles = (p->n + bn - 1) / bn;
        const int64_t tiles = (int64_t)m_tiles * n_tiles;
        // across the contraction B comes in boxes of 64, two to a CTA of any of these pairs: none is
        // cheaper than 256 columns
        const int cycles = kind.pair && p->b.across ? 540 : kind.cycles;
        for (int s = 1; s <= 64 && s <= p->blocks; ++s) {
            const int64_t rounds = (tiles * s + fit - 1) / fit;
            const double most = (p->blocks + s - 1) / s;   // blocks of a unit, below 2^25
            double cost = 2000. + (double)rounds * (most * cycles + 300.);
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
            case 128: return launch<128, false, T>(p, type, status, st);
            case 64: return launch<64, false, T>(p, type, status, st);
            case 32: return launch<32, false, T>(p, type, status, st);
            default: return launch<256, true, T>(p, type, status, st);
        }
    };
    return type == PSS_BF16 ? go(bf16()) : go(f16());
}

}  // namespace seq
}  // namespace pss
