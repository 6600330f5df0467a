// Attention over packed sequences, backward, on the tensor cores.
//
// With c = scale * log2 e, L = lse * log2 e and delta = sum_c grad * out of a
// query row:
//   P = exp2(c S - L),  S = Q K^T,     dP = dO V^T,     dS = P (dP - delta),
//   dQ = scale dS K,    dK = scale dS^T Q,    dV = P^T dO.
// Two kernels, each with its result resident in tensor memory:
//   dQ: a tile of 128 query rows over its key tiles (three products a tile);
//   it also leaves L and delta of each row for
//   dK, dV: a tile of 128 keys over its query tiles, S and dP transposed (four
//   products a tile), the heads that share the key head among the tile's rows.
// Together seven products where one kernel needs five; that one kernel would
// add dQ into memory with atomics, whose order changes the result, and has to
// keep five 128-column accumulators where tensor memory holds four.
//
// In both, eight warps share the elementwise work, a thread to half a row, and P or dS replaces S or dP in tensor memory as bf16, the first
// operand of the products after it.  The order of the products lets the
// elementwise work on one of them run under the others:
//   dQ:  S(n+1) | dQ += dS(n) K, dP(n+1)            (S twice in tensor memory)
//   dKV: dV += P(n) dO, S(n+1) | dK += dS(n) Q, dP(n+1)
// What a row does not see gets S = -infinity, hence P = 0; a row that sees
// nothing has L = +infinity.
// Non-finite rows are computed again by the definition, as in the forward pass.
#include <atomic>

#include "attention_rows.cuh"
#include "attention_tma.h"
#include "tc.cuh"

namespace pss {
namespace seq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
// A key that every query nearly ignores has a gradient of the size of its P, so
// the dK, dV kernel takes P and dS times 2^24: what exp2 flushes to zero is then
// below 2^-150, and the factor is taken off exactly at the end.  (A dO above
// 2^104 makes that row infinite, and it is computed by its definition.)
constexpr float kLift = 24.f, kUnlift = 1.f / 16777216.f;
constexpr int kCompute = 256;   // threads of the elementwise work

// HD: values of a head, padded; TN: rows of the tiles that an item runs over,
// the columns of S and dP.  With TN = 64 and HD = 64 everything takes half the
// tensor memory (256 columns) and 66 KB, and two CTAs share an SM, so one's
// start, end and waits run under the other's work; with HD = 128 the
// accumulators alone leave room for one CTA.
template <int HD, int TN>
struct Cfg {
    static constexpr int kHalves = HD / 64;
    static constexpr int kSlab = TN * 128;                     // TN rows of 64 values
    static constexpr int kTileBytes = kHalves * 16384;         // the resident 128 rows
    static constexpr int kUnit = kHalves * kSlab;              // a tile of the ring
    static constexpr int kUnits = 4;
    static constexpr int kSmem = 2 * kTileBytes + kUnits * kUnit + 1024;   // + alignment
    static constexpr int kThreads = kCompute + 64;
    static constexpr int kCtas = TN == 64 && HD == 64 ? 2 : 1; // to an SM
    static constexpr int kCols = kCtas == 2 ? 256 : 512;       // tensor-memory columns
    static constexpr int kChunks = TN / 64;                    // a thread's columns / 32
};

// Barrier of the elementwise warps alone.
__device__ __forceinline__ void compute_sync() {
    asm volatile("bar.sync 1, %0;" :: "n"(kCompute) : "memory");
}

// Loads one tile, `slab` bytes to 64 values of its rows.
template <int HD>
__device__ __forceinline__ void load_tile(uint8_t* to, int slab, const CUtensorMap* map, int head,
                                          int token, uint64_t* bar) {
#pragma unroll
    for (int h = 0; h < HD / 64; ++h)
        tma_load3(to + h * slab, map, 64 * h, head, token, bar);
}

// D = A B^T: 128 and TN rows of HD values in shared memory.
template <int HD, int TN>
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t a_at, uint32_t b_at) {
    constexpr uint32_t kDesc = mma_desc(128, TN, false);
#pragma unroll
    for (int i = 0; i < HD / 16; ++i)
        mma_ss(d, smem_desc(a_at + (i / 4) * 16384 + (i % 4) * 32, 16),
               smem_desc(b_at + (i / 4) * (TN * 128) + (i % 4) * 32, 16), kDesc, i > 0);
}
// D += A B: A 128 x TN bf16 in tensor memory, the first half of its columns at
// a, the second TN / 2 columns on (each thread packs into the columns that it
// read); B TN rows of HD values in shared memory.
template <int HD, int TN>
__device__ __forceinline__ void mma_columns(uint32_t d, uint32_t a, uint32_t b_at, bool add) {
    constexpr uint32_t kDesc = mma_desc(128, HD, true);
    constexpr int kHalf = TN / 32;
#pragma unroll
    for (int i = 0; i < TN / 16; ++i)
        mma_ts(d, a + (i / kHalf) * (TN / 2) + (i % kHalf) * 8,
               smem_desc(b_at + i * 2048, TN * 128), kDesc, add || i > 0);
}

// Packs values to bf16 and stores them over the columns at `at`.
template <int N>
__device__ __forceinline__ void store_bf16(uint32_t at, const float (&v)[N][32]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = pack2(v[i][2 * e], v[i][2 * e + 1], bf16());
        tmem_store16(at + 16 * i, w);
    }
}
template <int N>
__device__ __forceinline__ void load_columns(uint32_t at, float (&v)[N][32]) {
#pragma unroll
    for (int i = 0; i < N; ++i) tmem_load32(at + 32 * i, v[i]);
    tmem_wait_load();
#pragma unroll
    for (int i = 0; i < N; ++i) tmem_loaded(v[i]);
}

// Columns of one result row, times `scale`, to memory.  The columns are read
// once to see whether all are finite (the answer) and once to store.
template <int N>
__device__ __forceinline__ bool row_finite(uint32_t at) {
    float odd = 0.f;
#pragma unroll 1
    for (int i = 0; i < N; i += 32) {
        float v[32];
        tmem_load32(at + i, v);
        tmem_wait_load();
        tmem_loaded(v);
#pragma unroll
        for (int e = 0; e < 32; ++e) odd += v[e] * 0.f;
    }
    return odd == 0.f;
}
// load: whether there are columns to read (the same for the whole warp); a row
// with `zero` is zeros all the same.
template <int N>
__device__ __forceinline__ void row_out(uint32_t at, bf16* to, int from, int dim, float scale,
                                        bool load, bool store, bool zero) {
#pragma unroll 1
    for (int i = 0; i < N; i += 32) {
        float v[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = 0.f;
        __syncwarp();
        if (load) {
            tmem_load32(at + i, v);
            tmem_wait_load();
            tmem_loaded(v);
        }
        if (store) {
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
                if (from + i + e >= dim) break;
                float o[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) o[x] = zero ? 0.f : v[e + x] * scale;
                store8(to + from + i + e, o);
            }
        }
    }
}

template <int HD, int TN>
__global__ void __launch_bounds__(Cfg<HD, TN>::kThreads, Cfg<HD, TN>::kCtas)
k_attention_dq(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mg,
               const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
               Attn a, Plan p) {
    pdl_prologue();
    using C = Cfg<HD, TN>;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t q_full, full[C::kUnits], empty[C::kUnits], s_full[2], dp_full, ds_ready,
        done;
    __shared__ uint32_t tmem_at;
    __shared__ volatile int stop;
    __shared__ uint8_t bad[2][kTile];
    __shared__ float deltas[2][kTile];
    const int item = blockIdx.x / a.kv_heads, hk = blockIdx.x - item * a.kv_heads;
    const Item it = p.items[item];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = a.group, tokens = p.tokens, n_tiles = it.t1;

    uint8_t* smem = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    uint8_t* ring = smem + 2 * C::kTileBytes;
    if (threadIdx.x == 0) {
        stop = 0;
        bar_init(&q_full, 1);
        for (int i = 0; i < C::kUnits; ++i) {
            bar_init(&full[i], 1);
            bar_init(&empty[i], 1);
        }
        bar_init(&s_full[0], 1);
        bar_init(&s_full[1], 1);
        bar_init(&dp_full, 1);
        bar_init(&ds_ready, kCompute);
        bar_init(&done, 1);
        bar_init_done();
    }
    if (warp == 0) tmem_alloc(&tmem_at, C::kCols);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    // columns: S of even tiles, of odd ones, dP and dS, dQ
    const uint32_t tmem = tmem_at, dp_at = tmem + 2 * TN, dq_at = tmem + 3 * TN;

    if (warp == 8) {
        // ---- loads: Q and dO, then K and V tiles in turn ----
        if (lane == 0 && n_tiles > 0) {
            bar_expect(&q_full, 2 * C::kHalves * (uint32_t)(tokens * group) * 128);
            load_tile<HD>(smem, 16384, &mq, hk * group, it.q0, &q_full);
            load_tile<HD>(smem + C::kTileBytes, 16384, &mg, hk * group, it.q0, &q_full);
            int u = 0;
            for (; u < 2 * n_tiles; ++u) {
                const int slot = u % C::kUnits, turn = u / C::kUnits;
                if (turn > 0 && !bar_wait(&empty[slot], (turn - 1) & 1, &stop)) break;
                bar_expect(&full[slot], C::kUnit);
                load_tile<HD>(ring + slot * C::kUnit, C::kSlab, u & 1 ? &mv : &mk, hk,
                              it.k0 + (u / 2) * TN, &full[slot]);
            }
            if (stop) {   // the loads in flight must land before the CTA ends
                int never = 0;
                bar_wait(&q_full, 0, &never);
                for (int w = max(0, u - C::kUnits); w < u; ++w)
                    bar_wait(&full[w % C::kUnits], (w / C::kUnits) & 1, &never);
            }
        }
    } else if (warp == 9) {
        // ---- products ----
        if (lane == 0 && n_tiles > 0) {
            const uint32_t q_at = smem_addr(smem), g_at = q_at + C::kTileBytes;
            const uint32_t ring_at = smem_addr(ring);
            auto unit = [&](int u) { return ring_at + (u % C::kUnits) * C::kUnit; };
            auto loaded = [&](int u) {
                return bar_wait(&full[u % C::kUnits], (u / C::kUnits) & 1, &stop);
            };
            bool ok = bar_wait(&q_full, 0, &stop) && loaded(0) && loaded(1);
            if (ok) {
                tc_after_sync();
                mma_rows<HD, TN>(tmem, q_at, unit(0));
                tc_commit(&s_full[0]);
                mma_rows<HD, TN>(dp_at, g_at, unit(1));
                tc_commit(&dp_full);
                tc_commit(&empty[1]);
            }
            for (int n = 0; ok && n < n_tiles; ++n) {
                const int k = 2 * n, next = k + 2;
                const bool more = n + 1 < n_tiles;
                if (more) {
                    // its S was read before dS(n - 1) was announced
                    if (!(ok = loaded(next))) break;
                    mma_rows<HD, TN>(tmem + ((n + 1) & 1) * TN, q_at, unit(next));
                    tc_commit(&s_full[(n + 1) & 1]);
                }
                if (!(ok = bar_wait(&ds_ready, n & 1, &stop))) break;
                tc_after_sync();
                mma_columns<HD, TN>(dq_at, dp_at, unit(k), n > 0);
                tc_commit(&empty[k % C::kUnits]);
                if (more) {
                    if (!(ok = loaded(next + 1))) break;
                    mma_rows<HD, TN>(dp_at, g_at, unit(next + 1));
                    tc_commit(&dp_full);
                    tc_commit(&empty[(next + 1) % C::kUnits]);
                }
            }
            tc_commit(&done);
            if (!ok) {   // the products in flight must end before their memory is freed
                int never = 0;
                bar_wait(&done, 0, &never);
            }
        }
    } else if (warp < 8) {
        // ---- P and dS: thread = half a row ----
        const int r = (warp & 3) * 32 + lane, half = warp >> 2;
        const int tok = r / group, h = hk * group + r - tok * group, token = it.q0 + tok;
        // the keys that the row sees, counted from k0: see0 .. see1
        Range range{0, -1};
        if (tok < tokens && token < a.q_tokens) range = p.q_range[token];
        const bool live = range.live();
        const int see0 = live ? range.lo - it.k0 : 0, see1 = live ? range.hi - it.k0 : 0;
        const int64_t at_stats = ((int64_t)hk * a.q_tokens + token) * group + h - hk * group;
        float2 st = make_float2(INFINITY, 0.f);
        if (see1 > see0) {
            const float lse = a.lse[(int64_t)token * a.heads + h];
            st.x = lse == -INFINITY ? INFINITY : lse * kLog2e;
        }
        // delta = sum_c grad out, half a row to a thread; where the whole range is
        // one tile, sum_j p dp below: the same sum, without out's rounding to bf16
        if (n_tiles > 1) {
            const int from = half * (HD / 2), to = min(a.dim, from + HD / 2);
            if (see1 > see0)
                for (int e = from; e < to; e += 8) {
                    float g[8], o[8];
                    load8(a.grad.at(token, h) + e, g);
                    load8(a.out.at(token, h) + e, o);
#pragma unroll
                    for (int x = 0; x < 8; ++x) st.y += g[x] * o[x];
                }
            deltas[half][r] = st.y;
            compute_sync();
            st.y += deltas[half ^ 1][r];
        }
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const float c = a.scale * kLog2e;
        const float2 c2 = make_float2(c, c), l2 = make_float2(-st.x, -st.x);
        bool ok = true;
        for (int n = 0; n < n_tiles; ++n) {
            ok = bar_wait(&s_full[n & 1], (n >> 1) & 1, &stop);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_after_sync();
            float s[C::kChunks][32], d[C::kChunks][32];
            load_columns(tmem + (n & 1) * TN + half * (TN / 2) + lanes, s);
            const int first = n * TN + half * (TN / 2);
#pragma unroll
            for (int i = 0; i < C::kChunks; ++i)
                hide(s[i], see0 - first - 32 * i, see1 - first - 32 * i);
#pragma unroll
            for (int i = 0; i < C::kChunks; ++i)
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const float2 x = fma2(make_float2(s[i][e], s[i][e + 1]), c2, l2);
                    s[i][e] = exp2_fast(x.x);
                    s[i][e + 1] = exp2_fast(x.y);
                }
            ok = bar_wait(&dp_full, n & 1, &stop);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_after_sync();
            const uint32_t d_at = dp_at + half * (TN / 2) + lanes;
            load_columns(d_at, d);
            if (n_tiles == 1) {
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < C::kChunks; ++i)
#pragma unroll
                    for (int e = 0; e < 32; e += 2)
                        sum = fma2(make_float2(s[i][e], s[i][e + 1]),
                                   make_float2(d[i][e], d[i][e + 1]), sum);
                deltas[half][r] = sum.x + sum.y;
                compute_sync();
                st.y = deltas[0][r] + deltas[1][r];
            }
            const float2 d2 = make_float2(-st.y, -st.y);
#pragma unroll
            for (int i = 0; i < C::kChunks; ++i)
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const float2 x = mul2(make_float2(s[i][e], s[i][e + 1]),
                                          add2(make_float2(d[i][e], d[i][e + 1]), d2));
                    d[i][e] = x.x;
                    d[i][e + 1] = x.y;
                }
            store_bf16(d_at, d);
            tmem_wait_store();
            tc_before_sync();
            bar_arrive(&ds_ready);
        }
        if (live && half == 0) p.stats[at_stats] = st;   // for the dK, dV kernel
        // ---- epilogue: each half stores its half of the columns ----
        const bool any = n_tiles > 0;
        if (any && __all_sync(0xffffffffu, ok)) ok = bar_wait(&done, 0, &stop);
        ok = __all_sync(0xffffffffu, ok) != 0;
        tc_after_sync();
        constexpr int kHalf = HD / 2;
        const uint32_t at = dq_at + half * kHalf + lanes;
        bool fine = true;
        if (any && ok) fine = row_finite<kHalf>(at);
        bad[half][r] = see1 > see0 && !fine;
        compute_sync();
        const bool again = bad[0][r] | bad[1][r];
        if (ok) {
            row_out<kHalf>(at, live ? a.dq.at(token, h) : nullptr, half * kHalf, a.dim, a.scale,
                           any, live && !again, see1 <= see0);
            unsigned mask = half == 0 ? __ballot_sync(0xffffffffu, again) : 0;
            while (mask) {
                const int from = __ffs(mask) - 1;
                mask &= mask - 1;
                __syncwarp();
                dq_row(a, __shfl_sync(0xffffffffu, range.lo, from),
                       __shfl_sync(0xffffffffu, range.hi, from),
                       __shfl_sync(0xffffffffu, token, from),
                       __shfl_sync(0xffffffffu, h, from));
            }
        }
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    if (warp == 0) tmem_free(tmem, C::kCols);
    if (threadIdx.x == 0 && stop) report_stop(a.status);
}

template <int HD, int TN>
__global__ void __launch_bounds__(Cfg<HD, TN>::kThreads, Cfg<HD, TN>::kCtas)
k_attention_dkv(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mg,
                const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                Attn a, Plan p) {
    pdl_prologue();
    using C = Cfg<HD, TN>;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t kv_full, full[C::kUnits], empty[C::kUnits], s_full, dp_full, p_ready,
        ds_ready, stats_full[2], stats_free[2], done;
    __shared__ uint32_t tmem_at;
    __shared__ volatile int stop;
    __shared__ uint8_t bad[2][kTile];
    __shared__ alignas(16) float lses[2][TN], deltas[2][TN];
    const int item = blockIdx.x / a.kv_heads, hk = blockIdx.x - item * a.kv_heads;
    const Item it = p.key_items[item];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = a.group, tokens = p.key_tokens, n_tiles = it.t1;
    const int rows = tokens * group;   // of a query tile

    uint8_t* smem = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    uint8_t* ring = smem + 2 * C::kTileBytes;
    if (threadIdx.x == 0) {
        stop = 0;
        bar_init(&kv_full, 1);
        for (int i = 0; i < C::kUnits; ++i) {
            bar_init(&full[i], 1);
            bar_init(&empty[i], 1);
        }
        bar_init(&s_full, 1);
        bar_init(&dp_full, 1);
        bar_init(&p_ready, kCompute);
        bar_init(&ds_ready, kCompute);
        for (int i = 0; i < 2; ++i) {
            bar_init(&stats_full[i], 32);
            bar_init(&stats_free[i], kCompute);
        }
        bar_init(&done, 1);
        bar_init_done();
    }
    // rows that no load writes (TN is not a multiple of the group) enter the
    // products as zeros
    for (int i = threadIdx.x; i < C::kUnits * C::kHalves * (TN - rows) * 8; i += C::kThreads) {
        const int slab = i / ((TN - rows) * 8), at = i - slab * (TN - rows) * 8;
        reinterpret_cast<uint4*>(ring + slab * C::kSlab + rows * 128)[at] =
            make_uint4(0, 0, 0, 0);
    }
    fence_async();
    if (warp == 0) tmem_alloc(&tmem_at, C::kCols);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    // columns: S and P, dP and dS, dV, dK
    const uint32_t tmem = tmem_at, dp_at = tmem + TN, dv_at = tmem + 2 * TN, dk_at = dv_at + HD;

    if (warp == 8) {
        // ---- loads: K and V, then Q and dO tiles in turn, with their L and delta ----
        if (lane == 0 && n_tiles > 0) {
            bar_expect(&kv_full, 2 * C::kTileBytes);
            load_tile<HD>(smem, 16384, &mk, hk, it.k0, &kv_full);
            load_tile<HD>(smem + C::kTileBytes, 16384, &mv, hk, it.k0, &kv_full);
        }
        const float2* from = p.stats + ((int64_t)hk * a.q_tokens + it.q0) * group;
        const int64_t end = (int64_t)(a.q_tokens - it.q0) * group;
        int u = 0;
        bool ok = true;
        for (int n = 0; n < n_tiles; ++n) {
            if (lane == 0) {
                for (; u < 2 * n + 2; ++u) {
                    const int slot = u % C::kUnits, turn = u / C::kUnits;
                    ok = turn == 0 || bar_wait(&empty[slot], (turn - 1) & 1, &stop);
                    if (!ok) break;
                    bar_expect(&full[slot], C::kHalves * (uint32_t)rows * 128);
                    load_tile<HD>(ring + slot * C::kUnit, C::kSlab, u & 1 ? &mg : &mq, hk * group,
                                  it.q0 + n * tokens, &full[slot]);
                }
            }
            const int b = n & 1;
            ok = ok && (n < 2 || bar_wait(&stats_free[b], ((n >> 1) - 1) & 1, &stop));
            if (!__all_sync(0xffffffffu, ok)) break;
#pragma unroll
            for (int i = 0; i < TN; i += 32) {
                const int r = i + lane;
                const int64_t row = (int64_t)n * rows + r;
                float2 st = make_float2(INFINITY, 0.f);
                if (r < rows && row < end) st = from[row];
                lses[b][r] = st.x - kLift;
                deltas[b][r] = st.y;
            }
            bar_arrive(&stats_full[b]);
        }
        if (lane == 0 && stop) {   // the loads in flight must land before the CTA ends
            int never = 0;
            if (n_tiles > 0) bar_wait(&kv_full, 0, &never);
            for (int w = max(0, u - C::kUnits); w < u; ++w)
                bar_wait(&full[w % C::kUnits], (w / C::kUnits) & 1, &never);
        }
    } else if (warp == 9) {
        // ---- products ----
        if (lane == 0 && n_tiles > 0) {
            const uint32_t k_at = smem_addr(smem), v_at = k_at + C::kTileBytes;
            const uint32_t ring_at = smem_addr(ring);
            auto unit = [&](int u) { return ring_at + (u % C::kUnits) * C::kUnit; };
            auto loaded = [&](int u) {
                return bar_wait(&full[u % C::kUnits], (u / C::kUnits) & 1, &stop);
            };
            bool ok = bar_wait(&kv_full, 0, &stop) && loaded(0) && loaded(1);
            if (ok) {
                tc_after_sync();
                mma_rows<HD, TN>(tmem, k_at, unit(0));
                tc_commit(&s_full);
                mma_rows<HD, TN>(dp_at, v_at, unit(1));
                tc_commit(&dp_full);
            }
            for (int n = 0; ok && n < n_tiles; ++n) {
                const int q = 2 * n, next = q + 2;
                const bool more = n + 1 < n_tiles;
                if (!(ok = bar_wait(&p_ready, n & 1, &stop))) break;
                tc_after_sync();
                mma_columns<HD, TN>(dv_at, tmem, unit(q + 1), n > 0);
                if (more) {
                    if (!(ok = loaded(next))) break;
                    mma_rows<HD, TN>(tmem, k_at, unit(next));
                    tc_commit(&s_full);
                }
                if (!(ok = bar_wait(&ds_ready, n & 1, &stop))) break;
                tc_after_sync();
                mma_columns<HD, TN>(dk_at, dp_at, unit(q), n > 0);
                tc_commit(&empty[q % C::kUnits]);
                tc_commit(&empty[(q + 1) % C::kUnits]);
                if (more) {
                    if (!(ok = loaded(next + 1))) break;
                    mma_rows<HD, TN>(dp_at, v_at, unit(next + 1));
                    tc_commit(&dp_full);
                }
            }
            tc_commit(&done);
            if (!ok) {   // the products in flight must end before their memory is freed
                int never = 0;
                bar_wait(&done, 0, &never);
            }
        }
    } else {
        // ---- P and dS, transposed: thread = half of a key's row ----
        const int r = (warp & 3) * 32 + lane, half = warp >> 2;
        const int key = it.k0 + r;
        // the rows of the query side that see this key, counted from q0: see0 .. see1
        Range range{0, -1};
        if (key < a.k_tokens) range = p.k_range[key];
        const bool live = range.live();
        const int64_t see0 = live ? (int64_t)(range.lo - it.q0) * group : 0;
        const int64_t see1 = live ? (int64_t)(range.hi - it.q0) * group : 0;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const float c = a.scale * kLog2e;
        const float2 c2 = make_float2(c, c);
        bool ok = true;
        for (int n = 0; n < n_tiles; ++n) {
            const int b = n & 1;
            ok = bar_wait(&stats_full[b], (n >> 1) & 1, &stop) &&
                 bar_wait(&s_full, n & 1, &stop);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_after_sync();
            float s[C::kChunks][32], d[C::kChunks][32];
            const uint32_t s_at = tmem + half * (TN / 2) + lanes;
            const uint32_t d_at = dp_at + half * (TN / 2) + lanes;
            load_columns(s_at, s);
            const int64_t from = (int64_t)n * rows + half * (TN / 2);
            const int lo = (int)max((int64_t)0, min((int64_t)TN, see0 - from));
            const int hi = (int)max((int64_t)0, min((int64_t)TN, see1 - from));
#pragma unroll
            for (int i = 0; i < C::kChunks; ++i) hide(s[i], lo - 32 * i, hi - 32 * i);
            const float4* l4 = reinterpret_cast<const float4*>(&lses[b][half * (TN / 2)]);
            const float4* e4 = reinterpret_cast<const float4*>(&deltas[b][half * (TN / 2)]);
#pragma unroll
            for (int i = 0; i < C::kChunks; ++i)
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    const float4 l = l4[8 * i + e / 4];
                    const float2 x = fma2(make_float2(s[i][e], s[i][e + 1]), c2,
                                          make_float2(-l.x, -l.y));
                    const float2 y = fma2(make_float2(s[i][e + 2], s[i][e + 3]), c2,
                                          make_float2(-l.z, -l.w));
                    s[i][e] = exp2_fast(x.x);
                    s[i][e + 1] = exp2_fast(x.y);
                    s[i][e + 2] = exp2_fast(y.x);
                    s[i][e + 3] = exp2_fast(y.y);
                }
            store_bf16(s_at, s);
            tmem_wait_store();
            tc_before_sync();
            bar_arrive(&p_ready);
            ok = bar_wait(&dp_full, n & 1, &stop);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_after_sync();
            load_columns(d_at, d);
#pragma unroll
            for (int i = 0; i < C::kChunks; ++i)
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    const float4 m = e4[8 * i + e / 4];
                    const float2 x = mul2(make_float2(s[i][e], s[i][e + 1]),
                                          add2(make_float2(d[i][e], d[i][e + 1]),
                                               make_float2(-m.x, -m.y)));
                    const float2 y = mul2(make_float2(s[i][e + 2], s[i][e + 3]),
                                          add2(make_float2(d[i][e + 2], d[i][e + 3]),
                                               make_float2(-m.z, -m.w)));
                    d[i][e] = x.x;
                    d[i][e + 1] = x.y;
                    d[i][e + 2] = y.x;
                    d[i][e + 3] = y.y;
                }
            bar_arrive(&stats_free[b]);
            store_bf16(d_at, d);
            tmem_wait_store();
            tc_before_sync();
            bar_arrive(&ds_ready);
        }
        // ---- epilogue: the first four warps store dV, the others dK ----
        const bool any = n_tiles > 0;
        if (any && __all_sync(0xffffffffu, ok)) ok = bar_wait(&done, 0, &stop);
        ok = __all_sync(0xffffffffu, ok) != 0;
        tc_after_sync();
        const uint32_t at = (half == 0 ? dv_at : dk_at) + lanes;
        bool fine = true;
        if (any && ok) fine = row_finite<HD>(at);
        bad[half][r] = live && !fine;
        compute_sync();
        const bool again = bad[0][r] | bad[1][r];
        if (ok) {
            bf16* to = live ? (half == 0 ? a.dv : a.dk).at(key, hk) : nullptr;
            row_out<HD>(at, to, 0, a.dim, half == 0 ? kUnlift : a.scale * kUnlift, any,
                        live && !again, false);
            unsigned mask = half == 0 ? __ballot_sync(0xffffffffu, again) : 0;
            while (mask) {
                const int from = __ffs(mask) - 1;
                mask &= mask - 1;
                __syncwarp();
                dkv_row(a, __shfl_sync(0xffffffffu, range.lo, from),
                        __shfl_sync(0xffffffffu, range.hi, from), __shfl_sync(0xffffffffu, key, from), hk);
            }
        }
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    if (warp == 0) tmem_free(tmem, C::kCols);
    if (threadIdx.x == 0 && stop) report_stop(a.status);
}

template <int HD, int TN>
cudaError_t launch(const Attn& a, const Plan& p, cudaStream_t st) {
    using C = Cfg<HD, TN>;
    auto* dq = k_attention_dq<HD, TN>;
    auto* dkv = k_attention_dkv<HD, TN>;
    static std::atomic<uint64_t> ready[2];
    cudaError_t e = allow_smem(dq, C::kSmem, &ready[0]);
    if (e == cudaSuccess) e = allow_smem(dkv, C::kSmem, &ready[1]);
    CUtensorMap mq, mg, mk, mv;
    auto queries = [&](CUtensorMap* m, const Rows& r, int tokens) {
        if (e == cudaSuccess)
            e = tile_map(m, r, a.q_tokens, a.heads, a.dim, a.group, tokens, p.head);
    };
    auto keys = [&](CUtensorMap* m, const Rows& r, int n) {
        if (e == cudaSuccess) e = tile_map(m, r, a.k_tokens, a.kv_heads, a.dim, 1, n, p.head);
    };
    if (a.q_tokens > 0) {
        queries(&mq, a.q, p.tokens);
        queries(&mg, a.grad, p.tokens);
        keys(&mk, a.k, TN);
        keys(&mv, a.v, TN);
        if (e == cudaSuccess)
            e = launch_k(dq, dim3((unsigned)p.most_items * a.kv_heads), dim3(C::kThreads),
                         C::kSmem, st, mq, mg, mk, mv, a, p);
    }
    if (a.k_tokens > 0) {
        queries(&mq, a.q, p.key_tokens);
        queries(&mg, a.grad, p.key_tokens);
        keys(&mk, a.k, kTile);
        keys(&mv, a.v, kTile);
        if (e == cudaSuccess)
            e = launch_k(dkv, dim3((unsigned)p.key_tiles * a.kv_heads), dim3(C::kThreads),
                         C::kSmem, st, mq, mg, mk, mv, a, p);
    }
    return e;
}

}  // namespace

cudaError_t launch_tiles_backward(const Attn& a, const Plan& p, cudaStream_t st) {
    if (a.dim > 64) return launch<128, 128>(a, p, st);
    return p.keys == 64 ? launch<64, 64>(a, p, st) : launch<64, 128>(a, p, st);
}

}  // namespace seq
}  // namespace pss
