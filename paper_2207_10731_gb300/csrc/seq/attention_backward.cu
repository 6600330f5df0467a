// Attention over packed sequences, backward, on the tensor cores.
//
// With c = scale * log2 e, L = lse * log2 e and delta = sum_c grad * out of a
// query row (k_attention_ready, attention_plan.cu):
//   P = exp2(c S - L),  S = Q K^T,     dP = dO V^T,     dS = P (dP - delta),
//   dQ = scale dS K,    dK = scale dS^T Q,    dV = P^T dO.
// Two kernels, each with its result resident in tensor memory:
//   dQ: a tile of 128 query rows over its key tiles (three products a tile);
//   dK, dV: a tile of 128 keys over its query tiles, S and dP transposed (four
//   products a tile), the heads that share the key head among the tile's rows.
// Together seven products where one kernel needs five; that one kernel would
// add dQ into memory with atomics, whose order changes the result, and has to
// keep five 128-column accumulators where tensor memory holds four.
//
// In both, eight warps share the elementwise work, a thread to half a row, and
// pack P and dS as bf16 into columns of S and dP that they have read, the first
// operand of the products after it.  The order of the products lets the
// elementwise work of one half step run under the products of the other:
//   dQ:  S twice in tensor memory, dS(n) over S(n):
//        P(n+1) | dP(n+1), dQ += dS(n) K(n), S(n+2);
//   dKV: P(n) over S, dS(n) over dP:
//        dS(n) | dV += P(n) dO(n), S(n+1);   P(n+1) | dK += dS(n) Q(n), dP(n+1).
// So the first operand's tiles (K of dQ, Q of dKV) live for three steps and
// have three buffers, the others two.  Most buffers are freed by the elementwise
// warps, when they see S or dP of a later step, which the tensor core finished
// after it; K of dQ, which is wanted again soonest, by its last product.
//
// What a row does not see gets S = -infinity, hence P = 0; a row that sees
// nothing has L = +infinity.  Rows that are not finite, or whose tile did not
// come to its end, are computed again (attention_rows.cuh), as in the forward pass.
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
// 2^104 makes that row infinite, and it is computed again without the factor.)
constexpr float kLift = 24.f, kUnlift = 1.f / 16777216.f;
// The dQ kernel's second product takes dS as the sum of two bf16 for heads up to
// 64, where the products wait for the elementwise work anyway, and for heads of
// 128 in items of up to this many keys.  dQ's error against 64 bits is then 1.2
// to 1.4 times that of rounding dQ once instead of 1.6 (packed histories: 229
// instead of 221 us for the whole pass); on long rows of 128, where one part
// gives 1.4, it would cost a third more products.
constexpr int kTwiceKeys = 1024;
constexpr int kCompute = 256;   // threads of the elementwise work

// HD: values of a head, padded; TN: rows of the tiles that an item runs over,
// the columns of S and dP.  With TN = 64 and HD = 64 everything takes half the
// tensor memory (256 columns) and 74 KB, and two CTAs share an SM, so one's
// start, end and waits run under the other's work; with HD = 128 the
// accumulators alone leave room for one CTA.
template <int HD, int TN>
struct Cfg {
    static constexpr int kHalves = HD / 64;
    static constexpr int kSlab = TN * 128;                     // TN rows of 64 values
    static constexpr int kTileBytes = kHalves * 16384;         // a resident tile: 128 rows
    static constexpr int kUnit = kHalves * kSlab;              // a tile of the rings
    static constexpr int kA = 3, kB = 2;                       // buffers of the two rings
    static constexpr int kSmem = 2 * kTileBytes + (kA + kB) * kUnit;
    static constexpr int kCtas = TN == 64 && HD == 64 ? 2 : 1; // to an SM
    // dK, dV: threads that issue products, in turns (kAhead); where two CTAs share
    // the SM the other one's products fill the gaps, and registers are short.  dQ
    // has one long run of products a step: one thread (two were 16 % slower).
    static constexpr int kIssuers = kCtas == 2 ? 1 : 2;
    static constexpr int kThreads = kCompute + 64;
    static constexpr int kThreadsKV = kCompute + 32 + 32 * kIssuers;
    static constexpr int kCols = kCtas == 2 ? 256 : 512;       // tensor-memory columns
    static constexpr int kChunks = TN / 64;                    // a thread's columns / 32
};

// Both kernels' state in shared memory behind the tiles.
template <int TN>
struct Shared {
    uint64_t resident, a_full[3], a_empty[3], b_full[2], b_empty[2];
    uint64_t s_full[2], dp_full, p_ready, ds_ready, stats_full[2], stats_free[2], done, turn[2];
    union alignas(16) {
        struct {
            float lse[2][TN], delta[2][TN];   // dK, dV
        };
        float part[2][kTile];                 // dQ
    };
    uint32_t tmem;
    int stop;
    bool bad[2][kTile];
};

// Loads one tile, `slab` bytes to 64 values of its rows.
template <int HD>
__device__ __forceinline__ void load_tile(uint8_t* to, int slab, const CUtensorMap* map, int head,
                                          int token, uint64_t* bar) {
#pragma unroll
    for (int h = 0; h < HD / 64; ++h)
        tma_load3(to + h * slab, map, 64 * h, head, token, bar);
}

// The loads (na and nb tiles of the rings) must land before the CTA ends, also
// where nobody waits for them.
template <typename C, int TN>
__device__ __forceinline__ void loads_landed(Shared<TN>& sh, int na, int nb) {
    int never = 0;
    bar_wait(&sh.resident, 0, &never);
    for (int m = max(0, na - C::kA); m < na; ++m)
        bar_wait(&sh.a_full[m % C::kA], (m / C::kA) & 1, &never);
    for (int m = max(0, nb - C::kB); m < nb; ++m)
        bar_wait(&sh.b_full[m % C::kB], (m / C::kB) & 1, &never);
}

// D = A B^T: 128 and TN rows of HD values in shared memory.
// Products from .. to of its HD / 16.
template <int HD, int TN>
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t a_at, uint32_t b_at, int from = 0,
                                         int to = HD / 16) {
    constexpr uint32_t kDesc = mma_desc(128, TN, false);
#pragma unroll
    for (int i = from; i < to; ++i)
        mma_ss(d, smem_desc(a_at + (i / 4) * 16384 + (i % 4) * 32, 16),
               smem_desc(b_at + (i / 4) * (TN * 128) + (i % 4) * 32, 16), kDesc, i > 0);
}
// D += A B: A 128 x TN bf16 in tensor memory, the first half of its columns at
// a, the second TN / 2 columns on (each thread packs into the columns that it
// read); B TN rows of HD values in shared memory.
// Products from .. to of its TN / 16.
template <int HD, int TN>
__device__ __forceinline__ void mma_columns(uint32_t d, uint32_t a, uint32_t b_at, bool add,
                                            int from = 0, int to = TN / 16) {
    constexpr uint32_t kDesc = mma_desc(128, HD, true);
    constexpr int kHalf = TN / 32;
#pragma unroll
    for (int i = from; i < to; ++i)
        mma_ts(d, a + (i / kHalf) * (TN / 2) + (i % kHalf) * 8,
               smem_desc(b_at + i * 2048, TN * 128), kDesc, add || i > 0);
}

// Values less what their rounding to bf16 keeps.
template <int N>
__device__ __forceinline__ void bf16_rest(float (&v)[N][32]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float2 kept = unpack2(pack2(v[i][e], v[i][e + 1], bf16()), bf16());
            v[i][e] -= kept.x;
            v[i][e + 1] -= kept.y;
        }
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

template <int HD, int TN>
__global__ void __launch_bounds__(Cfg<HD, TN>::kThreads, Cfg<HD, TN>::kCtas)
k_attention_dq(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mg,
               const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
               const __grid_constant__ CUtensorMap mdq, const __grid_constant__ Attn a,
               const __grid_constant__ Plan p) {
    pdl_prologue();
    using C = Cfg<HD, TN>;
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared<TN>& sh = *reinterpret_cast<Shared<TN>*>(smem + C::kSmem);
    volatile int* stop = &sh.stop;
    const int item = blockIdx.x / a.kv_heads, hk = blockIdx.x - item * a.kv_heads;
    const Item it = p.items[item];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = a.group, tokens = p.tokens, n_tiles = it.t1;
    // rows of few keys have the largest dS and feel the rounding of both dS and
    // out (in delta) most
    const bool twice = HD == 64 || n_tiles * TN <= kTwiceKeys;

    // the thread's row and what it sees; asked for before the loads begin
    const int r = (warp & 3) * 32 + lane, tok = r / group, h = hk * group + r - tok * group;
    const int token = it.q0 + tok;
    Range range{0, -1};
    float2 st = make_float2(INFINITY, 0.f);
    const int64_t at_stats = ((int64_t)hk * a.q_tokens + token) * group + h - hk * group;
    if (warp < 8 && tok < tokens && token < a.q_tokens) {
        range = p.q_range[token];
        st = p.stats[at_stats];
    }

    uint8_t* ring_a = smem + 2 * C::kTileBytes;
    uint8_t* ring_b = ring_a + C::kA * C::kUnit;
    if (threadIdx.x == 0) {
        prefetch_map(&mq);
        prefetch_map(&mg);
        prefetch_map(&mk);
        prefetch_map(&mv);
        prefetch_map(&mdq);
        *stop = 0;
        bar_init(&sh.resident, 1);
        for (int i = 0; i < C::kA; ++i) bar_init(&sh.a_full[i], 1), bar_init(&sh.a_empty[i], 1);
        for (int i = 0; i < C::kB; ++i) bar_init(&sh.b_full[i], 1), bar_init(&sh.b_empty[i], 1);
        for (int i = 0; i < 2; ++i) bar_init(&sh.s_full[i], 1);
        bar_init(&sh.dp_full, 1);
        bar_init(&sh.ds_ready, kCompute);
        bar_init(&sh.done, 1);
        bar_init_done();
    }
    if (warp == 0) tmem_alloc(&sh.tmem, C::kCols);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    // columns: S and dS of even tiles, of odd ones, dP, dQ
    const uint32_t tmem = sh.tmem, dp_at = tmem + 2 * TN, dq_at = tmem + 3 * TN;

    if (warp == 8) {
        // ---- loads: Q and dO, then K and V tiles ----
        if (lane == 0 && n_tiles > 0) {
            const uint32_t box = C::kHalves * (uint32_t)(tokens * group) * 128;
            bar_expect(&sh.resident, 2 * box);
            load_tile<HD>(smem, 16384, &mq, hk * group, it.q0, &sh.resident);
            load_tile<HD>(smem + C::kTileBytes, 16384, &mg, hk * group, it.q0, &sh.resident);
            int na = 0, nb = 0;
            for (int n = 0; n < n_tiles; ++n) {
                const int sa = n % C::kA, sb = n % C::kB;
                if (n >= C::kA && !bar_wait(&sh.a_empty[sa], (n / C::kA - 1) & 1, stop)) break;
                bar_expect(&sh.a_full[sa], C::kUnit);
                load_tile<HD>(ring_a + sa * C::kUnit, C::kSlab, &mk, hk, it.k0 + n * TN,
                              &sh.a_full[sa]);
                ++na;
                if (n >= C::kB && !bar_wait(&sh.b_empty[sb], (n / C::kB - 1) & 1, stop)) break;
                bar_expect(&sh.b_full[sb], C::kUnit);
                load_tile<HD>(ring_b + sb * C::kUnit, C::kSlab, &mv, hk, it.k0 + n * TN,
                              &sh.b_full[sb]);
                ++nb;
            }
            loads_landed<C>(sh, na, nb);
        }
    } else if (warp == 9) {
        // ---- products ----
        if (lane == 0 && n_tiles > 0) {
            const uint32_t q_at = smem_addr(smem), g_at = q_at + C::kTileBytes;
            const uint32_t a_at = smem_addr(ring_a), b_at = smem_addr(ring_b);
            auto a_buf = [&](int n) { return a_at + (n % C::kA) * C::kUnit; };
            auto b_buf = [&](int n) { return b_at + (n % C::kB) * C::kUnit; };
            auto s_buf = [&](int n) { return tmem + (n & 1) * TN; };
            auto have_a = [&](int n) {
                return bar_wait(&sh.a_full[n % C::kA], (n / C::kA) & 1, stop);
            };
            auto have_b = [&](int n) {
                return bar_wait(&sh.b_full[n % C::kB], (n / C::kB) & 1, stop);
            };
            bool ok = bar_wait(&sh.resident, 0, stop) && have_a(0) && have_b(0) &&
                      (n_tiles == 1 || have_a(1));
            if (ok) {
                tc_after_sync();
                mma_rows<HD, TN>(s_buf(0), q_at, a_buf(0));
                tc_commit(&sh.s_full[0]);
                mma_rows<HD, TN>(dp_at, g_at, b_buf(0));
                tc_commit(&sh.dp_full);
                if (n_tiles > 1) {
                    mma_rows<HD, TN>(s_buf(1), q_at, a_buf(1));
                    tc_commit(&sh.s_full[1]);
                }
            }
            for (int n = 0; ok && n < n_tiles; ++n) {
                const bool more = n + 1 < n_tiles, more2 = n + 2 < n_tiles;
                if (!(ok = (!more || have_b(n + 1)) && bar_wait(&sh.ds_ready, n & 1, stop)))
                    break;
                tc_after_sync();
                if (more) {   // dP(n) was read before dS(n) was announced
                    mma_rows<HD, TN>(dp_at, g_at, b_buf(n + 1));
                    tc_commit(&sh.dp_full);
                }
                mma_columns<HD, TN>(dq_at, s_buf(n), a_buf(n), n > 0);
                if (twice) mma_columns<HD, TN>(dq_at, s_buf(n) + TN / 4, a_buf(n), true);
                tc_commit(&sh.a_empty[n % C::kA]);
                if (more2) {
                    if (!(ok = have_a(n + 2))) break;
                    mma_rows<HD, TN>(s_buf(n), q_at, a_buf(n + 2));
                    tc_commit(&sh.s_full[n & 1]);
                }
            }
            // the products must end before their memory is freed, also where the
            // other warps have given up
            int never = 0;
            tc_commit(&sh.done);
            bar_wait(&sh.done, 0, &never);
        }
    } else {
        // ---- P and dS: thread = half a row ----
        const int half = warp >> 2;
        // the keys that the row sees, counted from k0: see0 .. see1
        const bool live = range.live();
        const int see0 = live ? range.lo - it.k0 : 0, see1 = live ? range.hi - it.k0 : 0;
        if (see1 <= see0) st = make_float2(INFINITY, 0.f);
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const float c = a.scale * kLog2e;
        const float2 c2 = make_float2(c, c), l2 = make_float2(-st.x, -st.x);
        float2 ds_sum = make_float2(0.f, 0.f);
        bool ok = true;
        for (int n = 0; n < n_tiles; ++n) {
            ok = ok && bar_wait(&sh.s_full[n & 1], (n >> 1) & 1, stop);
            ok = __all_sync(0xffffffffu, ok) != 0;
            tc_after_sync();
            float s[C::kChunks][32], d[C::kChunks][32];
            const uint32_t s_at = tmem + (n & 1) * TN + half * (TN / 2) + lanes;
            load_columns(s_at, s);
            const int first = n * TN + half * (TN / 2);
            if (__any_sync(0xffffffffu, see0 > first || see1 < first + TN / 2)) {
#pragma unroll
                for (int i = 0; i < C::kChunks; ++i)
                    hide(s[i], see0 - first - 32 * i, see1 - first - 32 * i);
            }
#pragma unroll
            for (int i = 0; i < C::kChunks; ++i) {
                float2 x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    x[e] = fma2(make_float2(s[i][2 * e], s[i][2 * e + 1]), c2, l2);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    s[i][2 * e] = exp2_fast(x[e].x);
                    s[i][2 * e + 1] = exp2_fast(x[e].y);
                }
            }
            ok = ok && bar_wait(&sh.dp_full, n & 1, stop);
            ok = __all_sync(0xffffffffu, ok) != 0;
            if (threadIdx.x == 0) bar_arrive(&sh.b_empty[n % C::kB]);   // and that V
            tc_after_sync();
            load_columns(dp_at + half * (TN / 2) + lanes, d);
            if (n_tiles == 1) {
                // the row's whole range is here: delta = sum_j p dp, the same sum
                // without out's rounding to bf16
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < C::kChunks; ++i)
#pragma unroll
                    for (int e = 0; e < 32; e += 2)
                        sum = fma2(make_float2(s[i][e], s[i][e + 1]),
                                   make_float2(d[i][e], d[i][e + 1]), sum);
                sh.part[half][r] = sum.x + sum.y;
                part_sync(1, kCompute);
                const float delta = sh.part[0][r] + sh.part[1][r];
                if (isfinite(delta)) st.y = delta;   // a masked dp may not be
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
            if (n_tiles > 1) {
#pragma unroll
                for (int i = 0; i < C::kChunks; ++i)
#pragma unroll
                    for (int e = 0; e < 32; e += 2)
                        ds_sum = add2(ds_sum, make_float2(d[i][e], d[i][e + 1]));
            }
            store_bf16(s_at, d);
            if (twice) {
                bf16_rest(d);
                store_bf16(s_at + TN / 4, d);
            }
            tmem_wait_store();
            tc_before_sync();
            bar_arrive(&sh.ds_ready);
            if (!ok) break;
        }
        // For dK and dV: with sum_j p = 1, sum_j ds is what delta was short of for
        // out's rounding to bf16.
        if (n_tiles > 1) sh.part[half][r] = ds_sum.x + ds_sum.y;
        const bool lost = part_any(1, kCompute, !ok);
        if (n_tiles > 1) {
            const float rest = sh.part[0][r] + sh.part[1][r];
            if (isfinite(rest)) st.y += rest;
        }
        // Tokens in no sequence get L = +infinity: their rows may hold anything.
        if (!lost && half == 0 && tok < tokens && token < a.q_tokens) p.stats[at_stats] = st;
        // ---- epilogue: each half stages its half of the columns ----
        const bool any = n_tiles > 0;
        // (an issuing thread that gave up has announced its end, too)
        ok = ok && (!any || (bar_wait(&sh.done, 0, stop) && !*stop));
        ok = __all_sync(0xffffffffu, ok) != 0;
        tc_after_sync();
        bool fine = true;
        if (ok)
            fine = stage_row<HD / 2>(dq_at + half * (HD / 2) + lanes, smem, r, half * (HD / 16),
                                     a.scale, any);
        // rows that hold no token (128 is not a multiple of the group) come from what shared
        // memory held before
        fine = fine || tok >= tokens;
        // a row that is not to be stored now: dead, or to be computed again
        sh.bad[half][r] = !ok || !live || !fine;
        fence_async();
        // rows past the tile or the tensor are left out by the store itself
        if (!part_any(1, kCompute,
                      !ok || !fine || (!live && tok < tokens && token < a.q_tokens))) {
            if (threadIdx.x == 0) store_tile<HD>(&mdq, smem, hk * group, it.q0);
        } else {
            store_rows<HD, 16>(smem, warp * 16, a.dim, [&](int i) -> bf16* {
                const int t = i / group;
                return sh.bad[0][i] | sh.bad[1][i]
                           ? nullptr
                           : a.dq.at(it.q0 + t, hk * group + i - t * group);
            });
        }
        // the two warps that hold a row's halves take 16 of their 32 rows each
        const bool again = live && (sh.bad[0][r] | sh.bad[1][r]);
        if (__any_sync(0xffffffffu, again))
            dq_rows<HD>(a, hk, token, h, range.lo, range.hi, again, st, half);
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    if (warp == 0) tmem_free(tmem, C::kCols);
    if (threadIdx.x == 0 && *stop) report_stop(a.status);
}

template <int HD, int TN>
__global__ void __launch_bounds__(Cfg<HD, TN>::kThreadsKV, Cfg<HD, TN>::kCtas)
k_attention_dkv(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mg,
                const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                const __grid_constant__ CUtensorMap mdk, const __grid_constant__ CUtensorMap mdv,
                const __grid_constant__ Attn a, const __grid_constant__ Plan p) {
    pdl_prologue();
    using C = Cfg<HD, TN>;
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared<TN>& sh = *reinterpret_cast<Shared<TN>*>(smem + C::kSmem);
    volatile int* stop = &sh.stop;
    const int item = blockIdx.x / a.kv_heads, hk = blockIdx.x - item * a.kv_heads;
    const Item it = p.key_items[item];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = a.group, tokens = p.key_tokens, n_tiles = it.t1;
    const int rows = tokens * group;   // of a query tile

    // the thread's key and who sees it; asked for before the loads begin
    const int r = (warp & 3) * 32 + lane, key = it.k0 + r;
    Range range{0, -1};
    if (warp < 8 && key < a.k_tokens) range = p.k_range[key];

    uint8_t* ring_a = smem + 2 * C::kTileBytes;
    uint8_t* ring_b = ring_a + C::kA * C::kUnit;
    if (threadIdx.x == 0) {
        prefetch_map(&mq);
        prefetch_map(&mg);
        prefetch_map(&mk);
        prefetch_map(&mv);
        prefetch_map(&mdk);
        prefetch_map(&mdv);
        *stop = 0;
        bar_init(&sh.resident, 1);
        for (int i = 0; i < C::kA; ++i) bar_init(&sh.a_full[i], 1), bar_init(&sh.a_empty[i], 1);
        for (int i = 0; i < C::kB; ++i) bar_init(&sh.b_full[i], 1), bar_init(&sh.b_empty[i], 1);
        bar_init(&sh.s_full[0], 1);
        bar_init(&sh.dp_full, 1);
        bar_init(&sh.p_ready, kCompute);
        bar_init(&sh.ds_ready, kCompute);
        for (int i = 0; i < 2; ++i) {
            bar_init(&sh.stats_full[i], 32);
            bar_init(&sh.stats_free[i], kCompute);
        }
        bar_init(&sh.done, C::kIssuers);
        bar_init(&sh.turn[0], 1);
        bar_init(&sh.turn[1], 1);
        bar_init_done();
    }
    // rows that no load writes (TN is not a multiple of the group) enter the
    // products as zeros
    for (int i = threadIdx.x; i < (C::kA + C::kB) * C::kHalves * (TN - rows) * 8;
         i += C::kThreadsKV) {
        const int slab = i / ((TN - rows) * 8), at = i - slab * (TN - rows) * 8;
        reinterpret_cast<uint4*>(ring_a + slab * C::kSlab + rows * 128)[at] =
            make_uint4(0, 0, 0, 0);
    }
    fence_async();
    if (warp == 0) tmem_alloc(&sh.tmem, C::kCols);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    // columns: S and P, dP and dS, dV, dK
    const uint32_t tmem = sh.tmem, dp_at = tmem + TN, dv_at = tmem + 2 * TN, dk_at = dv_at + HD;

    if (warp == 8) {
        // ---- loads: K and V, then Q and dO tiles, with their L and delta ----
        if (lane == 0 && n_tiles > 0) {
            bar_expect(&sh.resident, 2 * C::kTileBytes);
            load_tile<HD>(smem, 16384, &mk, hk, it.k0, &sh.resident);
            load_tile<HD>(smem + C::kTileBytes, 16384, &mv, hk, it.k0, &sh.resident);
        }
        const uint32_t box = C::kHalves * (uint32_t)rows * 128;
        const float2* from = p.stats + ((int64_t)hk * a.q_tokens + it.q0) * group;
        const int64_t end = (int64_t)(a.q_tokens - it.q0) * group;
        int na = 0, nb = 0;
        bool ok = true;
        for (int n = 0; n < n_tiles; ++n) {
            if (lane == 0) {
                const int sa = n % C::kA, sb = n % C::kB;
                ok = n < C::kA || bar_wait(&sh.a_empty[sa], (n / C::kA - 1) & 1, stop);
                if (ok) {
                    bar_expect(&sh.a_full[sa], box);
                    load_tile<HD>(ring_a + sa * C::kUnit, C::kSlab, &mq, hk * group,
                                  it.q0 + n * tokens, &sh.a_full[sa]);
                    ++na;
                    ok = n < C::kB || bar_wait(&sh.b_empty[sb], (n / C::kB - 1) & 1, stop);
                }
                if (ok) {
                    bar_expect(&sh.b_full[sb], box);
                    load_tile<HD>(ring_b + sb * C::kUnit, C::kSlab, &mg, hk * group,
                                  it.q0 + n * tokens, &sh.b_full[sb]);
                    ++nb;
                }
            }
            const int b = n & 1;
            ok = ok && (n < 2 || bar_wait(&sh.stats_free[b], ((n >> 1) - 1) & 1, stop));
            if (!__all_sync(0xffffffffu, ok)) break;
#pragma unroll
            for (int i = 0; i < TN; i += 32) {
                const int row = i + lane;
                const int64_t at = (int64_t)n * rows + row;
                float2 st = make_float2(INFINITY, 0.f);
                if (row < rows && at < end) st = from[at];
                sh.lse[b][row] = st.x - kLift;
                sh.delta[b][row] = st.y;
            }
            bar_arrive(&sh.stats_full[b]);
        }
        if (lane == 0 && n_tiles > 0) loads_landed<C>(sh, na, nb);
    } else if (warp >= 9) {
        // ---- products ----
        if (lane == 0 && n_tiles > 0) {
            const uint32_t k_at = smem_addr(smem), v_at = k_at + C::kTileBytes;
            const uint32_t a_at = smem_addr(ring_a), b_at = smem_addr(ring_b);
            constexpr int kS = HD / 16;
            auto a_buf = [&](int n) { return a_at + (n % C::kA) * C::kUnit; };
            auto b_buf = [&](int n) { return b_at + (n % C::kB) * C::kUnit; };
            auto have_a = [&](int n) {
                return bar_wait(&sh.a_full[n % C::kA], (n / C::kA) & 1, stop);
            };
            auto have_b = [&](int n) {
                return bar_wait(&sh.b_full[n % C::kB], (n / C::kB) & 1, stop);
            };
            auto my_turn = [&](int i, int n) {
                return C::kIssuers == 1 || n < 0 || bar_wait(&sh.turn[i], n & 1, stop);
            };
            auto hand_over = [&](int i) {
                if (C::kIssuers == 2) bar_arrive(&sh.turn[i]);
            };
            const bool x = C::kIssuers == 1 || warp == 9, y = C::kIssuers == 1 || warp == 10;
            bool ok = bar_wait(&sh.resident, 0, stop);
            if (ok && x && (ok = have_a(0))) {
                tc_after_sync();
                mma_rows<HD, TN>(tmem, k_at, a_buf(0));
                tc_commit(&sh.s_full[0]);
            }
            if (ok && y && (ok = have_b(0))) {
                tc_after_sync();
                mma_rows<HD, TN>(dp_at, v_at, b_buf(0));
                tc_commit(&sh.dp_full);
            }
            for (int n = 0; ok && n < n_tiles; ++n) {
                const bool more = n + 1 < n_tiles;
                if (x) {   // dV += P(n) dO(n), then S(n + 1) over P(n)
                    if (!(ok = have_b(n) && (!more || have_a(n + 1)) &&
                               bar_wait(&sh.p_ready, n & 1, stop) && my_turn(0, n - 1)))
                        break;
                    tc_after_sync();
                    mma_columns<HD, TN>(dv_at, tmem, b_buf(n), n > 0);
                    if (more) {
                        mma_rows<HD, TN>(tmem, k_at, a_buf(n + 1), 0, kS - kAhead);
                        hand_over(1);
                        mma_rows<HD, TN>(tmem, k_at, a_buf(n + 1), kS - kAhead, kS);
                        tc_commit(&sh.s_full[0]);
                    } else {
                        hand_over(1);
                    }
                }
                if (y) {   // dK += dS(n) Q(n), then dP(n + 1) over dS(n)
                    if (!(ok = have_a(n) && (!more || have_b(n + 1)) &&
                               bar_wait(&sh.ds_ready, n & 1, stop) && my_turn(1, n)))
                        break;
                    tc_after_sync();
                    mma_columns<HD, TN>(dk_at, dp_at, a_buf(n), n > 0);
                    if (more) {
                        mma_rows<HD, TN>(dp_at, v_at, b_buf(n + 1), 0, kS - kAhead);
                        hand_over(0);
                        mma_rows<HD, TN>(dp_at, v_at, b_buf(n + 1), kS - kAhead, kS);
                        tc_commit(&sh.dp_full);
                    } else {
                        hand_over(0);
                    }
                }
            }
            // the products must end before their memory is freed, also where the
            // other warps have given up
            int never = 0;
            tc_commit(&sh.done);
            bar_wait(&sh.done, 0, &never);
        }
    } else {
        // ---- P and dS, transposed: thread = half of a key's row ----
        const int half = warp >> 2;
        // the rows of the query side that see this key, counted from q0: see0 .. see1
        const bool live = range.live();
        const int64_t see0 = live ? (int64_t)(range.lo - it.q0) * group : 0;
        const int64_t see1 = live ? (int64_t)(range.hi - it.q0) * group : 0;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const uint32_t s_at = tmem + half * (TN / 2) + lanes;
        const uint32_t d_at = dp_at + half * (TN / 2) + lanes;
        const float c = a.scale * kLog2e;
        const float2 c2 = make_float2(c, c);
        bool ok = true;
        for (int n = 0; n < n_tiles; ++n) {
            const int b = n & 1;
            ok = bar_wait(&sh.stats_full[b], (n >> 1) & 1, stop) &&
                 bar_wait(&sh.s_full[0], n & 1, stop);
            if (!__all_sync(0xffffffffu, ok)) break;
            // S(n) came after dV(n - 1): that dO may be overwritten
            if (threadIdx.x == 0 && n >= 1) bar_arrive(&sh.b_empty[(n - 1) % C::kB]);
            tc_after_sync();
            float s[C::kChunks][32], d[C::kChunks][32];
            load_columns(s_at, s);
            const int64_t from = (int64_t)n * rows + half * (TN / 2);
            const int lo = (int)max((int64_t)0, min((int64_t)TN, see0 - from));
            const int hi = (int)max((int64_t)0, min((int64_t)TN, see1 - from));
            if (__any_sync(0xffffffffu, lo > 0 || hi < TN / 2)) {
#pragma unroll
                for (int i = 0; i < C::kChunks; ++i) hide(s[i], lo - 32 * i, hi - 32 * i);
            }
            const float4* l4 = reinterpret_cast<const float4*>(&sh.lse[b][half * (TN / 2)]);
            const float4* e4 = reinterpret_cast<const float4*>(&sh.delta[b][half * (TN / 2)]);
#pragma unroll
            for (int i = 0; i < C::kChunks; ++i) {
                float2 x[16];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float4 l = l4[8 * i + e];
                    x[2 * e] = fma2(make_float2(s[i][4 * e], s[i][4 * e + 1]), c2,
                                    make_float2(-l.x, -l.y));
                    x[2 * e + 1] = fma2(make_float2(s[i][4 * e + 2], s[i][4 * e + 3]), c2,
                                        make_float2(-l.z, -l.w));
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    s[i][2 * e] = exp2_fast(x[e].x);
                    s[i][2 * e + 1] = exp2_fast(x[e].y);
                }
            }
            store_bf16(s_at, s);
            tmem_wait_store();
            tc_before_sync();
            bar_arrive(&sh.p_ready);
            ok = bar_wait(&sh.dp_full, n & 1, stop);
            if (!__all_sync(0xffffffffu, ok)) break;
            // dP(n) came after dK(n - 1): that Q may be overwritten
            if (threadIdx.x == 0 && n >= 1) bar_arrive(&sh.a_empty[(n - 1) % C::kA]);
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
            bar_arrive(&sh.stats_free[b]);
            store_bf16(d_at, d);
            tmem_wait_store();
            tc_before_sync();
            bar_arrive(&sh.ds_ready);
        }
        // ---- epilogue: the first four warps stage dV, the others dK ----
        const bool any = n_tiles > 0;
        // (an issuing thread that gave up has announced its end, too)
        ok = ok && (!any || (bar_wait(&sh.done, 0, stop) && !*stop));
        ok = __all_sync(0xffffffffu, ok) != 0;
        tc_after_sync();
        bool fine = true;
        uint8_t* tile = smem + half * C::kTileBytes;
        if (ok)
            fine = stage_row<HD>((half == 0 ? dv_at : dk_at) + lanes, tile, r, 0,
                                 half == 0 ? kUnlift : a.scale * kUnlift, any);
        sh.bad[half][r] = !ok || !live || !fine;
        fence_async();
        if (!part_any(1, kCompute, !ok || !fine || (!live && key < a.k_tokens))) {
            if (r == 0) store_tile<HD>(half == 0 ? &mdv : &mdk, tile, hk, it.k0);
        } else {
            store_rows<HD, 32>(tile, (warp & 3) * 32, a.dim, [&](int i) -> bf16* {
                return sh.bad[half][i] ? nullptr : (half == 0 ? a.dv : a.dk).at(it.k0 + i, hk);
            });
        }
        const bool again = live && sh.bad[half][r];
        if (__any_sync(0xffffffffu, again)) {
            if (half == 0)
                dkv_rows<HD, false>(a, p.stats, hk, key, range.lo, range.hi, again);
            else
                dkv_rows<HD, true>(a, p.stats, hk, key, range.lo, range.hi, again);
        }
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    if (warp == 0) tmem_free(tmem, C::kCols);
    if (threadIdx.x == 0 && *stop) report_stop(a.status);
}

template <int HD, int TN>
cudaError_t launch(const Attn& a, const Plan& p, cudaStream_t st) {
    using C = Cfg<HD, TN>;
    auto* dq = k_attention_dq<HD, TN>;
    auto* dkv = k_attention_dkv<HD, TN>;
    constexpr int kSmem = C::kSmem + (int)sizeof(Shared<TN>);
    static std::atomic<uint64_t> ready[2];
    cudaError_t e = allow_smem(dq, kSmem, &ready[0]);
    if (e == cudaSuccess) e = allow_smem(dkv, kSmem, &ready[1]);
    CUtensorMap mq, mg, mk, mv, mx, my;
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
        queries(&mx, a.dq, p.tokens);
        if (e == cudaSuccess)
            e = launch_k(dq, dim3((unsigned)p.most_items * a.kv_heads), dim3(C::kThreads), kSmem,
                         st, mq, mg, mk, mv, mx, a, p);
    }
    if (a.k_tokens > 0) {
        queries(&mq, a.q, p.key_tokens);
        queries(&mg, a.grad, p.key_tokens);
        keys(&mk, a.k, kTile);
        keys(&mv, a.v, kTile);
        keys(&mx, a.dk, kTile);
        keys(&my, a.dv, kTile);
        if (e == cudaSuccess)
            e = launch_k(dkv, dim3((unsigned)p.key_tiles * a.kv_heads), dim3(C::kThreadsKV),
                         kSmem, st, mq, mg, mk, mv, mx, my, a, p);
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
