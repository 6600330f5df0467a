// Attention over packed sequences, forward, on the tensor cores.
//
// For a tile of 128 query rows and the keys in tiles of 128:
//   S = Q K^T (fp32 in tensor memory),  P = exp2(c S - c m),  O += P V,
// c = scale * log2 e, m a running row maximum.  The 128 rows are the `group`
// query heads of 128 / group tokens: heads that share a key head share its
// tile, so a single new token's heads fill rows of one tile and K and V are
// read once.  K and V tiles arrive by TMA through a ring of shared-memory
// units; rows past a tensor's end arrive as zeros, rows of a neighbouring
// sequence are masked.
//
// Roles: one warp loads, one thread per query tile issues its products, four
// warps per tile do the softmax, a thread to a row (tensor-memory lane).  With two tiles
// to a CTA (NQ = 2) one tile's softmax runs under the other's products and both
// read the same K and V from shared memory; with one (NQ = 1) two CTAs share
// an SM.  P overwrites S in tensor memory, as bf16, and is the first operand of
// the second product from there.
//
// The running maximum is only raised when a row's new maximum exceeds it by
// more than 8 (in powers of two): until then P is at most 256, far inside
// bf16 and fp32, and the accumulator needs no rescaling.  The order "O += P V
// of tile j, then S of tile j + 1" makes one barrier say both that S is ready
// and that O may be touched.
//
// A row (or a piece of one) whose result is not finite is computed again
// (attention_rows.cuh): a product with a zero probability takes up an infinite or
// NaN value behind the mask.  So is a row whose tile did not come to its end (a
// wait gave up).
#include <atomic>

#include "attention_rows.cuh"
#include "attention_tma.h"
#include "tc.cuh"

namespace pss {
namespace seq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;   // see above

template <int HD, int NQ>
struct Cfg {
    static constexpr int kHalves = HD / 64;
    static constexpr int kUnit = kHalves * 16384;                      // one K or V tile
    static constexpr int kUnits = HD == 128 ? (NQ == 2 ? 4 : 2) : (NQ == 2 ? 8 : 4);
    static constexpr int kQ = NQ * kUnit;
    static constexpr int kSmem = kQ + kUnits * kUnit;
    static constexpr int kCols = NQ == 2 ? 512 : 256;                  // tensor-memory columns
    static constexpr int kO = NQ * 128;                                // O's first column
    // NQ = 2: three whole warpgroups, so that the two of the softmax can take
    // registers from the third (set_registers)
    static constexpr int kThreads = NQ == 2 ? 384 : 192;
    // registers a thread that the launch has to bring for the split
    static constexpr int kMore = 224, kLess = 56;
    static constexpr int kLaunch = NQ == 2 ? (2 * kMore + kLess) / 3 : 0;
};

template <int HD, int NQ>
__global__ void __launch_bounds__(Cfg<HD, NQ>::kThreads, NQ == 1 ? 2 : 1)
k_attention_forward(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                    const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mo,
                    const __grid_constant__ Attn a, const __grid_constant__ Plan p) {
    pdl_prologue();
    using C = Cfg<HD, NQ>;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ uint64_t q_full, full[C::kUnits], empty[C::kUnits], s_full[NQ], p_ready[NQ],
        drained[NQ], turn[2];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int stop;
    __shared__ bool keep[NQ][kTile];   // rows to be stored
    const int item = blockIdx.x / a.kv_heads, hk = blockIdx.x - item * a.kv_heads;
    if (p.most_slots > 0 && item >= p.head->items) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = a.group, tokens = p.tokens;
    Item it;
    if (NQ == 1 && p.direct) {
        it.q0 = item * tokens;
        it.k0 = range_of<false>(a, it.q0, a.q_off, a.k_off).lo;
        const int last = min(it.q0 + tokens, a.q_tokens) - 1;
        const int keys = range_of<false>(a, last, a.q_off, a.k_off).end() - it.k0;
        it.t0 = 0;
        it.t1 = keys > 0 ? (keys + kTile - 1) / kTile : 0;
        it.slot = -1;
    } else {
        it = p.items[item];
    }

    // key tiles of each query tile: t0 <= t < end[t]
    int end[NQ];
    end[NQ - 1] = it.t1;
    if (NQ == 2) {
        const int last = it.q0 + tokens - 1;
        const int n = last < a.q_tokens ? p.q_range[last].end() - it.k0 : 0;
        end[0] = last < a.q_tokens ? max(it.t0, min(it.t1, (n + kTile - 1) / kTile)) : it.t1;
        if (it.q0 + tokens >= a.q_tokens) end[1] = it.t0;
    }
    const int most = NQ == 2 ? max(end[0], end[NQ - 1]) : end[0];

    // the softmax's row; asked for first, the loads behind it take a while
    const int row = threadIdx.x & 127, tile = NQ == 2 ? (warp >> 2) & 1 : 0;
    const int row_tok = row / group, row_h = hk * group + row - row_tok * group;
    const int token = it.q0 + tile * tokens + row_tok;
    Range range{0, -1};
    if (warp < NQ * 4 && row_tok < tokens && token < a.q_tokens)
        range = NQ == 1 && p.direct ? range_of<false>(a, token, a.q_off, a.k_off)
                                    : p.q_range[token];

    uint8_t* ring = smem + C::kQ;
    if (threadIdx.x == 0) {
        prefetch_map(&mq);
        prefetch_map(&mk);
        prefetch_map(&mv);
        prefetch_map(&mo);
        stop = 0;
        bar_init(&q_full, 1);
        for (int i = 0; i < C::kUnits; ++i) {
            bar_init(&full[i], 1);
            bar_init(&empty[i], NQ);
        }
        for (int t = 0; t < NQ; ++t) {
            bar_init(&s_full[t], 1);
            bar_init(&drained[t], 1);
            bar_init(&turn[t], 1);
            bar_init(&p_ready[t], 128);
        }
        bar_init_done();
    }
    if (warp == 0) tmem_alloc(&tmem_at, C::kCols);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = tmem_at;

    // NQ = 2: 3 x 168 registers a thread at launch = 2 x 224 + 56 (kLaunch)
    if (warp == NQ * 4) {
        // ---- loads: Q, then K and V tiles in turn ----
        if (NQ == 2) set_registers<C::kLess, false>();
        if (lane == 0 && most > it.t0) {
            const uint32_t box = (uint32_t)(tokens * group) * 128;
            bar_expect(&q_full, NQ * C::kHalves * box);
            for (int t = 0; t < NQ; ++t)
                for (int h = 0; h < C::kHalves; ++h)
                    tma_load3(smem + t * C::kUnit + h * 16384, &mq, 64 * h, hk * group,
                              it.q0 + t * tokens, &q_full);
            const int units = 2 * (most - it.t0);
            int u = 0;
            for (; u < units; ++u) {
                const int slot = u % C::kUnits, turn = u / C::kUnits;
                if (turn > 0 && !bar_wait(&empty[slot], (turn - 1) & 1, &stop)) break;
                bar_expect(&full[slot], C::kUnit);
                for (int h = 0; h < C::kHalves; ++h)
                    tma_load3(ring + slot * C::kUnit + h * 16384, u & 1 ? &mv : &mk, 64 * h, hk,
                              it.k0 + (it.t0 + u / 2) * kTile, &full[slot]);
                // a query tile that does not use this unit frees it at once
                if (NQ == 2 && it.t0 + u / 2 >= end[0]) bar_arrive(&empty[slot]);
                if (NQ == 2 && it.t0 + u / 2 >= end[1]) bar_arrive(&empty[slot]);
            }
            // the loads must land before the CTA ends, also where nobody waits for them
            int never = 0;
            bar_wait(&q_full, 0, &never);
            for (int w = max(0, u - C::kUnits); w < u; ++w)
                bar_wait(&full[w % C::kUnits], (w / C::kUnits) & 1, &never);
        }
    } else if (warp > NQ * 4 && warp <= NQ * 5) {
        // ---- products: a thread to a query tile, in turns (kAhead) ----
        if (NQ == 2) set_registers<C::kLess, false>();
        const int t = warp - NQ * 4 - 1;
        const int steps = (t == 0 ? end[0] : end[NQ - 1]) - it.t0;
        const int others = NQ == 1 ? 0 : (t == 0 ? end[NQ - 1] : end[0]) - it.t0;
        if (lane == 0 && steps > 0) {
            constexpr uint32_t kQK = mma_desc(128, 128, false), kPV = mma_desc(128, HD, true);
            constexpr int kS = HD / 16;
            const uint32_t q_at = smem_addr(smem) + t * C::kUnit, ring_at = smem_addr(ring);
            const uint32_t s_at = tmem + t * 128, o_at = tmem + C::kO + t * HD;
            auto loaded = [&](int u) {
                return bar_wait(&full[u % C::kUnits], (u / C::kUnits) & 1, &stop);
            };
            auto scores = [&](int u, int from, int to) {
                const uint32_t k_at = ring_at + (u % C::kUnits) * C::kUnit;
#pragma unroll
                for (int i = from; i < to; ++i) {
                    const uint32_t off = (i / 4) * 16384 + (i % 4) * 32;
                    mma_ss(s_at, smem_desc(q_at + off, 16), smem_desc(k_at + off, 16), kQK, i > 0);
                }
            };
            auto values = [&](int u, int from, int to) {
                const uint32_t v_at = ring_at + (u % C::kUnits) * C::kUnit;
#pragma unroll
                for (int i = from; i < to; ++i)
                    mma_ts(o_at, s_at + i * 8, smem_desc(v_at + i * 2048, 16384), kPV,
                           u > 1 || i > 0);
            };
            bool ok = bar_wait(&q_full, 0, &stop) && loaded(0);
            if (ok) {
                tc_after_sync();
                scores(0, 0, kS);
                tc_commit(&s_full[t]);
            }
            for (int n = 0; ok && n < steps; ++n) {
                const bool more = n + 1 < steps;
                ok = loaded(2 * n + 1) && (!more || loaded(2 * n + 2)) &&
                     bar_wait(&p_ready[t], n & 1, &stop);
                // the other tile's products before these: of step n, or of n - 1
                const int before = t == 0 ? n - 1 : n;
                if (ok && before >= 0 && before < others)
                    ok = bar_wait(&turn[t], before & 1, &stop);
                if (!ok) break;
                tc_after_sync();
                if (more) {
                    values(2 * n + 1, 0, 8);
                    scores(2 * n + 2, 0, kS - kAhead);
                    if (NQ == 2) bar_arrive(&turn[t ^ 1]);
                    scores(2 * n + 2, kS - kAhead, kS);
                } else {
                    values(2 * n + 1, 0, 8 - kAhead);
                    if (NQ == 2) bar_arrive(&turn[t ^ 1]);
                    values(2 * n + 1, 8 - kAhead, 8);
                }
                tc_commit(&s_full[t]);
            }
            // the products must end before their memory is freed, also where the
            // softmax has given up
            int never = 0;
            tc_commit(&drained[t]);
            bar_wait(&drained[t], 0, &never);
        }
    } else if (warp < NQ * 4) {
        // ---- softmax: thread = row ----
        if (NQ == 2) set_registers<C::kMore, true>();
        const int t = tile, r = row, h = row_h;
        // the keys that the row sees, counted from k0: see0 .. see1
        const bool live = range.live();
        const int see0 = live ? range.lo - it.k0 : 0, see1 = live ? range.hi - it.k0 : 0;
        const int stop_at = NQ == 2 && t == 1 ? end[NQ - 1] : end[0];
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const uint32_t s_at = tmem + t * 128 + lanes, o_at = tmem + C::kO + t * HD + lanes;
        const float c = a.scale * kLog2e;
        float top = -INFINITY, sum = 0.f;
        bool ok = true;
        for (int j = it.t0; j < stop_at; ++j) {
            const int n = j - it.t0;
            ok = bar_wait(&s_full[t], n & 1, &stop);
            if (!__all_sync(0xffffffffu, ok)) break;
            // this query tile's products up to S(n) have ended: it frees K(n), V(n - 1)
            if (row == 0) {
                bar_arrive(&empty[(2 * n) % C::kUnits]);
                if (n > 0) bar_arrive(&empty[(2 * n - 1) % C::kUnits]);
            }
            tc_after_sync();
            float s[4][32];
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_load32(s_at + 32 * i, s[i]);
            tmem_wait_load();
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_loaded(s[i]);
            const int lo = see0 - j * kTile, hi = see1 - j * kTile;
            if (__any_sync(0xffffffffu, lo > 0 || hi < kTile)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) hide(s[i], lo - 32 * i, hi - 32 * i);
            }
            // eight chains side by side: one warp of a tile runs alone on its scheduler
            float m8[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) m8[i] = fmaxf(s[i >> 1][i & 1], s[i >> 1][2 + (i & 1)]);
#pragma unroll
            for (int e = 4; e < 32; e += 4)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    m8[i] = max3(m8[i], s[i >> 1][e + (i & 1)], s[i >> 1][e + 2 + (i & 1)]);
            const float m = fmaxf(max3(m8[0], m8[1], m8[2]),
                                  fmaxf(max3(m8[3], m8[4], m8[5]), fmaxf(m8[6], m8[7])));
            const bool raise = m * c > top * c + kSlack;   // also the first finite maximum
            if (__any_sync(0xffffffffu, raise)) {
                const float keep = raise ? (top == -INFINITY ? 0.f : exp2_fast((top - m) * c)) : 1.f;
                if (raise) top = m;
                sum *= keep;
                if (n > 0) {
#pragma unroll 1
                    for (int i = 0; i < HD; i += 32) {
                        float o[32];
                        tmem_load32(o_at + i, o);
                        tmem_wait_load();
                        tmem_loaded(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] *= keep;
                        tmem_store32(o_at + i, o);
                    }
                }
            }
            const float base = top == -INFINITY ? 0.f : -top * c;
            const float2 c2 = make_float2(c, c), base2 = make_float2(base, base);
            float2 add[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) add[i] = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    x[e] = fma2(make_float2(s[i][2 * e], s[i][2 * e + 1]), c2, base2);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    x[e].x = exp2_fast(x[e].x);
                    x[e].y = exp2_fast(x[e].y);
                }
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    add[e & 3] = add2(add[e & 3], x[e]);
                    w[e] = pack2(x[e].x, x[e].y, bf16());
                }
                tmem_store16(s_at + 16 * i, w);
            }
            add[0] = add2(add2(add[0], add[1]), add2(add[2], add[3]));
            sum += add[0].x + add[0].y;
            tmem_wait_store();
            tc_before_sync();
            bar_arrive(&p_ready[t]);
        }
        // ---- epilogue ----
        const bool any = stop_at > it.t0;
        if (any) {
            ok = __all_sync(0xffffffffu, ok) != 0;
            if (ok) ok = bar_wait(&s_full[t], (stop_at - it.t0) & 1, &stop);
            if (row == 0) bar_arrive(&empty[(2 * (stop_at - it.t0) - 1) % C::kUnits]);
            ok = __all_sync(0xffffffffu, ok) != 0;
            tc_after_sync();
        } else if (most > it.t0) {
            // the other tile has keys, so this tile's Q is on its way to where the zero
            // rows are about to be staged
            ok = bar_wait(&q_full, 0, &stop);
            ok = __all_sync(0xffffffffu, ok) != 0;
        }
        // ok: whether the waits of this warp ended well; a wait of another warp may
        // not have, so all of a tile's warps meet below either way
        const bool none = see1 <= see0;
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        // a row whose waits gave up counts as not finite
        const float lse = !ok          ? NAN
                          : sum > 0.f  ? top * a.scale + __log2f(sum) * kLn2
                          : sum == 0.f ? -INFINITY
                                       : NAN;
        if (it.slot >= 0) {
            // a piece: fp32, and nothing where it holds none of the row's keys
            const int from = max(see0, it.t0 * kTile), to = min(see1, it.t1 * kTile);
            const bool some = live && to > from;
            const int64_t first = ((int64_t)it.slot * a.kv_heads + hk) * kTile + (warp & 3) * 32;
            float* sums = p.partial + (first + lane) * a.dim;
            float odd = 0.f;   // NaN where a value is not finite
#pragma unroll 1
            for (int i = 0; i < HD; i += 32) {
                float o[32];
                __syncwarp();
                if (any) {
                    tmem_load32(o_at + i, o);
                    tmem_wait_load();
                    tmem_loaded(o);
                }
                if (ok && some) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        if (i + e >= a.dim) break;
                        float v[8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) {
                            v[x] = o[e + x] * inv;
                            odd = fmaf(v[x], 0.f, odd);
                        }
                        store8(sums + i + e, v);
                    }
                }
            }
            const bool again = some && !(ok && odd == 0.f && lse * 0.f == 0.f);
            if (!again) p.partial_lse[first + lane] = some ? lse : -INFINITY;
            __syncwarp();
            if (__any_sync(0xffffffffu, again))
                forward_rows<HD>(a, hk, token, h, it.k0 + from, it.k0 + to, again,
                                 p.partial + first * a.dim, p.partial_lse + first);
        } else {
            // through the tile's own Q, which no product reads any more
            uint8_t* out = smem + t * C::kUnit;
            const bool fine = ok && stage_row<HD>(o_at, out, r, 0, inv, any);
            const bool again = live && !(fine && (none || lse * 0.f == 0.f));
            if (live && !again) a.lse[(int64_t)token * a.heads + h] = lse;
            keep[t][r] = live && !again;
            fence_async();
            // rows past the tile or the tensor are left out by the store itself
            if (!part_any(1 + t, 128, !ok || again ||
                                          (!live && row_tok < tokens && token < a.q_tokens))) {
                if (r == 0 && it.q0 + t * tokens < a.q_tokens)
                    store_tile<HD>(&mo, out, hk * group, it.q0 + t * tokens);
            } else {
                store_rows<HD, 32>(out, (warp & 3) * 32, a.dim, [&](int i) -> bf16* {
                    const int tok = i / group;
                    return keep[t][i]
                               ? a.out.at(it.q0 + t * tokens + tok, hk * group + i - tok * group)
                               : nullptr;
                });
            }
            if (__any_sync(0xffffffffu, again))
                forward_rows<HD>(a, hk, token, h, range.lo, range.hi, again, nullptr, nullptr);
        }
    } else if (NQ == 2) {
        set_registers<C::kLess, false>();   // the warps without a role
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    if (warp == 0) tmem_free(tmem, C::kCols);
    if (threadIdx.x == 0 && stop) report_stop(a.status);
}

// The values 4l .. 4l+3 of a row are lane l's.
__device__ __forceinline__ void put4(bf16* p, float4 v, int dim) {
    const int c = 4 * (threadIdx.x & 31);
    if (c >= dim) return;
    uint2 w;
    w.x = pack2(v.x, v.y, bf16());
    w.y = pack2(v.z, v.w, bf16());
    *reinterpret_cast<uint2*>(p + c) = w;
}
__device__ __forceinline__ void add4(float4& a, float s, float4 b) {
    a.x += s * b.x;
    a.y += s * b.y;
    a.z += s * b.z;
    a.w += s * b.w;
}

// Joins the pieces of the split query tiles:
//   lse = log sum_i exp(lse_i),  out = sum_i exp(lse_i - lse) out_i,
// a warp to a row, lane l holding the values 4l .. 4l+3.  Most pieces of a tile
// of many short-query sequences hold nothing that a given row sees: the lanes
// read the pieces' lse side by side, and only the others' sums are read.
__global__ void __launch_bounds__(kThreads) k_attention_join(Attn a, Plan p) {
    pdl_prologue();
    constexpr int kParts = kTile / kWarps;   // CTAs to a tile and head
    const int part = blockIdx.x % kParts, rest = blockIdx.x / kParts;
    const int join = rest / a.kv_heads, hk = rest - join * a.kv_heads;
    if (join >= p.head->joins) return;
    const Join jn = p.joins[join];
    const int lane = threadIdx.x & 31, r = part * kWarps + (threadIdx.x >> 5);
    const int tok = r / a.group, token = jn.q0 + tok, h = hk * a.group + r - tok * a.group;
    if (tok >= p.tokens || token >= a.q_tokens) return;
    const Range range = p.q_range[token];
    if (!range.live()) return;
    if (range.hi <= range.lo) {
        put4(a.out.at(token, h), make_float4(0.f, 0.f, 0.f, 0.f), a.dim);
        if (lane == 0) a.lse[(int64_t)token * a.heads + h] = -INFINITY;
        return;
    }
    const int64_t base = ((int64_t)jn.slot * a.kv_heads + hk) * kTile + r;
    const int64_t step = (int64_t)a.kv_heads * kTile;
    // the pieces' lse, 32 at a time a lane each; the first 128 stay in registers
    constexpr int kHeld = 4;
    float held[kHeld], top = -INFINITY;
#pragma unroll
    for (int x = 0; x < kHeld; ++x) {
        const int i = 32 * x + lane;
        held[x] = i < jn.n ? p.partial_lse[base + i * step] : -INFINITY;
        top = fmaxf(top, held[x]);
    }
    for (int i = 32 * kHeld + lane; i < jn.n; i += 32)
        top = fmaxf(top, p.partial_lse[base + i * step]);
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
    float sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add_pieces = [&](int i0, float lse) {
        const float e = lse == -INFINITY ? 0.f : exp2_fast((lse - top) * kLog2e);
        sum += e;
        unsigned some = __ballot_sync(0xffffffffu, lse != -INFINITY);
        while (some) {
            // four pieces' sums in flight; a missing one is read as the first, times 0
            float w[4];
            float4 v[4];
            const int j0 = __ffs(some) - 1;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int j = some ? __ffs(some) - 1 : j0;
                w[x] = some ? __shfl_sync(0xffffffffu, e, j) : 0.f;
                some &= some - 1;
                v[x] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (4 * lane < a.dim)
                    v[x] = *reinterpret_cast<const float4*>(
                        p.partial + (base + (i0 + j) * step) * a.dim + 4 * lane);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) add4(o, w[x], v[x]);
        }
    };
#pragma unroll
    for (int x = 0; x < kHeld; ++x)
        if (32 * x < jn.n) add_pieces(32 * x, held[x]);
    for (int i0 = 32 * kHeld; i0 < jn.n; i0 += 32)
        add_pieces(i0, i0 + lane < jn.n ? p.partial_lse[base + (i0 + lane) * step] : -INFINITY);
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
    const float inv = 1.f / sum, lse = top + __log2f(sum) * kLn2;
    o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    put4(a.out.at(token, h), o, a.dim);
    if (lane == 0) a.lse[(int64_t)token * a.heads + h] = lse;
}

template <int HD, int NQ>
cudaError_t launch(const Attn& a, const Plan& p, cudaStream_t st) {
    using C = Cfg<HD, NQ>;
    CUtensorMap mq, mk, mv;
    cudaError_t e = tile_map(&mq, a.q, a.q_tokens, a.heads, a.dim, a.group, p.tokens, p.head);
    if (e == cudaSuccess) e = tile_map(&mk, a.k, a.k_tokens, a.kv_heads, a.dim, 1, kTile, p.head);
    if (e == cudaSuccess) e = tile_map(&mv, a.v, a.k_tokens, a.kv_heads, a.dim, 1, kTile, p.head);
    CUtensorMap mo;
    if (e == cudaSuccess)
        e = tile_map(&mo, a.out, a.q_tokens, a.heads, a.dim, a.group, p.tokens, p.head);
    if (e != cudaSuccess) return e;
    auto* k = k_attention_forward<HD, NQ>;
    static std::atomic<uint64_t> ready{0};
    e = allow_smem(k, C::kSmem, &ready, C::kLaunch);
    if (e != cudaSuccess) return e;
    return launch_k(k, dim3((unsigned)p.most_items * a.kv_heads), dim3(C::kThreads), C::kSmem, st,
                    mq, mk, mv, mo, a, p);
}

}  // namespace

cudaError_t launch_tiles_forward(const Attn& a, const Plan& p, cudaStream_t st) {
    cudaError_t e;
    if (a.dim <= 64)
        e = p.per_item == 2 ? launch<64, 2>(a, p, st) : launch<64, 1>(a, p, st);
    else
        e = p.per_item == 2 ? launch<128, 2>(a, p, st) : launch<128, 1>(a, p, st);
    if (e != cudaSuccess || p.most_slots == 0) return e;
    return launch_k(k_attention_join, dim3((unsigned)(p.tiles * a.kv_heads * (kTile / kWarps))),
                    dim3(kThreads), 0, st, a, p);
}

}  // namespace seq
}  // namespace pss
