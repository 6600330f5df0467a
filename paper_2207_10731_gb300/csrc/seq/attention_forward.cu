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
// Roles: one warp loads, one thread issues the products, four warps per query
// tile do the softmax, a thread to a row (tensor-memory lane).  With two tiles
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
// A row whose result is not finite is computed again by its definition
// (attention_rows.cuh): a product with a zero probability takes up an
// infinite or NaN value behind the mask, the definition does not.
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
    static constexpr int kSmem = kQ + kUnits * kUnit + 1024;           // + alignment
    static constexpr int kCols = NQ == 2 ? 512 : 256;                  // tensor-memory columns
    static constexpr int kO = NQ * 128;                                // O's first column
    static constexpr int kThreads = NQ * 128 + 64;
};

template <int HD, int NQ>
__global__ void __launch_bounds__(Cfg<HD, NQ>::kThreads, NQ == 1 ? 2 : 1)
k_attention_forward(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                    const __grid_constant__ CUtensorMap mv, Attn a, Plan p) {
    pdl_prologue();
    using C = Cfg<HD, NQ>;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t q_full, full[C::kUnits], empty[C::kUnits], s_full[NQ], p_ready[NQ], drained;
    __shared__ uint32_t tmem_at;
    __shared__ volatile int stop;
    const int item = blockIdx.x / a.kv_heads, hk = blockIdx.x - item * a.kv_heads;
    if (p.most_slots > 0 && item >= p.head->items) return;
    const Item it = p.items[item];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = a.group, tokens = p.tokens;

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

    uint8_t* smem = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    uint8_t* ring = smem + C::kQ;
    if (threadIdx.x == 0) {
        stop = 0;
        bar_init(&q_full, 1);
        bar_init(&drained, 1);
        for (int i = 0; i < C::kUnits; ++i) {
            bar_init(&full[i], 1);
            bar_init(&empty[i], 1);
        }
        for (int t = 0; t < NQ; ++t) {
            bar_init(&s_full[t], 1);
            bar_init(&p_ready[t], 128);
        }
        bar_init_done();
    }
    if (warp == 0) tmem_alloc(&tmem_at, C::kCols);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = tmem_at;

    if (warp == NQ * 4) {
        // ---- loads: Q, then K and V tiles in turn ----
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
            }
            if (stop) {   // the loads in flight must land before the CTA ends
                int never = 0;
                bar_wait(&q_full, 0, &never);
                for (int w = max(0, u - C::kUnits); w < u; ++w)
                    bar_wait(&full[w % C::kUnits], (w / C::kUnits) & 1, &never);
            }
        }
    } else if (warp == NQ * 4 + 1) {
        // ---- products ----
        if (lane == 0 && most > it.t0) {
            constexpr uint32_t kQK = mma_desc(128, 128, false), kPV = mma_desc(128, HD, true);
            const uint32_t q_at = smem_addr(smem), ring_at = smem_addr(ring);
            auto scores = [&](int t, int u) {
                const uint32_t k_at = ring_at + (u % C::kUnits) * C::kUnit;
#pragma unroll
                for (int i = 0; i < HD / 16; ++i) {
                    const uint32_t off = (i / 4) * 16384 + (i % 4) * 32;
                    mma_ss(tmem + t * 128, smem_desc(q_at + t * C::kUnit + off, 16),
                           smem_desc(k_at + off, 16), kQK, i > 0);
                }
            };
            auto values = [&](int t, int u, bool add) {
                const uint32_t v_at = ring_at + (u % C::kUnits) * C::kUnit;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    mma_ts(tmem + C::kO + t * HD, tmem + t * 128 + i * 8,
                           smem_desc(v_at + i * 2048, 16384), kPV, add || i > 0);
            };
            bool ok = bar_wait(&q_full, 0, &stop) && bar_wait(&full[0], 0, &stop);
            if (ok) {
                tc_after_sync();
#pragma unroll
                for (int t = 0; t < NQ; ++t)
                    if (it.t0 < end[t]) {
                        scores(t, 0);
                        tc_commit(&s_full[t]);
                    }
                tc_commit(&empty[0]);
            }
            for (int j = it.t0; ok && j < most; ++j) {
                const int n = j - it.t0, uv = 2 * n + 1, uk = 2 * n + 2;
                const bool more = j + 1 < most;
                ok = bar_wait(&full[uv % C::kUnits], (uv / C::kUnits) & 1, &stop) &&
                     (!more || bar_wait(&full[uk % C::kUnits], (uk / C::kUnits) & 1, &stop));
#pragma unroll
                for (int t = 0; t < NQ; ++t) {
                    if (!ok || j >= end[t]) continue;
                    ok = bar_wait(&p_ready[t], n & 1, &stop);
                    if (!ok) continue;
                    tc_after_sync();
                    values(t, uv, n > 0);
                    if (j + 1 < end[t]) scores(t, uk);
                    tc_commit(&s_full[t]);
                }
                if (!ok) break;
                tc_commit(&empty[uv % C::kUnits]);
                if (more) tc_commit(&empty[uk % C::kUnits]);
            }
            if (!ok) {   // the products in flight must end before their memory is freed
                int never = 0;
                tc_commit(&drained);
                bar_wait(&drained, 0, &never);
            }
        }
    } else {
        // ---- softmax: thread = row ----
        const int t = NQ == 2 ? warp >> 2 : 0;
        const int r = threadIdx.x & 127;
        const int tok = r / group, h = hk * group + r - tok * group;
        const int token = it.q0 + t * tokens + tok;
        // the keys that the row sees, counted from k0: see0 .. see1
        Range range{0, -1};
        if (tok < tokens && token < a.q_tokens) range = p.q_range[token];
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
            tc_after_sync();
            float s[4][32];
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_load32(s_at + 32 * i, s[i]);
            tmem_wait_load();
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_loaded(s[i]);
            const int lo = see0 - j * kTile, hi = see1 - j * kTile;
#pragma unroll
            for (int i = 0; i < 4; ++i) hide(s[i], lo - 32 * i, hi - 32 * i);
            float m4[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m4[i] = s[i][0];
#pragma unroll
                for (int e = 1; e < 32; ++e) m4[i] = fmaxf(m4[i], s[i][e]);
            }
            const float m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
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
            float2 add = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float2 x = fma2(make_float2(s[i][2 * e], s[i][2 * e + 1]), c2, base2);
                    x.x = exp2_fast(x.x);
                    x.y = exp2_fast(x.y);
                    add = add2(add, x);
                    w[e] = pack2(x.x, x.y, bf16());
                }
                tmem_store16(s_at + 16 * i, w);
            }
            sum += add.x + add.y;
            tmem_wait_store();
            tc_before_sync();
            bar_arrive(&p_ready[t]);
        }
        // ---- epilogue ----
        const bool any = stop_at > it.t0;
        if (any) {
            ok = __all_sync(0xffffffffu, ok) != 0;
            if (ok) ok = bar_wait(&s_full[t], (stop_at - it.t0) & 1, &stop);
            ok = __all_sync(0xffffffffu, ok) != 0;
            tc_after_sync();
        }
        if (ok) {
            const bool none = see1 <= see0;
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
            const float lse = sum > 0.f ? top * a.scale + __log2f(sum) * kLn2 : -INFINITY;
            float odd = none ? 0.f : lse * 0.f;   // NaN where something is not finite
            float* part = nullptr;
            if (it.slot >= 0) {
                const int64_t row = ((int64_t)it.slot * a.kv_heads + hk) * kTile + r;
                part = p.partial + row * a.dim;
                p.partial_lse[row] = lse;
            }
            // a piece that holds none of the keys that a row sees leaves it out
            const bool store = live && !(part && lse == -INFINITY);
#pragma unroll 1
            for (int i = 0; i < HD; i += 32) {
                float o[32];
                __syncwarp();
                if (any) {
                    tmem_load32(o_at + i, o);
                    tmem_wait_load();
                    tmem_loaded(o);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = 0.f;
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    o[e] *= inv;
                    odd += o[e] * 0.f;
                }
                if (store) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        if (i + e >= a.dim) break;
                        float v[8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) v[x] = none ? 0.f : o[e + x];
                        if (part)
                            store8(part + i + e, v);
                        else
                            store8(a.out.at(token, h) + i + e, v);
                    }
                }
            }
            if (it.slot < 0) {
                if (live) a.lse[(int64_t)token * a.heads + h] = lse;
                unsigned again = __ballot_sync(0xffffffffu, live && !none && odd != 0.f);
                while (again) {
                    const int from = __ffs(again) - 1;
                    again &= again - 1;
                    __syncwarp();
                    forward_row(a, __shfl_sync(0xffffffffu, range.lo, from),
                                __shfl_sync(0xffffffffu, range.hi, from),
                                __shfl_sync(0xffffffffu, token, from),
                                __shfl_sync(0xffffffffu, h, from));
                }
            }
        }
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    if (warp == 0) tmem_free(tmem, C::kCols);
    if (threadIdx.x == 0 && stop) report_stop(a.status);
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
    float top = -INFINITY;
    for (int i = lane; i < jn.n; i += 32) top = fmaxf(top, p.partial_lse[base + i * step]);
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
    float sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < jn.n; i0 += 32) {
        const int i = i0 + lane;
        const float lse = i < jn.n ? p.partial_lse[base + i * step] : -INFINITY;
        const float e = lse == -INFINITY ? 0.f : exp2_fast((lse - top) * kLog2e);
        sum += e;
        unsigned some = __ballot_sync(0xffffffffu, lse != -INFINITY);
        while (some) {
            const int j = __ffs(some) - 1;
            some &= some - 1;
            const float w = __shfl_sync(0xffffffffu, e, j);
            if (4 * lane < a.dim)
                add4(o, w, *reinterpret_cast<const float4*>(
                               p.partial + (base + (i0 + j) * step) * a.dim + 4 * lane));
        }
    }
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
    const float inv = 1.f / sum, lse = top + __log2f(sum) * kLn2;
    o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    const float odd = (o.x + o.y + o.z + o.w) * 0.f + lse * 0.f;
    if (__any_sync(0xffffffffu, odd != 0.f)) {
        forward_row(a, range.lo, range.hi, token, h);
        return;
    }
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
    if (e != cudaSuccess) return e;
    auto* k = k_attention_forward<HD, NQ>;
    static std::atomic<uint64_t> ready{0};
    e = allow_smem(k, C::kSmem, &ready);
    if (e != cudaSuccess) return e;
    return launch_k(k, dim3((unsigned)p.most_items * a.kv_heads), dim3(C::kThreads), C::kSmem, st,
                    mq, mk, mv, a, p);
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
