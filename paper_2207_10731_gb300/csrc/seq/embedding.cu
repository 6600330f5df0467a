// Rows of a dense table by id, and their gradient (pss_embedding_* of pss.h).
//
// Forward:  out[t] = scale * weight[ids[t]].
// Backward: dweight[v] = scale * sum over t with ids[t] = v of grad[t].
//
// Both are bound by memory.  Backward, the token positions are sorted by id, stable
// (by counting up to kSmall tokens, else by the radix sort of the shared array's
// backward), so that each row of the table is summed by one group of threads
// in the order of the tokens and stored once, rows without a token as zeros: no
// atomics, and equal inputs give equal bits.  A popular id's run would be one group's
// long chain: runs are cut at multiples of kChunk sorted places, the pieces that lie
// wholly in a run are summed beforehand side by side, kChunk of these again, and the
// row's group adds head, pieces and tail.
#include <cmath>

#include "seq_common.cuh"

using namespace pss;
using namespace pss::seq;

namespace {

constexpr int kPer = 8;          // values of a row that a thread holds
constexpr int kChunk = 32;       // sorted places of a piece
constexpr int kPieces = 64;      // pieces of a large piece
constexpr int kLarge = kChunk * kPieces;
constexpr int kRows = 8;         // rows of the table that a group sums, at most
constexpr int kSmall = 8192;     // tokens that are ranked instead of sorted
constexpr uint32_t kNone = 0xffffffffu;

// How a row is spread: `lanes` threads (a power of two up to 32) to a block of 8 * lanes
// values, `blocks` blocks to a row.
struct Spread {
    int log2_lanes, blocks, cols;
};

// The 8 values that a thread holds of block b: consecutive ones (VECTOR: rows start at
// multiples of 8 elements), else every lanes'th.
template <bool VECTOR>
struct Piece {
    int at, step, cols;
    __device__ __forceinline__ Piece(const Spread& s, int block) {
        const int lanes = 1 << s.log2_lanes, lane = threadIdx.x & (lanes - 1);
        cols = s.cols;
        step = VECTOR ? 1 : lanes;
        at = block * kPer * lanes + (VECTOR ? kPer * lane : lane);
    }
    __device__ __forceinline__ bool any() const { return at < cols; }
    template <typename T>
    __device__ __forceinline__ Raw8<T> load(const T* row) const {
        if constexpr (VECTOR) {
            return load_raw(row + at);
        } else {
            Raw8<T> r;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                set_raw(r, i, at + i * step < cols ? row[at + i * step] : round_to<T>(0.f));
            return r;
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T* row, const float (&v)[kPer]) const {
        if constexpr (VECTOR) {
            store8(row + at, v);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (at + i * step < cols) row[at + i * step] = round_to<T>(v[i]);
        }
    }
};

// A group's number and the block of its row's values.
__device__ __forceinline__ int64_t group_of(const Spread& s, unsigned cta, int* block) {
    const int64_t g = ((int64_t)cta * blockDim.x + threadIdx.x) >> s.log2_lanes;
    if (s.blocks == 1) {
        *block = 0;
        return g;
    }
    const int64_t of = g / s.blocks;
    *block = (int)(g - of * s.blocks);
    return of;
}

__device__ __forceinline__ void note_outside(unsigned long long* status, int64_t t) {
    if (status) atomicMin(status, (unsigned long long)t);
}

// The status of a call that has no value to read or write.
__global__ void __launch_bounds__(kThreads)
k_embedding_check(const int64_t* __restrict__ ids, int64_t tokens, int64_t rows,
                  unsigned long long* status) {
    pdl_prologue();
    const int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (t < tokens && (uint64_t)ids[t] >= (uint64_t)rows) note_outside(status, t);
}

// U tokens to a group, all their loads in flight (four in vectors: two 162 us and eight 197 for
// 1.7 M x 128; value by value two, 53 instead of 59 us for 100000 x 333).
template <typename TW, typename TO, bool VECTOR, int U>
__global__ void __launch_bounds__(kThreads)
k_embedding_forward(const TW* __restrict__ weight, int64_t ws, int64_t rows,
                    const int64_t* __restrict__ ids, int64_t tokens, float scale, TO* out,
                    int64_t os, unsigned long long* status, Spread s) {
    pdl_prologue();
    int block;
    const int64_t t0 = group_of(s, blockIdx.x, &block) * U;
    const Piece<VECTOR> piece(s, block);
    if (!piece.any() || t0 >= tokens) return;
    int64_t id[U];
    Raw8<TW> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = t0 + u < tokens ? ids[t0 + u] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool in = (uint64_t)id[u] < (uint64_t)rows;
        raw[u] = in ? piece.load(weight + id[u] * ws) : Raw8<TW>{};
        if (!in && piece.at == 0 && t0 + u < tokens) note_outside(status, t0 + u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (t0 + u >= tokens) break;
        float v[kPer];
        unpack(raw[u], v);
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] *= scale;
        piece.store(out + (t0 + u) * os, v);
    }
}

// ---- sorting -----------------------------------------------------------------

// The radix sort's input: each token's id (kNone: outside the table) and place.
__global__ void __launch_bounds__(kThreads)
k_embedding_keys(const int64_t* __restrict__ ids, int64_t tokens, int64_t rows, uint32_t* keys,
                 uint32_t* places, uint32_t* done, unsigned long long* status) {
    pdl_prologue();
    const int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (t == 0) *done = 0u;
    if (t >= tokens) return;
    const int64_t id = ids[t];
    const bool in = (uint64_t)id < (uint64_t)rows;
    if (!in) note_outside(status, t);
    keys[t] = in ? (uint32_t)id : kNone;
    places[t] = (uint32_t)t;
}

// Up to kSmall tokens: a token's place is the number of smaller ids and of equal ones in front
// of it, counted by a warp for kRanked tokens at a time against all ids in shared memory.
// (One CTA's bitonic sort of 2011: 15 us, its steps in turn, against 6.5; here CTAs know
// nothing of each other.)
constexpr int kRanked = 4;
__global__ void __launch_bounds__(kThreads)
k_embedding_rank(const int64_t* __restrict__ ids, int tokens, int64_t rows,
                 unsigned long long* __restrict__ sorted, unsigned long long* __restrict__ count,
                 unsigned long long* status) {
    pdl_prologue();
    extern __shared__ __align__(16) uint32_t keys[];   // kNone: outside the table, and past the end
    const int lane = threadIdx.x & 31, all = (tokens + 127) / 128 * 128;
    int valid = 0;
    for (int t0 = 0; t0 < all; t0 += kThreads) {
        const int t = t0 + threadIdx.x;
        const int64_t id = t < tokens ? ids[t] : -1;
        const bool in = (uint64_t)id < (uint64_t)rows;
        if (t < all) keys[t] = in ? (uint32_t)id : kNone;
        if (blockIdx.x == 0) {
            if (!in && t < tokens) note_outside(status, t);
            valid += __syncthreads_count(in);
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *count = (unsigned long long)valid;
    __syncthreads();
    const int t0 = (blockIdx.x * kWarps + (threadIdx.x >> 5)) * kRanked;
    if (t0 >= tokens) return;
    uint32_t k[kRanked];
    int rank[kRanked] = {};
#pragma unroll
    for (int x = 0; x < kRanked; ++x) k[x] = keys[t0 + x];
    for (int j = 4 * lane; j < all; j += 128) {
        const uint4 w = *reinterpret_cast<const uint4*>(keys + j);
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int x = 0; x < kRanked; ++x)
                rank[x] += v[e] < k[x] || (v[e] == k[x] && j + e < t0 + x);
    }
#pragma unroll
    for (int x = 0; x < kRanked; ++x) {
        rank[x] = __reduce_add_sync(0xffffffffu, rank[x]);
        if (lane == x && k[x] != kNone)
            sorted[rank[x]] = ((unsigned long long)k[x] << 32) | (unsigned)(t0 + x);
    }
}

// ---- sums --------------------------------------------------------------------

__device__ __forceinline__ uint32_t key_of(unsigned long long e) { return (uint32_t)(e >> 32); }

__device__ __forceinline__ void add_to(float (&sum)[kPer], const float (&v)[kPer]) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum[i] += v[i];
}

// A group to a piece of kChunk sorted places that belong to one id: its sum in fp32.
// Other pieces are left alone (and never read).
template <typename TG, bool VECTOR>
__global__ void __launch_bounds__(kThreads, 2)
k_embedding_pieces(const TG* __restrict__ grad, int64_t gs,
                   const unsigned long long* __restrict__ sorted,
                   const unsigned long long* __restrict__ count, float* __restrict__ sums,
                   int64_t sums_stride, Spread s) {
    pdl_prologue();
    int block;
    const int64_t c = group_of(s, blockIdx.x, &block), i0 = c * kChunk;
    const Piece<VECTOR> piece(s, block);
    if (!piece.any() || i0 + kChunk > (int64_t)*count ||
        key_of(sorted[i0]) != key_of(sorted[i0 + kChunk - 1]))
        return;
    constexpr int U = 32 / sizeof(TG);
    float sum[kPer] = {};
#pragma unroll 1
    for (int i = 0; i < kChunk; i += U) {
        uint32_t t[U];
        Raw8<TG> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) t[u] = (uint32_t)sorted[i0 + i + u];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = piece.load(grad + t[u] * gs);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[kPer];
            unpack(raw[u], v);
            add_to(sum, v);
        }
    }
    piece.store(sums + c * sums_stride, sum);
}

// kPieces pieces of one id again.
template <bool VECTOR>
__global__ void __launch_bounds__(kThreads)
k_embedding_large_pieces(const float* __restrict__ sums, int64_t sums_stride,
                         const unsigned long long* __restrict__ sorted,
                         const unsigned long long* __restrict__ count, float* __restrict__ large,
                         Spread s) {
    pdl_prologue();
    int block;
    const int64_t c = group_of(s, blockIdx.x, &block), i0 = c * kLarge;
    const Piece<VECTOR> piece(s, block);
    if (!piece.any() || i0 + kLarge > (int64_t)*count ||
        key_of(sorted[i0]) != key_of(sorted[i0 + kLarge - 1]))
        return;
    constexpr int U = 8;
    float sum[kPer] = {};
    for (int i = 0; i < kPieces; i += U) {
        Raw8<float> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = piece.load(sums + (c * kPieces + i + u) * sums_stride);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[kPer];
            unpack(raw[u], v);
            add_to(sum, v);
        }
    }
    piece.store(large + c * sums_stride, sum);
}

// The first place of lo .. hi whose key is at or behind v, or hi.
__device__ __forceinline__ int first_place(const unsigned long long* __restrict__ sorted, int lo,
                                           int hi, int64_t v) {
    while (lo < hi) {
        const int m = (int)(((unsigned)lo + (unsigned)hi) >> 1);
        if (key_of(sorted[m]) < v)
            lo = m + 1;
        else
            hi = m;
    }
    return lo;
}

// The same by a warp: 32 places a step.
__device__ __forceinline__ int first_place_warp(const unsigned long long* __restrict__ sorted,
                                                int lo, int hi, int64_t v) {
    const int lane = threadIdx.x & 31;
    while (lo < hi) {
        // places lo + step, lo + 2 step ..: the answer lies behind the last smaller key
        const int step = (hi - lo + 32) / 33, at = lo + (lane + 1) * step - 1;
        const unsigned less = __ballot_sync(0xffffffffu, at < hi && key_of(sorted[at]) < v);
        const int k = __popc(less);   // keys do not fall: the first k lanes say yes
        const int from = lo + k * step;
        if (k < 32) hi = min(hi, from + step - 1);
        lo = min(from, hi);
    }
    return lo;
}

// Whether the run from .. to holds a whole piece.
__device__ __forceinline__ bool is_long(int from, int to) {
    return (from + kChunk - 1) / kChunk * kChunk + kChunk <= to;
}

// The sums of the table's rows.  CTAs up to long_ctas: a group to a piece, which answers for
// its row where it is the first whole piece of the run: head, pieces and tail.  Runs of more than
// kAlone pieces are the CTA's, a part of the pieces to each group (kPieces of them at once where
// these were summed).  The other CTAs: a group to `per` rows, whose places its lanes find by
// bisection; then one pass over the short runs, U entries' loads in flight whichever rows
// these belong to.  (All runs in that pass: 943 us for the popular ids of a batch of
// 1.7 M x 128, the chains of a few groups; now 230, 82 % of the copy bandwidth.  Pieces of 16
// entries: 394 instead of 369 us for all of that call; two CTAs an SM 470, four 365.)
constexpr int kAlone = 16;
template <typename TG, typename TO, bool VECTOR>
__global__ void __launch_bounds__(kThreads, 4)
k_embedding_rows(const TG* __restrict__ grad, int64_t gs,
                 const unsigned long long* __restrict__ sorted,
                 const unsigned long long* __restrict__ count, const float* __restrict__ sums,
                 const float* __restrict__ large, int64_t sums_stride, float scale, TO* out,
                 int64_t os, int64_t rows, int per, unsigned long_ctas, Spread s) {
    pdl_prologue();
    constexpr int U = 4;
    __shared__ union {
        int places[kThreads][kRows + 1];
        float parts[kThreads][kPer + 1];
    } shared;
    __shared__ int ends[2], listed, list[kThreads][2];
    const int n = (int)*count;
    const int groups = kThreads >> s.log2_lanes, group = threadIdx.x >> s.log2_lanes;
    const int lanes = 1 << s.log2_lanes, lane = threadIdx.x & (lanes - 1);
    float sum[kPer] = {};
    int block;
    if (blockIdx.x < long_ctas) {
        const int64_t c64 = group_of(s, blockIdx.x, &block);
        if (threadIdx.x == 0) listed = 0;
        __syncthreads();
        // what this group sums: whole pieces first .. last of a run, entries head .. in front
        // of them and .. tail behind
        int head = 0, first = 0, last = 0, tail = 0;
        uint32_t k = 0;
        bool alone = false;
        if ((c64 + 1) * kChunk <= n) {
            const int c = (int)c64, at = c * kChunk;
            k = key_of(sorted[at]);
            if (k == key_of(sorted[at + kChunk - 1]) &&
                (at == 0 || key_of(sorted[at - kChunk]) != k)) {
                // the whole pieces behind it, all looked at at once
                unsigned whole = 0;
#pragma unroll
                for (int j = 0; j < kAlone; ++j) {
                    const int64_t to = at + (int64_t)(j + 2) * kChunk;
                    if (to <= n && key_of(sorted[to - 1]) == k) whole |= 1u << j;
                }
                const int more = __ffs(~whole) - 1;
                if (more == kAlone) {
                    if (lane == 0) {
                        const int i = atomicAdd(&listed, 1);
                        list[i][0] = c;
                        list[i][1] = block;
                    }
                } else {
                    alone = true;
                    first = c;
                    last = c + 1 + more;
                    head = first_place(sorted, at > 0 ? at - kChunk + 1 : 0, at, k);
                    tail = first_place(sorted, last * kChunk, min(n, last * kChunk + kChunk),
                                       (int64_t)k + 1);
                }
            }
        }
        __syncthreads();
        // its own run first, then the CTA's, whose order does not matter: each is a row of its own
        for (int x = -1; x < listed; ++x) {
            if (x >= 0) {
                const int c = list[x][0];
                block = list[x][1];
                k = key_of(sorted[c * kChunk]);
                const int end = first_place_warp(sorted, (c + kAlone) * kChunk, n, (int64_t)k + 1);
                const int pieces = end / kChunk - c;
                first = c + (int)((int64_t)pieces * group / groups);
                last = c + (int)((int64_t)pieces * (group + 1) / groups);
                head = group > 0 ? first * kChunk
                                 : first_place(sorted, c > 0 ? c * kChunk - kChunk + 1 : 0, c * kChunk, k);
                tail = group < groups - 1 ? last * kChunk : end;
#pragma unroll
                for (int e = 0; e < kPer; ++e) sum[e] = 0.f;
            }
            const Piece<VECTOR> piece(s, block);
            const bool work = (x >= 0 || alone) && piece.any();
            if (work) {
                int l0 = (first + kPieces - 1) / kPieces, l1 = last / kPieces;
                if (l1 <= l0) l0 = l1 = 0;
                for (int y = 0; y < 3; ++y) {   // pieces, large pieces, pieces
                    const float* from = y == 1 ? large : sums;
                    int i = y == 0 ? first : y == 1 ? l0 : l1 * kPieces;
                    int to = y == 0 ? l0 * kPieces : y == 1 ? l1 : last;
                    if (l1 == 0) i = first, to = y == 0 ? last : first;
                    constexpr int V = 4;
                    for (; i < to; i += V) {
                        Raw8<float> raw[V];
#pragma unroll
                        for (int u = 0; u < V; ++u)
                            raw[u] = i + u < to ? piece.load(from + (i + u) * sums_stride) : Raw8<float>{};
#pragma unroll
                        for (int u = 0; u < V; ++u) {
                            float v[kPer];
                            unpack(raw[u], v);
                            add_to(sum, v);
                        }
                    }
                }
                for (int y = 0; y < 2; ++y) {   // head, tail
                    const int to = y == 0 ? first * kChunk : tail;
                    for (int i = y == 0 ? head : last * kChunk; i < to; i += U) {
                        uint32_t t[U];
                        Raw8<TG> raw[U];
#pragma unroll
                        for (int u = 0; u < U; ++u) t[u] = i + u < to ? (uint32_t)sorted[i + u] : 0u;
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            raw[u] = i + u < to ? piece.load(grad + t[u] * gs) : Raw8<TG>{};
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            float v[kPer];
                            unpack(raw[u], v);
                            add_to(sum, v);
                        }
                    }
                }
            }
            if (x >= 0) {
                // the groups' parts, in their order
#pragma unroll
                for (int e = 0; e < kPer; ++e) shared.parts[threadIdx.x][e] = sum[e];
                __syncthreads();
                if (group == 0 && work)
                    for (int g = 1; g < groups; ++g)
#pragma unroll
                        for (int e = 0; e < kPer; ++e) sum[e] += shared.parts[g * lanes + lane][e];
                __syncthreads();
            }
            if (work && (x < 0 || group == 0)) {
                float v[kPer];
#pragma unroll
                for (int e = 0; e < kPer; ++e) v[e] = sum[e] * scale;
                piece.store(out + (int64_t)k * os, v);
            }
        }
        return;
    }
    int64_t v0 = group_of(s, blockIdx.x - long_ctas, &block) * per;
    const Piece<VECTOR> piece(s, block);
    const int some = rows - v0 < per ? (int)(rows - v0) : per;   // may be below 1
    int* place = shared.places[group];
    // the CTA's rows lie side by side: two warps find their ends in the list, and each row is
    // looked for between these (all in the whole list: 20 steps a row, 317 instead of 240 us for a
    // million rows; the runs' ends noted in a table beforehand: 233, and two launches more)
    {
        const int64_t cta = blockIdx.x - long_ctas;
        const int64_t first = cta * groups / s.blocks * per;
        const int64_t last = (((cta + 1) * groups - 1) / s.blocks + 1) * per;
        const int warp = threadIdx.x >> 5;
        if (warp < 2) {
            const int at = first_place_warp(sorted, 0, n, warp == 0 ? first : last);
            if ((threadIdx.x & 31) == 0) ends[warp] = at;
        }
    }
    __syncthreads();
    for (int j = lane; j <= some; j += lanes) place[j] = first_place(sorted, ends[0], ends[1], v0 + j);
    __syncthreads();
    // Rows of one block that are dense are dealt out instead: neighbours' runs are as long as
    // each other's, and a group's would add up.
    int step = 1, at = group;   // row r of the group is row at % per of group at / per, r by r
    if (s.blocks == 1 && per > 1 && ends[1] - ends[0] > 2 * groups * per) {
        step = groups;
    } else {
        at = group * per;
    }
    if (!piece.any()) return;
    const int64_t cta_v0 = (int64_t)(blockIdx.x - long_ctas) * groups * per;
    const float none[kPer] = {};
    const int count_rows = step == 1 ? some : per;
    for (int r = 0; r < count_rows; ++r) {
        int64_t row;
        int i, end, to = r;   // rows r .. to are short
        if (step == 1) {
            if (is_long(place[r], place[r + 1])) continue;
            while (to + 1 < some && !is_long(place[to + 1], place[to + 2])) ++to;
            i = place[r];
            end = place[to + 1];
            row = v0 + r;
        } else {
            const int x = at + r * step, g = x / per, y = x - g * per;
            row = cta_v0 + x;
            if (row >= rows) break;
            i = shared.places[g][y];
            end = shared.places[g][y + 1];
            if (is_long(i, end)) continue;
        }
        const int64_t behind = row + (to - r) + 1;
        auto leave = [&](int64_t next) {   // store the row, and zeros up to the next
            float v[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                v[e] = sum[e] * scale;
                sum[e] = 0.f;
            }
            piece.store(out + row * os, v);
            for (++row; row < next; ++row) piece.store(out + row * os, none);
        };
        while (i < end) {
            unsigned long long e[U];
            Raw8<TG> raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) e[u] = i + u < end ? sorted[i + u] : 0ull;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u < end) raw[u] = piece.load(grad + (uint32_t)e[u] * gs);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u >= end) break;
                if (key_of(e[u]) != row) leave(key_of(e[u]));
                float v[kPer];
                unpack(raw[u], v);
                add_to(sum, v);
            }
            i += U;
        }
        leave(behind);
        r = to;
    }
}

// ---- host --------------------------------------------------------------------

constexpr int64_t kMost = (int64_t(1) << 31) - 1024;   // rows, tokens
constexpr int64_t kMostCols = int64_t(1) << 20;

Spread spread(int64_t cols) {
    Spread s{0, 1, (int)cols};
    const int64_t vecs = (cols + kPer - 1) / kPer;
    while (s.log2_lanes < 5 && (1 << s.log2_lanes) < vecs) ++s.log2_lanes;
    s.blocks = (int)((vecs + (1 << s.log2_lanes) - 1) >> s.log2_lanes);
    return s;
}

// CTAs that hold a group to each of n * blocks parts; 0: more than a launch takes.
unsigned ctas(int64_t n, const Spread& s) {
    const int64_t per = kThreads >> s.log2_lanes;
    const int64_t c = (n * s.blocks + per - 1) / per;
    return c < (int64_t(1) << 31) ? (unsigned)c : 0u;
}

// The radix sort's tile: small ones while large ones leave SMs without any (the gradient of 100000
// tokens into a million rows of 128: 164 us with large ones, 144 with small; 1.7 M tokens 363 and 365).
int sort_tile(int64_t tokens) {
    return radix_tiles(tokens) < sm_count() ? kRadixSmallTile : kRadixTile;
}
struct Work {
    uint32_t *keys, *places, *cnt, *tot, *dstart, *done;
    unsigned long long *sorted, *other, *count;
    float *sums, *large;
    int64_t stride;   // of a piece's sum
};
// Where each part of the workspace lies; returns the bytes.
int64_t lay_out(int64_t tokens, int64_t rows, int64_t cols, void* base, Work* w) {
    Take take(base);
    *w = Work{};
    w->stride = (cols + kPer - 1) / kPer * kPer;
    w->count = static_cast<unsigned long long*>(take(16));
    w->done = static_cast<uint32_t*>(take(4));
    w->sorted = static_cast<unsigned long long*>(take(8 * tokens));
    w->sums = static_cast<float*>(take(tokens / kChunk * w->stride * 4));
    w->large = static_cast<float*>(take(tokens / kLarge * w->stride * 4));
    if (tokens > kSmall) {
        const RadixPlan plan = radix_plan((uint64_t)(rows > 0 ? rows : 1), 0);
        w->other = static_cast<unsigned long long*>(take(8 * tokens));
        w->keys = static_cast<uint32_t*>(take(4 * tokens));
        w->places = static_cast<uint32_t*>(take(4 * tokens));
        w->cnt = static_cast<uint32_t*>(take(4 * radix_tiles(tokens, sort_tile(tokens)) << plan.bits[0]));
        w->tot = static_cast<uint32_t*>(take(4 << kRadixMaxBits));
        w->dstart = static_cast<uint32_t*>(take(4 << kRadixMaxBits));
    }
    return take.bytes();
}

cudaError_t sort_tokens(const int64_t* ids, int64_t tokens, int64_t rows, const Work& w,
                        unsigned long long* status, cudaStream_t st) {
    if (tokens <= kSmall) {
        const int all = (int)(tokens + 127) / 128 * 128, per = kWarps * kRanked;
        return launch_k(k_embedding_rank, dim3((unsigned)((tokens + per - 1) / per)), dim3(kThreads),
                        (size_t)all * 4, st, ids, (int)tokens, rows, w.sorted, w.count, status);
    }
    cudaError_t e = launch_k(k_embedding_keys, dim3((unsigned)((tokens + kThreads - 1) / kThreads)),
                             dim3(kThreads), 0, st, ids, tokens, rows, w.keys, w.places, w.done,
                             status);
    if (e != cudaSuccess) return e;
    SortedBuffers sb{};
    sb.pair_x = w.keys;
    sb.q_row = w.places;
    sb.sorted_e = w.sorted;
    sb.tmp_e = w.other;
    sb.stats = w.count;
    sb.cnt = w.cnt;
    sb.tot = w.tot;
    sb.dstart = w.dstart;
    sb.done = w.done;
    return launch_radix_sort(sb, tokens, 1, 0u, radix_plan((uint64_t)rows, 0), st,
                             sort_tile(tokens));
}

bool sizes_ok(int64_t tokens, int64_t rows, int64_t cols) {
    return tokens >= 0 && rows >= 0 && cols >= 0 && tokens < kMost && rows < kMost;
}

pss_status clear_status(int64_t* status, cudaStream_t st) {
    return status ? status_of(cudaMemsetAsync(status, 0xff, 8, st)) : PSS_OK;
}

// For tables without rows or columns: the ids are looked at for the status alone.
pss_status check_only(const int64_t* ids, int64_t tokens, int64_t rows, int64_t* status,
                      cudaStream_t st) {
    if (!status || tokens == 0) return PSS_OK;
    return status_of(launch_k(k_embedding_check, dim3((unsigned)((tokens + kThreads - 1) / kThreads)),
                              dim3(kThreads), 0, st, ids, tokens, rows,
                              reinterpret_cast<unsigned long long*>(status)));
}

}  // namespace

extern "C" pss_status pss_embedding_forward(const void* weight, pss_dtype weight_type,
                                            int64_t weight_stride, int64_t rows, int64_t cols,
                                            const int64_t* ids, int64_t tokens, float scale,
                                            void* out, pss_dtype out_type, int64_t out_stride,
                                            int64_t* status, pss_stream stream) {
    if (!dtype_ok(weight_type) || !dtype_ok(out_type) || !sizes_ok(tokens, rows, cols) ||
        weight_stride < cols || out_stride < cols || !std::isfinite(scale))
        return PSS_ERR_INVALID_ARG;
    if (cols > kMostCols) return PSS_ERR_UNSUPPORTED;
    if (status && !(device_ptr(status) && aligned_to(status, 8))) return PSS_ERR_INVALID_ARG;
    const bool some = tokens > 0 && cols > 0;
    if ((some || (status && tokens > 0)) && (!device_ptr(ids) || !aligned_to(ids, 8)))
        return PSS_ERR_INVALID_ARG;
    if (some) {
        if (!device_ptr(out) || !aligned_to(out, dtype_size(out_type))) return PSS_ERR_INVALID_ARG;
        if (rows > 0 && (!device_ptr(weight) || !aligned_to(weight, dtype_size(weight_type))))
            return PSS_ERR_INVALID_ARG;
    }
    const Spread s = spread(cols > 0 ? cols : 1);
    // one token to a group while these do not fill the GPU
    const int64_t fill = (int64_t)sm_count() * 4 * (kThreads >> s.log2_lanes);
    const bool one = tokens * s.blocks <= fill;
    const bool vector = cols % 8 == 0 && aligned8(out, out_stride, dtype_size(out_type)) &&
                        aligned8(weight, weight_stride, dtype_size(weight_type));
    const int at_once = one ? 1 : vector ? 4 : 2;
    const unsigned n = ctas((tokens + at_once - 1) / at_once, s);
    if (some && n == 0) return PSS_ERR_UNSUPPORTED;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const pss_status rc = clear_status(status, st);
    if (rc != PSS_OK) return rc;
    if (!some) return check_only(ids, tokens, rows, status, st);
    return status_of(with_type(weight_type, [&](auto tw) {
        return with_type(out_type, [&](auto to) {
            using TW = decltype(tw);
            using TO = decltype(to);
            auto go = [&](auto* k) {
                return launch_k(k, dim3(n), dim3(kThreads), 0, st, static_cast<const TW*>(weight),
                                weight_stride, rows, ids, tokens, scale, static_cast<TO*>(out),
                                out_stride, reinterpret_cast<unsigned long long*>(status), s);
            };
            return vector ? one ? go(k_embedding_forward<TW, TO, true, 1>)
                                : go(k_embedding_forward<TW, TO, true, 4>)
                   : one  ? go(k_embedding_forward<TW, TO, false, 1>)
                          : go(k_embedding_forward<TW, TO, false, 2>);
        });
    }));
}

extern "C" int64_t pss_embedding_workspace(int64_t tokens, int64_t rows, int64_t cols) {
    if (!sizes_ok(tokens, rows, cols) || cols > kMostCols || tokens == 0 || rows == 0 || cols == 0)
        return 0;
    Work w;
    return lay_out(tokens, rows, cols, nullptr, &w);
}

extern "C" pss_status pss_embedding_backward(const void* grad, pss_dtype grad_type,
                                             int64_t grad_stride, const int64_t* ids,
                                             int64_t tokens, float scale, int64_t rows,
                                             int64_t cols, void* dweight, pss_dtype dweight_type,
                                             int64_t dweight_stride, void* workspace,
                                             int64_t workspace_bytes, int64_t* status,
                                             pss_stream stream) {
    if (!dtype_ok(grad_type) || !dtype_ok(dweight_type) || !sizes_ok(tokens, rows, cols) ||
        grad_stride < cols || dweight_stride < cols || !std::isfinite(scale))
        return PSS_ERR_INVALID_ARG;
    if (cols > kMostCols) return PSS_ERR_UNSUPPORTED;
    if (status && !(device_ptr(status) && aligned_to(status, 8))) return PSS_ERR_INVALID_ARG;
    if (tokens > 0 && (!device_ptr(ids) || !aligned_to(ids, 8))) return PSS_ERR_INVALID_ARG;
    const bool some = rows > 0 && cols > 0;
    const Spread s = spread(cols > 0 ? cols : 1);
    // as many rows to a group as have some 32 tokens, were these spread evenly
    int per = kRows;
    while (per > 1 && (int64_t)per * tokens > 32 * rows) per /= 2;
    const unsigned n = ctas((rows + per - 1) / per, s), pieces = ctas(tokens / kChunk, s);
    if (some) {
        if (!device_ptr(dweight) || !aligned_to(dweight, dtype_size(dweight_type)))
            return PSS_ERR_INVALID_ARG;
        if (tokens > 0 &&
            (!device_ptr(grad) || !aligned_to(grad, dtype_size(grad_type)) ||
             !device_ptr(workspace) || !aligned_to(workspace, 16) ||
             workspace_bytes < pss_embedding_workspace(tokens, rows, cols)))
            return PSS_ERR_INVALID_ARG;
        if (n == 0 || (tokens >= kChunk && pieces == 0) || (int64_t)n + pieces >= (int64_t(1) << 31))
            return PSS_ERR_UNSUPPORTED;
    }
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const pss_status rc = clear_status(status, st);
    if (rc != PSS_OK) return rc;
    if (!some) return check_only(ids, tokens, rows, status, st);
    if (tokens == 0)
        return status_of(cudaMemset2DAsync(dweight, dweight_stride * dtype_size(dweight_type), 0,
                                           cols * dtype_size(dweight_type), rows, st));
    Work w;
    lay_out(tokens, rows, cols, workspace, &w);
    cudaError_t e = sort_tokens(ids, tokens, rows, w,
                                reinterpret_cast<unsigned long long*>(status), st);
    if (e != cudaSuccess) return status_of(e);
    const bool vector = cols % 8 == 0 && aligned8(grad, grad_stride, dtype_size(grad_type)) &&
                        aligned8(dweight, dweight_stride, dtype_size(dweight_type));
    return status_of(with_type(grad_type, [&](auto tg) {
        using TG = decltype(tg);
        const TG* g = static_cast<const TG*>(grad);
        if (pieces > 0) {
            auto* k = vector ? k_embedding_pieces<TG, true> : k_embedding_pieces<TG, false>;
            e = launch_k(k, dim3(pieces), dim3(kThreads), 0, st, g, grad_stride, w.sorted, w.count,
                         w.sums, w.stride, s);
            if (e != cudaSuccess) return e;
        }
        if (tokens >= kLarge) {
            auto* k = vector ? k_embedding_large_pieces<true> : k_embedding_large_pieces<false>;
            e = launch_k(k, dim3(ctas(tokens / kLarge, s)), dim3(kThreads), 0, st, w.sums, w.stride,
                         w.sorted, w.count, w.large, s);
            if (e != cudaSuccess) return e;
        }
        return with_type(dweight_type, [&](auto to) {
            using TO = decltype(to);
            auto* k = vector ? k_embedding_rows<TG, TO, true> : k_embedding_rows<TG, TO, false>;
            return launch_k(k, dim3(n + pieces), dim3(kThreads), 0, st, g, grad_stride, w.sorted,
                            w.count, w.sums, w.large, w.stride, scale, static_cast<TO*>(dweight),
                            dweight_stride, rows, per, pieces, s);
        });
    }));
}
