// The next token's logits, bent by what each query's path holds (penalties for repeated tokens), by biases and by grammar masks.
// Every logit is read once and written once; which tokens stand on which path is worked out in LDS, never as a table of queries by
// vocabulary.  Bound by HBM where there are many queries (120 x 128000 float over a tree of 107000 tokens in 16-row pages 34.6 us, 7.1 of
// them to sort; the logits alone with a mask 22, a copy of them 25), by a chain of a few dependent loads where there are few (4 x
// 32000 4.2 us).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "deft_device.h"
#include "deft_internal.h"

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) int32_t i32x2;

// The pieces of the tree in its depth-first order, and the tokens that they hold.
struct Pieces {
    const int32_t *begin, *len, *qlo, *qhi;  // rows of the cache; queries that see them, in the plan's order
    const int32_t *off;                      // tokens in front
    const int32_t *tokens;
    uint32_t n;
};

// Tokens by tile of the vocabulary, as deft_sort_tokens leaves them: of every kRun of them, group g, those of tile i are
// events[g * kRun + table[i * groups + g]] up to where those of the next tile begin.
struct Sorted {
    u32x4 *events;  // {token, its queries, -}
    uint32_t *table;
    u32x2 *seen_by;  // of a group: queries that see any of its tokens lie in [x, y)
    uint32_t groups;
};

struct LogitsArgs {
    const void *logits;
    void *out;
    int64_t stride, out_stride;
    uint32_t vocab, nq, block, tiles;  // block: queries of a workgroup
    Pieces pieces;
    Sorted sorted;
    uint32_t history;        // pieces or groups to look through
    const int32_t *q_order;  // null: queries in the caller's order (no tokens are looked at)
    const float *repetition, *frequency, *presence;
    const float *bias;
    const uint32_t *mask;
    const int32_t *bias_row, *mask_row;
    int64_t bias_stride, mask_stride;
    uint32_t n_bias, n_masks;
};

// A thread has two logits side by side of every row of its workgroup, all in flight from the beginning: up to eight rows, since with
// more the counters of their tokens leave LDS for one workgroup to a compute unit (16 rows: 120 x 128000 44 -> 112 us) and with fewer
// the tokens are looked for more often (4: 50 us).  Kernels for one and for four rows have fewer loads and counters (one query, 8191
// tokens 12.4 -> 11.1 us).  256 or 1024 threads with four logits or one: 60 and 86 us where 512 took 47.
constexpr int kThreads = 512;
constexpr int kTile = 1024;       // logits of a row to a workgroup
constexpr int kMost = 8;          // rows
constexpr uint32_t kEach = kTile / kThreads;  // to a thread
constexpr int kPieces = 512;      // of the tree that are looked at together
constexpr int kGroups = 256;      // of sorted tokens that are
static_assert(kEach == 2, "a row ends behind a thread's logits, or behind the first of them");
constexpr int kSortThreads = 1024;
constexpr int kRun = 1024;        // tokens that deft_sort_tokens takes to a workgroup
constexpr int kMaxTiles = 2048;   // that it sorts by
constexpr int kFill = 512;        // workgroups that the chip holds with no trouble: two to a compute unit
constexpr int kFewTokens = 11000;  // are looked through unsorted by as many workgroups, see sorts
constexpr int kStepTokens = 3500;

// A value that is the same for all lanes, by a scalar load.
template <typename T>
__device__ __forceinline__ T uniform(const T *p, uint32_t i) {
    return *((const __attribute__((address_space(4))) T *)(uintptr_t)(p + i));
}

// Element i of what begins at a place that is the same for all lanes (so it stays in scalar registers); i * sizeof(T) is below 2^32.
template <typename T>
__device__ __forceinline__ T *element(T *p, uint32_t i) {
    return (T *)((char *)p + i * (uint32_t)sizeof(T));
}
template <typename T>
__device__ __forceinline__ const T *element(const T *p, uint32_t i) {
    return (const T *)((const char *)p + i * (uint32_t)sizeof(T));
}

struct Query {
    float repetition, inverse, frequency, presence;
    int32_t bias, mask;  // rows of the tables, -1: none
};

// The quotient by a repetition penalty is a product with its reciprocal, rounded twice (by a division in its place 64 x 50001 take
// 12.0 us, not 11.2, and 120 x 128000 39.4, not 36.4; with the reciprocal in two parts, which rounds once, 11.4 and 37.6).  By penalties
// whose reciprocal is none of fp32's normal numbers logits are divided.
constexpr float kLeastFactor = 0x1p-126f, kMostFactor = 0x1p126f;

// `N` elements side by side, as floats.  (Rows may have odd lengths: any element can be a row's first.)
template <typename T, int N>
__device__ __forceinline__ void get(const T *p, float *x) {
    typedef __attribute__((ext_vector_type(N), aligned(sizeof(T)))) T type;
    const type v = *reinterpret_cast<const type *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)v[i];
}
template <typename T, int N>
__device__ __forceinline__ void put(T *p, const float *x) {
    typedef __attribute__((ext_vector_type(N), aligned(sizeof(T)))) T type;
    type v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (T)x[i];
    __builtin_nontemporal_store(v, reinterpret_cast<type *>(p));  // (not read again here; measured over 61 MB, 39.8 -> 34.7 us)
}

// Queries are in the plan's depth-first order here, in which the queries whose path holds a token are neighbours: `bits` says which
// of the workgroup's queries they are.  With COUNTS a token adds one at the first of them and takes one away behind the last, so
// that the sum over the queries up to one is how often the token stands on that one's path.
template <bool COUNTS, int MOST>
struct Seen {
    uint32_t any[kTile];                        // bit q: on the path of query q
    uint32_t generated[COUNTS ? 4 : kTile];     // the same, prompt tokens left out
    int32_t change[COUNTS ? MOST : 1][COUNTS ? kTile : 4];
};

template <bool COUNTS, int MOST>
__device__ __forceinline__ void see(Seen<COUNTS, MOST> &seen, int32_t token, uint32_t first, uint32_t bits, uint32_t block) {
    const uint32_t at = ((uint32_t)token & (DEFT_TOKEN_PROMPT - 1)) - first;
    if (token < 0 || at >= kTile) return;
    if ((seen.any[at] & bits) != bits) atomicOr(&seen.any[at], bits);
    if (token & DEFT_TOKEN_PROMPT) return;
    if constexpr (COUNTS) {
        const uint32_t lo = __builtin_ctz(bits), hi = 32 - __builtin_clz(bits);
        atomicAdd(&seen.change[lo][at], 1);
        if (hi < block) atomicAdd(&seen.change[hi][at], -1);
    } else {
        if ((seen.generated[at] & bits) != bits) atomicOr(&seen.generated[at], bits);
    }
}

// Queries [qlo, qhi) as bits of a workgroup's that begin at q0.
__device__ __forceinline__ uint32_t bits_of(int32_t qlo, int32_t qhi, uint32_t q0, uint32_t block) {
    const int32_t lo = max(qlo - (int32_t)q0, 0), hi = min(qhi - (int32_t)q0, (int32_t)block);
    return lo < hi ? (0xffffffffu >> (32 - hi)) & (0xffffffffu << lo) : 0;
}

// Sum over the threads in front of this one, and over all, of two numbers each.
struct Sums {
    uint32_t x, y, all_x, all_y;
};
template <int THREADS>
__device__ __forceinline__ Sums sums_before(uint32_t x, uint32_t y, uint32_t (*part)[2]) {
    const uint32_t t = threadIdx.x, lane = t & 63;
    Sums s{x, y, 0, 0};
#pragma unroll
    for (uint32_t o = 1; o < 64; o <<= 1) {
        const uint32_t u = __shfl_up(s.x, o), v = __shfl_up(s.y, o);
        if (lane >= o) {
            s.x += u;
            s.y += v;
        }
    }
    if (lane == 63) {
        part[t / 64][0] = s.x;
        part[t / 64][1] = s.y;
    }
    s.x -= x;
    s.y -= y;
    __syncthreads();
#pragma unroll
    for (uint32_t w = 0; w < THREADS / 64; ++w) {
        const uint32_t u = part[w][0], v = part[w][1];
        if (w < t / 64) {
            s.x += u;
            s.y += v;
        }
        s.all_x += u;
        s.all_y += v;
    }
    return s;
}

// The last of n ascending numbers (n a power of two) that is not above f; the first is not.
__device__ __forceinline__ uint32_t last_not_above(const uint32_t *x, uint32_t n, uint32_t f) {
    uint32_t at = 0;
    for (uint32_t step = n / 2; step > 0; step /= 2)
        if (x[at + step] <= f) at += step;
    return at;
}

// Every workgroup of deft_logits would look through all tokens of its queries' paths for the few that are its tile's.  Where those are
// many they are sorted by tile first, kRun of them to a workgroup, in LDS: a counting sort, whose order within a tile is any, since
// what becomes of a tile's tokens (bits set, whole numbers added) does not depend on it.  Bound by latency: 5 us for 8000 tokens of 512
// pieces, 7 us for 107000 of 6700, whose first piece has to be searched for.
__global__ __launch_bounds__(kSortThreads) void deft_sort_tokens(Pieces p, Sorted to, uint32_t total, uint32_t tiles) {
    constexpr uint32_t kMine = kRun / kSortThreads, kBins = kMaxTiles / kSortThreads;
    __shared__ uint32_t off[kRun], bins[kMaxTiles], part[kSortThreads / 64][2];
    __shared__ int32_t begin[kRun], least, most;
    __shared__ i32x2 queries[kRun];
    const uint32_t t = threadIdx.x, f0 = blockIdx.x * kRun, end = min(f0 + kRun, total);
    uint32_t lo = 0, hi = p.n;  // the first token's piece is one of [lo, hi)
    while (p.n > kRun && hi - lo > 1) {  // (of no more pieces than that, all are taken)
        const uint32_t step = (hi - lo + kSortThreads - 1) / kSortThreads, probe = lo + (t + 1) * step;
        lo += step * (uint32_t)__syncthreads_count(probe < hi && (uint32_t)p.off[probe] <= f0);
        hi = min(hi, lo + step);
    }
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) {  // (a piece has a token at least: no more than kRun of them)
        const uint32_t k = t + kSortThreads * i, s = min(lo + k, p.n - 1);
        off[k] = lo + k < p.n ? (uint32_t)p.off[s] : 0xffffffffu;
        begin[k] = p.begin[s];
        queries[k] = i32x2{p.qlo[s], p.qhi[s]};
    }
    for (uint32_t i = t; i < tiles; i += kSortThreads) bins[i] = 0;
    if (t == 0) {
        least = INT32_MAX;
        most = 0;
    }
    __syncthreads();
    int32_t token[kMine], qlo[kMine], qhi[kMine];
    uint32_t rank[kMine];
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) {
        const uint32_t f = f0 + t + kSortThreads * i;
        token[i] = -1;
        if (f >= end) continue;
        const uint32_t k = last_not_above(off, kRun, f);
        token[i] = p.tokens[(int64_t)begin[k] + (f - off[k])];
        qlo[i] = queries[k][0];
        qhi[i] = queries[k][1];
    }
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) {
        const uint32_t tile = ((uint32_t)token[i] & (DEFT_TOKEN_PROMPT - 1)) / kTile;
        if (token[i] < 0 || tile >= tiles)
            token[i] = -1;
        else
            rank[i] = atomicAdd(&bins[tile], 1);
    }
    int32_t lowest = INT32_MAX, highest = 0;
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i)
        if (token[i] >= 0) {
            lowest = min(lowest, qlo[i]);
            highest = max(highest, qhi[i]);
        }
#pragma unroll
    for (uint32_t o = 1; o < 64; o <<= 1) {
        lowest = min(lowest, __shfl_xor(lowest, o));
        highest = max(highest, __shfl_xor(highest, o));
    }
    if (t % 64 == 0) {
        atomicMin(&least, lowest);
        atomicMax(&most, highest);
    }
    __syncthreads();
    uint32_t many[kBins], sum = 0;
#pragma unroll
    for (uint32_t i = 0; i < kBins; ++i) {
        const uint32_t k = kBins * t + i;
        many[i] = k < tiles ? bins[k] : 0;
        sum += many[i];
    }
    const Sums s = sums_before<kSortThreads>(sum, 0, part);
    uint32_t at = s.x;
#pragma unroll
    for (uint32_t i = 0; i < kBins; ++i) {
        const uint32_t k = kBins * t + i;
        if (k < tiles) {
            bins[k] = at;
            to.table[(uint64_t)k * to.groups + blockIdx.x] = at;
        }
        at += many[i];
    }
    if (t == 0) {
        to.table[(uint64_t)tiles * to.groups + blockIdx.x] = s.all_x;
        to.seen_by[blockIdx.x] = u32x2{(uint32_t)least, (uint32_t)most};
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i)
        if (token[i] >= 0) {
            const uint32_t tile = ((uint32_t)token[i] & (DEFT_TOKEN_PROMPT - 1)) / kTile;
            to.events[(uint64_t)f0 + bins[tile] + rank[i]] = u32x4{(uint32_t)token[i], (uint32_t)qlo[i], (uint32_t)qhi[i], 0};
        }
}

// A workgroup has kTile logits of `block` queries.  It first looks which of those tokens stand on the queries' paths: pieces of the
// tree that any of its queries sees, or the sorted tokens of its tile, are taken hundreds of stretches at a time into LDS, with the sum
// of their lengths in front of each, and every thread finds the stretch of its next token there by bisection.
template <typename I, typename O, bool COUNTS, bool SORTED, int MOST>
__global__ __launch_bounds__(kThreads) void deft_logits(LogitsArgs a) {
    __shared__ __align__(16) Seen<COUNTS, MOST> seen;
    constexpr uint32_t kStage = SORTED ? kGroups : kPieces;  // stretches at a time
    static_assert(kStage <= kThreads, "one to a thread");
    __shared__ uint32_t before[kStage + 1], bits[SORTED ? 1 : kStage], part[kThreads / 64][2];
    __shared__ int32_t begin[kStage];  // of a stretch, less `before`
    __shared__ Query queries[MOST];
    __shared__ float divisors[MOST];
    __shared__ uint32_t dividing;  // bit q: by query q's the logits are divided
    const uint32_t blocks = gridDim.x / a.tiles, tile = blockIdx.x / blocks, q0 = blockIdx.x % blocks * a.block, block = min(a.block, a.nq - q0);
    const uint32_t first = tile * kTile, t = threadIdx.x, mine = kEach * t, v = first + mine;
    const uint32_t n = v < a.vocab ? min(a.vocab - v, kEach) : 0;
    // What the first look at the tokens waits for is asked for first, and behind it all that does not wait for them.
    u32x4 stretch{};  // its length, where it begins, and the queries that see it
    auto look = [&](uint32_t s0) {
        const uint32_t s = min(s0 + t, a.history - 1);
        if constexpr (SORTED) {
            const uint32_t *from = a.sorted.table + (uint64_t)tile * a.sorted.groups + s;
            const u32x2 seen_by = a.sorted.seen_by[s];
            stretch = u32x4{from[a.sorted.groups], from[0], seen_by[0], seen_by[1]};
        } else {
            stretch = u32x4{(uint32_t)a.pieces.len[s], (uint32_t)a.pieces.begin[s], (uint32_t)a.pieces.qlo[s], (uint32_t)a.pieces.qhi[s]};
        }
    };
    if (a.history) look(0);
    // Queries behind the last are that one.
    uint32_t row[MOST];
#pragma unroll
    for (uint32_t q = 0; q < MOST; ++q) {
        const uint32_t at = q0 + min(q, block - 1);
        row[q] = a.q_order ? (uint32_t)uniform(a.q_order, at) : at;
    }
    if (t < MOST) {
        uint32_t r = row[0];
#pragma unroll
        for (uint32_t q = 1; q < MOST; ++q) r = t == q ? row[q] : r;
        Query q;
        q.repetition = a.repetition ? a.repetition[r] : 1.f;
        q.frequency = COUNTS ? a.frequency[r] : 0.f;
        q.presence = a.presence ? a.presence[r] : 0.f;
        q.bias = !a.bias ? -1 : a.bias_row ? a.bias_row[r] : 0;
        q.mask = !a.mask ? -1 : a.mask_row ? a.mask_row[r] : 0;
        if ((uint32_t)q.bias >= a.n_bias) q.bias = -1;
        if ((uint32_t)q.mask >= a.n_masks) q.mask = -1;
        // (penalties by which logits are divided are kept apart)
        const float given = q.repetition;
        const bool divides = !(given >= kLeastFactor && given <= kMostFactor);
        if (divides) q.repetition = 1.f;
        q.inverse = 1.f / q.repetition;
        divisors[t] = given;
        const uint32_t which = (uint32_t)__ballot(divides);
        if (t == 0) dividing = which;
        queries[t] = q;
    }
    float x[MOST][kEach];
    uint32_t word[MOST];
    const I *logits = static_cast<const I *>(a.logits);
    if (n == kEach) {
#pragma unroll
        for (uint32_t q = 0; q < MOST; ++q) get<I, kEach>(element(logits + (int64_t)row[q] * a.stride, v), x[q]);
    } else if (n) {
#pragma unroll
        for (uint32_t q = 0; q < MOST; ++q) get<I, 1>(element(logits + (int64_t)row[q] * a.stride, v), x[q]);
    }
    if (a.mask && n) {
#pragma unroll
        for (uint32_t q = 0; q < MOST; ++q) {
            const uint32_t m = a.mask_row ? (uint32_t)uniform(a.mask_row, row[q]) : 0;
            word[q] = *element(a.mask + (int64_t)(m < a.n_masks ? m : 0) * a.mask_stride, v / 32) >> (v % 32);
        }
    }
    static_assert(sizeof(seen) % 16 == 0, "cleared in 128-bit words");
    for (uint32_t i = t; i < sizeof(seen) / 16; i += kThreads) reinterpret_cast<u32x4 *>(&seen)[i] = u32x4{0, 0, 0, 0};
    for (uint32_t s0 = 0; s0 < a.history; s0 += kStage) {
        if (s0) look(s0);
        uint32_t on = t < kStage && s0 + t < a.history ? bits_of((int32_t)stretch[2], (int32_t)stretch[3], q0, block) : 0;
        if (SORTED && stretch[0] == stretch[1]) on = 0;
        const uint32_t len = !on ? 0 : SORTED ? stretch[0] - stretch[1] : stretch[0];
        for (uint32_t i = t; i <= kStage; i += kThreads) before[i] = 0xffffffffu;
        const Sums sums = sums_before<kThreads>(len, on != 0, part);
        if (on) {
            before[sums.y] = sums.x;
            begin[sums.y] = (int32_t)((SORTED ? (s0 + t) * kRun : 0) + stretch[1] - sums.x);
            if constexpr (!SORTED) bits[sums.y] = on;
        }
        __syncthreads();
        const uint32_t steps = sums.all_y > 1 ? 1u << (32 - __builtin_clz(sums.all_y - 1)) : 1;
        auto take = [&](auto ahead) {
            constexpr uint32_t kAhead = decltype(ahead)::value;
            for (uint32_t f = kAhead * t; f < sums.all_x; f += kAhead * kThreads) {
                uint32_t k[kAhead];
                u32x4 e[kAhead];
#pragma unroll
                for (uint32_t u = 0; u < kAhead; ++u) {  // (a stretch has a token at least)
                    k[u] = u == 0 ? last_not_above(before, steps, f) : k[u - 1] + (before[k[u - 1] + 1] <= f + u);
                    k[u] = min(k[u], sums.all_y - 1);
                    const uint32_t g = min(f + u, sums.all_x - 1);
                    if constexpr (SORTED)
                        e[u] = a.sorted.events[(uint32_t)(begin[k[u]] + (int32_t)g)];
                    else
                        e[u][0] = (uint32_t)a.pieces.tokens[(int64_t)begin[k[u]] + g];
                }
#pragma unroll
                for (uint32_t u = 0; u < kAhead; ++u) {
                    if (f + u >= sums.all_x) break;
                    const uint32_t which = SORTED ? bits_of((int32_t)e[u][1], (int32_t)e[u][2], q0, block) : bits[k[u]];
                    if (which) see(seen, (int32_t)e[u][0], first, which, block);
                }
            }
        };
        // a thread's tokens side by side, one bisection for all: as many as still leave work for every thread (8000 tokens of one query
        // two by two 11.1 us, four by four 9.8, eight by eight 9.1; 1000 tokens 4.5 and 4.9 by two and four); with eight rows, whose
        // logits are in registers, no more than four (64 x 50001, 4000 tokens, 11.1 -> 12.3 with eight); sorted ones are larger, and
        // two by two is best throughout
        if (sums.all_x <= kThreads)
            take(std::integral_constant<uint32_t, 1>{});
        else if (SORTED || sums.all_x <= 2 * kThreads)
            take(std::integral_constant<uint32_t, 2>{});
        else if (MOST == kMost || sums.all_x <= 4 * kThreads)
            take(std::integral_constant<uint32_t, 4>{});
        else
            take(std::integral_constant<uint32_t, MOST == kMost ? 4 : 8>{});
        __syncthreads();
    }
    __syncthreads();
    if (n == 0) return;
    uint32_t any[kEach], generated[kEach];
    int32_t count[kEach] = {};
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        any[i] = seen.any[mine + i];
        generated[i] = COUNTS ? 0 : seen.generated[mine + i];
    }
    if (const uint32_t which = __builtin_amdgcn_readfirstlane(dividing)) {
#pragma unroll
        for (uint32_t q = 0; q < MOST; ++q) {
            const uint32_t on = which >> q & 1 ? any[0] >> q & 1 | (any[1] >> q & 1) << 1 : 0;
            const float by = divisors[q];
#pragma unroll
            for (uint32_t i = 0; i < kEach; ++i)
                if (on >> i & 1) x[q][i] = x[q][i] > 0 ? x[q][i] / by : x[q][i] * by;
        }
    }
#pragma unroll
    for (uint32_t q = 0; q < MOST; ++q) {
        if (q >= block) break;
        const Query query = queries[q];
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            if ((any[i] >> q) & 1) x[q][i] *= x[q][i] > 0 ? query.inverse : query.repetition;
            if constexpr (COUNTS) {
                count[i] += seen.change[q][mine + i];
                if (count[i] > 0) x[q][i] -= query.frequency * (float)count[i] + query.presence;
            } else {
                if ((generated[i] >> q) & 1) x[q][i] -= query.presence;
            }
        }
        if (query.bias >= 0) {
            const float *from = element(a.bias + (int64_t)__builtin_amdgcn_readfirstlane(query.bias) * a.bias_stride, v);
            float y[kEach];
            if (n == kEach)
                get<float, kEach>(from, y);
            else
                get<float, 1>(from, y);
#pragma unroll
            for (uint32_t i = 0; i < kEach; ++i) x[q][i] += y[i];
        }
        if (query.mask >= 0) {
#pragma unroll
            for (uint32_t i = 0; i < kEach; ++i)
                if (!((word[q] >> i) & 1)) x[q][i] = -__builtin_inff();
        }
        O *to = element(static_cast<O *>(a.out) + (int64_t)row[q] * a.out_stride, v);
        if (n == kEach)
            put<O, kEach>(to, x[q]);
        else
            put<O, 1>(to, x[q]);
    }
}

template <typename I, typename O, int MOST>
void launch(const LogitsArgs &a, bool counts, bool sorted, uint32_t groups, hipStream_t st) {
    auto *kernel = counts ? (sorted ? &deft_logits<I, O, true, true, MOST> : &deft_logits<I, O, true, false, MOST>)
                          : (sorted ? &deft_logits<I, O, false, true, MOST> : &deft_logits<I, O, false, false, MOST>);
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(kThreads), 0, st, a);
}
template <typename I, typename O>
void launch(const LogitsArgs &a, bool counts, bool sorted, uint32_t groups, hipStream_t st) {
    if (a.block == 1)
        launch<I, O, 1>(a, counts, sorted, groups, st);
    else if (a.block <= kMost / 2)
        launch<I, O, kMost / 2>(a, counts, sorted, groups, st);
    else
        launch<I, O, kMost>(a, counts, sorted, groups, st);
}

// Tokens of all pieces, a query's own time and again where pieces are grouped by query.
int64_t tokens_of(const deft_plan_t *plan) {
    int64_t total = plan->tokens.load(std::memory_order_relaxed);
    if (total < 0) {  // (a plan never changes)
        total = 0;
        for (const int32_t len : plan->seg_len) total += len;
        plan->tokens.store(total, std::memory_order_relaxed);
    }
    return total;
}
// A row is cut into tiles, and as many rows to a workgroup as still leave kFill of them (us with 256, 512, 768 and 1024 of them: 20 x
// 128000 12.0, 11.3, 10.9, 13.9, 64 x 50001 14.0, 14.2, 16.1, 18.8, one query the same with all).
struct Shape {
    uint32_t tiles, block;
    uint64_t groups;
};
Shape shape_of(uint32_t nq, uint32_t vocab) {
    Shape s;
    s.tiles = (vocab + kTile - 1) / kTile;
    s.block = (uint32_t)std::clamp<uint64_t>(((uint64_t)nq * s.tiles + kFill - 1) / kFill, 1, kMost);
    s.groups = (uint64_t)s.tiles * ((nq + s.block - 1) / s.block);
    return s;
}
// Whether tokens are sorted before they are looked for.  us, unsorted -> sorted: one query x 128000, 125 workgroups, 9500 tokens 11.1 ->
// 10.9, 13000 13.2 -> 11.6; 4 x 32000 9500 tokens 11.3 -> 12.6, 13000 13.5 -> 13.6; 64 x 50001, 490 workgroups, 9500 tokens 13.9 -> 14.8,
// 13000 16.3 -> 15.9; 80 x 128000, 1250 workgroups, 2000 tokens 16.4 -> 19.0, 4000 19.9 -> 19.1; 200 x 128000, 3125 workgroups, 1200
// tokens 30.5 -> 33.3, 2200 34.4 -> 33.9.  That is in a graph; otherwise the host has a second launch to make, 3 us, so the line is
// drawn somewhat later.
// Pieces beyond the first kPieces are looked through in further steps, each of which costs as much as 2000 tokens where there are few
// workgroups and 4000 where there are 500, and counts as kStepTokens.  In pages of one row: one query x 128000, 600 tokens 6.4 -> 8.4, 1000 6.5 ->
// 8.8, 1500 8.3 -> 9.9, 2000 10.0 -> 10.2, 4000 17.2 -> 11.0; 20 x 128000, 1160 11.0 -> 12.4, 1660 13.3 -> 12.4, 2160 15.4 -> 12.6; 64 x 50001, 1512 12.1 -> 13.6,
// 2012 14.2 -> 13.7; 120 x 128000, 1360 28.7 -> 25.1.  In pages of 16 rows: one query x 128000, 8000 tokens (500 pieces) 9.4 -> 10.9, 8193 (513) 10.5 -> 10.9,
// 8400 11.8 -> 11.1; 4 x 32000, 8225 11.0 -> 12.2, 12000 13.5 -> 13.9; 20 x 128000, 8353 14.5 -> 12.9; 64 x 50001, 8912 16.0 -> 14.6.  In pages of 64, one
// query x 128000: 8400 11.2 -> 11.0, 12000 12.7 -> 11.9.
bool sorts(const deft_plan_t *plan, int64_t total, const Shape &s) {
    if (s.tiles > kMaxTiles || total >= (int64_t(1) << 30)) return false;
    const int64_t steps = (plan->n_segs() + kPieces - 1) / kPieces, cost = total + kStepTokens * std::max<int64_t>(steps - 1, 0);
    return cost * (int64_t)std::max<uint64_t>(s.groups, kFill) > (int64_t)kFewTokens * kFill;
}
struct Space {
    uint64_t groups, table, seen_by, bytes;  // places
};
Space space_of(int64_t total, uint32_t tiles) {
    Space s;
    s.groups = (uint64_t)(total + kRun - 1) / kRun;
    s.table = s.groups * kRun * sizeof(u32x4);
    s.seen_by = s.table + (s.groups * (tiles + 1) + 1) / 2 * 2 * sizeof(uint32_t);
    s.bytes = s.seen_by + s.groups * sizeof(u32x2);
    return s;
}

constexpr int64_t kMaxStride = int64_t(1) << 31;

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

}  // namespace

extern "C" size_t deft_logits_workspace_bytes(const deft_plan_t *plan, int32_t vocab) {
    if (!plan || vocab < 1 || vocab > DEFT_MAX_VOCAB) return 0;
    const Shape shape = shape_of((uint32_t)plan->nq, (uint32_t)vocab);
    const int64_t total = tokens_of(plan);
    return sorts(plan, total, shape) ? (size_t)space_of(total, shape.tiles).bytes : 0;
}

extern "C" int deft_adjust_logits(const deft_plan_t *plan, const void *dev_image, int32_t group, const deft_logits_t *l, void *workspace,
                                  size_t workspace_bytes, void *stream) {
    if (!plan || !l || l->vocab < 1 || l->vocab > DEFT_MAX_VOCAB) return DEFT_EINVAL;
    const int32_t nq = plan->nq;
    const bool history = l->repetition || l->frequency || l->presence;
    if (history && (!l->tokens || !aligned4(l->tokens) || l->n_tokens < deft_plan_rows(plan))) return DEFT_EINVAL;
    if (!aligned4(l->repetition) || !aligned4(l->frequency) || !aligned4(l->presence) || !aligned4(l->bias) || !aligned4(l->mask) ||
        !aligned4(l->bias_row) || !aligned4(l->mask_row))
        return DEFT_EINVAL;
    if (l->reserved != 0) return DEFT_EINVAL;
    if (l->bias && (l->n_bias < 1 || l->bias_stride < (l->n_bias > 1 ? l->vocab : 0) || l->bias_stride > kMaxStride)) return DEFT_EINVAL;
    if (l->mask && (l->n_masks < 1 || l->mask_stride < (l->n_masks > 1 ? (l->vocab + 31) / 32 : 0) || l->mask_stride > kMaxStride)) return DEFT_EINVAL;
    if ((l->bias_row && !l->bias) || (l->mask_row && !l->mask)) return DEFT_EINVAL;
    const deft::Schedule *S = nullptr;
    if (history) {
        if (!dev_image || !deft::aligned16(dev_image) || group <= 0) return DEFT_EINVAL;
        S = deft::find_schedule(plan, group);
        if (!S) return DEFT_ENOTREADY;
    }
    if (nq == 0) return DEFT_OK;
    if (!l->logits || !l->out || (l->logits_f32 && !l->out_f32)) return DEFT_EINVAL;
    const int in_bytes = l->logits_f32 ? 4 : 2, out_bytes = l->out_f32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(l->logits) % in_bytes || reinterpret_cast<uintptr_t>(l->out) % out_bytes) return DEFT_EINVAL;
    if (nq > 1 && (l->stride < 0 || l->out_stride < l->vocab || l->stride > kMaxStride || l->out_stride > kMaxStride)) return DEFT_EINVAL;
    if (nq > 1 && (double)nq * (double)std::max(l->stride, l->out_stride) > 0x1p60) return DEFT_EINVAL;
    if ((double)l->n_bias * (double)l->bias_stride > 0x1p60 || (double)l->n_masks * (double)l->mask_stride > 0x1p60) return DEFT_EINVAL;
    const bool in_place = l->out == l->logits && in_bytes == out_bytes && (nq == 1 || l->stride == l->out_stride);
    const uintptr_t in = reinterpret_cast<uintptr_t>(l->logits), out = reinterpret_cast<uintptr_t>(l->out);
    const uint64_t in_size = in_bytes * ((uint64_t)(nq - 1) * (uint64_t)l->stride + l->vocab), out_size = out_bytes * ((uint64_t)(nq - 1) * (uint64_t)l->out_stride + l->vocab);
    auto meets = [&](const void *p, uint64_t bytes) {  // what is written
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        return p && at < out + out_size && out < at + bytes;
    };
    if (!in_place && in < out + out_size && out < in + in_size) return DEFT_EINVAL;
    const uint64_t words = ((uint64_t)l->vocab + 31) / 32, of_queries = 4 * (uint64_t)nq;
    if (meets(l->bias, 4 * ((uint64_t)(l->n_bias - 1) * (uint64_t)l->bias_stride + l->vocab)) || meets(l->bias_row, of_queries) ||
        meets(l->mask, 4 * ((uint64_t)(l->n_masks - 1) * (uint64_t)l->mask_stride + words)) || meets(l->mask_row, of_queries) ||
        meets(l->repetition, of_queries) || meets(l->frequency, of_queries) || meets(l->presence, of_queries) ||
        (history && meets(l->tokens, 4 * (uint64_t)l->n_tokens)))
        return DEFT_EINVAL;
    LogitsArgs a{};
    a.logits = l->logits;
    a.out = l->out;
    a.stride = l->stride;
    a.out_stride = l->out_stride;
    a.vocab = (uint32_t)l->vocab;
    a.nq = (uint32_t)nq;
    const Shape shape = shape_of(a.nq, a.vocab);
    a.tiles = shape.tiles;
    a.block = shape.block;
    a.repetition = l->repetition;
    a.frequency = l->frequency;
    a.presence = l->presence;
    a.bias = l->bias;
    a.bias_row = l->bias_row;
    a.bias_stride = l->bias_stride;
    a.n_bias = (uint32_t)l->n_bias;
    a.mask = static_cast<const uint32_t *>(l->mask);
    a.mask_row = l->mask_row;
    a.mask_stride = l->mask_stride;
    a.n_masks = (uint32_t)l->n_masks;
    const bool counts = l->frequency != nullptr;
    if (shape.groups * kThreads > UINT32_MAX) return DEFT_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    bool sorted = false;
    if (history && plan->n_segs() > 0) {
        auto at = [&](size_t off) { return reinterpret_cast<const int32_t *>(static_cast<const uint8_t *>(dev_image) + off); };
        a.pieces = {at(S->off_seg_tok_begin), at(S->off_seg_len), at(S->off_seg_qlo), at(S->off_seg_qhi), at(S->off_seg_off), l->tokens, (uint32_t)plan->n_segs()};
        a.q_order = at(S->off_q_order);
        a.history = a.pieces.n;
        const int64_t total = tokens_of(plan);
        sorted = workspace && sorts(plan, total, shape);
        if (sorted) {
            const Space space = space_of(total, a.tiles);
            if (!deft::aligned16(workspace)) return DEFT_EINVAL;
            if (workspace_bytes < space.bytes) return DEFT_EWORKSPACE;
            a.sorted = {static_cast<u32x4 *>(workspace), reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(workspace) + space.table),
                        reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(workspace) + space.seen_by), (uint32_t)space.groups};
            a.history = a.sorted.groups;
            hipLaunchKernelGGL(deft_sort_tokens, dim3(a.sorted.groups), dim3(kSortThreads), 0, st, a.pieces, a.sorted, (uint32_t)total, a.tiles);
            if (!deft::hip_ok(hipGetLastError(), "deft_sort_tokens launch")) return DEFT_EHIP;
        }
    }
    if (l->logits_f32)
        launch<float, float>(a, counts, sorted, (uint32_t)shape.groups, st);
    else if (l->out_f32)
        launch<__bf16, float>(a, counts, sorted, (uint32_t)shape.groups, st);
    else
        launch<__bf16, __bf16>(a, counts, sorted, (uint32_t)shape.groups, st);
    return deft::hip_ok(hipGetLastError(), "deft_logits launch") ? DEFT_OK : DEFT_EHIP;
}
