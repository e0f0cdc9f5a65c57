// The next token's logits, bent by what each query's path holds (penalties for repeated tokens), by biases and by grammar masks.
// Every logit is read once and written once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "deft_device.h"
#include "deft_internal.h"

namespace {

struct LogitsArgs {
    const void *logits;
    void *out;
    int64_t stride, out_stride;
    uint32_t vocab, nq, block, tiles;  // block: queries of a workgroup
    const int32_t *seg_begin, *seg_len, *seg_qlo, *seg_qhi;
    const int32_t *q_order;  // null: queries in the caller's order (no tokens are looked at)
    uint32_t n_segs;         // 0: none are
    const int32_t *tokens;
    const float *repetition, *frequency, *presence;
    const float *bias;
    const uint32_t *mask;
    const int32_t *bias_row, *mask_row;
    int64_t bias_stride, mask_stride;
    uint32_t n_bias, n_masks;
};

constexpr int kThreads = 256, kEach = 4;     // logits of a row to a thread, side by side
constexpr int kTile = kThreads * kEach;      // of a workgroup
constexpr int kMost = 32, kMostCounted = 8;  // queries of a workgroup: bits of a word, and counters that LDS has room for
constexpr int kStage = 1024;                 // pieces at a time

struct Query {
    int32_t row;
    float repetition, inverse, frequency, presence;
    int32_t bias, mask;  // rows of the tables, -1: none
};

template <typename T>
struct Vec;
template <>
struct Vec<float> {
    typedef __attribute__((ext_vector_type(4), aligned(4))) float type;  // (rows of odd length: any element can be a row's first)
    static __device__ __forceinline__ float get(const float *p) { return *p; }
    static __device__ __forceinline__ void get4(const float *p, float *x) {
        const type v = *reinterpret_cast<const type *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i];
    }
    static __device__ __forceinline__ void put(float *p, float x) { *p = x; }
    static __device__ __forceinline__ void put4(float *p, const float *x) { *reinterpret_cast<type *>(p) = type{x[0], x[1], x[2], x[3]}; }
};
template <>
struct Vec<__bf16> {
    typedef __attribute__((ext_vector_type(4), aligned(2))) __bf16 type;
    static __device__ __forceinline__ float get(const __bf16 *p) { return (float)*p; }
    static __device__ __forceinline__ void get4(const __bf16 *p, float *x) {
        const type v = *reinterpret_cast<const type *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)v[i];
    }
    static __device__ __forceinline__ void put(__bf16 *p, float x) { *p = (__bf16)x; }
    static __device__ __forceinline__ void put4(__bf16 *p, const float *x) {
        *reinterpret_cast<type *>(p) = type{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
    }
};

// Queries are in the plan's depth-first order here, in which the queries whose path holds a token are neighbours: `bits` says which
// of the workgroup's queries they are.  With COUNTS a token adds one at the first of them and takes one away behind the last, so
// that the sum over the queries up to one is how often the token stands on that one's path.
template <bool COUNTS>
struct Seen {
    uint32_t any[kTile];                        // bit q: on the path of query q
    uint32_t generated[COUNTS ? 1 : kTile];     // the same, prompt tokens left out
    int32_t change[COUNTS ? kMostCounted : 1][COUNTS ? kTile : 1];
};

template <bool COUNTS>
__device__ __forceinline__ void see(Seen<COUNTS> &seen, int32_t token, uint32_t first, uint32_t bits, uint32_t block) {
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

// A workgroup has kTile logits of `block` queries.  It first looks which of those tokens stand on the queries' paths: pieces of the
// tree that any of its queries sees are taken kStage at a time into LDS, with the sum of their lengths in front of each, and every
// thread finds the piece of its next token there by bisection.
template <typename I, typename O, bool COUNTS>
__global__ __launch_bounds__(kThreads) void deft_logits(LogitsArgs a) {
    __shared__ Seen<COUNTS> seen;
    __shared__ uint32_t before[kStage + 1], bits[kStage];
    __shared__ int32_t begin[kStage];  // row of a piece's first token, less `before`
    __shared__ uint32_t part[kThreads / 64];
    __shared__ Query queries[kMost];
    const uint32_t tile = blockIdx.x % a.tiles, q0 = blockIdx.x / a.tiles * a.block, block = min(a.block, a.nq - q0);
    const uint32_t first = tile * kTile, t = threadIdx.x, lane = t & 63;
    if (t < block) {
        Query q;
        q.row = a.q_order ? a.q_order[q0 + t] : (int32_t)(q0 + t);
        q.repetition = a.repetition ? a.repetition[q.row] : 1.f;
        q.inverse = 1.f / q.repetition;
        q.frequency = a.frequency ? a.frequency[q.row] : 0.f;
        q.presence = a.presence ? a.presence[q.row] : 0.f;
        q.bias = a.bias ? (a.bias_row ? a.bias_row[q.row] : 0) : -1;
        q.mask = a.mask ? (a.mask_row ? a.mask_row[q.row] : 0) : -1;
        if ((uint32_t)q.bias >= a.n_bias) q.bias = -1;
        if ((uint32_t)q.mask >= a.n_masks) q.mask = -1;
        queries[t] = q;
    }
    for (uint32_t i = t; i < sizeof(seen) / 4; i += kThreads) reinterpret_cast<uint32_t *>(&seen)[i] = 0;
    for (uint32_t s0 = 0; s0 < a.n_segs; s0 += kStage) {
        uint32_t len[4], on[4], sum = 0, many = 0;
        int32_t at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t s = s0 + 4 * t + i;
            len[i] = on[i] = 0;
            at[i] = 0;
            if (s < a.n_segs) {
                const int32_t lo = max(a.seg_qlo[s] - (int32_t)q0, 0), hi = min(a.seg_qhi[s] - (int32_t)q0, (int32_t)block);
                if (lo < hi) {
                    on[i] = (0xffffffffu >> (32 - hi)) & (0xffffffffu << lo);
                    len[i] = (uint32_t)a.seg_len[s];
                    at[i] = a.seg_begin[s];
                }
            }
            sum += len[i];
            many += on[i] != 0;
        }
        // sums over the threads in front, of lengths and of pieces; both are below 2^32 in all
        uint32_t sums = sum, pieces = many;
#pragma unroll
        for (uint32_t o = 1; o < 64; o <<= 1) {
            const uint32_t x = __shfl_up(sums, o), y = __shfl_up(pieces, o);
            if (lane >= o) {
                sums += x;
                pieces += y;
            }
        }
        __shared__ uint32_t part_pieces[kThreads / 64];
        if (lane == 63) {
            part[t / 64] = sums;
            part_pieces[t / 64] = pieces;
        }
        __syncthreads();
        uint32_t total = 0, all = 0, base = sums - sum, slot = pieces - many;
#pragma unroll
        for (uint32_t w = 0; w < kThreads / 64; ++w) {
            if (w < t / 64) {
                base += part[w];
                slot += part_pieces[w];
            }
            total += part[w];
            all += part_pieces[w];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!on[i]) continue;
            before[slot] = base;
            begin[slot] = at[i] - (int32_t)base;
            bits[slot++] = on[i];
            base += len[i];
        }
        __syncthreads();
        for (uint32_t f = t; f < total; f += kThreads) {
            uint32_t lo = 0, hi = all;  // before[lo] <= f < before[hi]
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) / 2;
                (before[mid] <= f ? lo : hi) = mid;
            }
            see(seen, a.tokens[(int64_t)begin[lo] + f], first, bits[lo], block);
        }
        __syncthreads();
    }
    __syncthreads();
    const uint32_t mine = kEach * t, v = first + mine;
    if (v >= a.vocab) return;
    const uint32_t n = min(a.vocab - v, (uint32_t)kEach);
    uint32_t any[kEach], generated[kEach];
    int32_t count[kEach] = {};
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        any[i] = seen.any[mine + i];
        generated[i] = COUNTS ? 0 : seen.generated[mine + i];
    }
    for (uint32_t q = 0; q < block; ++q) {
        const Query &query = queries[q];
        const I *from = static_cast<const I *>(a.logits) + (int64_t)query.row * a.stride + v;
        O *to = static_cast<O *>(a.out) + (int64_t)query.row * a.out_stride + v;
        float x[kEach] = {};
        if (n == kEach)
            Vec<I>::get4(from, x);
        else
            for (uint32_t i = 0; i < n; ++i) x[i] = Vec<I>::get(from + i);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if ((any[i] >> q) & 1) x[i] *= x[i] > 0 ? query.inverse : query.repetition;
            if constexpr (COUNTS) {
                count[i] += seen.change[q][mine + i];
                if (count[i] > 0) x[i] -= query.frequency * (float)count[i] + query.presence;
            } else {
                if ((generated[i] >> q) & 1) x[i] -= query.presence;
            }
        }
        if (query.bias >= 0) {
            const float *b = a.bias + (int64_t)query.bias * a.bias_stride + v;
            for (uint32_t i = 0; i < n; ++i) x[i] += b[i];
        }
        if (query.mask >= 0) {
            const uint32_t word = a.mask[(int64_t)query.mask * a.mask_stride + v / 32] >> (v % 32);
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (!((word >> i) & 1)) x[i] = -__builtin_inff();
        }
        if (n == kEach)
            Vec<O>::put4(to, x);
        else
            for (uint32_t i = 0; i < n; ++i) Vec<O>::put(to + i, x[i]);
    }
}

template <typename I, typename O>
void launch(const LogitsArgs &a, bool counts, uint32_t groups, hipStream_t st) {
    if (counts)
        hipLaunchKernelGGL((deft_logits<I, O, true>), dim3(groups), dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((deft_logits<I, O, false>), dim3(groups), dim3(kThreads), 0, st, a);
}

constexpr int64_t kMaxStride = int64_t(1) << 31;  // times 2^31 queries of 4 bytes: within 64 bits

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

}  // namespace

extern "C" int deft_adjust_logits(const deft_plan_t *plan, const void *dev_image, int32_t group, const deft_logits_t *l, void *stream) {
    if (!plan || !l || l->vocab < 1 || l->vocab > DEFT_MAX_VOCAB) return DEFT_EINVAL;
    const int32_t nq = plan->nq;
    const bool history = l->repetition || l->frequency || l->presence;
    if (history && (!l->tokens || !aligned4(l->tokens) || l->n_tokens < deft_plan_rows(plan))) return DEFT_EINVAL;
    if (!aligned4(l->repetition) || !aligned4(l->frequency) || !aligned4(l->presence) || !aligned4(l->bias) || !aligned4(l->mask) ||
        !aligned4(l->bias_row) || !aligned4(l->mask_row))
        return DEFT_EINVAL;
    if (l->bias && (l->n_bias < 1 || l->bias_stride < (l->n_bias > 1 ? l->vocab : 0))) return DEFT_EINVAL;
    if (l->mask && (l->n_masks < 1 || l->mask_stride < (l->n_masks > 1 ? (l->vocab + 31) / 32 : 0))) return DEFT_EINVAL;
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
    const bool in_place = l->out == l->logits && in_bytes == out_bytes && (nq == 1 || l->stride == l->out_stride);
    const uintptr_t in = reinterpret_cast<uintptr_t>(l->logits), out = reinterpret_cast<uintptr_t>(l->out);
    const uint64_t in_size = in_bytes * ((uint64_t)(nq - 1) * (uint64_t)l->stride + l->vocab), out_size = out_bytes * ((uint64_t)(nq - 1) * (uint64_t)l->out_stride + l->vocab);
    if (!in_place && in < out + out_size && out < in + in_size) return DEFT_EINVAL;
    LogitsArgs a{};
    a.logits = l->logits;
    a.out = l->out;
    a.stride = l->stride;
    a.out_stride = l->out_stride;
    a.vocab = (uint32_t)l->vocab;
    a.nq = (uint32_t)nq;
    a.tiles = (a.vocab + kTile - 1) / kTile;
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
    if (history) {
        auto at = [&](size_t off) { return reinterpret_cast<const int32_t *>(static_cast<const uint8_t *>(dev_image) + off); };
        a.seg_begin = at(S->off_seg_tok_begin);
        a.seg_len = at(S->off_seg_len);
        a.seg_qlo = at(S->off_seg_qlo);
        a.seg_qhi = at(S->off_seg_qhi);
        a.q_order = at(S->off_q_order);
        a.n_segs = (uint32_t)plan->n_segs();
        a.tokens = l->tokens;
    }
    const bool counts = l->frequency != nullptr;
    const uint64_t work = (uint64_t)a.nq * a.tiles;
    a.block = (uint32_t)std::clamp<uint64_t>((work + 1023) / 1024, 1, counts ? kMostCounted : kMost);
    const uint64_t groups = (uint64_t)a.tiles * ((a.nq + a.block - 1) / a.block);
    if (groups * kThreads > UINT32_MAX) return DEFT_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (l->logits_f32)
        launch<float, float>(a, counts, (uint32_t)groups, st);
    else if (l->out_f32)
        launch<__bf16, float>(a, counts, (uint32_t)groups, st);
    else
        launch<__bf16, __bf16>(a, counts, (uint32_t)groups, st);
    return deft::hip_ok(hipGetLastError(), "deft_logits launch") ? DEFT_OK : DEFT_EHIP;
}
