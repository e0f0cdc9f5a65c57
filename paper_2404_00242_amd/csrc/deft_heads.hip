// What happens to the heads of a projection's output before attention reads them: RMS norms of queries and keys, rotation by their
// positions, keys and values into the rows of a cache.  One pass: every head is read once and written once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "deft_device.h"
#include "deft_lists.h"

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// floor(n / d), given inverse(d)
uint32_t inverse(uint32_t d) { return d == 1 ? 0xffffffffu : (uint32_t)((uint64_t(1) << 32) / d); }
__device__ __forceinline__ uint32_t divide(uint32_t n, uint32_t d, uint32_t inv) {
    const uint32_t q = __umulhi(n, inv);  // floor(n / d) or one less
    return n - q * d >= d ? q + 1 : q;
}

enum { kQ, kK, kV, kParts };
enum Turn { kNoTurn, kHalf, kInterleaved };

// Heads of one kind.  Strides in elements.
struct Part {
    const uint16_t *x;
    uint16_t *out;
    const void *weight;  // null: not normalised
    int64_t token, head, out_token, out_head, weight_head;
};

struct HeadsArgs {
    Part part[kParts];
    const int32_t *positions;
    const u32x2 *entries;  // {row of k's and v's out, token}; null: every token, and its row is its own number
    uint32_t waves, chunks, inv_chunks;  // of the launch; of a token
    uint32_t k_begin, v_begin, heads;    // of a token's heads, q's before k's before v's
    uint32_t rot, wide;                  // wide: weights are float
    float eps, offset, factor;
    uint64_t turns[64];  // of a turn a position, in 2^-64
};

// cos and sin of 2 pi phase / 2^32: the nearest quarter turn is taken off exactly, and what is left, at most pi / 4, goes through the
// Taylor polynomials of degree 8 and 9 (their first term left out is below 3e-8; with the roundings 1.5e-7 all in all).
__device__ __forceinline__ void cos_sin(uint32_t phase, float &c, float &s) {
    const uint32_t quarter = (phase + 0x20000000u) >> 30;
    const float t = (float)(int32_t)(phase - (quarter << 30)) * 1.46291807926715968e-9f;  // 2 pi / 2^32
    const float t2 = t * t;
    const float sn = fmaf(t * t2, fmaf(t2, fmaf(t2, fmaf(t2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), t);
    const float cs = fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, 1.f / 40320, -1.f / 720), 1.f / 24), -0.5f), 1.f);
    c = quarter & 1 ? sn : cs;
    s = quarter & 1 ? cs : sn;
    if ((quarter + 1) & 2) c = -c;
    if (quarter & 2) s = -s;
}

__device__ __forceinline__ float lower(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
__device__ __forceinline__ float upper(uint32_t x) { return __builtin_bit_cast(float, x & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 r = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ void unpack8(const u32x4 &x, float *y) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[2 * i] = lower(x[i]);
        y[2 * i + 1] = upper(x[i]);
    }
}
__device__ __forceinline__ u32x4 pack8(const float *y) { return u32x4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])}; }
__device__ __forceinline__ void load8(const void *p, uint32_t at, bool wide, float *y) {
    if (wide) {
        const f32x4 *w = reinterpret_cast<const f32x4 *>(static_cast<const float *>(p) + at);
        const f32x4 a = w[0], b = w[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = a[i];
            y[4 + i] = b[i];
        }
    } else {
        unpack8(*reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p) + at), y);
    }
}

// A wave has one token and 64 / (D / 16) of its heads, sixteen elements of a head to a lane: two groups of eight that in the half layout
// are partners of one another, so that no lane needs another's elements.  The angles of a token are the same for all its heads: a
// lane makes one pair's cosine and sine, and the wave's LDS hands them round.
template <int D, int TURN, bool NORM>
__global__ __launch_bounds__(256) void deft_heads(HeadsArgs a) {
    constexpr uint32_t kLanes = D / 16, kHeads = 64 / kLanes;
    __shared__ float table[4][2][64];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * 4 + wave;
    if (unit >= a.waves) return;
    const uint32_t entry = divide(unit, a.chunks, a.inv_chunks);
    uint32_t token = entry, row = entry;
    if (a.entries) {
        const u32x2 e = a.entries[entry];
        row = e[0];
        token = e[1];
    }
    const uint32_t j = lane % kLanes, asked = (unit - entry * a.chunks) * kHeads + lane / kLanes, at = min(asked, a.heads - 1);
    const int kind = at >= a.v_begin ? kV : at >= a.k_begin ? kK : kQ;
    const Part &p = a.part[kind];
    const uint32_t head = at - (kind == kV ? a.v_begin : kind == kK ? a.k_begin : 0);
    // the lane's two groups: interleaved anywhere in the head, in the half layout partners, and of the elements that do not turn the same
    const bool turned = TURN == kHalf && kind != kV && 16 * j < a.rot;
    const uint32_t begin = turned || TURN != kHalf || kind == kV ? 0 : a.rot, width = turned ? a.rot : D - begin;
    const uint32_t first = begin + 8 * (j - begin / 16), second = first + width / 2;
    const bool turned0 = TURN == kInterleaved ? kind != kV && first < a.rot : turned, turned1 = TURN == kInterleaved ? kind != kV && second < a.rot : turned;
    const uint16_t *x = p.x + ((int64_t)token * p.token + (int64_t)head * p.head);
    const u32x4 x0 = *reinterpret_cast<const u32x4 *>(x + first), x1 = *reinterpret_cast<const u32x4 *>(x + second);
    float (*cs)[64] = table[wave];
    if (TURN != kNoTurn && 2 * lane < a.rot) {
        const int32_t position = a.positions[token];
        const uint64_t turns = a.turns[lane];
        const uint32_t low = (uint32_t)turns, high = (uint32_t)(turns >> 32);
        uint32_t phase = __umulhi((uint32_t)position, low) + (uint32_t)position * high;
        if (position < 0) phase -= low;
        float c, s;
        cos_sin(phase, c, s);
        cs[0][lane] = c * a.factor;
        cs[1][lane] = s * a.factor;
    }
    float y0[8], y1[8];
    unpack8(x0, y0);
    unpack8(x1, y1);
    const bool normed = NORM && p.weight;
    if (NORM) {
        float w0[8], w1[8];
        if (normed) {
            const uint32_t w = (uint32_t)(head * p.weight_head);
            load8(p.weight, w + first, a.wide, w0);
            load8(p.weight, w + second, a.wide, w1);
        }
        auto mean = [&](float eps) {
            float sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(y0[i], y0[i], fmaf(y1[i], y1[i], sum));
#pragma unroll
            for (uint32_t o = 1; o < kLanes; o <<= 1) sum += __shfl_xor(sum, o);
            return fmaf(sum, 1.f / D, eps);
        };
        float m = mean(a.eps);
        if (normed && (m > 0x1p100f || m < 0x1p-80f)) {  // squares near the ends of fp32: the head is taken by a power of two of itself
            const float by = m > 1.f ? 0x1p-70f : 0x1p90f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y0[i] *= by;
                y1[i] *= by;
            }
            m = mean(a.eps * by * by);
        }
        const float r = __builtin_amdgcn_rsqf(m);
        if (normed) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y0[i] *= r * (w0[i] + a.offset);
                y1[i] *= r * (w1[i] + a.offset);
            }
        }
    }
    auto turn = [](float &u, float &v, float c, float s) {
        const float t = u * c - v * s;
        v = v * c + u * s;
        u = t;
    };
    auto cosines = [&](uint32_t i) { return *reinterpret_cast<const f32x4 *>(&cs[0][i]); };
    auto sines = [&](uint32_t i) { return *reinterpret_cast<const f32x4 *>(&cs[1][i]); };
    if (TURN == kHalf && turned) {
        const f32x4 c0 = cosines(first), c1 = cosines(first + 4), s0 = sines(first), s1 = sines(first + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            turn(y0[i], y1[i], c0[i], s0[i]);
            turn(y0[4 + i], y1[4 + i], c1[i], s1[i]);
        }
    }
    if (TURN == kInterleaved && turned0) {
        const f32x4 c = cosines(first / 2), s = sines(first / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) turn(y0[2 * i], y0[2 * i + 1], c[i], s[i]);
    }
    if (TURN == kInterleaved && turned1) {
        const f32x4 c = cosines(second / 2), s = sines(second / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) turn(y1[2 * i], y1[2 * i + 1], c[i], s[i]);
    }
    if (asked >= a.heads) return;
    uint16_t *out = p.out + ((int64_t)(kind == kQ ? token : row) * p.out_token + (int64_t)head * p.out_head);
    // bits as they are where nothing is done to them; none of it is read again here
    __builtin_nontemporal_store(turned0 || normed ? pack8(y0) : x0, reinterpret_cast<u32x4 *>(out + first));
    __builtin_nontemporal_store(turned1 || normed ? pack8(y1) : x1, reinterpret_cast<u32x4 *>(out + second));
}

// ---- host ----

constexpr uint64_t kMaxWaves = 1u << 22;  // of a launch

template <int D, int TURN, bool NORM>
void launch(const HeadsArgs &a, hipStream_t st) {
    hipLaunchKernelGGL((deft_heads<D, TURN, NORM>), dim3((a.waves + 3) / 4), dim3(256), 0, st, a);
}
template <int D, int TURN>
void launch(const HeadsArgs &a, bool norm, hipStream_t st) {
    norm ? launch<D, TURN, true>(a, st) : launch<D, TURN, false>(a, st);
}
template <int D>
void launch(const HeadsArgs &a, int turn, bool norm, hipStream_t st) {
    turn == kNoTurn ? launch<D, kNoTurn>(a, norm, st) : turn == kHalf ? launch<D, kHalf>(a, norm, st) : launch<D, kInterleaved>(a, norm, st);
}

// Memory that a part is read from or written to: `rows` times `heads` stretches of d elements.
struct Area {
    uintptr_t begin, end;
    int64_t row, head;  // strides, bytes
    int64_t heads, d;   // d in bytes
    bool same(const Area &o) const { return begin == o.begin && end == o.end && row == o.row && head == o.head; }
};
Area area(const void *p, int64_t rows, int64_t heads, int64_t d, int64_t row, int64_t head) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return {at, rows && heads ? at + 2 * (uint64_t)((rows - 1) * row + (heads - 1) * head + d) : at, 2 * row, 2 * head, heads, 2 * d};
}
// Whether two have no byte in common: apart altogether, or slices of the same rows or heads of a wider tensor.
bool apart(const Area &a, const Area &b) {
    if (a.begin >= b.end || b.begin >= a.end) return true;
    const Area &l = a.begin <= b.begin ? a : b, &h = a.begin <= b.begin ? b : a;
    const int64_t by = (int64_t)(h.begin - l.begin);
    if (l.row == h.row && l.row > 0) {
        const int64_t at = by % l.row;
        if (at >= (l.heads - 1) * l.head + l.d && at + (h.heads - 1) * h.head + h.d <= l.row) return true;
    }
    if (l.head == h.head && l.head > 0 && l.row % l.head == 0 && h.row % l.head == 0) {
        const int64_t at = by % l.head;
        return at >= l.d && at + h.d <= l.head;
    }
    return false;
}
// Whether no element of a tensor is another's memory.
bool plain(int64_t n, const deft_heads_t &p, int64_t d) {
    if (n > 1 && p.heads > 1)
        return (p.head_stride >= d && p.token_stride >= (p.heads - 1) * p.head_stride + d) ||
               (p.token_stride >= d && p.head_stride >= (n - 1) * p.token_stride + d);
    return (n <= 1 || p.token_stride >= d) && (p.heads <= 1 || p.head_stride >= d);
}

constexpr int64_t kMaxStride = int64_t(1) << 40;

// One call.  parts: q, k, v, each may be null; pool: rows of k's and v's out where the call has a list.
int run(const deft_heads_t *const (&parts)[kParts], int64_t n, int32_t d, float eps, float offset, const int32_t *positions,
        const deft_rope_t *rope, const u32x2 *entries, int64_t pool, void *stream) {
    if (n < 0 || (d != 64 && d != 128)) return DEFT_EINVAL;
    if (rope && (rope->rot < 16 || rope->rot > d || rope->rot % 16 || (rope->layout != DEFT_ROPE_HALF && rope->layout != DEFT_ROPE_INTERLEAVED)))
        return DEFT_EINVAL;
    if (rope && ((!positions && n > 0) || (reinterpret_cast<uintptr_t>(positions) & 3))) return DEFT_EINVAL;
    HeadsArgs a{};
    Area in[kParts], out[kParts];
    uint32_t begin[kParts + 1] = {};
    bool norm = false, wide = false;
    for (int i = 0; i < kParts; ++i) {
        const deft_heads_t *p = parts[i];
        in[i] = out[i] = Area{};
        begin[i + 1] = begin[i];
        if (!p || p->heads == 0) continue;
        if (p->heads < 0 || p->heads > DEFT_MAX_Q8_HEADS) return DEFT_EINVAL;
        if (p->weight) {
            if (i == kV || !(eps >= 0) || !std::isfinite(eps) || !std::isfinite(offset)) return DEFT_EINVAL;
            if (!deft::aligned16(p->weight) || p->weight_stride < 0 || p->weight_stride % 8 || p->weight_stride > 4096) return DEFT_EINVAL;
            if (norm && wide != (p->weight_f32 != 0)) return DEFT_EINVAL;
            norm = true;
            wide = p->weight_f32 != 0;
        }
        if (n == 0) continue;
        if (!p->x || !p->out || !deft::aligned16(p->x) || !deft::aligned16(p->out)) return DEFT_EINVAL;
        if ((p->token_stride | p->head_stride) & 7) return DEFT_EINVAL;
        if (p->token_stride < 0 || p->head_stride < 0 || p->token_stride > kMaxStride || p->head_stride > kMaxStride) return DEFT_EINVAL;
        if ((double)n * (double)p->token_stride + (double)p->heads * (double)p->head_stride > 0x1p60) return DEFT_EINVAL;
        const bool stored = entries && i != kQ, in_place = !stored && p->out == p->x;
        if (in_place && !plain(n, *p, d)) return DEFT_EINVAL;
        Part &t = a.part[i];
        t.x = static_cast<const uint16_t *>(p->x);
        t.out = static_cast<uint16_t *>(p->out);
        t.weight = p->weight;
        t.weight_head = p->weight_stride;
        t.token = p->token_stride;
        t.head = p->head_stride;
        t.out_token = in_place ? t.token : (int64_t)p->heads * d;
        t.out_head = in_place ? t.head : d;
        in[i] = area(p->x, n, p->heads, d, t.token, t.head);
        out[i] = area(p->out, stored ? pool : n, p->heads, d, t.out_token, t.out_head);
        begin[i + 1] += (uint32_t)p->heads;
    }
    for (int i = 0; i < kParts; ++i)
        for (int j = 0; j < kParts; ++j) {
            if (out[i].begin == out[i].end) continue;
            if (!(i == j && out[i].same(in[i])) && !apart(out[i], in[j])) return DEFT_EINVAL;
            if (j < i && !apart(out[i], out[j])) return DEFT_EINVAL;
        }
    if (n == 0 || begin[kParts] == 0) return DEFT_OK;
    a.k_begin = begin[kK];
    a.v_begin = begin[kV];
    a.heads = begin[kParts];
    a.chunks = (a.heads + 64 / (d / 16) - 1) / (64 / (d / 16));
    a.inv_chunks = inverse(a.chunks);
    a.positions = positions;
    a.entries = entries;
    a.eps = eps;
    a.offset = offset;
    a.wide = wide;
    if (rope) {
        a.rot = (uint32_t)rope->rot;
        a.factor = rope->factor;
        std::copy(rope->turns, rope->turns + rope->rot / 2, a.turns);
    }
    const int turn = !rope ? kNoTurn : rope->layout == DEFT_ROPE_HALF ? kHalf : kInterleaved;
    const int64_t most = (int64_t)(kMaxWaves / a.chunks);
    for (int64_t left = n, now; left > 0; left -= now) {
        now = std::min(left, most);
        a.waves = (uint32_t)now * a.chunks;
        d == 128 ? launch<128>(a, turn, norm, static_cast<hipStream_t>(stream)) : launch<64>(a, turn, norm, static_cast<hipStream_t>(stream));
        if (!deft::hip_ok(hipGetLastError(), "deft_heads launch")) return DEFT_EHIP;
        if (a.entries) {
            a.entries += now;
            continue;
        }
        if (a.positions) a.positions += now;
        for (Part &p : a.part) {
            p.x += now * p.token;
            p.out += now * p.out_token;
        }
    }
    return DEFT_OK;
}

}  // namespace

extern "C" int deft_rotate(const deft_heads_t *x, int32_t n, int32_t d, const int32_t *positions, const deft_rope_t *rope, void *stream) {
    if (!x || !rope || x->weight) return DEFT_EINVAL;
    return run({x, nullptr, nullptr}, n, d, 0, 0, positions, rope, nullptr, 0, stream);
}

extern "C" int deft_qk_norm_rotate(const deft_heads_t *q, const deft_heads_t *k, int32_t n, int32_t d, float eps, float weight_offset,
                                   const int32_t *positions, const deft_rope_t *rope, void *stream) {
    return run({q, k, nullptr}, n, d, eps, weight_offset, positions, rope, nullptr, 0, stream);
}

extern "C" int deft_qkv_store(const deft_kv_list_t *list, const void *dev_image, const deft_heads_t *q, const deft_heads_t *k, const deft_heads_t *v,
                              int32_t n_rows, int32_t d, float eps, float weight_offset, const int32_t *positions, const deft_rope_t *rope,
                              void *stream) {
    if (!list || list->copies || !dev_image || !deft::aligned16(dev_image) || !k || !v || k->heads < 1 || k->heads != v->heads) return DEFT_EINVAL;
    if (n_rows < 0 || list->pool > n_rows) return DEFT_EINVAL;
    const u32x2 *entries = reinterpret_cast<const u32x2 *>(static_cast<const uint8_t *>(dev_image) + list->off_entries);
    return run({q, k, v}, list->entries, d, eps, weight_offset, positions, rope, entries, n_rows, stream);
}
