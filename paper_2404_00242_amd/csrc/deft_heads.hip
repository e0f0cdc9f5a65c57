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
    uint32_t heads, chunk;  // a token's first wave for them
};

struct HeadsArgs {
    Part part[kParts];
    const int32_t *positions;
    const u32x2 *entries;  // {row of k's and v's out, token}; null: every token, and its row is its own number
    uint32_t waves, chunks, inv_chunks;  // of the launch; of a token
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

// Eight weights as they lie in memory, and as floats.
struct Weights {
    u32x4 a, b;  // b: the second four floats
};
__device__ __forceinline__ Weights weights_at(const void *p, uint32_t at, bool wide) {
    Weights w;
    if (wide) {
        const u32x4 *x = reinterpret_cast<const u32x4 *>(static_cast<const float *>(p) + at);
        w.a = x[0];
        w.b = x[1];
    } else {
        w.a = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p) + at);
    }
    return w;
}
__device__ __forceinline__ void unpack_weights(const Weights &w, bool wide, float offset, float *y) {
    if (wide) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = __builtin_bit_cast(float, (uint32_t)w.a[i]);
            y[4 + i] = __builtin_bit_cast(float, (uint32_t)w.b[i]);
        }
    } else {
        unpack8(w.a, y);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] += offset;
}

// A value that is the same for all lanes, by a scalar load.
template <typename T>
__device__ __forceinline__ T uniform(const T *p, uint32_t i) {
    return *((const __attribute__((address_space(4))) T *)(uintptr_t)(p + i));
}

// A wave has one token and 64 / (D / 16) of its heads of one kind (what tells queries, keys and values apart is then in scalar registers:
// 8192 tokens x 40 heads normalised and turned 32.0 -> 28.1 us), sixteen elements of a head to a lane: two groups of eight that in the
// half layout are partners of one another, so that no lane needs another's elements.  The angles of a token are the same for all its
// heads: a lane makes one pair's cosine and sine, and the wave's LDS hands them round.
// Bound by HBM where calls are large: 8192 tokens x 40 heads of 128, us: copied by this kernel 26.8, turned 27.1, normalised 27.1, both
// 28.0 (6.0 TB/s); by the host's call, and 3 to 4 us of launch and dependent loads, where they are a decode iteration's.  Two or more
// batches of heads to a wave, 8192 x 32 turned: 21.0 -> 21.8.  Stores that stay in the caches: 8192 x 32 20.7 -> 25.1.
template <int D, int TURN, bool NORM>
__global__ __launch_bounds__(256) void deft_heads(HeadsArgs a) {
    constexpr uint32_t kLanes = D / 16, kHeads = 64 / kLanes;
    __shared__ float table[4][2][64];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * 4 + wave;
    if (unit >= a.waves) return;
    const uint32_t entry = divide(unit, a.chunks, a.inv_chunks), chunk = unit - entry * a.chunks;
    const int kind = chunk >= a.part[kV].chunk ? kV : chunk >= a.part[kK].chunk ? kK : kQ;
    const Part &p = a.part[kind];
    uint32_t token = entry, row = entry;
    if (a.entries) {
        const u32x2 e = uniform(a.entries, entry);
        row = kind == kQ ? e[1] : e[0];
        token = e[1];
    }
    // the lane's two groups: interleaved anywhere in the head, in the half layout partners, and of the elements that do not turn the same
    const uint32_t j = lane % kLanes, rot = kind == kV ? 0 : a.rot;
    const bool turned = TURN == kHalf && 16 * j < rot;
    const uint32_t begin = turned || TURN != kHalf ? 0 : rot, width = turned ? rot : D - begin;
    const uint32_t first = begin + 8 * (j - begin / 16), second = first + width / 2;
    const bool turned0 = TURN == kInterleaved ? first < rot : turned, turned1 = TURN == kInterleaved ? second < rot : turned;
    const uint32_t head = (chunk - p.chunk) * kHeads + lane / kLanes, at = min(head, p.heads - 1);  // (heads behind the last are that one)
    const uint16_t *x = p.x + ((int64_t)token * p.token + (int64_t)at * p.head);
    // What the angles and the norm wait for is asked for in front of the heads, by vector loads: those come back in order, and a scalar
    // load of the position would hold up everything behind the next wait for any scalar load.
    int32_t position = 0;
    uint64_t turns = 0;
    if (TURN != kNoTurn && 2 * lane < rot) {
        uint32_t of = token;
        asm("" : "+v"(of));
        position = a.positions[of];
        turns = a.turns[lane];
    }
    const bool normed = NORM && p.weight;
    Weights v0, v1;
    if (normed) {
        const uint32_t w = at * (uint32_t)p.weight_head;
        v0 = weights_at(p.weight, w + first, a.wide);
        v1 = weights_at(p.weight, w + second, a.wide);
    }
    const u32x4 x0 = *reinterpret_cast<const u32x4 *>(x + first), x1 = *reinterpret_cast<const u32x4 *>(x + second);
    float (*cs)[64] = table[wave];
    if (TURN != kNoTurn && 2 * lane < rot) {
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
    if (normed) {
        float w0[8], w1[8];
        unpack_weights(v0, a.wide, a.offset, w0);
        unpack_weights(v1, a.wide, a.offset, w1);
        auto mean = [&](float eps) {
            float sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(y0[i], y0[i], fmaf(y1[i], y1[i], sum));
#pragma unroll
            for (uint32_t o = 1; o < kLanes; o <<= 1) sum += __shfl_xor(sum, o);
            return fmaf(sum, 1.f / D, eps);
        };
        float m = mean(a.eps);
        if (m > 0x1p100f || m < 0x1p-80f) {  // squares near the ends of fp32: the head is taken by a power of two of itself
            const float by = m > 1.f ? 0x1p-70f : 0x1p90f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y0[i] *= by;
                y1[i] *= by;
            }
            m = mean(a.eps * by * by);
        }
        const float r = __builtin_amdgcn_rsqf(m);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y0[i] *= r * w0[i];
            y1[i] *= r * w1[i];
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
    if (head >= p.heads) return;
    uint16_t *out = p.out + ((int64_t)row * p.out_token + (int64_t)head * p.out_head);
    // bits as they are where nothing is done to them; none of it is read again here
    __builtin_nontemporal_store(turned0 || normed ? pack8(y0) : x0, reinterpret_cast<u32x4 *>(out + first));
    __builtin_nontemporal_store(turned1 || normed ? pack8(y1) : x1, reinterpret_cast<u32x4 *>(out + second));
}

// ---- host ----

constexpr uint64_t kMaxWaves = 1u << 22;  // of a launch

template <int D, int TURN>
void launch(const HeadsArgs &a, bool norm, hipStream_t st) {
    auto *kernel = norm ? &deft_heads<D, TURN, true> : &deft_heads<D, TURN, false>;
    hipLaunchKernelGGL(kernel, dim3((a.waves + 3) / 4), dim3(256), 0, st, a);
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
    uint32_t heads = 0;
    bool norm = false, wide = false;
    for (int i = 0; i < kParts; ++i) {
        const deft_heads_t *p = parts[i];
        in[i] = out[i] = Area{};
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
        t.heads = (uint32_t)p->heads;
        heads += t.heads;
    }
    for (int i = 0; i < kParts; ++i)  // what is written is nobody else's, and nobody's input but the part's own, in place
        for (int j = 0; j < kParts; ++j) {
            if (out[i].begin == out[i].end) continue;
            if (!(i == j && out[i].same(in[i])) && !apart(out[i], in[j])) return DEFT_EINVAL;
            if (j < i && !apart(out[i], out[j])) return DEFT_EINVAL;
        }
    for (int i = 0; i < kParts; ++i) {  // nor a weight or position
        auto meets = [&](const void *p, int64_t bytes) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(p);
            return p && at < out[i].end && out[i].begin < at + (uint64_t)bytes;
        };
        if (out[i].begin == out[i].end) continue;
        if (rope && meets(positions, 4 * n)) return DEFT_EINVAL;
        for (int j = 0; j < kParts; ++j)
            if (parts[j] && meets(parts[j]->weight, ((parts[j]->heads - 1) * parts[j]->weight_stride + d) * (wide ? 4 : 2))) return DEFT_EINVAL;
    }
    if (n == 0 || heads == 0) return DEFT_OK;
    const uint32_t at_once = 64 / ((uint32_t)d / 16);  // heads of a wave
    for (Part &p : a.part) {
        p.chunk = a.chunks;
        a.chunks += (p.heads + at_once - 1) / at_once;
    }
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
