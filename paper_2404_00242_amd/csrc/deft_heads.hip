// What happens to the heads of a projection's output before attention reads them: RMS norms of queries and keys, rotation by their
// positions, keys and values into the rows of a cache.  One pass: every head is read once and written once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "deft_device.h"
#include "deft_lists.h"
#include "deft_q8_device.h"

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;

enum { kQ, kK, kV, kParts };
enum Turn { kNoTurn, kHalf, kInterleaved, kAny };  // kAny: as the arguments say

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
    uint32_t rot, wide, turn;            // wide: weights are float; turn: a Turn
    float eps, offset, factor;
    uint64_t turns[64];  // of a turn a position, in 2^-64
};

// The upper half of position x turns modulo 2^64.
__device__ __forceinline__ uint32_t phase_of(int32_t position, uint64_t turns) {
    const uint32_t low = (uint32_t)turns, high = (uint32_t)(turns >> 32);
    const uint32_t phase = __umulhi((uint32_t)position, low) + (uint32_t)position * high;
    return position < 0 ? phase - low : phase;
}

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

// A head whose elements D / 16 neighbouring lanes have, sixteen each.
template <int D>
__device__ __forceinline__ void normalise(float *y0, float *y1, const float *w0, const float *w1, float eps) {
    auto mean = [&](float eps) {
        float sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(y0[i], y0[i], fmaf(y1[i], y1[i], sum));
#pragma unroll
        for (uint32_t o = 1; o < D / 16; o <<= 1) sum += __shfl_xor(sum, o);
        return fmaf(sum, 1.f / D, eps);
    };
    float m = mean(eps);
    if (m > 0x1p100f || m < 0x1p-80f) {  // squares near the ends of fp32: the head is taken by a power of two of itself
        const float by = m > 1.f ? 0x1p-70f : 0x1p90f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y0[i] *= by;
            y1[i] *= by;
        }
        m = mean(eps * by * by);
    }
    const float r = __builtin_amdgcn_rsqf(m);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y0[i] *= r * w0[i];
        y1[i] *= r * w1[i];
    }
}
// (which of the products is rounded by itself is said here, so that every kernel gives the same bits)
__device__ __forceinline__ void turn(float &u, float &v, float c, float s) {
    const float t = fmaf(u, c, -(v * s));
    v = fmaf(v, c, u * s);
    u = t;
}

// A lane's two groups of eight elements: interleaved anywhere in the head, in the half layout partners, and of the elements that do not
// turn the same.
struct Groups {
    uint32_t first, second;
    bool turned0, turned1;
};
template <int D>
__device__ __forceinline__ Groups groups_of(uint32_t j, int turn, uint32_t rot) {
    const bool turned = turn == kHalf && 16 * j < rot;
    const uint32_t begin = turned || turn != kHalf ? 0 : rot, width = turned ? rot : D - begin;
    Groups g;
    g.first = begin + 8 * (j - begin / 16);
    g.second = g.first + width / 2;
    g.turned0 = turn == kInterleaved ? g.first < rot : turned;
    g.turned1 = turn == kInterleaved ? g.second < rot : turned;
    return g;
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
// batches of heads to a wave, 8192 x 32 turned: 21.0 -> 21.8.  Stores that stay in the caches: 8192 x 32 (67 MB) 20.7 -> 25.1; of a few
// tokens, whose heads the attention reads next, the two are not compared.
template <int D, int TURN, bool NORM>
__device__ __forceinline__ void heads_of_wave(const HeadsArgs &a, uint32_t unit, float (*cs)[64]) {
    constexpr uint32_t kLanes = D / 16, kHeads = 64 / kLanes;
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t entry = divide(unit, a.chunks, a.inv_chunks), chunk = unit - entry * a.chunks;
    const int kind = chunk >= a.part[kV].chunk ? kV : chunk >= a.part[kK].chunk ? kK : kQ;
    const Part &p = a.part[kind];
    uint32_t token = entry, row = entry;
    if (a.entries) {
        const u32x2 e = uniform(a.entries, entry);
        row = kind == kQ ? e[1] : e[0];
        token = e[1];
    }
    const int how = TURN == kAny ? (int)a.turn : TURN;
    const uint32_t j = lane % kLanes, rot = how == kNoTurn || kind == kV ? 0 : a.rot;
    const Groups g = groups_of<D>(j, how, rot);
    const uint32_t first = g.first, second = g.second;
    const uint32_t head = (chunk - p.chunk) * kHeads + lane / kLanes, at = min(head, p.heads - 1);  // (heads behind the last are that one)
    const uint16_t *x = p.x + ((int64_t)token * p.token + (int64_t)at * p.head);
    // What the angles and the norm wait for is asked for in front of the heads, by vector loads: those come back in order, and a scalar
    // load of the position would hold up everything behind the next wait for any scalar load.
    int32_t position = 0;
    uint64_t turns = 0;
    if (2 * lane < rot) {
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
    if (2 * lane < rot) {
        float c, s;
        cos_sin(phase_of(position, turns), c, s);
        cs[0][lane] = c * a.factor;
        cs[1][lane] = s * a.factor;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // other lanes' angles are read from here on (a wave's LDS operations stay in
    __builtin_amdgcn_wave_barrier();                        // order: neither costs an instruction)
    float y0[8], y1[8];
    unpack8(x0, y0);
    unpack8(x1, y1);
    if (normed) {
        float w0[8], w1[8];
        unpack_weights(v0, a.wide, a.offset, w0);
        unpack_weights(v1, a.wide, a.offset, w1);
        normalise<D>(y0, y1, w0, w1, a.eps);
    }
    auto cosines = [&](uint32_t i) { return *reinterpret_cast<const f32x4 *>(&cs[0][i]); };
    auto sines = [&](uint32_t i) { return *reinterpret_cast<const f32x4 *>(&cs[1][i]); };
    if (how == kHalf && g.turned0) {
        const f32x4 c0 = cosines(first), c1 = cosines(first + 4), s0 = sines(first), s1 = sines(first + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            turn(y0[i], y1[i], c0[i], s0[i]);
            turn(y0[4 + i], y1[4 + i], c1[i], s1[i]);
        }
    }
    if (how == kInterleaved && g.turned0) {
        const f32x4 c = cosines(first / 2), s = sines(first / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) turn(y0[2 * i], y0[2 * i + 1], c[i], s[i]);
    }
    if (how == kInterleaved && g.turned1) {
        const f32x4 c = cosines(second / 2), s = sines(second / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) turn(y1[2 * i], y1[2 * i + 1], c[i], s[i]);
    }
    if (head >= p.heads) return;
    uint16_t *out = p.out + ((int64_t)row * p.out_token + (int64_t)head * p.out_head);
    // bits as they are where nothing is done to them; none of it is read again here
    __builtin_nontemporal_store(g.turned0 || normed ? pack8(y0) : x0, reinterpret_cast<u32x4 *>(out + first));
    __builtin_nontemporal_store(g.turned1 || normed ? pack8(y1) : x1, reinterpret_cast<u32x4 *>(out + second));
}

template <int D, int TURN, bool NORM>
__global__ __launch_bounds__(256) void deft_heads(HeadsArgs a) {
    __shared__ float table[4][2][64];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), unit = blockIdx.x * 4 + wave;
    if (unit < a.waves) heads_of_wave<D, TURN, NORM>(a, unit, table[wave]);
}

// ---- into an 8-bit cache ----

struct StoreArgs {
    HeadsArgs h;            // its entries are null; k's and v's parts have no out
    const u32x4 *groups;    // {block, first, count, low}, see deft::RowGroup
    const u32x2 *entries;   // {row, token}
    CacheArgs c;
    uint32_t units, parts, inv_parts, workgroups;  // the queries' workgroups come behind the others
};

// How a launch is cut: a row takes D / 16 lanes, so that a lane has a key's partners, and a unit, the new rows of a block and head, as many
// waves as that makes or a part of one.  Eight waves to a workgroup everywhere, us (32 + 8 heads of 128): a token in each of 20 blocks
// of 32 rows 4.6 -> 5.1, 1024 tokens in blocks of 16 6.4 -> 6.9, 8192 in blocks of 32 33.1 -> 32.9.
template <int D, int BLOCK>
struct Cut {
    static constexpr int kRowLanes = D / 16, kWaveRows = 64 / kRowLanes;
    static constexpr bool kWhole = BLOCK >= kWaveRows;  // whole waves: a workgroup has heads of one block; otherwise units in order
    static constexpr int kUnitLanes = kWhole ? 64 : kRowLanes * BLOCK;  // of a wave
    static constexpr int kUnitWaves = kWhole ? BLOCK / kWaveRows : 1;
    static constexpr int kWaves = kUnitWaves > 4 ? kUnitWaves : 4, kThreads = 64 * kWaves;  // of a workgroup
    static constexpr int kHeads = kWhole ? kWaves / kUnitWaves : 0;  // of a workgroup
    static constexpr int kPitch = 68;                                // floats of a row of angles, so that rows begin in different banks
    static constexpr int kTable = kWhole && 2 * BLOCK * kPitch > kWaves * 128 ? 2 * BLOCK * kPitch : kWaves * 128;
};

// Keys normalised and turned as by deft_heads and then, with the values, stored as by deft_store_q8, byte for byte what the two do one after
// the other; the queries in the same launch.  Each lane has one row's sixteen elements of K and of V: a wave that has all rows of a block
// of 32 one step after the other, as that kernel's have, takes three times the registers here and its steps wait for one another
// (32 + 8 heads of 128, 300 tokens 9.7 -> 5.9 us, 8192 37.3 -> 33.1).  So the waves of a unit tell each other their scales, and those of
// a workgroup make the angles of a block's rows together (8192 tokens, 32 heads: 5 % of the time is theirs).
// Bound by HBM where calls are large and most heads are queries: 8192 tokens, 32 + 8 heads of 128, 184 MB: 33.1 us, 5.6 TB/s, where
// deft_heads and deft_store_q8 need 38.5.  Where most are stored, by what stands between a row's loads and its stores: 32 KV heads of 128
// alone, 201 MB, in blocks of 32 rows 45.5 us, 4.4 TB/s (a workgroup has one head, so that the angles and both barriers are each head's
// own, and no loads follow a lane's first four), in blocks of 8 40.6; 32 + 8 heads of 64, 92 MB, 19.7 us, 4.7 TB/s.  By the launch and
// dependent loads where calls are an iteration's: 20 tokens 4.6 us, 6.5 by the two.  Queries by a launch of their own in front, 8192
// tokens: 36.6 -> 39.5 (2048: 13.1 -> 17.6).
template <int D, int BLOCK>
__global__ __launch_bounds__((Cut<D, BLOCK>::kThreads)) void deft_store_heads_q8(StoreArgs a) {
    using C = Cut<D, BLOCK>;
    constexpr int kRowLanes = C::kRowLanes, kPitch = C::kPitch;
    __shared__ __attribute__((aligned(16))) float table[C::kTable];
    __shared__ uint32_t scales[C::kWaves];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (blockIdx.x >= a.workgroups) {
        const uint32_t unit = (blockIdx.x - a.workgroups) * C::kWaves + wave;
        if (unit < a.h.waves) heads_of_wave<D, kAny, true>(a.h, unit, reinterpret_cast<float (*)[64]>(table + wave * 128));
        return;
    }
    uint32_t group, h, sub = lane % C::kUnitLanes / kRowLanes;  // sub: which of the unit's rows
    if (C::kWhole) {
        group = divide(blockIdx.x, a.parts, a.inv_parts);
        h = (blockIdx.x - group * a.parts) * C::kHeads + wave / C::kUnitWaves;
        sub += wave % C::kUnitWaves * C::kWaveRows;
    } else {
        const uint32_t unit = (blockIdx.x * C::kThreads + threadIdx.x) / C::kUnitLanes;
        if (unit >= a.units) return;  // (whole units, and all lanes that exchange values below belong to one)
        group = divide(unit, a.c.Hkv, a.c.inv_Hkv);
        h = unit - group * a.c.Hkv;
    }
    const uint32_t j = lane % kRowLanes;
    const int how = (int)a.h.turn;
    const uint32_t rot = how == kNoTurn ? 0 : a.h.rot;
    const Groups g = groups_of<D>(j, how, rot);
    const uint32_t v_first = 8 * j, v_second = D / 2 + 8 * j;
    const Part &kp = a.h.part[kK], &vp = a.h.part[kV];
    const bool normed = kp.weight;
    const u32x4 head = a.groups[group];
    const uint32_t block = head[0], first = head[1], count = head[2], low = head[3];
    // Waves behind the last head or the last row make angles all the same, and wait with the others.
    const bool ours = !C::kWhole || h < a.c.Hkv, live = !C::kWhole || (ours && wave % C::kUnitWaves * C::kWaveRows < __builtin_amdgcn_readfirstlane(count));
    const size_t scale_at = (size_t)block * a.c.Hkv + h;
    int ek = kScaleMin, ev = kScaleMin;
    const bool kept = low > 0 && ours;
    if (kept) {
        ek = a.c.k_scale[scale_at];
        ev = a.c.v_scale[scale_at];
    }
    // A lane's pairs: those of its first group, or of its first four and its second group's.
    const uint32_t pair0 = how == kHalf ? g.first : g.first / 2, pair1 = how == kHalf ? g.first + 4 : g.second / 2;
    uint64_t turns[8] = {};
    int32_t position = 0;
    Weights w0, w1;
    uint32_t row = 0;
    u32x4 k0, k1, v0, v1;
    if (C::kWhole && rot) {
        if (2 * lane < rot) turns[0] = a.h.turns[lane];
        position = a.h.positions[a.entries[first + min(lane, count - 1)][1]];  // of row `lane`
    }
    if (live) {
        const u32x2 e = a.entries[first + min(sub, count - 1)];  // rows past the last repeat it
        row = e[0];
        if (normed) {
            const uint32_t w = h * (uint32_t)kp.weight_head;
            w0 = weights_at(kp.weight, w + g.first, a.h.wide);
            w1 = weights_at(kp.weight, w + g.second, a.h.wide);
        }
        if (!C::kWhole && rot) {
            position = a.h.positions[e[1]];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (g.turned0) turns[i] = a.h.turns[pair0 + i];
                if (g.turned1) turns[4 + i] = a.h.turns[pair1 + i];
            }
        }
        const uint16_t *k = kp.x + ((int64_t)e[1] * kp.token + (int64_t)h * kp.head), *v = vp.x + ((int64_t)e[1] * vp.token + (int64_t)h * vp.head);
        k0 = load_once(reinterpret_cast<const u32x4 *>(k + g.first));
        k1 = load_once(reinterpret_cast<const u32x4 *>(k + g.second));
        v0 = load_once(reinterpret_cast<const u32x4 *>(v + v_first));
        v1 = load_once(reinterpret_cast<const u32x4 *>(v + v_second));
    }
    if (C::kWhole && rot) {  // the angles of the block's rows, once for all its heads here: a wave makes a row's, a lane one pair's
        const uint32_t rows = __builtin_amdgcn_readfirstlane(count);
        for (uint32_t r = wave; r < rows; r += C::kWaves) {
            float c, s;
            cos_sin(phase_of(__builtin_amdgcn_readlane(position, r), turns[0]), c, s);
            table[2 * r * kPitch + lane] = c * a.h.factor;
            table[(2 * r + 1) * kPitch + lane] = s * a.h.factor;
        }
        __syncthreads();
    }
    const int old_k = ek, old_v = ev;
    bool spoiled = false;  // an infinity or a NaN in the row
    if (live) {
        if (normed || rot) {
            float y0[8], y1[8];
            unpack8(k0, y0);
            unpack8(k1, y1);
            if (normed) {
                float f0[8], f1[8];
                unpack_weights(w0, a.h.wide, a.h.offset, f0);
                unpack_weights(w1, a.h.wide, a.h.offset, f1);
                normalise<D>(y0, y1, f0, f1, a.h.eps);
            }
            f32x4 c[2], s[2];
            if (C::kWhole) {
                const float *of = table + 2 * min(sub, count - 1) * kPitch;
                if (g.turned0) {
                    c[0] = *reinterpret_cast<const f32x4 *>(of + pair0);
                    s[0] = *reinterpret_cast<const f32x4 *>(of + kPitch + pair0);
                }
                if (g.turned1) {
                    c[1] = *reinterpret_cast<const f32x4 *>(of + pair1);
                    s[1] = *reinterpret_cast<const f32x4 *>(of + kPitch + pair1);
                }
            } else if (g.turned0 || g.turned1) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float cs, sn;
                    cos_sin(phase_of(position, turns[i]), cs, sn);
                    c[i / 4][i % 4] = cs * a.h.factor;
                    s[i / 4][i % 4] = sn * a.h.factor;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (how == kHalf && g.turned0) {
                    turn(y0[i], y1[i], c[0][i], s[0][i]);
                    turn(y0[4 + i], y1[4 + i], c[1][i], s[1][i]);
                }
                if (how == kInterleaved && g.turned0) turn(y0[2 * i], y0[2 * i + 1], c[0][i], s[0][i]);
                if (how == kInterleaved && g.turned1) turn(y1[2 * i], y1[2 * i + 1], c[1][i], s[1][i]);
            }
            if (g.turned0 || normed) k0 = pack8(y0);
            if (g.turned1 || normed) k1 = pack8(y1);
        }
        uint32_t mk = 0, mv = 0;  // magnitudes as pairs of bf16 bits
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            mk = pk_max(pk_max(mk, k0[i] & 0x7fff7fffu), k1[i] & 0x7fff7fffu);
            mv = pk_max(pk_max(mv, v0[i] & 0x7fff7fffu), v1[i] & 0x7fff7fffu);
        }
        const uint32_t both = pk_max(mk, mv);
        const uint64_t bad = __ballot(max(both & 0xffffu, both >> 16) >= 0x7f80u);
        spoiled = ((bad >> (lane / kRowLanes * kRowLanes)) & ((uint64_t(1) << kRowLanes) - 1)) != 0;
        uint32_t top = spoiled ? 0u : max(mk & 0xffffu, mk >> 16) | max(mv & 0xffffu, mv >> 16) << 16;
#pragma unroll
        for (int o = C::kUnitLanes / 2; o > 0; o >>= 1) top = pk_max(top, (uint32_t)__shfl_xor((int)top, o));
        ek = max(ek, scale_byte(top & 0xffffu));
        ev = max(ev, scale_byte(top >> 16));
    }
    if (C::kUnitWaves > 1) {
        if (lane == 0) scales[wave] = (uint32_t)ek | (uint32_t)ev << 16;
        __syncthreads();
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < C::kUnitWaves; ++i) most = pk_max(most, scales[wave / C::kUnitWaves * C::kUnitWaves + i]);
        ek = (int)(most & 0xffffu);
        ev = (int)(most >> 16);
    }
    const size_t pitch = (size_t)a.c.Hkv * D;
    if (kept) {
        const size_t begin = (size_t)block * BLOCK * pitch + h * D;
        constexpr uint32_t step = C::kWhole ? BLOCK : C::kUnitLanes / kRowLanes;  // (of the unit's rows a lane has one)
        for (const uint32_t col : {v_first, v_second}) {
            if (ek > old_k) rescale_kept(a.c.k + begin + col, sub, step, low, pitch, power(max(127 + old_k - ek, 0)));
            if (ev > old_v) rescale_kept(a.c.v + begin + col, sub, step, low, pitch, power(max(127 + old_v - ev, 0)));
        }
    }
    if (!ours) return;
    if (sub < count) {
        const float inv_k = power(254 - ek), inv_v = power(254 - ev);
        const u32x2 nan = {0x7f7f7f7fu, 0x7f7f7f7fu}, zero = {0u, 0u};
        const size_t at = row * pitch + h * D;
        *reinterpret_cast<u32x2 *>(a.c.k + at + g.first) = spoiled ? nan : round8(k0, inv_k);
        *reinterpret_cast<u32x2 *>(a.c.k + at + g.second) = spoiled ? nan : round8(k1, inv_k);
        *reinterpret_cast<u32x2 *>(a.c.v + at + v_first) = spoiled ? zero : round8(v0, inv_v);
        *reinterpret_cast<u32x2 *>(a.c.v + at + v_second) = spoiled ? zero : round8(v1, inv_v);
    }
    if (sub == 0 && j == 0) {
        a.c.k_scale[scale_at] = (uint8_t)ek;
        a.c.v_scale[scale_at] = (uint8_t)ev;
    }
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

// A call as it was checked.
struct Call {
    HeadsArgs a{};
    uint32_t heads = 0;
    bool norm = false;
    Area in[kParts]{}, out[kParts]{};
};
enum Where { kOwnOut, kPool, kCache };  // where keys and values go: as queries do, into rows of a bf16 cache, or elsewhere

// parts: q, k, v, each may be null; pool: rows of k's and v's out where they are a bf16 cache's.
int check(const deft_heads_t *const (&parts)[kParts], int64_t n, int32_t d, float eps, float offset, const int32_t *positions,
          const deft_rope_t *rope, Where where, int64_t pool, Call &call) {
    if (n < 0 || (d != 64 && d != 128)) return DEFT_EINVAL;
    if (rope && (rope->rot < 16 || rope->rot > d || rope->rot % 16 || (rope->layout != DEFT_ROPE_HALF && rope->layout != DEFT_ROPE_INTERLEAVED)))
        return DEFT_EINVAL;
    if (rope && ((!positions && n > 0) || (reinterpret_cast<uintptr_t>(positions) & 3))) return DEFT_EINVAL;
    HeadsArgs &a = call.a;
    auto &in = call.in;
    auto &out = call.out;
    bool wide = false;
    for (int i = 0; i < kParts; ++i) {
        const deft_heads_t *p = parts[i];
        const bool stored = where != kOwnOut && i != kQ, writes = where != kCache || i == kQ;
        if (!p || p->heads == 0) continue;
        if (p->heads < 0 || p->heads > DEFT_MAX_Q8_HEADS) return DEFT_EINVAL;
        if (p->weight) {
            if (i == kV || !(eps >= 0) || !std::isfinite(eps) || !std::isfinite(offset)) return DEFT_EINVAL;
            if (!deft::aligned16(p->weight) || p->weight_stride < 0 || p->weight_stride % 8 || p->weight_stride > 4096) return DEFT_EINVAL;
            if (call.norm && wide != (p->weight_f32 != 0)) return DEFT_EINVAL;
            call.norm = true;
            wide = p->weight_f32 != 0;
        }
        if (n == 0) continue;
        if (!p->x || !deft::aligned16(p->x) || (writes && (!p->out || !deft::aligned16(p->out)))) return DEFT_EINVAL;
        if ((p->token_stride | p->head_stride) & 7) return DEFT_EINVAL;
        if (p->token_stride < 0 || p->head_stride < 0 || p->token_stride > kMaxStride || p->head_stride > kMaxStride) return DEFT_EINVAL;
        if ((double)n * (double)p->token_stride + (double)p->heads * (double)p->head_stride > 0x1p60) return DEFT_EINVAL;
        const bool in_place = !stored && p->out == p->x;
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
        if (writes) out[i] = area(p->out, stored ? pool : n, p->heads, d, t.out_token, t.out_head);
        t.heads = (uint32_t)p->heads;
        call.heads += t.heads;
    }
    for (int i = 0; i < kParts; ++i)  // what is written is nobody else's, and nobody's input but the part's own, in place (not in a pool,
        for (int j = 0; j < kParts; ++j) {  // whose rows are others than the tokens')
            if (out[i].begin == out[i].end) continue;
            const bool own = i == j && (where == kOwnOut || i == kQ) && out[i].same(in[i]);
            if (!own && !apart(out[i], in[j])) return DEFT_EINVAL;
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
    const uint32_t at_once = 64 / ((uint32_t)d / 16);  // heads of a wave
    for (int i = 0; i < kParts; ++i) {
        a.part[i].chunk = a.chunks;
        if (where != kCache || i == kQ) a.chunks += (a.part[i].heads + at_once - 1) / at_once;
    }
    if (a.chunks) a.inv_chunks = inverse(a.chunks);
    a.positions = positions;
    a.eps = eps;
    a.offset = offset;
    a.wide = wide;
    a.turn = !rope ? kNoTurn : rope->layout == DEFT_ROPE_HALF ? kHalf : kInterleaved;
    if (rope) {
        a.rot = (uint32_t)rope->rot;
        a.factor = rope->factor;
        std::copy(rope->turns, rope->turns + rope->rot / 2, a.turns);
    }
    return DEFT_OK;
}

// The waves of a call, in launches.
int launch_waves(HeadsArgs a, bool norm, int64_t n, int32_t d, hipStream_t st) {
    if (n == 0 || a.chunks == 0) return DEFT_OK;
    const int turn = (int)a.turn;
    const int64_t most = (int64_t)(kMaxWaves / a.chunks);
    for (int64_t left = n, now; left > 0; left -= now) {
        now = std::min(left, most);
        a.waves = (uint32_t)now * a.chunks;
        d == 128 ? launch<128>(a, turn, norm, st) : launch<64>(a, turn, norm, st);
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

int run(const deft_heads_t *const (&parts)[kParts], int64_t n, int32_t d, float eps, float offset, const int32_t *positions,
        const deft_rope_t *rope, const u32x2 *entries, int64_t pool, void *stream) {
    Call call;
    const int rc = check(parts, n, d, eps, offset, positions, rope, entries ? kPool : kOwnOut, pool, call);
    if (rc != DEFT_OK || call.heads == 0) return rc;
    call.a.entries = entries;
    return launch_waves(call.a, call.norm, n, d, static_cast<hipStream_t>(stream));
}

// Threads of a launch of stores at most (they are counted in 32 bits); longer lists take several launches.
constexpr uint64_t kMaxThreads = 1u << 28;

template <int D, int BLOCK>
bool launch_store(StoreArgs a, uint32_t groups, hipStream_t st) {
    using C = Cut<D, BLOCK>;
    constexpr uint32_t units = C::kThreads / C::kUnitLanes;
    a.parts = C::kWhole ? (a.c.Hkv + C::kHeads - 1) / std::max(C::kHeads, 1) : 0;
    if (C::kWhole) a.inv_parts = inverse(a.parts);
    const uint32_t most = (uint32_t)(C::kWhole ? kMaxThreads / C::kThreads / a.parts : kMaxThreads / C::kUnitLanes / a.c.Hkv);
    for (uint32_t n; groups > 0; groups -= n, a.groups += n) {
        n = std::min(groups, most);
        a.units = n * a.c.Hkv;
        a.workgroups = C::kWhole ? n * a.parts : (a.units + units - 1) / units;
        const uint32_t queries = (a.h.waves + C::kWaves - 1) / C::kWaves;
        hipLaunchKernelGGL((deft_store_heads_q8<D, BLOCK>), dim3(a.workgroups + queries), dim3(C::kThreads), 0, st, a);
        if (!deft::hip_ok(hipGetLastError(), "deft_store_heads_q8 launch")) return false;
        a.h.waves = 0;
    }
    return true;
}
template <int D>
bool launch_store(const StoreArgs &a, uint32_t groups, int block_rows, hipStream_t st) {
    switch (block_rows) {
        case 1: return launch_store<D, 1>(a, groups, st);
        case 2: return launch_store<D, 2>(a, groups, st);
        case 4: return launch_store<D, 4>(a, groups, st);
        case 8: return launch_store<D, 8>(a, groups, st);
        case 16: return launch_store<D, 16>(a, groups, st);
        case 32: return launch_store<D, 32>(a, groups, st);
        default: return launch_store<D, 64>(a, groups, st);
    }
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

extern "C" int deft_qkv_store_q8(const deft_kv_list_t *list, const void *dev_image, const deft_heads_t *q, const deft_heads_t *k, const deft_heads_t *v,
                                 const deft_cache_q8_t *cache, float eps, float weight_offset, const int32_t *positions, const deft_rope_t *rope,
                                 void *stream) {
    if (!rows_fit(list, dev_image, cache) || !k || !v || k->heads != cache->Hkv || v->heads != cache->Hkv) return DEFT_EINVAL;
    if (cache->n_rows > 0 && (cache->k == cache->v || cache->k_scale == cache->v_scale)) return DEFT_EINVAL;
    const int64_t n = list->entries, d = cache->d;
    Call call;
    const int rc = check({q, k, v}, n, (int32_t)d, eps, weight_offset, positions, rope, kCache, 0, call);
    if (rc != DEFT_OK || n == 0) return rc;
    // what the cache is made of is nobody's input, nor the queries' output
    const int64_t bytes = (int64_t)cache->n_rows * cache->Hkv * d, scales = ((int64_t)cache->n_rows + cache->block_rows - 1) / cache->block_rows * cache->Hkv;
    const struct { const void *p; int64_t bytes; } own[] = {{cache->k, bytes}, {cache->v, bytes}, {cache->k_scale, scales}, {cache->v_scale, scales}};
    auto meets = [&](uintptr_t begin, uintptr_t end) {
        for (const auto &o : own) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(o.p);
            if (begin < at + (uint64_t)o.bytes && at < end) return true;
        }
        return false;
    };
    for (int i = 0; i < kParts; ++i) {
        if (meets(call.in[i].begin, call.in[i].end) || meets(call.out[i].begin, call.out[i].end)) return DEFT_EINVAL;
        const Part &p = call.a.part[i];
        const uintptr_t w = reinterpret_cast<uintptr_t>(p.weight);
        if (w && meets(w, w + (uint64_t)((p.heads - 1) * p.weight_head + d) * (call.a.wide ? 4 : 2))) return DEFT_EINVAL;
    }
    const uintptr_t at = reinterpret_cast<uintptr_t>(positions);
    if (rope && meets(at, at + 4 * (uint64_t)n)) return DEFT_EINVAL;
    StoreArgs a{};
    a.h = call.a;
    a.groups = static_cast<const u32x4 *>(dev_image);
    a.entries = reinterpret_cast<const u32x2 *>(static_cast<const uint8_t *>(dev_image) + list->off_entries);
    a.c = cache_args(cache);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint64_t waves = (uint64_t)n * call.a.chunks;
    if (waves > kMaxWaves) {
        const int done = launch_waves(call.a, call.norm, n, (int32_t)d, st);
        if (done != DEFT_OK) return done;
    } else {
        a.h.waves = (uint32_t)waves;
    }
    const bool ok = d == 128 ? launch_store<128>(a, (uint32_t)list->heads, cache->block_rows, st) : launch_store<64>(a, (uint32_t)list->heads, cache->block_rows, st);
    return ok ? DEFT_OK : DEFT_EHIP;
}
