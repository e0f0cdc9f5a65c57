// The calls that fill, read back and rearrange a KV cache: rows into and out of an 8-bit cache, copies of pages inside pools of
// any kind.  All of them are bound by HBM where they are large and by a few dependent round trips where they are not.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <vector>

#include "deft_device.h"
#include "deft_lists.h"
#include "deft_q8_device.h"

namespace {

// ---- rows into an 8-bit cache ----
// One unit = (block, KV head), K and V: a block's scale is that of all its rows, so one wave (or a part of one, where a block has
// few rows) holds the new rows of a block in registers, finds their largest magnitudes, and rounds.  A row takes D/8 lanes, eight
// values (128 bits of bf16, 64 of e4m3) to a lane.
// The scale is a power of two 2^(e - 127) because nothing is then rounded twice: x / scale is exact, and when a scale grows the
// kept rows are moved by whole binary places, so that a value loses bits only where it becomes subnormal.  It costs no accuracy: the
// error of rounding to four significant bits does not depend on the scale as long as nothing over- or underflows.
struct StoreArgs {
    const u32x4 *groups;    // {block, first, count, low}, see deft::RowGroup
    const u32x2 *entries;   // {row, token}
    const uint16_t *k, *v;
    int64_t k_stride, v_stride;
    CacheArgs c;
    uint32_t units;
};

// BLOCK: rows of a block.  A prompt of 8192 tokens x 32 heads, us: 1 row 37.9, 16 36.3, 32 36.8; with 64 rows a wave has them in 237
// registers at D = 128, two waves to a SIMD, and takes 40.4.
template <int D, int BLOCK>
__global__ __launch_bounds__(256) void deft_store_q8(StoreArgs a) {
    constexpr int kRowLanes = D / 8;
    constexpr int kUnitLanes = kRowLanes * BLOCK < 64 ? kRowLanes * BLOCK : 64;
    constexpr int kUnitRows = kUnitLanes / kRowLanes;  // rows of a unit at a time
    constexpr int kSteps = BLOCK / kUnitRows;
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t unit = (blockIdx.x * 256 + threadIdx.x) / kUnitLanes;
    if (unit >= a.units) return;  // (whole units, and all lanes that exchange values below belong to one)
    const uint32_t group = divide(unit, a.c.Hkv, a.c.inv_Hkv), h = unit - group * a.c.Hkv;
    const uint32_t in_unit = lane % kUnitLanes, sub = in_unit / kRowLanes, col = 8 * (in_unit % kRowLanes);
    const u32x4 head = a.groups[group];
    const uint32_t block = head[0], first = head[1], count = head[2], low = head[3];
    const size_t scale_at = (size_t)block * a.c.Hkv + h;
    int ek = kScaleMin, ev = kScaleMin;
    const bool kept = low > 0;
    if (kept) {
        ek = a.c.k_scale[scale_at];
        ev = a.c.v_scale[scale_at];
    }
    uint32_t row[kSteps];
    u32x4 k[kSteps], v[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        const u32x2 e = a.entries[first + min((uint32_t)(u * kUnitRows) + sub, count - 1)];  // rows past the last repeat it
        row[u] = e[0];
        k[u] = load_once(reinterpret_cast<const u32x4 *>(a.k + (int64_t)e[1] * a.k_stride + (h * D + col)));
        v[u] = load_once(reinterpret_cast<const u32x4 *>(a.v + (int64_t)e[1] * a.v_stride + (h * D + col)));
    }
    uint32_t top_k = 0, top_v = 0, spoiled = 0;  // magnitudes as pairs of bf16 bits; rows with an infinity or a NaN
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        uint32_t mk = 0, mv = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            mk = pk_max(mk, k[u][i] & 0x7fff7fffu);
            mv = pk_max(mv, v[u][i] & 0x7fff7fffu);
        }
        const uint32_t both = pk_max(mk, mv);
        const uint64_t bad = __ballot(max(both & 0xffffu, both >> 16) >= 0x7f80u);
        const bool mine = ((bad >> (lane / kRowLanes * kRowLanes)) & ((uint64_t(1) << kRowLanes) - 1)) != 0;
        spoiled |= (uint32_t)mine << u;
        top_k = pk_max(top_k, mine ? 0u : mk);
        top_v = pk_max(top_v, mine ? 0u : mv);
    }
    uint32_t top = max(top_k & 0xffffu, top_k >> 16) | max(top_v & 0xffffu, top_v >> 16) << 16;
#pragma unroll
    for (int o = kUnitLanes / 2; o > 0; o >>= 1) top = pk_max(top, (uint32_t)__shfl_xor((int)top, o));
    const int old_k = ek, old_v = ev;
    ek = max(ek, scale_byte(top & 0xffffu));
    ev = max(ev, scale_byte(top >> 16));
    const size_t pitch = (size_t)a.c.Hkv * D;
    if (kept) {
        const size_t begin = (size_t)block * BLOCK * pitch + h * D + col;
        if (ek > old_k) rescale_kept(a.c.k + begin, sub, kUnitRows, low, pitch, power(max(127 + old_k - ek, 0)));
        if (ev > old_v) rescale_kept(a.c.v + begin, sub, kUnitRows, low, pitch, power(max(127 + old_v - ev, 0)));
    }
    const float inv_k = power(254 - ek), inv_v = power(254 - ev);
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
        if ((uint32_t)(u * kUnitRows) + sub >= count) continue;
        const bool bad = (spoiled >> u) & 1;
        const u32x2 nan = {0x7f7f7f7fu, 0x7f7f7f7fu}, zero = {0u, 0u};
        const size_t at = row[u] * pitch + h * D + col;
        *reinterpret_cast<u32x2 *>(a.c.k + at) = bad ? nan : round8(k[u], inv_k);
        *reinterpret_cast<u32x2 *>(a.c.v + at) = bad ? zero : round8(v[u], inv_v);
    }
    if (in_unit == 0) {
        a.c.k_scale[scale_at] = (uint8_t)ek;
        a.c.v_scale[scale_at] = (uint8_t)ev;
    }
}

// ---- rows out of an 8-bit cache ----
// 16 values of one of K and V to a thread: one load, two stores.
struct LoadArgs {
    const u32x2 *entries;
    uint16_t *k, *v;  // v's threads come behind those of k; either may be null
    CacheArgs c;
    uint32_t per_row, inv_per_row;  // threads per row of all heads
    uint32_t threads, all;          // of one of the two, of those that are asked for
    uint32_t shift;                 // rows of a block, log2
};

template <int D>
__global__ __launch_bounds__(256) void deft_load_q8(LoadArgs a) {
    uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= a.all) return;
    const bool second = !a.k || i >= a.threads;
    if (i >= a.threads) i -= a.threads;
    const uint32_t entry = divide(i, a.per_row, a.inv_per_row), part = i - entry * a.per_row, h = part / (D / 16);
    const u32x2 e = a.entries[entry];
    const uint8_t *from = second ? a.c.v : a.c.k, *scales = second ? a.c.v_scale : a.c.k_scale;
    uint16_t *to = second ? a.v : a.k;
    const float scale = power(scales[(size_t)(e[0] >> a.shift) * a.c.Hkv + h]);
    const u32x4 x = *reinterpret_cast<const u32x4 *>(from + ((size_t)e[0] * a.per_row + part) * 16);
    u32x4 *out = reinterpret_cast<u32x4 *>(to + ((size_t)e[1] * a.per_row + part) * 16);
#pragma unroll
    for (int i2 = 0; i2 < 2; ++i2) {
        u32x4 y;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t w = x[2 * i2 + j];
            y[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
            y[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
        }
        out[i2] = y;
    }
}

// ---- copies of pages ----
// A thread owns the same few bytes of every page of one pool, and makes a chain's copies of them one after the other in the
// list's order: pages may be read and overwritten in one call without a second copy of anything, because no other thread ever
// touches those bytes.  That no page is overwritten before it was read makes it right to ask for later pages ahead of the stores.
// Most chains are one copy long (forks), so a thread takes four words where that leaves enough threads; all lanes of a wave have
// one chain where pages are that large.  The stores are not kept in the caches.  Bound by HBM: 40 pages of 16 rows in 64 bf16
// pools, 168 MB moved, a word to a thread 51 us, four 38, and with such stores 30.6 (5.5 TB/s; with
// pools that the memory-side cache does not hold 35.9, 4.7 TB/s, where a plain copy of 134 MB reaches 6.3).
constexpr int kMaxPools = 256;  // to a launch, 2 KB of its arguments
constexpr int kMaxClasses = 4;  // sizes of pages among them
constexpr uint32_t kMaxGroups = 1u << 16;  // workgroups to a pool; more work goes round
// Waves of four words to a thread from which on a thread takes four: a quarter of what the chip holds.  us, one word -> four: 1024
// waves 5.6 -> 6.1, 5.3 -> 6.1 and 5.2 -> 4.8; 2048 8.0 -> 7.6 and 7.6 -> 6.1; 4096 13.8 -> 10.4; 20480 51 -> 30; 65536 152 -> 87.
constexpr uint32_t kManyWaves = 2048;

struct PoolClass {
    uint32_t begin_group, begin_pool;  // first workgroup, first pool
    uint32_t groups, inv_groups;       // workgroups of a pool
    uint32_t width;                    // bytes that a thread moves at a time: 16, 8, 4, 2 or 1
    uint32_t per_thread;               // such words to a thread, of 64 * per_thread consecutive ones to a wave; 0: see below
    uint32_t words;                    // of a page
    uint32_t per_page, inv_per_page;   // waves to a page; with per_thread = 0 threads, of any number of pages to a wave
    uint32_t unused;
    uint64_t items;                    // waves or threads of a pool
    int64_t page_bytes;
};
struct CopyArgs {
    const u32x4 *chains;   // {first, count, held, -}, see deft::CopyChain
    const u32x2 *steps;    // {src, dst}
    uint32_t n_classes;
    PoolClass classes[kMaxClasses];
    uint8_t *pools[kMaxPools];
};
static_assert(sizeof(CopyArgs) <= 4096, "arguments of a kernel");

// The copies of one chain, W words to a thread: this lane's first is `word`, the others come 64 behind each other.  `kAhead` steps'
// words are in flight.  UNIFORM: the chain is all lanes'; they fetch 64 of its steps at a time, one each.  A cycle of 150 64-KB pages in 16 pools, 315 MB moved, 79 us; with a scalar load
// in front of every copy and a branch around each word 136.
template <typename T, int W, bool UNIFORM>
__device__ __forceinline__ void copy_chain(const CopyArgs &a, uint8_t *pool, int64_t page_bytes, uint32_t chain, uint32_t word, uint32_t words) {
    constexpr int kAhead = W == 1 ? 16 : 4;
    const u32x4 head = a.chains[chain];
    // Lanes past the page's end do what the one with its last word does, in the same instructions: the same bytes, and no branch.
    uint32_t at[W];
#pragma unroll
    for (int w = 0; w < W; ++w) at[w] = min(word + 64 * w, words - 1);
    const u32x2 *steps = a.steps + head[0];
    auto load = [&](T(&x)[W], uint32_t page) {
        const T *p = reinterpret_cast<const T *>(pool + (int64_t)page * page_bytes);
#pragma unroll
        for (int w = 0; w < W; ++w) x[w] = p[at[w]];
    };
    auto store = [&](const T(&x)[W], uint32_t page) {
        T *p = reinterpret_cast<T *>(pool + (int64_t)page * page_bytes);
#pragma unroll
        for (int w = 0; w < W; ++w) __builtin_nontemporal_store(x[w], p + at[w]);
    };
    T held[W];
    uint32_t n = head[1];
    if (head[2]) {  // the last step's page is overwritten before its turn: read now, and here before anything is stored
        load(held, steps[--n][0]);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    for (uint32_t first = 0; first < n; first += 64) {
        const uint32_t m = min(64u, n - first);
        u32x2 mine{};
        if (UNIFORM) mine = steps[first + min(threadIdx.x & 63, m - 1)];
        auto step = [&](uint32_t i) {
            if (UNIFORM) return u32x2{(uint32_t)__builtin_amdgcn_readlane((int)mine[0], (int)i), (uint32_t)__builtin_amdgcn_readlane((int)mine[1], (int)i)};
            return steps[first + i];
        };
        T x[kAhead][W];
        uint32_t i = 0;
        for (; i + kAhead <= m; i += kAhead) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) load(x[u], step(i + u)[0]);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) store(x[u], step(i + u)[1]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < m) load(x[u], step(i + u)[0]);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < m) store(x[u], step(i + u)[1]);
    }
    if (head[2]) store(held, steps[n][1]);
}

template <typename T>
__device__ __forceinline__ void copy_part(const CopyArgs &a, const PoolClass &c, uint8_t *pool, uint32_t group) {
    if (c.per_thread == 0) {  // pages of less than a wave
        for (uint64_t i = (uint64_t)group * 256 + threadIdx.x; i < c.items; i += (uint64_t)c.groups * 256) {
            const uint32_t chain = i >> 32 ? (uint32_t)(i / c.per_page) : divide((uint32_t)i, c.per_page, c.inv_per_page);
            copy_chain<T, 1, false>(a, pool, c.page_bytes, chain, (uint32_t)(i - (uint64_t)chain * c.per_page), c.words);
        }
        return;
    }
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (uint64_t i = (uint64_t)group * 4 + wave; i < c.items; i += (uint64_t)c.groups * 4) {
        const uint32_t chain = i >> 32 ? (uint32_t)(i / c.per_page) : divide((uint32_t)i, c.per_page, c.inv_per_page);
        const uint32_t first = (uint32_t)(i - (uint64_t)chain * c.per_page) * 64;
        if (c.per_thread == 4)
            copy_chain<T, 4, true>(a, pool, c.page_bytes, chain, 4 * first + lane, c.words);
        else
            copy_chain<T, 1, true>(a, pool, c.page_bytes, chain, first + lane, c.words);
    }
}

__global__ __launch_bounds__(256) void deft_copy_pages(CopyArgs a) {
    uint32_t k = 0;
    while (k + 1 < a.n_classes && blockIdx.x >= a.classes[k + 1].begin_group) ++k;
    const PoolClass &c = a.classes[k];
    const uint32_t group = blockIdx.x - c.begin_group, pool = divide(group, c.groups, c.inv_groups);
    uint8_t *base = a.pools[c.begin_pool + pool];
    const uint32_t part = group - pool * c.groups;
    switch (c.width) {
        case 16: copy_part<u32x4>(a, c, base, part); break;
        case 8: copy_part<u32x2>(a, c, base, part); break;
        case 4: copy_part<uint32_t>(a, c, base, part); break;
        case 2: copy_part<uint16_t>(a, c, base, part); break;
        default: copy_part<uint8_t>(a, c, base, part); break;
    }
}

// Threads of a launch of store and load at most (they are counted in 32 bits); longer lists take several launches.
constexpr uint64_t kMaxThreads = 1u << 28;
static_assert(kMaxThreads / 64 >= DEFT_MAX_Q8_HEADS, "a group's units go into one launch");

template <int D, int BLOCK>
bool launch_store(StoreArgs a, uint32_t groups, hipStream_t st) {
    constexpr uint32_t lanes = D / 8 * BLOCK < 64 ? D / 8 * BLOCK : 64, units = 256 / lanes;
    const uint32_t most = (uint32_t)(kMaxThreads / lanes / a.c.Hkv);
    for (uint32_t n; groups > 0; groups -= n, a.groups += n) {
        n = std::min(groups, most);
        a.units = n * a.c.Hkv;
        hipLaunchKernelGGL((deft_store_q8<D, BLOCK>), dim3((a.units + units - 1) / units), dim3(256), 0, st, a);
        if (!deft::hip_ok(hipGetLastError(), "deft_store_q8 launch")) return false;
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

extern "C" int deft_kv_list_upload(const deft_kv_list_t *list, void *dev_image, size_t bytes, void *stream) {
    if (!list || !dev_image || !deft::aligned16(dev_image)) return DEFT_EINVAL;
    if (bytes < list->image.size()) return DEFT_EWORKSPACE;
    return deft::upload_image(dev_image, list->image.data(), list->image.size(), static_cast<hipStream_t>(stream));
}

extern "C" int deft_kv_store_q8(const deft_kv_list_t *list, const void *dev_image, const void *k, const void *v, int64_t k_stride,
                                int64_t v_stride, const deft_cache_q8_t *cache, void *stream) {
    if (!rows_fit(list, dev_image, cache)) return DEFT_EINVAL;
    if (list->entries == 0) return DEFT_OK;
    if (cache->k == cache->v || cache->k_scale == cache->v_scale) return DEFT_EINVAL;
    const int64_t least = (int64_t)cache->Hkv * cache->d;
    if (!k || !v || !deft::aligned16(k) || !deft::aligned16(v)) return DEFT_EINVAL;
    if (k_stride < least || v_stride < least || (k_stride & 7) || (v_stride & 7)) return DEFT_EINVAL;
    const uint8_t *img = static_cast<const uint8_t *>(dev_image);
    StoreArgs a{};
    a.groups = reinterpret_cast<const u32x4 *>(img);
    a.entries = reinterpret_cast<const u32x2 *>(img + list->off_entries);
    a.k = static_cast<const uint16_t *>(k);
    a.v = static_cast<const uint16_t *>(v);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.c = cache_args(cache);
    const uint32_t groups = (uint32_t)list->heads;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool ok = cache->d == 128 ? launch_store<128>(a, groups, cache->block_rows, st) : launch_store<64>(a, groups, cache->block_rows, st);
    return ok ? DEFT_OK : DEFT_EHIP;
}

extern "C" int deft_kv_load_q8(const deft_kv_list_t *list, const void *dev_image, const deft_cache_q8_t *cache, void *k, void *v, void *stream) {
    if (!rows_fit(list, dev_image, cache)) return DEFT_EINVAL;
    if (list->entries == 0 || (!k && !v)) return DEFT_OK;
    if (!deft::aligned16(k) || !deft::aligned16(v) || k == v) return DEFT_EINVAL;
    const uint32_t per_row = (uint32_t)cache->Hkv * (uint32_t)cache->d / 16, both = k && v ? 2 : 1;
    const uint8_t *img = static_cast<const uint8_t *>(dev_image);
    LoadArgs a{};
    a.entries = reinterpret_cast<const u32x2 *>(img + list->off_entries);
    a.k = static_cast<uint16_t *>(k);
    a.v = static_cast<uint16_t *>(v);
    a.c = cache_args(cache);
    a.per_row = per_row;
    a.inv_per_row = inverse(per_row);
    a.shift = (uint32_t)__builtin_ctz((unsigned)cache->block_rows);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint32_t most = (uint32_t)(kMaxThreads / both / per_row);
    for (uint32_t left = (uint32_t)list->entries, n; left > 0; left -= n, a.entries += n) {
        n = std::min(left, most);
        a.threads = n * per_row;
        a.all = both * a.threads;
        const uint32_t groups = (a.all + 255) / 256;
        if (cache->d == 128)
            hipLaunchKernelGGL((deft_load_q8<128>), dim3(groups), dim3(256), 0, st, a);
        else
            hipLaunchKernelGGL((deft_load_q8<64>), dim3(groups), dim3(256), 0, st, a);
        if (!deft::hip_ok(hipGetLastError(), "deft_load_q8 launch")) return DEFT_EHIP;
    }
    return DEFT_OK;
}

extern "C" int deft_kv_copy_pages(const deft_kv_list_t *list, const void *dev_image, void *const *pools, const int64_t *page_bytes,
                                  int32_t n_pools, void *stream) {
    if (!list || !list->copies || !dev_image || !deft::aligned16(dev_image) || n_pools < 0) return DEFT_EINVAL;
    if (n_pools > 0 && (!pools || !page_bytes)) return DEFT_EINVAL;
    struct Pool {
        uint8_t *at;
        int64_t page;
        uint32_t width;
    };
    std::vector<Pool> todo;
    try {
        todo.reserve((size_t)n_pools);
        for (int32_t i = 0; i < n_pools; ++i) {
            if (!pools[i] || page_bytes[i] < 1 || page_bytes[i] > INT64_MAX / std::max(1, list->pool)) return DEFT_EINVAL;
            const uint64_t bits = reinterpret_cast<uintptr_t>(pools[i]) | (uint64_t)page_bytes[i] | 16;
            const int64_t width = (int64_t)(bits & -bits);
            if (page_bytes[i] / width > INT32_MAX) return DEFT_EINVAL;
            todo.push_back({static_cast<uint8_t *>(pools[i]), page_bytes[i], (uint32_t)width});
        }
        std::sort(todo.begin(), todo.end(), [](const Pool &a, const Pool &b) { return a.at < b.at; });
        for (size_t i = 1; i < todo.size(); ++i)
            if (todo[i].at - todo[i - 1].at < todo[i - 1].page * list->pool) return DEFT_EINVAL;
        if (list->heads == 0) return DEFT_OK;
        std::stable_sort(todo.begin(), todo.end(), [](const Pool &a, const Pool &b) { return a.page != b.page ? a.page > b.page : a.width > b.width; });
    } catch (...) {
        return DEFT_ENOMEM;
    }
    const uint8_t *img = static_cast<const uint8_t *>(dev_image);
    for (size_t i = 0; i < todo.size();) {
        CopyArgs a{};
        a.chains = reinterpret_cast<const u32x4 *>(img);
        a.steps = reinterpret_cast<const u32x2 *>(img + list->off_entries);
        uint32_t n = 0, groups = 0;
        for (; i < todo.size() && n < kMaxPools; ++i) {
            const Pool &p = todo[i];
            if (a.n_classes == 0 || a.classes[a.n_classes - 1].page_bytes != p.page || a.classes[a.n_classes - 1].width != p.width) {
                if (a.n_classes == kMaxClasses) break;
                PoolClass &c = a.classes[a.n_classes++];
                c.begin_group = groups;
                c.begin_pool = n;
                c.width = p.width;
                c.words = (uint32_t)(p.page / p.width);
                c.page_bytes = p.page;
                size_t alike = 1;  // pools of this class
                while (i + alike < todo.size() && todo[i + alike].page == p.page && todo[i + alike].width == p.width) ++alike;
                const uint64_t chains = (uint64_t)list->heads, wide = (c.words + 255) / 256;
                c.per_thread = c.words < 64 ? 0 : wide * chains * alike >= kManyWaves ? 4 : 1;
                c.per_page = c.per_thread == 0 ? c.words : c.per_thread == 4 ? (uint32_t)wide : (c.words + 63) / 64;
                c.inv_per_page = inverse(c.per_page);
                c.items = chains * c.per_page;
                const uint64_t per_group = c.per_thread == 0 ? 256 : 4;
                c.groups = (uint32_t)std::min<uint64_t>((c.items + per_group - 1) / per_group, kMaxGroups / 2);
                c.inv_groups = inverse(c.groups);
            }
            a.pools[n++] = p.at;
            groups += a.classes[a.n_classes - 1].groups;
        }
        hipLaunchKernelGGL(deft_copy_pages, dim3(groups), dim3(256), 0, static_cast<hipStream_t>(stream), a);
        if (!deft::hip_ok(hipGetLastError(), "deft_copy_pages launch")) return DEFT_EHIP;
    }
    return DEFT_OK;
}
