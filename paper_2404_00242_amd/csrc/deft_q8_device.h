// What the kernels that write and read an 8-bit cache share (deft_cache.hip, deft_heads.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "deft_device.h"
#include "deft_lists.h"

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

// floor(n / d), given inverse(d)
uint32_t inverse(uint32_t d) { return d == 1 ? 0xffffffffu : (uint32_t)((uint64_t(1) << 32) / d); }
__device__ __forceinline__ uint32_t divide(uint32_t n, uint32_t d, uint32_t inv) {
    const uint32_t q = __umulhi(n, inv);  // floor(n / d) or one less
    return n - q * d >= d ? q + 1 : q;
}

// What is read once is not kept in the caches (prompt of 8192 tokens x 32 heads stored, 201 MB: 51.7 -> 36.7 us).
template <typename T>
__device__ __forceinline__ T load_once(const T *p) {
    return __builtin_nontemporal_load(p);
}

constexpr int kScaleMin = 10;   // 2^-117: the cache's smallest value, 2^-9 of it, is a normal bf16 number
constexpr int kScaleMax = 246;  // 2^119: the cache's largest value, 448 of it, is a finite bf16 number

struct CacheArgs {
    uint8_t *k, *v, *k_scale, *v_scale;
    uint32_t Hkv, inv_Hkv;
};

// largest magnitude as bf16 bits -> scale byte: the smallest power of two that brings it to 448 = 1.75 * 2^8 or below
__device__ __forceinline__ int scale_byte(uint32_t bits) {
    const int e = (int)(bits >> 7) - 8 + ((bits & 0x7f) > 0x60);
    return min(max(e, kScaleMin), kScaleMax);
}
__device__ __forceinline__ float power(int byte) { return __builtin_bit_cast(float, (uint32_t)byte << 23); }
__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// rounds to nearest, ties to even; past 448 only where the scale is at its largest
__device__ __forceinline__ uint32_t round4(float a, float b, float c, float d) {
    a = fminf(fmaxf(a, -448.f), 448.f);
    b = fminf(fmaxf(b, -448.f), 448.f);
    c = fminf(fmaxf(c, -448.f), 448.f);
    d = fminf(fmaxf(d, -448.f), 448.f);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ u32x2 round8(const u32x4 &x, float inv) {
    auto lo = [&](int i) { return __builtin_bit_cast(float, x[i] << 16) * inv; };
    auto hi = [&](int i) { return __builtin_bit_cast(float, x[i] & 0xffff0000u) * inv; };
    return u32x2{round4(lo(0), hi(0), lo(1), hi(1)), round4(lo(2), hi(2), lo(3), hi(3))};
}
// e4m3 values times a power of two that is below one, rounded again; a NaN stays one
__device__ __forceinline__ uint32_t rescale4(uint32_t x, float by) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * by, b[1] * by, __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * by, a[1] * by, 0, false), true);
}
__device__ __forceinline__ void rescale_kept(uint8_t *rows, uint32_t first, uint32_t step, uint32_t low, size_t pitch, float by) {
    for (uint32_t r = first; r < low; r += step) {
        u32x2 *p = reinterpret_cast<u32x2 *>(rows + r * pitch);
        const u32x2 x = *p;
        *p = u32x2{rescale4(x[0], by), rescale4(x[1], by)};
    }
}

// ---- host ----

CacheArgs cache_args(const deft_cache_q8_t *c) {
    return {static_cast<uint8_t *>(c->k), static_cast<uint8_t *>(c->v), static_cast<uint8_t *>(c->k_scale), static_cast<uint8_t *>(c->v_scale),
            (uint32_t)c->Hkv, inverse((uint32_t)c->Hkv)};
}

// A list of rows and the cache that it is for.
bool rows_fit(const deft_kv_list_t *list, const void *dev_image, const deft_cache_q8_t *cache) {
    return list && !list->copies && dev_image && deft::aligned16(dev_image) && deft::cache_ok(cache) && list->block_rows == cache->block_rows &&
           list->pool <= cache->n_rows;
}

}  // namespace
