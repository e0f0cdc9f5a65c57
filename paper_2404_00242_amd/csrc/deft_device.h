// What the device sides of the library (deft_decode.hip, deft_cache.hip) share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "deft.h"

namespace deft {
// False, and the text for deft_last_hip_error, where a runtime call failed.
bool hip_ok(hipError_t e, const char *what);
// Sends a plan's or a list's image to device memory on a stream (see deft_plan_upload).  Returns a deft_status.
int upload_image(void *dev_image, const uint8_t *src, size_t bytes, hipStream_t st);

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Whether a cache's description is one: what any call on it asks for before it reads from it.
inline bool cache_ok(const deft_cache_q8_t *c) {
    if (!c || !aligned16(c->k) || !aligned16(c->v)) return false;
    if (c->n_rows > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return false;
    if ((reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale)) & 3) return false;
    if (c->n_rows < 0 || c->Hkv <= 0 || c->Hkv > DEFT_MAX_Q8_HEADS || (c->d != 64 && c->d != 128)) return false;
    return c->block_rows >= 1 && c->block_rows <= 64 && (c->block_rows & (c->block_rows - 1)) == 0;
}
}  // namespace deft
