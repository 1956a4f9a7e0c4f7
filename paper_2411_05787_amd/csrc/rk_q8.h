// The cache of 8 bits (rk_kv8): argument checks, its values.
#pragma once

#include "rk_attn_common.h"

namespace rk {

constexpr int kQ8MaxBlock = 128;

static inline int check_kv8(const rk_kv8* c) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail) return RK_ERR_INVALID_ARG;
    if (c->format != RK_Q8_E4M3 && c->format != RK_Q8_INT8) return RK_ERR_UNSUPPORTED;
    if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != kQ8MaxBlock) return RK_ERR_UNSUPPORTED;
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_tail) || !aligned16(c->v_tail)) return RK_ERR_INVALID_ARG;
    if (((uintptr_t)c->k_scale & 3u) || ((uintptr_t)c->v_scale & 3u)) return RK_ERR_INVALID_ARG;
    if (c->stride_b < 0 || c->stride_h < 0 || c->stride_b % 16 != 0 || c->stride_h % 16 != 0) return RK_ERR_INVALID_ARG;
    if (c->capacity <= 0 || c->capacity % c->block != 0 || c->capacity > INT32_MAX - 2 * kMaxChunks * kMinChunk) return RK_ERR_INVALID_ARG;
    if (c->stride_b >= (1ll << 56) || c->stride_h > INT32_MAX) return RK_ERR_UNSUPPORTED;
    return RK_OK;
}

}  // namespace rk
