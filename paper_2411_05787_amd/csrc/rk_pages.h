// A cache in pages (rk_pages): argument checks.
#pragma once

#include "rk_attn_common.h"

namespace rk {

static inline int page_shift(int32_t page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7; }

static inline int check_pages(const rk_pages* c, bool rows, bool bounds) {
    if (!c || c->n_pages <= 0) return RK_ERR_INVALID_ARG;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return RK_ERR_UNSUPPORTED;
    if (rows && (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v))) return RK_ERR_INVALID_ARG;
    if (rows && (c->stride_p < 0 || c->stride_h < 0 || c->stride_p % 8 != 0 || c->stride_h % 8 != 0)) return RK_ERR_INVALID_ARG;
    if (rows && (c->stride_p > (1ll << 46) / c->n_pages || c->stride_h >= (1ll << 40))) return RK_ERR_UNSUPPORTED;      // (places in bytes: 48 bits)
    if ((c->k_min != nullptr) != (c->k_max != nullptr) || (bounds && !c->k_min)) return RK_ERR_INVALID_ARG;
    if (!aligned16(c->k_min) || !aligned16(c->k_max)) return RK_ERR_INVALID_ARG;
    return RK_OK;
}
// What a launch takes along its first axis: fewer than 2^32 threads.
static inline bool fits_launch(int64_t workgroups, int64_t threads) { return workgroups <= (int64_t)UINT32_MAX / threads; }
// A table of `width` page numbers to a sequence: its rows are numbered in 32 bits, and the kernels step past the end by up to kMaxChunks * kMinChunk.
static inline int check_table(const rk_pages* c, const int32_t* table, int32_t width) {
    if (!table || ((uintptr_t)table & 3u) || width <= 0) return RK_ERR_INVALID_ARG;
    return (int64_t)width * c->page > INT32_MAX - 2 * kMaxChunks * kMinChunk ? RK_ERR_UNSUPPORTED : RK_OK;
}

}  // namespace rk
