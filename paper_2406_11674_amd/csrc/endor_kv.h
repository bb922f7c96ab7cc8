// The paged key-value cache as the device code of the decode side sees it, and the host's checks of it.
#ifndef ENDOR_KV_H_
#define ENDOR_KV_H_

#include <hip/hip_runtime.h>

#include <cstdint>

#include "endor.h"

namespace endor_kv {

struct Cache {
    uint16_t *k, *v;
    int64_t page_stride, head_stride, slot_stride;
    const int32_t *pages;
    int64_t pages_stride;
    uint32_t num_pages, page_shift, max_pages;
    int32_t batch, kv_heads, dim;
};

inline int32_t capacity_of(const endor_kv_cache &c) { return c.max_pages * c.page_size; }

// ENDOR_OK and *out, or what is wrong with the caller's description.
inline endor_status read_cache(const endor_kv_cache *c, Cache *out) {
    if (!c) return ENDOR_ERR_INVALID_ARG;
    if (c->batch < 0 || c->kv_heads < 1 || c->max_pages < 0 || c->num_pages < 0 || c->num_pages > 0x7fffffff) return ENDOR_ERR_INVALID_ARG;
    if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 != 0) return ENDOR_ERR_UNSUPPORTED;
    if (c->page_size < 8 || c->page_size > 32768 || (c->page_size & (c->page_size - 1)) != 0) return ENDOR_ERR_UNSUPPORTED;
    if (c->dtype != ENDOR_F16 && c->dtype != ENDOR_BF16) return ENDOR_ERR_UNSUPPORTED;
    if (int64_t(c->max_pages) * c->page_size > (1 << 30)) return ENDOR_ERR_UNSUPPORTED;
    // a launch has at most 65535 workgroups in y and z, and a program of a few heads never comes near it
    if (c->batch > 65535 || c->kv_heads > 65535) return ENDOR_ERR_UNSUPPORTED;
    for (int64_t s : {c->page_stride, c->head_stride, c->slot_stride})
        if (s < c->head_dim || s % 8 != 0) return ENDOR_ERR_INVALID_ARG;
    if (c->max_pages > 0 && c->batch > 0) {
        if (!c->d_pages || (reinterpret_cast<uintptr_t>(c->d_pages) & 3) || c->pages_stride < c->max_pages) return ENDOR_ERR_INVALID_ARG;
        if (c->num_pages > 0)
            for (const void *p : {c->d_k, c->d_v})
                if (!p || (reinterpret_cast<uintptr_t>(p) & 15)) return ENDOR_ERR_INVALID_ARG;
    }
    out->k = static_cast<uint16_t *>(c->d_k);
    out->v = static_cast<uint16_t *>(c->d_v);
    out->page_stride = c->page_stride;
    out->head_stride = c->head_stride;
    out->slot_stride = c->slot_stride;
    out->pages = c->d_pages;
    out->pages_stride = c->pages_stride;
    out->num_pages = static_cast<uint32_t>(c->num_pages);
    out->page_shift = static_cast<uint32_t>(__builtin_ctz(static_cast<unsigned>(c->page_size)));
    out->max_pages = static_cast<uint32_t>(c->max_pages);
    out->batch = c->batch;
    out->kv_heads = c->kv_heads;
    out->dim = c->head_dim;
    return ENDOR_OK;
}

inline bool aligned(const void *p, uintptr_t to) { return p && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// The page of a slot below the capacity, and whether it is there.
__device__ __forceinline__ bool page_of(const Cache &C, const int32_t *row, uint32_t slot, uint32_t *page) {
    *page = static_cast<uint32_t>(row[slot >> C.page_shift]);
    return *page < C.num_pages;
}
// Element offset of a slot's first element: pools pass 2^32 elements, so it is formed in 64 bits.
__device__ __forceinline__ int64_t slot_at(const Cache &C, uint32_t page, uint32_t head, uint32_t slot) {
    return int64_t(page) * C.page_stride + int64_t(head) * C.head_stride + int64_t(slot & ((1u << C.page_shift) - 1)) * C.slot_stride;
}

__device__ __forceinline__ int32_t clamp_length(int32_t n, int32_t most) { return n < 0 ? 0 : n > most ? most : n; }

}  // namespace endor_kv

#endif  // ENDOR_KV_H_
