// A paged K/V cache as the kernels and their host code see it (opttree.h: ot_paged_cache).
#pragma once

#include "common.hpp"

namespace ot {

// Argument rules of a cache; pointers included when `pointers`.
inline int validate_cache(const ot_paged_cache* c, bool pointers) {
    if (!c) return OT_ERR_INVALID_ARG;
    if (c->num_pages < 1 || c->kv_heads < 1 || c->max_pages < 1 || c->page_size < 1) return OT_ERR_INVALID_ARG;
    if (c->dtype != OT_BF16 && c->dtype != OT_E4M3) return OT_ERR_INVALID_ARG;
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return OT_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128) return OT_ERR_UNSUPPORTED;
    if ((long long)c->max_pages * c->page_size >= 1 << 30 || (long long)c->num_pages * c->kv_heads > 0x7fffffffLL) return OT_ERR_UNSUPPORTED;
    const int vec = c->dtype == OT_BF16 ? 8 : 16;
    const int64_t* st[2] = {c->k_strides, c->v_strides};
    for (int t = 0; t < 2; ++t) {
        for (int i = 0; i < 3; ++i)
            if (st[t][i] < 0 || st[t][i] % vec) return OT_ERR_INVALID_ARG;
        if (st[t][2] < c->head_dim) return OT_ERR_INVALID_ARG;
        if (st[t][2] > (1 << 22) || st[t][0] / vec > 0xffffffffLL) return OT_ERR_UNSUPPORTED;      // 32-bit arithmetic in the kernels
    }
    if (!pointers) return OT_OK;
    if (!c->k_pages || !c->v_pages || !c->page_table) return OT_ERR_INVALID_ARG;
    if ((uintptr_t)c->k_pages % 16 || (uintptr_t)c->v_pages % 16 || (uintptr_t)c->page_table % 4) return OT_ERR_INVALID_ARG;
    if (c->dtype == OT_E4M3 && (!c->k_exp || !c->v_exp || (uintptr_t)c->k_exp % 4 || (uintptr_t)c->v_exp % 4)) return OT_ERR_INVALID_ARG;
    return OT_OK;
}

inline int log2_of(int power) { return __builtin_ctz((unsigned)power); }

}  // namespace ot
