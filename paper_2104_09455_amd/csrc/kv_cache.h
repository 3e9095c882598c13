// The paged cache as its kernels see it, and the host's checks of a cache descriptor.
#pragma once
#include "../../include/abft.h"
#include "gemm_common.h"

namespace abft {

constexpr int KV_MAX_DIM = 128, KV_MAX_PAGE = 4096;

// ABFT_OK, or why the descriptor cannot be used with 16-bit values of type `dtype`
inline int kv_validate(const abft_kv_cache_t* c, int dtype) {
    if (!c) return ABFT_E_NULL;
    if (dtype != ABFT_F16 && dtype != ABFT_BF16) return ABFT_E_ENUM;
    if (c->dtype != ABFT_I8 && c->dtype != dtype) return ABFT_E_ENUM;
    if (c->pages <= 0 || c->heads <= 0 || c->head_dim <= 0 || c->head_dim % 16 != 0 || c->head_dim > KV_MAX_DIM) return ABFT_E_SHAPE;
    if (c->page_size <= 0 || c->page_size % 16 != 0 || c->page_size > KV_MAX_PAGE) return ABFT_E_VALUE;
    if ((long long)c->pages * c->page_size > 0x7fffffffll || (long long)c->pages * c->heads > 0x7fffffffll) return ABFT_E_SHAPE;
    if (!c->k || !c->v || (c->dtype == ABFT_I8 && (!c->k_scale || !c->v_scale))) return ABFT_E_NULL;
    uintptr_t at = reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v);
    if (c->dtype == ABFT_I8) at |= reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale);
    if ((at & 15u) != 0) return ABFT_E_LD;
    return ABFT_OK;
}

}  // namespace abft
