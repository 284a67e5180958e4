// Shared pieces of the calls that read and write the paged K/V pool.
#pragma once
#include <stdint.h>

#include "../../include/gift.h"
#include "gift_batch.cuh"

namespace gift {

// Host checks of a pool.
inline int pool_args_ok(const gift_kv_pool* p)
{
    if (!p || !p->pages) return GIFT_E_INVAL;
    if (p->dtype != GIFT_BF16 && p->dtype != GIFT_FP16) return GIFT_E_INVAL;
    if (p->page_tokens == 0 || p->n_heads == 0 || p->head_dim == 0) return GIFT_E_INVAL;
    if (p->page_tokens > GIFT_MAX_PAGE_TOKENS || p->n_heads > GIFT_MAX_HEADS || p->head_dim > 1024u) return GIFT_E_RANGE;
    if ((uint64_t)p->n_pages * p->page_tokens > 0x7FFFFFFFu) return GIFT_E_RANGE;
    if (((uintptr_t)p->pages & 15) || p->head_dim % 8 != 0) return GIFT_E_ALIGN;
    return GIFT_OK;
}

// Host checks of a [rows][heads][head_dim] array with contiguous heads' elements: 16-byte accesses.
inline int rows_args_ok(const void* p, uint64_t row_stride, uint64_t head_stride)
{
    if (!p) return GIFT_E_INVAL;
    // tensor maps take strides below 2^40 bytes
    if (row_stride >= ((uint64_t)1 << 38) || head_stride >= ((uint64_t)1 << 38)) return GIFT_E_RANGE;
    if (((uintptr_t)p & 15) || row_stride % 8 != 0 || head_stride % 8 != 0) return GIFT_E_ALIGN;
    return GIFT_OK;
}

}  // namespace gift
