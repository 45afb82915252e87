// Argument checks shared by the C ABI layers of rrq_serve.h and rrq_draft.h.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "rrq_serve.h"

namespace rrq_detail {

inline bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// The cache's sizes, and (buffers) its pointers.
inline int check_cache(const rrq_cache *c, bool buffers)
{
    if (!c) return RRQ_ERR_NULL;
    if (c->code_type != RRQ_CODE_INT8 && c->code_type != RRQ_CODE_FP8) return RRQ_ERR_FORMAT;
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 1024) return RRQ_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return RRQ_ERR_SHAPE;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
        return RRQ_ERR_SHAPE;
    // byte offsets into the codes fit in int64
    if (c->n_pages > INT64_MAX / ((int64_t)c->n_kv_heads * c->head_dim * c->page_size))
        return RRQ_ERR_SHAPE;
    if (!buffers) return RRQ_OK;
    if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return RRQ_ERR_NULL;
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scales, 4) ||
        !aligned(c->v_scales, 4))
        return RRQ_ERR_ALIGN;
    return RRQ_OK;
}

inline int check_batch(const rrq_batch *b, bool buffers)
{
    if (!b) return RRQ_ERR_NULL;
    if (b->n_seqs < 0 || b->n_seqs > (int64_t(1) << 20) || b->n_tokens < 0 ||
        b->n_tokens > (int64_t(1) << 26))
        return RRQ_ERR_SHAPE;
    if (b->n_seqs == 0) return RRQ_OK;
    if (b->max_pages < 1 || b->table_stride < b->max_pages ||
        b->table_stride > (int64_t(1) << 40))
        return RRQ_ERR_SHAPE;
    if (!buffers) return RRQ_OK;
    if (!b->page_table || !b->lengths || !b->offsets) return RRQ_ERR_NULL;
    if (!aligned(b->page_table, 4) || !aligned(b->lengths, 4) || !aligned(b->offsets, 4))
        return RRQ_ERR_ALIGN;
    return RRQ_OK;
}

// Dense rows read with caller's strides: 16-byte aligned pieces.
inline int check_rows(const void *p, int32_t dtype, int64_t token, int64_t head)
{
    const int64_t per = dtype == RRQ_F32 ? 4 : 8;       // elements in 16 bytes
    if (!p) return RRQ_ERR_NULL;
    if (token < 0 || head < 0 || token > (int64_t(1) << 32) || head > (int64_t(1) << 32))
        return RRQ_ERR_SHAPE;
    if (!aligned(p, 16) || token % per != 0 || head % per != 0) return RRQ_ERR_ALIGN;
    return RRQ_OK;
}

inline bool known_dtype(int32_t t) { return t == RRQ_F32 || t == RRQ_BF16; }

inline int status(hipError_t e) { return e == hipSuccess ? RRQ_OK : RRQ_ERR_HIP; }

inline int check_heads(const rrq_cache *c, const rrq_batch *b, int32_t n_heads)
{
    if (n_heads < 1 || n_heads > (1 << 16) || n_heads % c->n_kv_heads != 0) return RRQ_ERR_SHAPE;
    if (b->n_tokens * (n_heads / c->n_kv_heads) > (int64_t(1) << 26)) return RRQ_ERR_SHAPE;
    return RRQ_OK;
}

}  // namespace rrq_detail
