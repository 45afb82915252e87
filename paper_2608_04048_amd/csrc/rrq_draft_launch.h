// Internal launch interface between the C ABI layer of rrq_draft.h
// (rrq_draft_api.cpp) and its kernels. Arguments are already validated.
#pragma once

#include "rrq_draft.h"
#include "rrq_serve_launch.h"

namespace rrq_detail {

// Longest row of the norm: 1024 threads of 8 pieces of 8 elements hold it.
constexpr int64_t kNormHidden = 65536;

struct BlockNorm {
    rrq_norm norm;
    const void *residual, *y, *gate;
    void *out, *h;
    int64_t r_stride, y_stride, gate_stride, n_rows;
    int32_t hidden, out_bf16;
};
hipError_t launch_block_norm(const BlockNorm &a, bool r_bf16, bool y_bf16, hipStream_t stream);

// The append: rows as in CacheWrite, and the queries.
struct CacheAppend {
    rrq_cache cache;
    rrq_batch batch;
    const void *K, *V, *Q;
    void *Q_out;
    const double *frequencies;
    const int32_t *positions;       // NULL: the rows' places in their sequences
    double amplitude;
    int64_t k_token, k_head, v_token, v_head, q_token, q_head;      // strides in elements
    int32_t n_heads, rot, interleaved;
    // filled in by the launch: workgroups of pages, tokens a group of queries
    // has, groups, workgroups that take them
    int32_t query_tokens;
    uint32_t page_slots;
    int64_t query_groups, query_blocks;
};
hipError_t launch_cache_append(CacheAppend a, bool bf16, hipStream_t stream);

}  // namespace rrq_detail
