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
    int64_t r_stride, y_stride, gate_stride, n_rows, row0;
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

// Verification. The workspace: a segment's largest logit and sum (greedy: the place
// of the largest) of each row; where a sequence's walk ended; sums over a block of the
// vocabulary of what the next token is drawn from.
struct VerifySum {
    float m;
    int32_t unused;
    double sum;
};
struct VerifyChoice {
    int32_t row, first, n, at;      // of the logits (-1: nothing to draw from); of the sequence
    int32_t draft;                  // the draft's row that was rejected, -1: none
    int32_t removed;                // the children's tokens are
    int32_t last;                   // the last of them that had any weight, -1: none
    float m, mq;                    // with a rejected draft: largest logits and sums
    double l, lq;
};
struct VerifyBlock {
    double p, q, sp, sq;            // of p, of q, of both where p > q
    float m;                        // p's weights are relative to it
    int32_t unused;
};
struct Verify {
    const void *logits, *draft;
    const int64_t *tokens;
    const int32_t *offsets, *parents;
    const float *uniforms;
    int32_t *counts, *paths;
    int64_t *following;
    VerifySum *sums;
    VerifyChoice *choices;
    VerifyBlock *blocks;
    int64_t n_rows, n_seqs, vocab, row_stride, draft_seq_stride, draft_row_stride, segment;
    double inv_temperature, inv_draft_temperature;      // 0: greedy
    int32_t max_accept, segments, draw_segments, bf16;
};
// Logits a workgroup takes at a time, and the most segments (of whole blocks) of a row.
constexpr int64_t kVerifySumBlock = 8192, kVerifyDrawBlock = 4096;
constexpr int kVerifySegments = 64;
// Logits of a segment where `units` rows are summed.
int64_t verify_segment(int64_t units, int64_t vocab);
hipError_t launch_verify(const Verify &a, hipStream_t stream);

}  // namespace rrq_detail
