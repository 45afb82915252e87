// Internal launch interface between the C ABI layer of rrq_serve.h
// (rrq_serve_api.cpp) and its kernels (rrq_cache.hip, rrq_attention.hip,
// rrq_logprobs.hip). Arguments are already validated.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "rrq_serve.h"

namespace rrq_detail {

// Compute units of an MI355X: how far small calls are split. A constant, so
// that a call's workspace does not depend on the device it is asked on.
constexpr int64_t kServeCus = 256;

// Workgroups of the write and read kernels: at most pages(b) = offsets[b + 1]
// / P - offsets[b] / P + 2 pages hold rows offsets[b] .. offsets[b + 1] - 1
// of a sequence, so n_tokens / P + 2 n_seqs page slots cover every batch; a
// workgroup finds its sequence from the offsets and leaves if its slot is
// empty.
inline int64_t cache_page_slots(const rrq_batch &b, int page_size)
{
    return b.n_tokens / page_size + 2 * b.n_seqs;
}

struct CacheWrite {
    rrq_cache cache;
    rrq_batch batch;
    const void *K, *V;
    int64_t k_token, k_head, v_token, v_head;   // strides in elements
};
hipError_t launch_cache_write(const CacheWrite &a, bool bf16, hipStream_t stream);

struct CacheRead {
    rrq_cache cache;
    rrq_batch batch;
    void *K, *V;
};
hipError_t launch_cache_read(const CacheRead &a, bool bf16, hipStream_t stream);

// Attention. Rows of a sequence and kv head are (token, query head of the
// group): row r is token r / ratio, head kv * ratio + r % ratio. Two forms: few
// rows a sequence (row tiles of 16 or 32, rrq_attention.hip) and many (row tiles
// of 128, rrq_attention_rows.hip). At most offsets[b + 1] * ratio / R - offsets[b]
// * ratio / R + 1 tiles of R rows hold a sequence's rows.
constexpr int kWideTile = 32, kRowsTile = 128;
inline int64_t attend_row_tiles(const rrq_batch &b, int ratio, int tile)
{
    return b.n_tokens * ratio / tile + b.n_seqs;
}
// How a call is served: the form and its rows a tile; the key ranges a row tile is split into at
// most, of min_tiles 64-key tiles at least, about target workgroups in all;
// waves a workgroup and rows a tile of the few-row form.
struct AttendPlan {
    bool rows_form;
    int tile, splits, target, min_tiles, waves, lds_rows;
};
AttendPlan attend_plan(const rrq_cache &c, const rrq_batch &b, int n_heads, int64_t window);
struct Attend {
    rrq_cache cache;
    rrq_batch batch;
    const void *Q;
    int64_t q_token, q_head;
    void *out;
    float *part_o;      // [n_splits][n_tokens][n_heads][D], n_splits > 1
    float *part_ml;     // [n_splits][n_tokens][n_heads][2]
    int64_t window;     // 0: none
    float scale;
    int32_t n_heads, ratio, causal, q_bf16, out_bf16;
    int32_t n_splits, target, min_tiles, lds_rows;
};
hipError_t launch_attend(const Attend &a, const AttendPlan &p, hipStream_t stream);
hipError_t launch_attend_rows(const Attend &a, hipStream_t stream);

struct Logprobs {
    const void *logits;
    const int64_t *targets;
    float *logprobs, *entropy, *top_logprobs;
    int64_t *top_ids;
    void *workspace;
    int64_t n_rows, vocab, row_stride;
    int32_t n_top, segments;
};
// Segments (workgroups) a row is split into, and the workspace of one row's
// segments.
int logprobs_segments(int64_t n_rows, int64_t vocab);
size_t logprobs_row_bytes(int segments, int n_top);
hipError_t launch_logprobs(const Logprobs &a, bool bf16, hipStream_t stream);

}  // namespace rrq_detail
