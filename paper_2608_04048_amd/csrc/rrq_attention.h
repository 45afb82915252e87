// What the forms of attention over the 8-bit cache share: which rows and keys
// a workgroup has, and the queries' scaling.
#pragma once

#include "rrq_serve_device.h"
#include "rrq_serve_launch.h"

namespace rrq_detail {
namespace {

constexpr int kTileKeys = 64;
// Positions are ints; tiles may reach past the last one.
constexpr int64_t kMaxPositions = (int64_t(1) << 31) - 4096;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The rows of a workgroup: rows row0 .. of sequence seq, which has n_rows
// rows (tokens x ratio) from dense row o0 on, its first token at position
// start of len.
struct RowTile {
    int64_t seq, row0;
    int64_t o0, n_rows;
    int64_t len, start;
};

__device__ __forceinline__ int64_t clamp_length(const Attend &a, int64_t len)
{
    int64_t cap = a.batch.max_pages * a.cache.page_size;
    if (cap > kMaxPositions) cap = kMaxPositions;
    return len < 0 ? 0 : (len > cap ? cap : len);
}

// The rows of tile slot u, tiles of R rows.
template <int R>
__device__ __forceinline__ bool find_rows(const Attend &a, int64_t u, RowTile &r)
{
    const int64_t s = find_sequence(a.batch, u, a.ratio, R, 1);
    r.seq = s;
    r.o0 = clamp_row(a.batch, s);
    const int64_t n = clamp_row(a.batch, s + 1) - r.o0;
    r.row0 = (u - (r.o0 * a.ratio / R + s)) * R;
    r.n_rows = n * a.ratio;
    if (n <= 0 || r.row0 < 0 || r.row0 >= r.n_rows) return false;   // < 0: before the first sequence
    const int64_t len = a.batch.lengths[s];
    r.start = len - n;
    r.len = clamp_length(a, len);
    return true;
}

// Keys row token i sees: [lo, hi).
__device__ __forceinline__ void row_keys(const Attend &a, const RowTile &r, int64_t i, int &lo,
                                         int &hi)
{
    const int64_t pos = r.start + i;
    int64_t h = a.causal && pos + 1 < r.len ? pos + 1 : r.len;
    int64_t l = a.window > 0 && pos + 1 > a.window ? pos + 1 - a.window : 0;
    if (h < 0) h = 0;
    if (l > h) l = h;
    lo = (int)l;
    hi = (int)h;
}

// Keys any row and every row of the tile sees: tokens ascend with rows, and so
// do both ends of what they see.
template <int R>
__device__ __forceinline__ void tile_keys(const Attend &a, const RowTile &r, int &lo_any,
                                          int &hi_any, int &lo_all, int &hi_all)
{
    const int64_t end = r.row0 + R < r.n_rows ? r.row0 + R : r.n_rows;
    row_keys(a, r, r.row0 / a.ratio, lo_any, hi_all);
    row_keys(a, r, (end - 1) / a.ratio, lo_all, hi_any);
}

// Key tiles of the whole batch, times the row tiles that read them (one kv
// head): what the splits share out. Every lane calls it.
template <int R>
__device__ __forceinline__ int64_t batch_tiles(const Attend &a)
{
    int64_t sum = 0;
    for (int64_t s = threadIdx.x & 63; s < a.batch.n_seqs; s += 64) {
        const int64_t n = clamp_row(a.batch, s + 1) - clamp_row(a.batch, s);
        if (n <= 0) continue;
        int64_t keys = clamp_length(a, a.batch.lengths[s]);
        if (a.window > 0 && keys > a.window + n) keys = a.window + n;
        sum += (keys + kTileKeys - 1) / kTileKeys * ((n * a.ratio + R - 1) / R);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    return sum;
}

// The key tiles [tb, te) of split number `split` of a row tile that sees
// [lo, hi). Splits are of one size over the whole batch as far as their
// number allows, so that long sequences take more of them.
template <int R>
__device__ __forceinline__ void split_tiles(const Attend &a, int lo, int hi, int split, int &tb,
                                            int &te)
{
    const int t0 = lo / kTileKeys;
    const int tiles = hi > lo ? (hi + kTileKeys - 1) / kTileKeys - t0 : 0;
    int per = tiles;
    if (a.n_splits > 1) {
        const int64_t even = (batch_tiles<R>(a) * a.cache.n_kv_heads + a.target - 1) / a.target;
        per = (tiles + a.n_splits - 1) / a.n_splits;
        per = per < even ? (int)even : per;
        per = per < a.min_tiles ? a.min_tiles : per;
    }
    tb = split * per < tiles ? t0 + split * per : t0 + tiles;
    te = tb + per < t0 + tiles ? tb + per : t0 + tiles;
}

// N query values of the element offset `at` on.
template <int N>
__device__ __forceinline__ void load_query(const Attend &a, int64_t at, float (&x)[N])
{
    if (a.q_bf16) {
#pragma unroll
        for (int v = 0; v < N / 8; ++v) {
            const u32x4v w = *reinterpret_cast<const u32x4v *>(
                static_cast<const uint16_t *>(a.Q) + at + 8 * v);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[8 * v + 2 * e] = __uint_as_float(w[e] << 16);
                x[8 * v + 2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int v = 0; v < N / 4; ++v) {
            const f32x4 y = *reinterpret_cast<const f32x4 *>(
                static_cast<const float *>(a.Q) + at + 4 * v);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * v + e] = y[e];
        }
    }
}

// Queries go to binary16 times `up`, a power of two that brings the row's
// largest magnitude to [2^13, 2^14) (smaller values keep 11 bits down to
// 2^-27 of it), with the sign of the softmax scale; products times qf >= 0 are
// the scores in units of log 2. A row that holds an infinity gives no number.
__device__ __forceinline__ void query_factors(const Attend &a, float amax, float &up, float &qf)
{
    int e = (int)(__float_as_uint(amax) >> 23) - 127;
    e = e < -100 ? -100 : (e > 120 ? 120 : e);
    up = __uint_as_float((uint32_t)(13 - e + 127) << 23);
    if (a.scale < 0.0f) up = -up;
    qf = __uint_as_float((uint32_t)(e - 13 + 127) << 23) * (fabsf(a.scale) * kLog2e);
    if (amax == kInf) qf = __builtin_nanf("");
}

}  // namespace
}  // namespace rrq_detail
