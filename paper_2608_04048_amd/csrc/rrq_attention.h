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
    int seq, row0;
    int o0, n_rows;
    int len, start;
};

__device__ __forceinline__ int clamp_length(const Attend &a, int len)
{
    int64_t cap = a.batch.max_pages * a.cache.page_size;
    if (cap > kMaxPositions) cap = kMaxPositions;
    return len < 0 ? 0 : (len > cap ? (int)cap : len);
}

// A value that is the same in every lane, told so to the compiler: in a scalar
// register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The rows of tile slot u, tiles of R rows.
template <int R>
__device__ __forceinline__ bool find_rows(const Attend &a, int u, RowTile &r)
{
    constexpr int shift = __builtin_ctz(R);
    const int s = uniform(find_sequence(a.batch, u, a.ratio, shift, 1));
    r.seq = s;
    r.o0 = uniform(clamp_row(a.batch, s));
    const int n = uniform(clamp_row(a.batch, s + 1)) - r.o0;
    const int given = uniform(a.batch.lengths[s]), len = given < 0 ? 0 : given;
    r.row0 = (u - ((r.o0 * a.ratio >> shift) + s)) * R;
    r.n_rows = n * a.ratio;
    if (n <= 0 || r.row0 < 0 || r.row0 >= r.n_rows) return false;   // < 0: before the first sequence
    r.start = len - n;
    r.len = clamp_length(a, len);
    return true;
}

// A row's token and query head within the kv head's group.
struct RowPlace {
    int token, member;
};
__device__ __forceinline__ RowPlace place_of(const Attend &a, int row)
{
    const uint32_t token = (uint32_t)row / (uint32_t)a.ratio;
    return RowPlace{(int)token, row - (int)token * a.ratio};
}

// Keys row token i sees: [lo, hi).
__device__ __forceinline__ void row_keys(const Attend &a, const RowTile &r, int i, int &lo,
                                         int &hi)
{
    const int64_t end = (int64_t)r.start + i + 1;       // one past the token's position
    int64_t h = a.causal && end < r.len ? end : r.len;
    int64_t l = a.window > 0 && end > a.window ? end - a.window : 0;
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
    const int end = r.row0 + R < r.n_rows ? r.row0 + R : r.n_rows;
    row_keys(a, r, uniform(place_of(a, r.row0).token), lo_any, hi_all);
    row_keys(a, r, uniform(place_of(a, end - 1).token), lo_all, hi_any);
}

// Key tiles of the whole batch, times the row tiles that read them (one kv
// head), about: what the splits share out. Every lane calls it.
template <int R>
__device__ __forceinline__ float batch_tiles(const Attend &a)
{
    const int span = R / a.ratio + 1;           // tokens of a row tile
    float sum = 0.0f;
    for (int s = threadIdx.x & 63; s < a.batch.n_seqs; s += 64) {
        const int n = clamp_row(a.batch, s + 1) - clamp_row(a.batch, s);
        if (n <= 0) continue;
        int64_t keys = clamp_length(a, a.batch.lengths[s]);
        if (a.causal) keys -= n / 2 < keys ? n / 2 : keys;
        if (a.window > 0 && keys > a.window + span) keys = a.window + span;
        sum += (float)((keys + kTileKeys - 1) / kTileKeys) * (float)((n * a.ratio + R - 1) / R);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    return sum;
}

// The key tiles [tb, te) of split number `split` of a row tile that sees
// [lo, hi). Splits are of about one size over the whole batch as far as their
// number allows, so that long sequences take more of them; a range of up to
// 1.5 times that size stays whole (two halves would cost more in written and
// joined outputs than they save). Returns whether split 0 has the whole range:
// it then writes the result itself and leaves kAlone where the join looks for
// its sum.
constexpr float kAlone = -1.0f;
template <int R>
__device__ __forceinline__ bool split_tiles(const Attend &a, int lo, int hi, int split, int &tb,
                                            int &te)
{
    const int t0 = lo / kTileKeys;
    const int tiles = hi > lo ? (hi + kTileKeys - 1) / kTileKeys - t0 : 0;
    int per = tiles, n = 1;
    if (a.n_splits > 1) {
        float share = batch_tiles<R>(a) * (float)a.cache.n_kv_heads / (float)a.target;
        share = fmaxf(share, (float)a.min_tiles);
        if ((float)tiles > 1.5f * share) {
            const float want = floorf((float)tiles / share + 0.5f);
            n = want < (float)a.n_splits ? (int)want : a.n_splits;
            per = (int)((uint32_t)(tiles + n - 1) / (uint32_t)n);
        }
    }
    n = uniform(n);
    per = uniform(per);
    tb = split * per < tiles ? t0 + split * per : t0 + tiles;
    te = tb + per < t0 + tiles ? tb + per : t0 + tiles;
    return n == 1;
}

// What a range without keys leaves for the join: a sum of 0, no mean. Grids
// are as deep as the longest sequence may need, so most workgroups of a ragged
// batch end here; they load no queries and pass no barrier.
template <int R>
__device__ __forceinline__ void empty_range(const Attend &a, const RowTile &r, int kvh, int split)
{
    const int row = r.row0 + (int)threadIdx.x;
    if (threadIdx.x >= R || row >= r.n_rows) return;
    const RowPlace place = place_of(a, row);
    const int64_t at = (int64_t)(r.o0 + place.token) * a.n_heads + kvh * a.ratio + place.member;
    const int64_t part = (int64_t)split * a.batch.n_tokens * a.n_heads + at;
    *reinterpret_cast<f32x2 *>(a.part_ml + 2 * part) = f32x2{-kInf, 0.0f};
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

// Value scales are taken relative to vref, the largest of a wave's first keys
// that are not all zeros. One that passes it by more than kReferAgain makes it
// move (so that exponents stay far from binary32's ends): m falls by the
// logarithm of the step and the sum l, in units of 2^m, grows by it; outputs
// stay, as value scale and m move alike. The step ends at 2^90, past which
// l could overflow: what went before then counts 2^-90 of the new scale.
constexpr float kReferAgain = 0x1p60f;
__device__ __forceinline__ void refer(float vmax, float vref, float &m, float &l)
{
    if (vref == 0.0f) return;           // nothing but zeros so far
    const float up = fminf(vmax / vref, 0x1p90f);
    m -= __builtin_amdgcn_logf(up);
    l *= up;
}
// vref / vs: what a weight that carries vs counts in the sum, 2^100 at most, in
// kSumUnit, which undoes the weights' largest factor (so a sum of 2^27 of them
// is finite; the unit also shifts m, by a constant that falls out). A block of
// zeros (vs = 0) may take any scale: a small one, which does not push the other
// blocks' weights down.
constexpr float kSumUnit = 0x1p-14f;
__device__ __forceinline__ float scale_back(float vs, float vref)
{
    return vs > 0.0f ? fminf(vref * kSumUnit * __builtin_amdgcn_rcpf(vs), 0x1p86f) : 0x1p46f;
}

// What turns a sum of weighted codes, in kSumUnit, into their mean value. At
// most the scale of the largest contribution, as the sum counts that one with
// vref / vs: a mean passes the largest value by its rounding at most, where
// the sum times vref may pass binary32's range.
__device__ __forceinline__ float mean_factor(float vref, float sum)
{
    return sum == 0.0f ? 0.0f : vref / sum;
}

// Operands of the products: codes are exact in binary16; queries and weights are
// rounded to it (11 bits) where the result is rounded to bfloat16's 8, and go
// in as two such parts, the rounded value and what the rounding left (22 bits),
// where it is binary32. Off by (norm of the difference to 64 bits over the
// norm) 4e-4 with one part and 6e-7 with two; plain binary32 operations make 5e-7.
// Two parts double the matrix instructions and take more registers: with few
// rows 12.2 us for 10.9 (one short step), 170 for 168 (64 sequences), 26.6 for 22.9
// (drafted tokens); with many 2530 for 1311 (4096 rows of 40 heads on 16384) and
// 230 for 105 (chunks, heads of 256), with one workgroup a compute unit for two.

// Queries go to binary16 times `up`, a power of two that brings the row's
// largest magnitude to [2^13, 2^14) (smaller values keep 11 bits a part down
// to 2^-27 of it), with the sign of the softmax scale; products times qf >= 0 are
// the scores in units of log 2. A row that holds an infinity gives no number.
__device__ __forceinline__ void query_factors(const Attend &a, float amax, float &up, float &qf)
{
    int e = (int)(__float_as_uint(amax) >> 23) - 127;
    e = e < -100 ? -100 : (e > 127 ? 127 : e);
    up = __uint_as_float((uint32_t)(13 - e + 127) << 23);
    if (a.scale < 0.0f) up = -up;
    qf = __uint_as_float((uint32_t)(e - 13 + 127) << 23) * (fabsf(a.scale) * kLog2e);
    if (amax == kInf) qf = __builtin_nanf("");
}

}  // namespace
}  // namespace rrq_detail
