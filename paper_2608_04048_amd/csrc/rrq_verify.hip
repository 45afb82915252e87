// Verification of drafted tokens against the target's distributions
// (rrq_draft.h: rrq_verify_drafts).
//
// A row's probabilities are e^(x / T) / l, l the sum over the vocabulary. Four steps:
//   1. sums: l of every row that has children (only those are asked whether to accept
//      one), and of the draft's rows: segments of a row, each with a large logit m and
//      its sum relative to that;
//   2. decide: one wave a sequence walks down from the root. Rows are 64 at a time in
//      the lanes; a lane has its token's probability under its parent, the walk itself
//      is a ballot and a broadcast a tried token;
//   3. weights: of the one row a sequence ends at, sums of what the next token is drawn
//      from, a block of the vocabulary a workgroup, in 64 bits;
//   4. draw: the block in which the running sum passes the random number's share, and
//      the token in it.
// Greedy calls (T = 0) end with step 2, on each row's first largest logit.
//
// Precision. Whether u q < p or a running sum passes u times the total is a border
// that any input may come near, and the results are whole numbers. Step 1 has
// binary32 exponentials (each off by 2^-24 or so at random) and corrects what is
// systematic, the rounding of log2(e) / T, by the sum of e d; sums of more than eight
// are 64 bits. A logit's distance d to its thread's reference is rounded, and so is its
// product with log2(e) / T: 2^-24 of the exponent each, so the reference is the largest of
// 2048 logits and moves up where a later one passes it by 6 powers of two. l is good to
// 2^-24 as a rule, a decision off in one of some 10^7 cases; at worst, with all of l in one
// such logit, to 18 x 2^-24 (2 x 6 ln 2 of those roundings, 2 of the exponential, 7 of the
// additions). A reference that stays put until 2^60 gives 50 x 2^-24 there and saves no time.
// Running sums of a vocabulary pass borders that lie 10^-5 apart: steps 3 and 4 are 64
// bits throughout, exponentials good to 2 10^-13. The residual (p - q)+ needs both rows'
// sums before it can be formed; step 3 leaves the sums of p and of q over the tokens
// where p > q (by step 1's sums; a token whose sign these get wrong adds nothing) for
// step 4 to scale and subtract.
//
// Measured. Step 1 is bound by memory: 96 sequences of 3 to 7 drafts with the draft's
// distributions, 150001 tokens in bfloat16, 290 MB in 59 us (4.9 TB/s), its vector
// instructions (ten a logit) 70% of that time; of 16 trees of 29 to 48 drafts and 131072
// tokens in binary32 the 264 rows that have children, 138 MB in 30 us. Step 3 is bound by
// issue: 58 MB and 14 million pairs of exponentials in 28 us, the vector units busy 72% of
// it. Steps 2 and 4 are chains of dependent loads: 6 to 7 and 7 to 9 us. Five drafts of
// one sequence take 4.0, 8.0 (steps 2 and 3 together) and 7.8 us.
#include <hip/hip_runtime.h>

#include "rrq_draft_launch.h"
#include "rrq_serve_device.h"
#include "rrq_wave.h"

namespace rrq_detail {
namespace {

constexpr float kInf = __builtin_inff();
constexpr double kLn2 = 0.69314718055994530942, kLog2e = 1.44269504088896340736;
constexpr int kThreads = 256;
// A block's sum from which on step 1's reference moves up to the block's largest logit.
// (32 logits up to the reference make 32 at most.)
constexpr double kFar = 64.0;
// Logits a thread takes: in step 1; in step 3, and in step 4, whose one workgroup a
// sequence has twice the threads, as its time is a single wave's.
constexpr int kSumLane = 32, kWeightLane = 16, kDrawLane = 8, kDrawThreads = 512;
constexpr int kSumBlock = kThreads * kSumLane, kDrawBlock = kThreads * kWeightLane;
static_assert(kSumBlock == kVerifySumBlock && kDrawBlock == kVerifyDrawBlock &&
                  kDrawBlock == kDrawThreads * kDrawLane, "blocks of the workspace");

// 2^y, y of any size; a NaN stays one.
__device__ __forceinline__ double exp2_64(double y)
{
    y = y < -1100.0 ? -1100.0 : (y > 1100.0 ? 1100.0 : y);
    const double n = __builtin_rint(y);
    const double r = (y - n) * kLn2;
    double p = 1.0 / 39916800.0;
    p = __builtin_fma(p, r, 1.0 / 3628800.0);
    p = __builtin_fma(p, r, 1.0 / 362880.0);
    p = __builtin_fma(p, r, 1.0 / 40320.0);
    p = __builtin_fma(p, r, 1.0 / 5040.0);
    p = __builtin_fma(p, r, 1.0 / 720.0);
    p = __builtin_fma(p, r, 1.0 / 120.0);
    p = __builtin_fma(p, r, 1.0 / 24.0);
    p = __builtin_fma(p, r, 1.0 / 6.0);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}
// e^((x - m) / T), c = log2(e) / T.
__device__ __forceinline__ double weight(float x, float m, double c)
{
    return exp2_64(((double)x - (double)m) * c);
}

// The same from a table of 2^(i / 256) in LDS and a series of degree 3 (2e-13): half
// the instructions of the whole one. (32 entries, no two of which share a bank, and
// degree 5: two instructions of 20 more.)
constexpr int kTable = 256;
__device__ __forceinline__ void fill_table(double *table)
{
    if (threadIdx.x < kTable) table[threadIdx.x] = exp2_64(threadIdx.x * (1.0 / kTable));
    __syncthreads();
}
// c: kTable log2(e) / T. The sum with 1.5 2^52 rounds y to a whole number, which its
// low bits are.
__device__ __forceinline__ double weight(const double *table, float x, float m, double c)
{
    constexpr double kRound = 6755399441055744.0, L = kLn2 / kTable;
    const double y = ((double)x - (double)m) * c;
    const double t = y + kRound;
    const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, t);
    const double r = y - (t - kRound);
    double p = __builtin_fma(L * L * L / 6.0, r, L * L / 2.0);
    p = __builtin_fma(p, r, L);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_amdgcn_ldexp(table[n & (kTable - 1)] * p, n >> 8);
    return y < -1000.0 * kTable ? 0.0 : p;
}

__device__ __forceinline__ float logit(const void *row, bool bf16, int64_t i)
{
    if (bf16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(row)[i] << 16);
    return static_cast<const float *>(row)[i];
}

// Sequence b's rows: the first, and how many.
__device__ __forceinline__ int rows_of(const Verify &a, int b, int &n)
{
    const int N = (int)a.n_rows;
    int o0 = a.offsets[b], o1 = a.offsets[b + 1];
    o0 = o0 < 0 ? 0 : (o0 > N ? N : o0);
    o1 = o1 < 0 ? 0 : (o1 > N ? N : o1);
    n = o1 > o0 ? o1 - o0 : 0;
    return o0;
}
// Row j's parent among its sequence's rows; -1: none that counts.
__device__ __forceinline__ int parent_of(const Verify &a, int o0, int j)
{
    if (j <= 0) return -1;
    if (!a.parents) return j - 1;
    const int p = a.parents[o0 + j];
    return p >= 0 && p < j ? p : -1;
}

__device__ __forceinline__ const void *target_row(const Verify &a, int64_t row)
{
    return static_cast<const char *>(a.logits) + row * a.row_stride * (a.bf16 ? 2 : 4);
}
__device__ __forceinline__ const void *draft_row(const Verify &a, int64_t b, int64_t j)
{
    return static_cast<const char *>(a.draft) +
           (b * a.draft_seq_stride + j * a.draft_row_stride) * (a.bf16 ? 2 : 4);
}

// Where in a block of T threads' N logits a thread's i-th stands: VEC (16 bytes) in a
// row; RUNS: N in a row.
template <bool BF16, int N, bool RUNS, int T>
__device__ __forceinline__ int place(int i)
{
    constexpr int VEC = BF16 ? 8 : 4;
    return RUNS ? (int)threadIdx.x * N + i : ((i / VEC) * T + (int)threadIdx.x) * VEC + i % VEC;
}

// A thread's N logits of the block from `base` on, as they are loaded: 16 bytes at a
// time, without a branch between them. Rows may start at any multiple of their type; a
// piece that passes the vocabulary's end is read from inside it and put right by unpack.
struct __attribute__((packed, aligned(2))) Wide {
    uint32_t w[4];
};
template <bool BF16, bool RUNS, int N, int T>
struct Block {
    static constexpr int VEC = BF16 ? 8 : 4, SIZE = BF16 ? 2 : 4;
    Wide piece[N / VEC];

    __device__ __forceinline__ void load(const void *row, int64_t base, int64_t vocab)
    {
        const char *x = static_cast<const char *>(row);
        const bool whole = base + (int64_t)T * N <= vocab;
        if (!whole && vocab < VEC) return;
        const int64_t end = vocab - VEC;
#pragma unroll
        for (int i = 0; i < N / VEC; ++i) {
            const int64_t at = base + place<BF16, N, RUNS, T>(i * VEC);
            piece[i] = *reinterpret_cast<const Wide *>(x + (whole || at < end ? at : end) * SIZE);
        }
    }
    // -inf past the vocabulary
    __device__ __forceinline__ void unpack(const void *row, int64_t base, int64_t vocab,
                                           float (&v)[N]) const
    {
#pragma unroll
        for (int i = 0; i < N / VEC; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t w = piece[i].w[e];
                if (BF16) {
                    v[i * VEC + 2 * e] = __uint_as_float(w << 16);
                    v[i * VEC + 2 * e + 1] = __uint_as_float(w & 0xFFFF0000u);
                } else {
                    v[i * VEC + e] = __uint_as_float(w);
                }
            }
        if (base + (int64_t)T * N <= vocab) return;
#pragma unroll
        for (int i = 0; i < N / VEC; ++i) {
            const int64_t at = base + place<BF16, N, RUNS, T>(i * VEC);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[i * VEC + e] = at + e < vocab ? v[i * VEC + e] : -kInf;
            if (at >= vocab || at + VEC <= vocab) continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e)       // (of one thread)
                if (at + e < vocab) v[i * VEC + e] = logit(row, BF16, at + e);
        }
    }
};

// Over a workgroup of W waves; lds is used by nothing else between two barriers.
template <int W>
__device__ __forceinline__ float block_max(float x, float (&lds)[W])
{
    x = wave_max(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int w = 1; w < W; ++w) x = fmaxf(x, lds[w]);
    return x;
}
template <int W>
__device__ __forceinline__ double block_sum(double x, double (&lds)[W])
{
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int w = 1; w < W; ++w) x += lds[w];
    return x;
}

// Whether anything asks for the sums of a row: a child that may be accepted.
__device__ __forceinline__ bool has_child(const Verify &a, int o0, int n, int j)
{
    if (!a.parents) return j + 1 < n;
    bool found = false;
    for (int k = j + 1 + (int)(threadIdx.x & 63); k < n && !found; k += 64)
        found = a.parents[o0 + k] == j;
    return __any(found);
}

// Step 1. One workgroup a segment of a row; the target's rows, then the draft's.
template <bool BF16, bool GREEDY>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(Verify a)
{
    constexpr int W = kThreads / 64;
    __shared__ float lds_max[W];
    __shared__ double lds_sum[W];
    const int64_t unit = blockIdx.x / (uint32_t)a.segments;
    const int seg = blockIdx.x % (uint32_t)a.segments;
    const void *row;
    double c = kLog2e * a.inv_temperature;
    if (unit < a.n_rows) {
        row = target_row(a, unit);
        if (!GREEDY) {
            rrq_batch b = {};
            b.offsets = a.offsets;
            b.n_seqs = a.n_seqs;
            b.n_tokens = a.n_rows;
            const int s = find_sequence(b, (int)unit, 1, 0, 0);
            int n;
            const int o0 = rows_of(a, s, n);
            const int j = (int)unit - o0;
            if (j < 0 || j >= n || !has_child(a, o0, n, j)) return;
        }
    } else {
        const int64_t d = unit - a.n_rows;
        const int b = (int)(d / (uint32_t)a.max_accept), j = (int)(d % (uint32_t)a.max_accept);
        int n;
        rows_of(a, b, n);
        if (j + 1 >= n) return;
        row = draft_row(a, b, j);
        c = kLog2e * a.inv_draft_temperature;
    }
    const float ch = (float)c;
    const double cl = c - (double)ch;
    const int64_t end = (int64_t)(seg + 1) * a.segment < a.vocab ? (int64_t)(seg + 1) * a.segment
                                                                 : a.vocab;
    float m = -kInf;
    double sum = 0.0;
    int64_t best = a.vocab;
    Block<BF16, false, kSumLane, kThreads> block;
    int64_t base = (int64_t)seg * a.segment;
    block.load(row, base, a.vocab);
    for (;;) {
        float v[kSumLane];
        block.unpack(row, base, a.vocab, v);
        // the next block is on its way under this one's sums
        const int64_t next = base + kSumBlock;
        if (next < end) block.load(row, next, a.vocab);
        auto largest = [&] {
            float x = v[0] == v[0] ? v[0] : -kInf;
#pragma unroll
            for (int i = 1; i < kSumLane; ++i) x = fmaxf(x, v[i]);
            return x;
        };
        if (GREEDY) {
            // the first place of a thread's largest (blocks ascend)
            const float bm = largest();
            if (bm > m || best == a.vocab) {
#pragma unroll
                for (int i = kSumLane - 1; i >= 0; --i) {
                    const int64_t at = base + place<BF16, kSumLane, false, kThreads>(i);
                    if (v[i] == bm && at < a.vocab) best = at;
                }
                m = bm;
            }
        } else {
            // s = sum w, t = sum w d, w = e^(d / T), d relative to m
            double s;
            float t;
            auto add = [&](auto cut) {
                s = 0.0;
                t = 0.0f;
#pragma unroll
                for (int i = 0; i < kSumLane; i += 8) {
                    float part = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float d = v[i + e] - m, x = __builtin_amdgcn_exp2f(d * ch);
                        part += x;
                        t = __builtin_fmaf(x, cut(d), t);
                    }
                    s += (double)part;
                }
            };
            // m is the largest logit of the wave's first block that has any: later ones
            // need no maximum of their own until a thread's sum says that they do (from
            // its own first block, sums say so often: 113 us where this takes 96). It is
            // -inf in all lanes or in none.
            if (m == -kInf) m = wave_max(largest());
            if (m > -kInf) {
                add([](float d) { return d; });
                const bool far = !(s < kFar);
                // (a logit of -inf makes t no number; so may one that is none)
                if (far || t != t) {
                    if (far) {
                        const float more = fmaxf(m, largest());
                        sum *= exp2_64(((double)m - (double)more) * c);
                        m = more;
                    }
                    add([](float d) { return fmaxf(d, -1e30f); });
                }
                sum += s + kLn2 * cl * (double)t;
            } else {
                // nothing but -inf and what is no number
#pragma unroll
                for (int i = 0; i < kSumLane; ++i) sum += v[i] == v[i] ? 0.0 : (double)v[i];
            }
        }
        if (next >= end) break;
        base = next;
    }
    VerifySum *out = a.sums + unit * a.segments + seg;
    const float most = block_max(m, lds_max);
    if (GREEDY) {
        // the largest logit, and of equal ones the first
        double at = m == most && best < a.vocab ? (double)best : (double)a.vocab;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) at = fmin(at, __shfl_xor(at, d));
        if ((threadIdx.x & 63) == 0) lds_sum[threadIdx.x >> 6] = at;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int w = 1; w < W; ++w) at = fmin(at, lds_sum[w]);
            *out = VerifySum{most, 0, at};
        }
        return;
    }
    if (m < most && m != -kInf) sum *= exp2_64(((double)m - (double)most) * c);
    sum = block_sum(sum, lds_sum);
    if (threadIdx.x == 0) *out = VerifySum{most, 0, sum};
}

// A row's largest logit and sum, from its segments, by kRowLanes neighbouring lanes.
constexpr int kRowLanes = 16;       // (a row of the wave)
__device__ __forceinline__ void row_sum(const Verify &a, int64_t unit, double c, float &m,
                                        double &l)
{
    const VerifySum *s = a.sums + unit * a.segments;
    const int lane = threadIdx.x % kRowLanes;
    constexpr int kMost = kVerifySegments / kRowLanes;
    VerifySum x[kMost];
    m = -kInf;
#pragma unroll
    for (int k = 0; k < kMost; ++k) {
        x[k] = VerifySum{-kInf, 0, 0.0};
        if (lane + k * kRowLanes < a.segments) x[k] = s[lane + k * kRowLanes];
        m = fmaxf(m, x[k].m);
    }
    m = row_max(m);
    l = 0.0;
#pragma unroll
    for (int k = 0; k < kMost; ++k)
        l += x[k].m == -kInf ? x[k].sum
                             : x[k].sum * exp2_64(((double)x[k].m - (double)m) * c);
    l = row_total(l);
}
// A row's first largest logit, by as many lanes; the vocabulary's size for none.
__device__ __forceinline__ int64_t row_best(const Verify &a, int64_t unit)
{
    const VerifySum *s = a.sums + unit * a.segments;
    float m = -kInf;
    double at = (double)a.vocab;
    auto better = [&](float om, double oat) {
        if (oat < (double)a.vocab && (at == (double)a.vocab || om > m || (om == m && oat < at))) {
            m = om;
            at = oat;
        }
    };
    for (int i = threadIdx.x % kRowLanes; i < a.segments; i += kRowLanes) better(s[i].m, s[i].sum);
#pragma unroll
    for (int d = 1; d < kRowLanes; d *= 2) {
        const float om = __shfl_xor(m, d);
        const double oat = __shfl_xor(at, d);
        better(om, oat);
    }
    return (int64_t)at;
}

// Lane i's value in every lane, i the same in all.
__device__ __forceinline__ double lane_value(double x, int i)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)b, i);
    const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(b >> 32), i);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Step 2, by a workgroup of T threads: where the walk of sequence b ends. Of 64 rows at
// a time, kRowLanes lanes a row find the token's probability under its parent; the first
// wave walks. write: whether this workgroup writes what is known then.
template <int T>
__device__ __forceinline__ VerifyChoice decide(const Verify &a, int b, bool write)
{
    struct Row {
        double w, q, l, lq;
        float m, mq;
    };
    __shared__ Row rows[64];
    __shared__ int at_shared, count_shared, rejected_shared, last_shared;
    __shared__ bool spoilt_shared;
    const int t = threadIdx.x, lane = t & 63;
    const bool greedy = a.inv_temperature == 0.0, given = a.draft && !greedy;
    int n;
    const int o0 = rows_of(a, b, n);
    int32_t *path = a.paths + (int64_t)b * (a.max_accept + 1);
    for (int i = t; write && i <= a.max_accept; i += T) path[i] = i == 0 && n > 0 ? 0 : -1;
    const double c = kLog2e * a.inv_temperature, cq = kLog2e * a.inv_draft_temperature;
    int at = 0, count = 0, rejected = -1, last = -1;
    // A row without a distribution accepts nothing, and the weights must not be asked
    // whether it has one: the token that spoils it may be a child's, which they leave out.
    bool spoilt = false;
    double mass = 1.0;
    for (int base = 0; base < n && count < a.max_accept && rejected < 0; base += 64) {
        for (int k = t / kRowLanes; k < 64 && base + k < n; k += T / kRowLanes) {
            const int j = base + k, parent = parent_of(a, o0, j);
            if (parent < 0) continue;
            const int64_t token = a.tokens[o0 + j];
            const bool inside = token >= 0 && token < a.vocab;
            Row r = {};
            if (greedy) {
                r.w = token == row_best(a, o0 + parent) && inside ? 1.0 : 0.0;
            } else {
                const float x = inside ? logit(target_row(a, o0 + parent), a.bf16, token) : -kInf;
                float y = -kInf;
                if (given && j <= a.max_accept) {
                    if (inside) y = logit(draft_row(a, b, j - 1), a.bf16, token);
                    row_sum(a, a.n_rows + (int64_t)b * a.max_accept + j - 1, cq, r.mq, r.lq);
                    r.q = inside ? weight(y, r.mq, cq) / r.lq : 0.0;
                }
                row_sum(a, o0 + parent, c, r.m, r.l);
                r.w = inside ? weight(x, r.m, c) / r.l : 0.0;
            }
            if (t % kRowLanes == 0) rows[k] = r;
        }
        // (the path's first entries are written before the walk's)
        __syncthreads();
        if (t < 64) {
            const int j = base + lane;
            const int parent = j < n ? parent_of(a, o0, j) : -1;
            double w = 0.0, q = 0.0, u = 0.0;
            int64_t token = -1;
            if (parent >= 0) {
                w = rows[lane].w;
                q = rows[lane].q;
                token = a.tokens[o0 + j];
                u = (double)a.uniforms[o0 + j];
            }
            // a token that an earlier sibling has was rejected there: by rows of
            // earlier rounds, and below by those of this one
            for (int k0 = at & ~63; a.parents && k0 < base; k0 += 64) {
                const bool sibling = parent_of(a, o0, k0 + lane) == at;
                const int64_t gone = sibling ? a.tokens[o0 + k0 + lane] : -1;
                for (uint64_t left = __ballot(sibling); left; left &= left - 1)
                    if (token == __shfl(gone, __builtin_ctzll(left)) && parent == at) w = 0.0;
            }
            const double l = parent >= 0 ? rows[lane].l : 1.0;
            const uint64_t none = __ballot(!(l > 0.0 && l < (double)kInf));
            uint64_t tried = __ballot(parent == at);
            while (tried) {
                const int i = __builtin_ctzll(tried);
                spoilt = !greedy && (none >> i & 1);
                const double wi = lane_value(w, i), ui = lane_value(u, i);
                if (given ? ui * lane_value(q, i) < wi : ui * mass < wi) {
                    at = base + i;
                    mass = 1.0;
                    last = -1;
                    ++count;
                    if (write && lane == 0) path[count] = at;
                    if (count == a.max_accept) break;
                    tried = __ballot(parent == at);
                    continue;
                }
                if (given) {
                    rejected = base + i;
                    break;
                }
                mass -= wi;
                if (wi > 0.0) last = base + i;
                tried &= tried - 1;
                if (parent == at && token == __shfl(token, i)) w = 0.0;
            }
            if (lane == 0) {
                at_shared = at;
                count_shared = count;
                rejected_shared = rejected;
                last_shared = last;
                spoilt_shared = spoilt;
            }
        }
        __syncthreads();
        last = last_shared;
        spoilt = spoilt_shared;
        at = at_shared;
        count = count_shared;
        rejected = rejected_shared;
    }
    VerifyChoice choice = {};
    choice.row = n > 0 && !spoilt ? o0 + at : -1;
    choice.first = o0;
    choice.n = n;
    choice.at = at;
    choice.draft = rejected >= 0 ? rejected - 1 : -1;
    // children were all tried and rejected
    choice.removed = !given && count < a.max_accept;
    choice.last = last;
    if (rejected >= 0) {
        const Row &r = rows[rejected & 63];
        choice.m = r.m;
        choice.l = r.l;
        choice.mq = r.mq;
        choice.lq = r.lq;
    }
    int64_t following = -1;
    if (greedy && n > 0) {
        following = row_best(a, choice.row);
        if (following >= a.vocab) following = -1;
    }
    if (write && t == 0) {
        a.counts[b] = count;
        if (greedy || choice.row < 0) a.following[b] = following;
        a.choices[b] = choice;
    }
    return choice;
}

// One workgroup a sequence.
constexpr int kDecideThreads = 64 * kRowLanes;
__global__ __launch_bounds__(kDecideThreads) void verify_decide_kernel(Verify a)
{
    decide<kDecideThreads>(a, blockIdx.x, true);
}


// A thread's logits v of block `seg` of the sequence's row, and with a rejected draft
// the draft's, y. RUNS: as in place(). A token that was taken out is -inf.
template <bool BF16, bool RUNS, int T, int N>
__device__ __forceinline__ void load_logits(const Verify &a, int b, const VerifyChoice &c, int seg,
                                            float (&v)[N], float (&y)[N])
{
    static_assert(T * N == kDrawBlock, "a block");
    const int64_t base = (int64_t)seg * kDrawBlock;
    const void *p = target_row(a, c.row), *q = draft_row(a, b, c.draft < 0 ? 0 : c.draft);
    Block<BF16, RUNS, N, T> x, z;
    x.load(p, base, a.vocab);
    if (c.draft >= 0) z.load(q, base, a.vocab);
    x.unpack(p, base, a.vocab, v);
    if (c.draft >= 0) z.unpack(q, base, a.vocab, y);
    if (!c.removed) return;
    // children of the row: 64 at a time, each wave on its own
    const int lane = threadIdx.x & 63;
    for (int k0 = c.at + 1; k0 < c.n; k0 += 64) {
        const int k = k0 + lane;
        int64_t token = -1;
        if (k < c.n && parent_of(a, c.first, k) == c.at) token = a.tokens[c.first + k];
        uint64_t here = __ballot(token >= base && token < base + kDrawBlock);
        while (here) {
            const int i = __builtin_ctzll(here);
            here &= here - 1;
            const int at = (int)(__shfl(token, i) - base);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (at == place<BF16, N, RUNS, T>(e)) v[e] = -kInf;
        }
        if (!a.parents) break;      // a chain's row has one child, the next
    }
}
// Factors of weight() for the target's logits and the draft's.
__device__ __forceinline__ double weight_factor(double inv_temperature)
{
    return kTable * kLog2e * inv_temperature;
}

// Step 3: one workgroup a block of the vocabulary. DECIDE: each of a sequence's decides
// for itself first, which in few sequences takes no longer than a kernel before this
// one and saves its launch: up to a block a compute unit. The call so, and with a kernel
// before: 4 and 8 sequences of five drafts (128 and 256 blocks) 21.8 and 27.4 us, 23.6 and
// 29.9; of trees of 29 to 48 drafts 29.0 and 34.4, 28.1 and 34.4. Past that bound 16
// sequences 36.5 and 39.5, 16 trees 47.7 and 47.1, 32 chains of 150001 tokens 49.1 and
// 48.2. (Letting the workgroup that ends last go on with step 4
// would save another, but its fences write the L2 caches back: 20 us for 20 with one
// sequence, 225 for 102 with 96.)
template <bool BF16, bool DECIDE>
__global__ __launch_bounds__(kThreads) void verify_weights_kernel(Verify a)
{
    constexpr int W = kThreads / 64;
    __shared__ float lds_max[W];
    __shared__ double lds[4][W], table[kTable];
    const int b = blockIdx.x / (uint32_t)a.draw_segments;
    const int seg = blockIdx.x % (uint32_t)a.draw_segments;
    const VerifyChoice c = DECIDE ? decide<kThreads>(a, b, seg == 0) : a.choices[b];
    if (c.row < 0) return;
    float v[kWeightLane], y[kWeightLane];
    load_logits<BF16, false, kThreads>(a, b, c, seg, v, y);
    fill_table(table);
    float m = c.m;
    if (c.draft < 0) {
        m = -kInf;
#pragma unroll
        for (int i = 0; i < kWeightLane; ++i) m = fmaxf(m, v[i]);
        m = block_max(m, lds_max);
    }
    const float ms = m == -kInf ? 0.0f : m;
    const double f = weight_factor(a.inv_temperature);
    double p = 0.0, q = 0.0, sp = 0.0, sq = 0.0;
    if (c.draft >= 0) {
        const double fq = weight_factor(a.inv_draft_temperature);
#pragma unroll
        for (int i = 0; i < kWeightLane; ++i) {
            const double w = weight(table, v[i], ms, f), x = weight(table, y[i], c.mq, fq);
            p += w;
            q += x;
            if (w * c.lq > x * c.l) {
                sp += w;
                sq += x;
            }
        }
        q = wave_sum(q);
        sp = wave_sum(sp);
        sq = wave_sum(sq);
    } else {
#pragma unroll
        for (int i = 0; i < kWeightLane; ++i) p += weight(table, v[i], ms, f);
    }
    p = wave_sum(p);
    if ((threadIdx.x & 63) == 0) {
        const int w = threadIdx.x >> 6;
        lds[0][w] = p;
        lds[1][w] = q;
        lds[2][w] = sp;
        lds[3][w] = sq;
    }
    __syncthreads();
    if (threadIdx.x > 0) return;
    double all[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        all[i] = lds[i][0];
#pragma unroll
        for (int w = 1; w < W; ++w) all[i] += lds[i][w];
    }
    a.blocks[(int64_t)b * a.draw_segments + seg] =
        VerifyBlock{all[0], all[1], all[2], all[3], m, 0};
}

// Inclusive sum over the workgroup's threads; total: of all.
template <int W>
__device__ __forceinline__ double block_scan(double x, double (&lds)[W], double &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    x = wave_scan(x);
    __syncthreads();
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    double before = 0.0;
    total = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        if (w < wave) before += lds[w];
        total += lds[w];
    }
    return before + x;
}

// The first thread that has `is`, of it `at`, and the last that has `was`, of it `to`;
// `none` and -1 for none. Places ascend with threads.
template <int W>
__device__ __forceinline__ void first_and_last(bool is, int at, bool was, int to, int none,
                                               int (&lds)[2][W], int &first, int &last)
{
    const int wave = threadIdx.x >> 6;
    const uint64_t i = __ballot(is), w = __ballot(was);
    const int f = i ? __shfl(at, __builtin_ctzll(i)) : none;
    const int l = w ? __shfl(to, 63 - __builtin_clzll(w)) : -1;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        lds[0][wave] = f;
        lds[1][wave] = l;
    }
    __syncthreads();
    first = none;
    last = -1;
#pragma unroll
    for (int k = 0; k < W; ++k) {
        first = lds[0][k] < first ? lds[0][k] : first;
        last = lds[1][k] > last ? lds[1][k] : last;
    }
}

// Step 4: one workgroup a sequence.
template <bool BF16>
__global__ __launch_bounds__(kDrawThreads) void verify_draw_kernel(Verify a)
{
    constexpr int W = kDrawThreads / 64;
    __shared__ float lds_max[W];
    __shared__ double lds[W], table[kTable];
    __shared__ int lds_place[2][W];
    __shared__ double before_picked;
    const int b = blockIdx.x, t = threadIdx.x;
    const VerifyChoice c = a.choices[b];
    if (c.row < 0) return;
    const VerifyBlock *blocks = a.blocks + (int64_t)b * a.draw_segments;
    const double f = kLog2e * a.inv_temperature;
    const double u = (double)a.uniforms[c.first];
    // this thread's block of the first round, read once
    VerifyBlock mine = {0.0, 0.0, 0.0, 0.0, -kInf, 0};
    if (t < a.draw_segments) mine = blocks[t];
    fill_table(table);
    auto block = [&](int i) { return i < kDrawThreads ? mine : blocks[i]; };
    float m = mine.m;
    for (int i = t + kDrawThreads; i < a.draw_segments; i += kDrawThreads) m = fmaxf(m, blocks[i].m);
    m = block_max(m, lds_max);
    // a block's weights relative to the row's largest logit
    auto whole = [&](const VerifyBlock &k) {
        return k.m == -kInf ? k.p : k.p * exp2_64(((double)k.m - (double)m) * f);
    };
    double lp = 0.0, lq = 0.0, res = 0.0;
    for (int i = t; i < a.draw_segments; i += kDrawThreads) {
        const VerifyBlock k = block(i);
        lp += whole(k);
        lq += k.q;
    }
    lp = block_sum(lp, lds);
    bool residual = c.draft >= 0;
    if (residual) {
        lq = block_sum(lq, lds);
        for (int i = t; i < a.draw_segments; i += kDrawThreads) {
            const VerifyBlock k = block(i);
            res += fmax(k.sp / lp - k.sq / lq, 0.0);
        }
        res = block_sum(res, lds);
        residual = res > 0.0;           // (else p itself)
    }
    const double total = residual ? res : lp;
    if (!(total > 0.0) || total > 1e300) {
        // Nothing left of a sound row: its children are all that it has. By the formulas
        // the last one that has any probability is accepted then, and only the roundings
        // of step 1's sum can have rejected it: it comes as the next token.
        const bool all = total == 0.0 && c.removed && c.last >= 0;
        if (t == 0) a.following[b] = all ? a.tokens[c.first + c.last] : -1;
        return;
    }
    const double goal = u * total;
    // the first block past which the sum exceeds the goal, the last that has any
    int seg = a.draw_segments, last = -1;
    double before = 0.0;
    for (int i0 = 0; i0 < a.draw_segments && seg == a.draw_segments; i0 += kDrawThreads) {
        const int i = i0 + t;
        double x = 0.0;
        if (i < a.draw_segments) {
            const VerifyBlock k = block(i);
            x = residual ? fmax(k.sp / lp - k.sq / lq, 0.0) : whole(k);
        }
        double sum;
        const double upto = before + block_scan(x, lds, sum);
        int some;
        first_and_last(x > 0.0 && upto > goal, i, x > 0.0, i, a.draw_segments, lds_place, seg,
                       some);
        last = some >= 0 ? some : last;
        if (i == seg) before_picked = upto - x;
        before += sum;
    }
    __syncthreads();
    // a goal past the sum's last digit: the last token that has any weight
    const bool past = seg == a.draw_segments;
    if (past) seg = last;
    if (seg < 0) {
        if (t == 0) a.following[b] = -1;
        return;
    }
    float v[kDrawLane], y[kDrawLane];
    load_logits<BF16, true, kDrawThreads>(a, b, c, seg, v, y);
    const float ms = m == -kInf ? 0.0f : m;
    double w[kDrawLane];
    {
        const double fp = weight_factor(a.inv_temperature);
        const double fq = weight_factor(a.inv_draft_temperature);
#pragma unroll
        for (int i = 0; i < kDrawLane; ++i) {
            w[i] = weight(table, v[i], ms, fp);
            if (residual) {
                const double q = weight(table, y[i], c.mq, fq);
                w[i] = w[i] * c.lq > q * c.l ? fmax(w[i] / lp - q / lq, 0.0) : 0.0;
            }
        }
    }
    double x = 0.0, sum;
#pragma unroll
    for (int i = 0; i < kDrawLane; ++i) x += w[i];
    double upto = (past ? 0.0 : before_picked) + block_scan(x, lds, sum) - x;
    int first = kDrawBlock, end = -1;
#pragma unroll
    for (int i = 0; i < kDrawLane; ++i) {
        upto += w[i];
        if (w[i] > 0.0) {
            end = t * kDrawLane + i;
            if (!past && upto > goal && first == kDrawBlock) first = end;
        }
    }
    int picked, some;
    first_and_last(first < kDrawBlock, first, end >= 0, end, kDrawBlock, lds_place, picked, some);
    if (t == 0) {
        const int at = picked < kDrawBlock ? picked : some;
        a.following[b] = at < 0 ? -1 : (int64_t)seg * kDrawBlock + at;
    }
}

template <bool BF16>
hipError_t launch_type(const Verify &a, hipStream_t stream)
{
    const bool greedy = a.inv_temperature == 0.0;
    const int64_t units = a.n_rows + (a.draft ? a.n_seqs * a.max_accept : 0);
    const unsigned grid = (unsigned)(units * a.segments);
    if (grid > 0) {
        if (greedy)
            verify_sums_kernel<BF16, true><<<grid, kThreads, 0, stream>>>(a);
        else
            verify_sums_kernel<BF16, false><<<grid, kThreads, 0, stream>>>(a);
    }
    const unsigned blocks = (unsigned)(a.n_seqs * a.draw_segments);
    const bool few = !greedy && blocks <= kServeCus;
    if (!few) verify_decide_kernel<<<(unsigned)a.n_seqs, kDecideThreads, 0, stream>>>(a);
    if (!greedy) {
        if (few)
            verify_weights_kernel<BF16, true><<<blocks, kThreads, 0, stream>>>(a);
        else
            verify_weights_kernel<BF16, false><<<blocks, kThreads, 0, stream>>>(a);
        verify_draw_kernel<BF16><<<(unsigned)a.n_seqs, kDrawThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

int64_t verify_segment(int64_t units, int64_t vocab)
{
    const int64_t blocks = (vocab + kSumBlock - 1) / kSumBlock;
    int64_t n = units > 0 ? (16 * kServeCus + units - 1) / units : 1;
    n = n > kVerifySegments ? kVerifySegments : n;
    n = n > blocks ? blocks : n;
    return (blocks + n - 1) / n * kSumBlock;
}

hipError_t launch_verify(const Verify &a, hipStream_t stream)
{
    return a.bf16 ? launch_type<true>(a, stream) : launch_type<false>(a, stream);
}

}  // namespace rrq_detail
