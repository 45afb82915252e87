// Verification of drafted tokens against the target's distributions
// (rrq_draft.h: rrq_verify_drafts).
//
// A row's probabilities are e^(x / T) / l, l the sum over the vocabulary. Four steps:
//   1. sums: l of every row that has children (only those are asked whether to accept
//      one), and of the draft's rows: segments of a row, each with its largest logit m
//      and its sum relative to that;
//   2. decide: one wave a sequence walks down from the root. Rows are 64 at a time in
//      the lanes; a lane has its token's probability under its parent, the walk itself
//      is a ballot and a broadcast a tried token;
//   3. weights: of the one row a sequence ends at, sums of what the next token is drawn
//      from, a segment a workgroup, in 64 bits;
//   4. draw: the segment in which the running sum passes the random number's share, and
//      the token in it.
// Greedy calls (T = 0) end with step 2, on each row's first largest logit.
//
// Precision. Whether u q < p or a running sum passes u times the total is a border
// that any input may come near, and the results are whole numbers. Step 1 has
// binary32 exponentials (each off by 2^-24 or so at random) and corrects what is
// systematic, the rounding of log2(e) / T, by the sum of e d; sums of more than eight
// are 64 bits: l is good to about 2^-24, and a decision off in one of some 10^7 cases.
// Running sums of a vocabulary pass borders that lie 10^-5 apart: steps 3 and 4 are 64
// bits throughout, exponentials (Taylor's series) good to 10^-14. The residual
// (p - q)+ needs both rows' sums before it can be formed; step 3 leaves the sums of p and
// of q over the tokens where p > q (by step 1's sums; a token whose sign these get wrong
// adds nothing) for step 4 to scale and subtract.
#include <hip/hip_runtime.h>

#include "rrq_draft_launch.h"
#include "rrq_serve_device.h"

namespace rrq_detail {
namespace {

constexpr float kInf = __builtin_inff();
constexpr double kLn2 = 0.69314718055994530942, kLog2e = 1.44269504088896340736;
constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kSumLane = 32, kSumBlock = kThreads * kSumLane;       // logits of step 1
constexpr int kDrawLane = 16, kDrawBlock = kThreads * kDrawLane;    // of steps 3 and 4
static_assert(kSumBlock == kVerifySumBlock && kDrawBlock == kVerifyDrawBlock, "workspace");

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

// A thread's N logits of the block from `base` on, VEC (16 bytes) in a row each:
// logit (i * kThreads + thread) * VEC + e of the block is v[i * VEC + e]. -inf past the
// vocabulary. Rows may start at any multiple of their type.
template <bool BF16, int N>
__device__ __forceinline__ void load_block(const void *row, int64_t base, int64_t vocab,
                                           float (&v)[N])
{
    constexpr int VEC = BF16 ? 8 : 4, SIZE = BF16 ? 2 : 4;
    struct __attribute__((packed, aligned(2))) Wide { uint32_t w[4]; };
    const char *x = static_cast<const char *>(row);
    const bool whole = base + (int64_t)kThreads * N <= vocab;
#pragma unroll
    for (int i = 0; i < N / VEC; ++i) {
        const int64_t at = base + (int64_t)(i * kThreads + (int)threadIdx.x) * VEC;
        if (whole || at + VEC <= vocab) {
            const Wide w = *reinterpret_cast<const Wide *>(x + at * SIZE);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (BF16) {
                    v[i * VEC + 2 * e] = __uint_as_float(w.w[e] << 16);
                    v[i * VEC + 2 * e + 1] = __uint_as_float(w.w[e] & 0xFFFF0000u);
                } else {
                    v[i * VEC + e] = __uint_as_float(w.w[e]);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                v[i * VEC + e] = at + e < vocab ? logit(row, BF16, at + e) : -kInf;
        }
    }
}

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}
__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}
// Over the workgroup; lds: kWaves places, used by nothing else between two barriers.
__device__ __forceinline__ float block_max(float x, float *lds)
{
    x = wave_max(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) x = fmaxf(x, lds[w]);
    return x;
}
__device__ __forceinline__ double block_sum(double x, double *lds)
{
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) x += lds[w];
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
    __shared__ float lds_max[kWaves];
    __shared__ double lds_sum[kWaves];
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
    for (int64_t base = (int64_t)seg * a.segment; base < end; base += kSumBlock) {
        float v[kSumLane];
        load_block<BF16>(row, base, a.vocab, v);
        float bm = -kInf;
#pragma unroll
        for (int i = 0; i < kSumLane; ++i) bm = fmaxf(bm, v[i]);
        if (GREEDY) {
            // the first place of a thread's largest (blocks ascend)
            constexpr int VEC = BF16 ? 8 : 4;
            if (bm > m || best == a.vocab) {
#pragma unroll
                for (int i = kSumLane - 1; i >= 0; --i) {
                    const int64_t at = base + (int64_t)((i / VEC) * kThreads + (int)threadIdx.x) *
                                                  VEC + i % VEC;
                    if (v[i] == bm && at < a.vocab) best = at;
                }
                m = bm;
            }
            continue;
        }
        const float mn = fmaxf(m, block_max(bm, lds_max));
        const float ms = mn == -kInf ? 0.0f : mn;
        if (mn > m) sum *= m == -kInf ? 0.0 : exp2_64(((double)m - (double)mn) * c);
        m = mn;
        float t = 0.0f;
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < kSumLane; i += 8) {
            float part = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = v[i + e] - ms, w = __builtin_amdgcn_exp2f(d * ch);
                part += w;
                // (-inf times 0 is kept out)
                t = __builtin_fmaf(w, fmaxf(d, -1e30f), t);
            }
            s += (double)part;
        }
        sum += s + kLn2 * cl * (double)t;
    }
    VerifySum *out = a.sums + unit * a.segments + seg;
    if (GREEDY) {
        // the largest logit, and of equal ones the first
        const float most = block_max(m, lds_max);
        double at = m == most && best < a.vocab ? (double)best : (double)a.vocab;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) at = fmin(at, __shfl_xor(at, d));
        if ((threadIdx.x & 63) == 0) lds_sum[threadIdx.x >> 6] = at;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int w = 1; w < kWaves; ++w) at = fmin(at, lds_sum[w]);
            *out = VerifySum{most, 0, at};
        }
        return;
    }
    sum = block_sum(sum, lds_sum);
    if (threadIdx.x == 0) *out = VerifySum{m, 0, sum};
}

// A row's largest logit and sum, from its segments (one thread).
__device__ __forceinline__ void row_sum(const Verify &a, int64_t unit, double c, float &m,
                                        double &l)
{
    const VerifySum *s = a.sums + unit * a.segments;
    m = -kInf;
    for (int i = 0; i < a.segments; ++i) m = fmaxf(m, s[i].m);
    l = 0.0;
    for (int i = 0; i < a.segments; ++i)
        l += s[i].m == -kInf ? s[i].sum : s[i].sum * exp2_64(((double)s[i].m - (double)m) * c);
}
// A row's first largest logit (one thread); the vocabulary's size for none.
__device__ __forceinline__ int64_t row_best(const Verify &a, int64_t unit)
{
    const VerifySum *s = a.sums + unit * a.segments;
    float m = -kInf;
    double at = (double)a.vocab;
    for (int i = 0; i < a.segments; ++i)
        if (s[i].sum < (double)a.vocab && (s[i].m > m || at == (double)a.vocab)) {
            m = s[i].m;
            at = s[i].sum;
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

// Step 2: one wave a sequence.
__global__ __launch_bounds__(64) void verify_decide_kernel(Verify a)
{
    const int b = blockIdx.x, lane = threadIdx.x;
    const bool greedy = a.inv_temperature == 0.0;
    int n;
    const int o0 = rows_of(a, b, n);
    int32_t *path = a.paths + (int64_t)b * (a.max_accept + 1);
    for (int i = lane; i <= a.max_accept; i += 64) path[i] = i == 0 && n > 0 ? 0 : -1;
    const double c = kLog2e * a.inv_temperature, cq = kLog2e * a.inv_draft_temperature;
    int at = 0, count = 0, rejected = -1;
    double mass = 1.0;
    for (int base = 0; base < n && count < a.max_accept; base += 64) {
        // this lane's row: its token's probability w under its parent, and q
        const int j = base + lane;
        const int parent = j < n ? parent_of(a, o0, j) : -1;
        double w = 0.0, q = 1.0, u = 0.0;
        int64_t token = -1;
        if (parent >= 0) {
            token = a.tokens[o0 + j];
            u = (double)a.uniforms[o0 + j];
            const bool inside = token >= 0 && token < a.vocab;
            if (greedy) {
                w = inside && token == row_best(a, o0 + parent) ? 1.0 : 0.0;
            } else {
                const float x = inside ? logit(target_row(a, o0 + parent), a.bf16, token) : -kInf;
                float m;
                double l;
                row_sum(a, o0 + parent, c, m, l);
                w = weight(x, m, c) / l;
                if (a.draft) {
                    q = 0.0;
                    if (j <= a.max_accept) {
                        const float y = inside ? logit(draft_row(a, b, j - 1), a.bf16, token)
                                               : -kInf;
                        row_sum(a, a.n_rows + (int64_t)b * a.max_accept + j - 1, cq, m, l);
                        q = weight(y, m, cq) / l;
                    }
                }
                if (!inside) w = 0.0;
            }
        }
        // a token that an earlier sibling has was rejected there: by rows of earlier
        // rounds, and below by those of this one
        for (int k0 = at & ~63; a.parents && k0 < base; k0 += 64) {
            const bool sibling = parent_of(a, o0, k0 + lane) == at;
            const int64_t gone = sibling ? a.tokens[o0 + k0 + lane] : -1;
            for (uint64_t left = __ballot(sibling); left; left &= left - 1)
                if (token == __shfl(gone, __builtin_ctzll(left)) && parent == at) w = 0.0;
        }
        uint64_t tried = __ballot(parent == at);
        while (tried) {
            const int i = __builtin_ctzll(tried);
            const double wi = lane_value(w, i), ui = lane_value(u, i);
            const bool accept = a.draft && !greedy ? ui * lane_value(q, i) < wi : ui * mass < wi;
            if (accept) {
                at = base + i;
                mass = 1.0;
                ++count;
                if (lane == 0) path[count] = at;
                if (count == a.max_accept) break;
                tried = __ballot(parent == at);
                continue;
            }
            if (a.draft && !greedy) {
                rejected = base + i;
                break;
            }
            mass -= wi;
            tried &= tried - 1;
            if (parent == at && token == __shfl(token, i)) w = 0.0;
        }
        if (rejected >= 0) break;
    }
    VerifyChoice choice = {};
    choice.row = n > 0 ? o0 + at : -1;
    choice.first = o0;
    choice.n = n;
    choice.at = at;
    choice.draft = rejected >= 0 ? rejected - 1 : -1;
    // children were all tried and rejected
    choice.removed = !a.draft && count < a.max_accept;
    if (lane == 0) {
        a.counts[b] = count;
        if (greedy || n == 0) {
            const int64_t t = n > 0 ? row_best(a, choice.row) : a.vocab;
            a.following[b] = t < a.vocab ? t : -1;
        }
        if (rejected >= 0) {
            float m;
            double l;
            row_sum(a, choice.row, c, m, l);
            choice.m = m;
            choice.l = l;
            row_sum(a, a.n_rows + (int64_t)b * a.max_accept + choice.draft, cq, m, l);
            choice.mq = m;
            choice.lq = l;
        }
        a.choices[b] = choice;
    }
}

// Weights of a thread's logits of block `seg` of the sequence's row: w[i], of v[i] less m.
// With a rejected draft also q's.
struct Weights {
    double w[kDrawLane], q[kDrawLane];
    float m;
};
template <bool BF16>
__device__ __forceinline__ void load_weights(const Verify &a, int b, const VerifyChoice &c, int seg,
                                             float ref, bool given, float *lds, Weights &r)
{
    constexpr int VEC = BF16 ? 8 : 4;
    const int64_t base = (int64_t)seg * kDrawBlock;
    float v[kDrawLane], y[kDrawLane];
    load_block<BF16>(target_row(a, c.row), base, a.vocab, v);
    if (c.draft >= 0) load_block<BF16>(draft_row(a, b, c.draft), base, a.vocab, y);
    r.m = ref;
    if (!given) {
        float bm = -kInf;
#pragma unroll
        for (int i = 0; i < kDrawLane; ++i) bm = fmaxf(bm, v[i]);
        r.m = block_max(bm, lds);
    }
    const float ms = r.m == -kInf ? 0.0f : r.m;
    const double f = kLog2e * a.inv_temperature;
#pragma unroll
    for (int i = 0; i < kDrawLane; ++i) r.w[i] = weight(v[i], ms, f);
    if (c.draft >= 0) {
        const double fq = kLog2e * a.inv_draft_temperature;
#pragma unroll
        for (int i = 0; i < kDrawLane; ++i) r.q[i] = weight(y[i], c.mq, fq);
    }
    if (c.removed) {
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
                for (int e = 0; e < kDrawLane; ++e)
                    if (at == ((e / VEC) * kThreads + (int)threadIdx.x) * VEC + e % VEC)
                        r.w[e] = 0.0;
            }
            if (!a.parents) break;      // a chain's row has one child, the next
        }
    }
}

// Step 3: one workgroup a block of the vocabulary.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void verify_weights_kernel(Verify a)
{
    __shared__ float lds_max[kWaves];
    __shared__ double lds[kWaves];
    const int b = blockIdx.x / (uint32_t)a.draw_segments;
    const int seg = blockIdx.x % (uint32_t)a.draw_segments;
    const VerifyChoice c = a.choices[b];
    if (c.row < 0) return;
    Weights r;
    load_weights<BF16>(a, b, c, seg, c.m, c.draft >= 0, lds_max, r);
    double p = 0.0, q = 0.0, sp = 0.0, sq = 0.0;
#pragma unroll
    for (int i = 0; i < kDrawLane; ++i) p += r.w[i];
    if (c.draft >= 0) {
#pragma unroll
        for (int i = 0; i < kDrawLane; ++i) {
            q += r.q[i];
            if (r.w[i] * c.lq > r.q[i] * c.l) {
                sp += r.w[i];
                sq += r.q[i];
            }
        }
        q = block_sum(q, lds);
        sp = block_sum(sp, lds);
        sq = block_sum(sq, lds);
    }
    p = block_sum(p, lds);
    if (threadIdx.x == 0)
        a.blocks[(int64_t)b * a.draw_segments + seg] = VerifyBlock{p, q, sp, sq, r.m, 0};
}

// Inclusive sum over the workgroup's threads; total: of all.
__device__ __forceinline__ double block_scan(double x, double *lds, double &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    double before = 0.0;
    total = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += lds[w];
        total += lds[w];
    }
    return before + x;
}

// Step 4: one workgroup a sequence.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void verify_draw_kernel(Verify a)
{
    __shared__ float lds_max[kWaves];
    __shared__ double lds[kWaves];
    __shared__ int picked, last;
    __shared__ double before_picked;
    const int b = blockIdx.x, t = threadIdx.x;
    const VerifyChoice c = a.choices[b];
    if (c.row < 0) return;
    const VerifyBlock *blocks = a.blocks + (int64_t)b * a.draw_segments;
    const double f = kLog2e * a.inv_temperature;
    float m = -kInf;
    for (int i = t; i < a.draw_segments; i += kThreads) m = fmaxf(m, blocks[i].m);
    m = block_max(m, lds_max);
    // a block's weights relative to the row's largest logit
    auto whole = [&](const VerifyBlock &k) {
        return k.m == -kInf ? k.p : k.p * exp2_64(((double)k.m - (double)m) * f);
    };
    double lp = 0.0, lq = 0.0, res = 0.0;
    for (int i = t; i < a.draw_segments; i += kThreads) {
        lp += whole(blocks[i]);
        lq += blocks[i].q;
    }
    lp = block_sum(lp, lds);
    bool residual = c.draft >= 0;
    if (residual) {
        lq = block_sum(lq, lds);
        for (int i = t; i < a.draw_segments; i += kThreads)
            res += fmax(blocks[i].sp / lp - blocks[i].sq / lq, 0.0);
        res = block_sum(res, lds);
        residual = res > 0.0;           // (else p itself)
    }
    auto of_block = [&](const VerifyBlock &k) {
        return residual ? fmax(k.sp / lp - k.sq / lq, 0.0) : whole(k);
    };
    const double total = residual ? res : lp;
    if (t == 0) {
        picked = a.draw_segments;
        last = -1;
    }
    __syncthreads();
    if (!(total > 0.0) || total > 1e300) {
        if (t == 0) a.following[b] = -1;
        return;
    }
    const double goal = (double)a.uniforms[c.first] * total;
    // the first block past which the sum exceeds the goal, the last that has any
    double before = 0.0;
    for (int i0 = 0; i0 < a.draw_segments; i0 += kThreads) {
        const int i = i0 + t;
        const double x = i < a.draw_segments ? of_block(blocks[i]) : 0.0;
        double sum;
        const double upto = before + block_scan(x, lds, sum);
        if (x > 0.0) {
            atomicMax(&last, i);
            if (upto > goal) atomicMin(&picked, i);
        }
        __syncthreads();
        if (picked < a.draw_segments) {
            if (i == picked) before_picked = upto - x;
            break;
        }
        before += sum;
    }
    __syncthreads();
    // a goal past the sum's last digit: the last token that has any weight
    const bool past = picked >= a.draw_segments;
    const int seg = past ? last : picked;
    if (seg < 0) {
        if (t == 0) a.following[b] = -1;
        return;
    }
    const double start = past ? 0.0 : before_picked;
    Weights r;
    load_weights<BF16>(a, b, c, seg, m, true, lds_max, r);
    if (residual) {
#pragma unroll
        for (int i = 0; i < kDrawLane; ++i)
            r.w[i] = r.w[i] * c.lq > r.q[i] * c.l ? fmax(r.w[i] / lp - r.q[i] / lq, 0.0) : 0.0;
    }
    // pieces of VEC logits a thread, in the order of the vocabulary
    constexpr int VEC = BF16 ? 8 : 4;
    __syncthreads();
    if (t == 0) {
        picked = kDrawBlock;
        last = -1;
    }
    __syncthreads();
    before = start;
#pragma unroll
    for (int i = 0; i < kDrawLane / VEC; ++i) {
        double x = 0.0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) x += r.w[i * VEC + e];
        double sum;
        double upto = before + block_scan(x, lds, sum) - x;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const double w = r.w[i * VEC + e];
            const int at = (i * kThreads + t) * VEC + e;
            upto += w;
            if (w > 0.0) {
                atomicMax(&last, at);
                if (!past && upto > goal) atomicMin(&picked, at);
            }
        }
        before += sum;
    }
    __syncthreads();
    if (t == 0) {
        const int at = picked < kDrawBlock ? picked : last;
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
    verify_decide_kernel<<<(unsigned)a.n_seqs, 64, 0, stream>>>(a);
    if (!greedy) {
        verify_weights_kernel<BF16>
            <<<(unsigned)(a.n_seqs * a.draw_segments), kThreads, 0, stream>>>(a);
        verify_draw_kernel<BF16><<<(unsigned)a.n_seqs, kThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_verify(const Verify &a, hipStream_t stream)
{
    return a.bf16 ? launch_type<true>(a, stream) : launch_type<false>(a, stream);
}

}  // namespace rrq_detail
