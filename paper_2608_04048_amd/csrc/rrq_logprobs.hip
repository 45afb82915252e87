// Scoring of tokens from logits (rrq_serve.h: rrq_token_logprobs): one pass
// over the logits for the log-sum-exp, the entropy and the largest few.
//
// A workgroup of four waves takes a segment of a row, each wave a contiguous
// part of it in blocks of 64 x 32 logits (32 a lane, in registers). A lane
// keeps its own running maximum m, l = sum exp(x - m) and t = sum exp(x - m)
// (x - m); when a block raises m by d, l and t become f l and f (t + d' l)
// with f = exp(-d), d' = -d. Lanes, waves and segments are joined by the same
// rule, so
//   lse = m + log l,  entropy = log l - t / l.
// The largest few: a logit and its index make a 64-bit key whose order is
// "larger logit first, then lower index". Each wave keeps a buffer of keys
// that beat its n-th best so far; only blocks whose lane maxima beat it are
// looked at again, about n log(N / n) keys of N in random order. A full
// buffer is cut back to its best n by counting, for every key, the larger
// ones.
#include <hip/hip_runtime.h>

#include "rrq_serve_device.h"
#include "rrq_serve_launch.h"

namespace rrq_detail {
namespace {

constexpr float kInf = __builtin_inff();
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kPerLane = 32;
constexpr int kBlock = 64 * kPerLane;
constexpr int kWaves = 4;
constexpr int kBuffer = 128;            // keys a wave buffers
typedef unsigned long long key_t;

// Ascending order of floats as unsigned; NaN first.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x);
    if (x != x) return 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ key_t make_key(uint32_t ord, uint32_t index)
{
    return ((key_t)ord << 32) | (uint32_t)~index;
}

// Running sums of one lane, wave, segment or row.
struct Sums {
    float m, l, t;
};

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

__device__ __forceinline__ Sums join(const Sums &a, const Sums &b)
{
    Sums r;
    r.m = fmaxf(a.m, b.m);
    if (r.m == -kInf) return Sums{-kInf, a.l + b.l, a.t + b.t};     // both empty (or NaN)
    const float da = fmaxf(a.m - r.m, -1e30f), db = fmaxf(b.m - r.m, -1e30f);
    const float fa = exp_of(da), fb = exp_of(db);
    r.l = fa * a.l + fb * b.l;
    r.t = fa * (a.t + da * a.l) + fb * (b.t + db * b.l);
    return r;
}

__device__ __forceinline__ Sums wave_join(Sums s)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const Sums o = {__shfl_xor(s.m, d), __shfl_xor(s.l, d), __shfl_xor(s.t, d)};
        s = join(s, o);
    }
    return s;
}

// Orders the wave's own LDS accesses (they complete in order; this keeps the
// compiler from moving them).
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A wave's key buffer in LDS; count and floor are the same in every lane.
// floor is a key that n others reach or beat: only larger keys can matter.
struct Top {
    key_t *buf;
    int n, count;
    key_t floor;

    // Cuts the buffer to its n best, in order. Keys are distinct.
    __device__ void cut()
    {
        const int lane = threadIdx.x & 63;
        wave_sync();
        const key_t a = lane < count ? buf[lane] : 0;
        const key_t b = lane + 64 < count ? buf[lane + 64] : 0;
        int ra = 0, rb = 0;
        for (int i = 0; i < count; ++i) {
            const key_t o = buf[i];
            ra += o > a;
            rb += o > b;
        }
        wave_sync();
        if (lane < count && ra < n) buf[ra] = a;
        if (lane + 64 < count && rb < n) buf[rb] = b;
        wave_sync();
        if (count >= n) {
            count = n;
            floor = buf[n - 1];
        }
    }

    // Adds the lanes' keys that beat the floor (every lane calls it).
    __device__ void add(bool has, key_t k)
    {
        const uint64_t who = __ballot(has && k > floor);
        if (!who) return;
        if (count > kBuffer - 64) cut();
        // the cut may have raised the floor: some keys stay without need
        const int lane = threadIdx.x & 63;
        const int at = count + __popcll(who & ((1ull << lane) - 1));
        if ((who >> lane) & 1) buf[at] = k;
        count += __popcll(who);
    }
};

// The n-th largest of the lanes' values (n <= 64).
__device__ __forceinline__ uint32_t nth_largest(uint32_t v, int n)
{
    uint32_t r = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t c = r | (1u << bit);
        if (__popcll(__ballot(v >= c)) >= n) r = c;
    }
    return r;
}

template <bool BF16>
__device__ __forceinline__ float load_logit(const void *row, int64_t i)
{
    if (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(row)[i] << 16);
    return static_cast<const float *>(row)[i];
}

// Results of a segment, in the workspace: n_top keys (0: none), then m, l, t.
__device__ __forceinline__ key_t *segment_keys(const Logprobs &a, int64_t row, int seg)
{
    char *base = static_cast<char *>(a.workspace) +
                 (row * a.segments + seg) * (8 * (int64_t)a.n_top + 16);
    return reinterpret_cast<key_t *>(base);
}

// The row's results, from its joined sums and its sorted keys (one wave).
template <bool BF16>
__device__ __forceinline__ void write_row(const Logprobs &a, int64_t row, const Sums &s,
                                          const key_t *keys)
{
    const int lane = threadIdx.x & 63;
    const void *x = static_cast<const char *>(a.logits) + row * a.row_stride * (BF16 ? 2 : 4);
    // a row of -inf only: l and t are 0 (or NaN, if it holds one)
    const bool empty = s.m == -kInf;
    const float log_l = empty ? s.l : logf(s.l);
    if (lane == 0) {
        if (a.entropy) a.entropy[row] = empty ? s.l : log_l - s.t / s.l;
        if (a.targets) {
            const int64_t t = a.targets[row];
            float r = 0.0f;
            if (t >= 0 && t < a.vocab)
                r = (empty ? load_logit<BF16>(x, t) : load_logit<BF16>(x, t) - s.m) - log_l;
            a.logprobs[row] = r;
        }
    }
    if (lane < a.n_top) {       // n_top <= vocab: every key is a logit's
        const uint32_t i = ~(uint32_t)keys[lane];
        const float v = load_logit<BF16>(x, i);
        a.top_ids[row * a.n_top + lane] = i;
        a.top_logprobs[row * a.n_top + lane] = (empty ? v : v - s.m) - log_l;
    }
}

template <bool BF16>
__global__ __launch_bounds__(64 * kWaves) void logprobs_kernel(Logprobs a)
{
    __shared__ key_t lds_keys[kWaves][kBuffer];
    __shared__ float lds_sums[kWaves][3];
    constexpr int VEC = BF16 ? 8 : 4;           // logits a load
    constexpr int NV = kPerLane / VEC;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x / a.segments;
    const int seg = blockIdx.x % a.segments;
    const char *x = static_cast<const char *>(a.logits) + row * a.row_stride * (BF16 ? 2 : 4);
    // parts of whole blocks, one a wave
    const int64_t parts = (int64_t)a.segments * kWaves;
    const int64_t blocks = (a.vocab + kBlock - 1) / kBlock;
    const int64_t p = (int64_t)seg * kWaves + wave;
    const int64_t b0 = blocks * p / parts, b1 = blocks * (p + 1) / parts;

    Sums s = {-kInf, 0.0f, 0.0f};
    Top top = {lds_keys[wave], a.n_top, 0, 0};
    for (int64_t b = b0; b < b1; ++b) {
        const int64_t base = b * kBlock;
        float v[kPerLane];
        if (base + kBlock <= a.vocab) {
            // rows may start at any multiple of their type: 16-byte loads
            // without that alignment
            struct __attribute__((packed, aligned(2))) Wide { uint32_t w[4]; };
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const Wide w = *reinterpret_cast<const Wide *>(
                    x + (base + (i * 64 + lane) * VEC) * (BF16 ? 2 : 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (BF16) {
                        v[i * VEC + 2 * e] = __uint_as_float(w.w[e] << 16);
                        v[i * VEC + 2 * e + 1] = __uint_as_float(w.w[e] & 0xFFFF0000u);
                    } else {
                        v[i * VEC + e] = __uint_as_float(w.w[e]);
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) {
                const int64_t at = base + ((i / VEC) * 64 + lane) * VEC + i % VEC;
                v[i] = at < a.vocab ? load_logit<BF16>(x, at) : -kInf;
            }
        }
        float bm = -kInf;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) bm = fmaxf(bm, v[i]);
        const float mn = fmaxf(s.m, bm);
        const float ms = mn == -kInf ? 0.0f : mn;
        const float d = fmaxf(s.m - ms, -1e30f), f = exp_of(d);
        float l = 0.0f, t = 0.0f;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            // a logit of -inf: exp is 0 and the finite difference keeps 0 out
            // of 0 times infinity
            const float di = v[i] - ms, e = exp_of(di);
            l += e;
            t += e * fmaxf(di, -1e30f);
        }
        s.t = f * (s.t + d * s.l) + t;
        s.l = f * s.l + l;
        s.m = mn;
        if (a.n_top == 0) continue;
        // a later block has higher indices: an equal logit does not matter
        const uint32_t bo = ordered(bm);
        if (top.floor != 0 && !__any(bo > (uint32_t)(top.floor >> 32))) continue;
        if (top.floor == 0 && top.count == 0) {
            // The wave's first block: the n-th largest lane maximum is a
            // floor that at least n logits reach. Lanes without a logit
            // count as 0.
            uint32_t lm = 0;
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) {
                const int64_t at = base + ((i / VEC) * 64 + lane) * VEC + i % VEC;
                const uint32_t o = at < a.vocab ? ordered(v[i]) : 0;
                lm = o > lm ? o : lm;
            }
            const uint32_t nth = nth_largest(lm, a.n_top);
            if (nth > 0) top.floor = ((key_t)nth << 32) - 1;
        }
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            const int64_t at = base + ((i / VEC) * 64 + lane) * VEC + i % VEC;
            top.add(at < a.vocab, make_key(ordered(v[i]), (uint32_t)at));
        }
        top.cut();
    }
    s = wave_join(s);
    if (lane == 0) {
        lds_sums[wave][0] = s.m;
        lds_sums[wave][1] = s.l;
        lds_sums[wave][2] = s.t;
    }
    // unused places of the first n hold no key
    if (lane >= top.count && lane < a.n_top) top.buf[lane] = 0;
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < kWaves; ++w)
        s = join(s, Sums{lds_sums[w][0], lds_sums[w][1], lds_sums[w][2]});
    if (a.n_top > 0) {
        for (int w = 1; w < kWaves; ++w) {
            const key_t k = lane < a.n_top ? lds_keys[w][lane] : 0;
            top.add(k != 0, k);
        }
        top.cut();
    }
    if (a.segments == 1) {
        write_row<BF16>(a, row, s, top.buf);
        return;
    }
    key_t *out = segment_keys(a, row, seg);
    if (lane < a.n_top) out[lane] = lane < top.count ? top.buf[lane] : 0;
    float *sums = reinterpret_cast<float *>(out + a.n_top);
    if (lane == 0) {
        sums[0] = s.m;
        sums[1] = s.l;
        sums[2] = s.t;
    }
}

// Joins a row's segments: one wave a row.
template <bool BF16>
__global__ __launch_bounds__(64) void logprobs_join_kernel(Logprobs a)
{
    __shared__ key_t lds_keys[kBuffer];
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    Sums s = {-kInf, 0.0f, 0.0f};
    for (int seg = lane; seg < a.segments; seg += 64) {
        const float *sums = reinterpret_cast<const float *>(segment_keys(a, row, seg) + a.n_top);
        s = join(s, Sums{sums[0], sums[1], sums[2]});
    }
    s = wave_join(s);
    Top top = {lds_keys, a.n_top, 0, 0};
    if (a.n_top > 0) {
        const int total = a.segments * a.n_top;
        for (int i0 = 0; i0 < total; i0 += 64) {
            const int i = i0 + lane;
            key_t k = 0;
            if (i < total) k = segment_keys(a, row, i / a.n_top)[i % a.n_top];
            top.add(k != 0, k);
        }
        top.cut();
    }
    write_row<BF16>(a, row, s, lds_keys);
}

}  // namespace

int logprobs_segments(int64_t n_rows, int64_t vocab)
{
    // four workgroups a compute unit, each wave at least one block
    const int64_t most = (vocab + kBlock * kWaves - 1) / (kBlock * kWaves);
    int64_t n = (kServeCus * 4 + n_rows - 1) / n_rows;
    n = n > most ? most : n;
    return n < 1 ? 1 : (int)n;
}

size_t logprobs_row_bytes(int segments, int n_top)
{
    return segments == 1 ? 0 : (size_t)segments * (8 * (size_t)n_top + 16);
}

hipError_t launch_logprobs(const Logprobs &a, bool bf16, hipStream_t stream)
{
    const unsigned grid = (unsigned)(a.n_rows * a.segments);
    if (bf16)
        logprobs_kernel<true><<<grid, 64 * kWaves, 0, stream>>>(a);
    else
        logprobs_kernel<false><<<grid, 64 * kWaves, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.segments == 1) return e;
    if (bf16)
        logprobs_join_kernel<true><<<(unsigned)a.n_rows, 64, 0, stream>>>(a);
    else
        logprobs_join_kernel<false><<<(unsigned)a.n_rows, 64, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace rrq_detail
