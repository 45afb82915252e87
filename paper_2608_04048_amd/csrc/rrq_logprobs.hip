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
//
// Long calls are bound by reading the logits: 2000 rows of 131072 in binary32,
// 1.05 GB in 200 us (5.2 TB/s; a kernel that only reads makes 5.3). 96 rows of
// 150001 in bfloat16 with 20 alternatives: 20 us and 6 of the join where the bytes
// need 6; every wave has two blocks, so the selection's start is most of its 27
// vector instructions a logit. One row of 131072: 8 + 4 us of latency.
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
constexpr int kSlots = kBuffer + 8;     // and what a cut pads them with
typedef unsigned long long key_t;

// Ascending order of floats as unsigned; NaN first. The two zeros are equal:
// -0 + 0 is +0, and the sum is every other number itself.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    if (x != x) return 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// The logit of an ordered() value (0: of no number).
__device__ __forceinline__ float logit_of(uint32_t o)
{
    return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
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
        if (lane < 8) buf[count + lane] = 0;        // to whole groups of 8
        wave_sync();
        const key_t a = lane < count ? buf[lane] : 0;
        int ra = 0;
        if (count <= 64) {
            for (int i = 0; i < count; i += 8) {
                key_t o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = buf[i + e];
#pragma unroll
                for (int e = 0; e < 8; ++e) ra += o[e] > a;
            }
            wave_sync();
        } else {
            const key_t b = lane + 64 < count ? buf[lane + 64] : 0;
            int rb = 0;
            for (int i = 0; i < count; i += 8) {
                key_t o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = buf[i + e];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ra += o[e] > a;
                    rb += o[e] > b;
                }
            }
            wave_sync();
            if (lane + 64 < count && rb < n) buf[rb] = b;
        }
        if (lane < count && ra < n) buf[ra] = a;
        wave_sync();
        if (count >= n) {
            count = n;
            floor = buf[n - 1];
        }
    }

    // A value below this cannot beat the floor (no number if anything can:
    // nothing is below that).
    __device__ float floor_value() const
    {
        return logit_of((uint32_t)(floor >> 32));
    }

    // Adds the keys of the lanes that have one (every lane calls it); there is
    // room.
    __device__ void add(bool has, key_t k)
    {
        const uint64_t who = __ballot(has);
        const int lane = threadIdx.x & 63;
        const int at = count + __popcll(who & ((1ull << lane) - 1));
        if ((who >> lane) & 1) buf[at] = k;
        count += __popcll(who);
    }
    // Raises the floor to just below the largest of the lanes' keys, each the
    // n-th best of some list (0: of a shorter list).
    __device__ void raise(key_t nth)
    {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const key_t o = __shfl_xor(nth, d);
            nth = o > nth ? o : nth;
        }
        if (nth > floor + 1) floor = nth - 1;
    }
    __device__ void add_or_cut(bool has, key_t k)
    {
        if (count > kBuffer - 64) cut();
        add(has && k > floor, k);
    }
};

// A value that n lanes reach (n <= 64): the n-th largest in its upper 16 bits.
__device__ __forceinline__ uint32_t nth_largest(uint32_t v, int n)
{
    uint32_t r = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
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

// The row's target logit (lane 0; loaded before it is needed). inside: the
// target is a token.
template <bool BF16>
__device__ __forceinline__ float target_logit(const Logprobs &a, int64_t row, bool &inside)
{
    inside = false;
    if ((threadIdx.x & 63) != 0 || !a.targets) return 0.0f;
    const int64_t t = a.targets[row];
    inside = t >= 0 && t < a.vocab;
    const void *x = static_cast<const char *>(a.logits) + row * a.row_stride * (BF16 ? 2 : 4);
    return inside ? load_logit<BF16>(x, t) : 0.0f;
}

// The row's results, from its joined sums and its sorted keys (one wave).
__device__ __forceinline__ void write_row(const Logprobs &a, int64_t row, const Sums &s,
                                          const key_t *keys, float target, bool inside)
{
    const int lane = threadIdx.x & 63;
    // a row of -inf only: l and t are 0 (or NaN, if it holds one)
    const bool empty = s.m == -kInf;
    const float log_l = empty ? s.l : logf(s.l);
    if (lane == 0) {
        if (a.entropy) a.entropy[row] = empty ? s.l : log_l - s.t / s.l;
        if (a.targets)
            a.logprobs[row] = inside ? (empty ? target : target - s.m) - log_l : 0.0f;
    }
    if (lane < a.n_top) {       // n_top <= vocab: every key is a logit's
        const key_t k = keys[lane];
        const float v = logit_of((uint32_t)(k >> 32));
        a.top_ids[row * a.n_top + lane] = (uint32_t)~(uint32_t)k;
        a.top_logprobs[row * a.n_top + lane] = (empty ? v : v - s.m) - log_l;
    }
}

// W: waves; kWaves, or one for rows too short to give each of them a block.
template <bool BF16, int W>
__global__ __launch_bounds__(64 * W, 5) void logprobs_kernel(Logprobs a)
{
    __shared__ key_t lds_keys[W][kSlots];
    __shared__ float lds_sums[W][3];
    __shared__ uint32_t lds_nth[W];
    constexpr int VEC = BF16 ? 8 : 4;           // logits a load
    constexpr int NV = kPerLane / VEC;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x / (uint32_t)a.segments;
    const int seg = blockIdx.x % (uint32_t)a.segments;
    const char *x = static_cast<const char *>(a.logits) + row * a.row_stride * (BF16 ? 2 : 4);
    // parts of whole blocks, one a wave
    const uint32_t vocab = (uint32_t)a.vocab;       // at most 2^30
    const uint32_t parts = a.segments * W, blocks = (vocab + kBlock - 1) / kBlock;
    const uint32_t p = seg * W + wave, each = blocks / parts, more = blocks % parts;
    const uint32_t b0 = each * p + (p < more ? p : more), b1 = b0 + each + (p < more ? 1 : 0);

    // every wave of the workgroup has a block: their first ones share a floor
    const bool shared = each > 0 || seg * W + W - 1 < more;

    Sums s = {-kInf, 0.0f, 0.0f};
    Top top = {lds_keys[wave], a.n_top, 0, 0};
    // rows may start at any multiple of their type: 16-byte loads without that
    // alignment
    struct __attribute__((packed, aligned(2))) Wide { uint32_t w[4]; };
    for (uint32_t b = b0; b < b1; ++b) {
        const uint32_t base = b * kBlock;
        float v[kPerLane];
        const bool whole = base + kBlock <= vocab;
        if (whole || vocab >= VEC) {
            // of a row's last block, pieces that pass the row's end are read
            // from inside it and then put right
            const char *src = x + ((int64_t)base + lane * VEC) * (BF16 ? 2 : 4);
            const uint32_t end = vocab - VEC;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t at = base + (i * 64 + lane) * VEC;
                const char *from = whole ? src + i * 1024
                                         : x + (int64_t)(at < end ? at : end) * (BF16 ? 2 : 4);
                const Wide w = *reinterpret_cast<const Wide *>(from);
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
        }
        if (!whole) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const uint32_t at = base + (i * 64 + lane) * VEC;
                if (vocab >= VEC && at <= vocab - VEC) continue;
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    v[i * VEC + e] = at + e < vocab ? load_logit<BF16>(x, at + e) : -kInf;
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
            t = __builtin_fmaf(e, fmaxf(di, -1e30f), t);
        }
        s.t = f * (s.t + d * s.l) + t;
        s.l = f * s.l + l;
        s.m = mn;
        if (a.n_top == 0) continue;
        // (opaque, so that the slots' indices are formed where they are used
        // and not kept in registers)
        uint32_t at0 = base + lane * VEC;
        asm volatile("" : "+v"(at0));
        // a later block has higher indices: an equal logit does not matter
        const uint32_t bo = ordered(bm);
        if (top.floor != 0 && !__any(bo > (uint32_t)(top.floor >> 32))) continue;
        // What n lanes' maxima reach is a floor that n logits reach; so is, in
        // the first blocks, what ceil(n / 4) lanes of each wave reach. A maximum
        // of -inf counts if it is a logit's, not just where the lane began.
        const bool has = bm > -kInf || (at0 < vocab && v[0] == -kInf);
        const bool first = shared && b == b0;
        uint32_t nth = nth_largest(has ? bo : 0,
                                   first ? (a.n_top + W - 1) / W : a.n_top);
        if (first) {
            if (lane == 0) lds_nth[wave] = nth;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < W; ++w) nth = lds_nth[w] < nth ? lds_nth[w] : nth;
        }
        const key_t least = ((key_t)nth << 32) - 1;
        if (nth > 0 && least > top.floor) top.floor = least;
        const float fv = top.floor_value();
        int full = kPerLane;        // slot at which the buffer had no room
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            if (full < kPerLane || !__any(!(v[i] < fv))) continue;
            if (top.count > kBuffer - 64) {
                full = i;
                continue;
            }
            const uint32_t at = at0 + (i / VEC) * 64 * VEC + i % VEC;
            top.add(at < vocab && !(v[i] < fv), make_key(ordered(v[i]), at));
        }
        // rows in order, or many equal logits: slot by slot, read again
#pragma unroll 1
        for (int i = full; i < kPerLane; ++i) {
            const uint32_t at = at0 + (i / VEC) * 64 * VEC + i % VEC;
            const float y = at < vocab ? load_logit<BF16>(x, at) : 0.0f;
            top.add_or_cut(at < vocab, make_key(ordered(y), at));
        }
        top.cut();
    }
    bool inside = false;
    float target = 0.0f;
    if (a.segments == 1 && wave == 0) target = target_logit<BF16>(a, row, inside);
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
    for (int w = 1; w < W; ++w)
        s = join(s, Sums{lds_sums[w][0], lds_sums[w][1], lds_sums[w][2]});
    if (a.n_top > 0) {
        top.raise(lane < W ? lds_keys[lane][a.n_top - 1] : 0);
#pragma unroll 1
        for (int w = 1; w < W; ++w) {
            const key_t k = lane < a.n_top ? lds_keys[w][lane] : 0;
            top.add_or_cut(k != 0, k);
        }
        top.cut();
    }
    if (a.segments == 1) {
        write_row(a, row, s, top.buf, target, inside);
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
    __shared__ key_t lds_keys[kSlots];
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    // every load that waits for nothing first
    bool inside;
    const float target = target_logit<BF16>(a, row, inside);
    const uint32_t n = a.n_top, total = a.segments * n;
    key_t k[4] = {}, nth = 0;
    auto load_keys = [&](uint32_t i0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t i = i0 + 64 * e + lane;
            k[e] = i < total ? segment_keys(a, row, i / n)[i % n] : 0;
        }
    };
    if (n > 0) {
        load_keys(0);
        for (int seg = lane; seg < a.segments; seg += 64) {
            const key_t o = segment_keys(a, row, seg)[n - 1];
            nth = o > nth ? o : nth;
        }
    }
    Sums s = {-kInf, 0.0f, 0.0f};
    for (int seg = lane; seg < a.segments; seg += 64) {
        const float *sums = reinterpret_cast<const float *>(segment_keys(a, row, seg) + n);
        s = join(s, Sums{sums[0], sums[1], sums[2]});
    }
    s = wave_join(s);
    Top top = {lds_keys, a.n_top, 0, 0};
    if (n > 0) {
        top.raise(nth);
        for (uint32_t i0 = 0;;) {
#pragma unroll
            for (int e = 0; e < 4; ++e) top.add_or_cut(k[e] != 0, k[e]);
            if ((i0 += 256) >= total) break;
            load_keys(i0);
        }
        top.cut();
    }
    write_row(a, row, s, lds_keys, target, inside);
}

}  // namespace

int logprobs_segments(int64_t n_rows, int64_t vocab)
{
    // four workgroups a compute unit, each wave at least one block: 300 rows of
    // 131072 40 us (45 at two, 42 at eight), 96 of 150001 27 us (32, 28), 20 of
    // 131072 16 us (17.5, 16)
    const int64_t most = (vocab + kBlock * kWaves - 1) / (kBlock * kWaves);
    int64_t n = (kServeCus * 4 + n_rows - 1) / n_rows;
    n = n > most ? most : n;
    if (n < 1) n = 1;
    // and no more than the longest part needs: 96 rows of 150001 in 10 segments
    // of two blocks a wave, not 11 with some waves at one (27.8 -> 26.9 us)
    const int64_t blocks = (vocab + kBlock - 1) / kBlock;
    const int64_t longest = (blocks + n * kWaves - 1) / (n * kWaves);
    return (int)((blocks + longest * kWaves - 1) / (longest * kWaves));
}

size_t logprobs_row_bytes(int segments, int n_top)
{
    return segments == 1 ? 0 : (size_t)segments * (8 * (size_t)n_top + 16);
}

hipError_t launch_logprobs(const Logprobs &a, bool bf16, hipStream_t stream)
{
    const unsigned grid = (unsigned)(a.n_rows * a.segments);
    // Rows that give some of four waves no block: one wave a row, 3641 rows of
    // 2003 14.6 us (31.8 with four), 3000 of 5000 21.1 (27.1); 8 rows of 5000 14.9
    // (14.0).
    if (a.vocab <= (kWaves - 1) * kBlock) {
        if (bf16)
            logprobs_kernel<true, 1><<<grid, 64, 0, stream>>>(a);
        else
            logprobs_kernel<false, 1><<<grid, 64, 0, stream>>>(a);
    } else {
        if (bf16)
            logprobs_kernel<true, kWaves><<<grid, 64 * kWaves, 0, stream>>>(a);
        else
            logprobs_kernel<false, kWaves><<<grid, 64 * kWaves, 0, stream>>>(a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.segments == 1) return e;
    if (bf16)
        logprobs_join_kernel<true><<<(unsigned)a.n_rows, 64, 0, stream>>>(a);
    else
        logprobs_join_kernel<false><<<(unsigned)a.n_rows, 64, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace rrq_detail
