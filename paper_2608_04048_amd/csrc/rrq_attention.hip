// Attention over the 8-bit cache (rrq_serve.h: rrq_cache_attention): the form
// for few query rows a sequence (single tokens, drafted tokens), the join of
// split key ranges, and the choice of form.
//
// One workgroup takes a tile of 16 or 32 rows (token, query head of the kv
// head's group) and a range of key positions; its waves take 64-key tiles of the
// range in turn, each with its own running maximum, sum and output, and are
// joined at the end. The cache's bytes bound it: codes go from memory to
// registers, each read once. A row tile whose range is split over several
// workgroups is joined by a second kernel.
//
// Both products run on the matrix cores in binary16 with binary32 sums, with
// the keys as rows: S^T = K Q^T and O^T = V^T P^T, so that the layout of the
// first's result (a lane holds 4 consecutive rows of a column) is the second's
// operand without any exchange between lanes. That fixes which key stands in
// which matrix row: in a tile of 64 keys lane group g (16 lanes) owns keys 16 g
// .. 16 g + 15, and row m of the i-th product takes key 16 (m / 4) + 4 i + m % 4.
// A run of 16 keys never spans pages, so a lane group has one key scale and one
// value scale a tile; the scales stay out of the operands (codes are exact in
// binary16): the key scale multiplies the product, the value scale the weight.
//
// Measured (keys and values in 8 bits, 8 kv heads of 128): a step of 64
// sequences of 90 to 12000 positions, 40 query heads, 796 MB in 163 us and 6 of
// the join (4.7 TB/s; a device copy makes 4.67, a kernel that only reads 5.3); a
// step of three of 99000 to 131072, 749 MB in 137 + 5 us (5.3 TB/s). One sequence
// of 1000 positions: 11.5 us, the latency of two tiles a wave on 8 compute units.
// 16 sequences of 300 to 9000 with 60 rows each, 2 kv heads of 64: 19.5 + 4 us,
// some 40% of it the issue of vector instructions (softmax and widening), the
// rest memory latency: two or three tiles a wave. Loading a tile's keys under
// the softmax of the one before gains 1% there and makes the step of 64
// sequences 186 us (fewer waves a SIMD, the last tile read twice).
#include "rrq_attention.h"

namespace rrq_detail {
namespace {

// Weights are scaled by 2^14 before rounding to binary16, whose normal range
// then reaches 2^-28 below the largest weight.
constexpr float kWeightBits = 14.0f;

// Maximum over the four lane groups: the swaps exchange the second halves of
// rows (of the wave) of one copy with the first of the other.
__device__ __forceinline__ float group_max(float a)
{
    const uint32_t x = __float_as_uint(a);
    const auto u = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    a = fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
    const uint32_t y = __float_as_uint(a);
    const auto v = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    return fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1]));
}
__device__ __forceinline__ float group_sum(float a)
{
    a += __shfl_xor(a, 16);
    return a + __shfl_xor(a, 32);
}

// LDS of a workgroup of `waves` waves and row tiles of at most `rows` rows:
// each wave's outputs (rows padded by 4 values, so that 16 rows start in
// different banks) and its maximum and sum.
constexpr unsigned few_lds(int D, int waves, int rows)
{
    return (unsigned)(waves * rows * (D + 4 + 2) * 4);
}

// Waves of a workgroup that takes a short range alone: as many as the
// registers of a compute unit hold.
constexpr int many_waves(int D) { return D == 64 ? 16 : 8; }

// NW: waves; NQ: blocks of 16 rows of the row tile; PARTS: of an operand
// (rrq_attention.h); TREE: rows see of their step what their bits say.
template <int D, int CODE, int NW, int NQ, int PARTS, bool TREE>
__global__ __launch_bounds__(64 * NW, NW > 4 || D == 256 || PARTS > 1 ? 1 : 2)
void attend_kernel(Attend a)
{
    constexpr int KL = D / 64;      // 16-byte key loads a lane and key row
    constexpr int ND = D / 16;      // 16-channel tiles of the output
    constexpr int R = 16 * NQ;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int rows_max = a.lds_rows;
    float *lds_ml = lds + NW * rows_max * (D + 4);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int kvh = blockIdx.y, split = blockIdx.z;
    RowTile r;
    if (!find_rows<R>(a, blockIdx.x, r)) return;
    int lo_any, hi_any, lo_all, hi_all, tb, te;
    if (TREE)
        tile_past<R>(a, r, lo_any, hi_any, lo_all, hi_all);
    else
        tile_keys<R>(a, r, lo_any, hi_any, lo_all, hi_all);
    const bool alone = split_tiles<R>(a, lo_any, hi_any, split, tb, te);
    if (alone && split > 0) return;
    if (!alone && te <= tb) {
        empty_range<R>(a, r, kvh, split);
        return;
    }

    const int P = a.cache.page_size, H = a.cache.n_kv_heads;
    const int shift = __builtin_ctz(P);
    const int32_t *table = a.batch.page_table + r.seq * a.batch.table_stride;
    // page number of the run of 16 keys at `key`, -1 if no row sees one of them
    auto page_of = [&](int key) {
        return key < hi_any && key + 16 > lo_any ? table[key >> shift] : -1;
    };
    // of the run this lane loads keys of (matrix rows col: run col / 4) and of
    // the run it owns (g), one tile ahead
    int kpage = -1, opage = -1;
    if (tb + wave < te) {
        kpage = page_of((tb + wave) * kTileKeys + 16 * (col >> 2));
        opage = page_of((tb + wave) * kTileKeys + 16 * g);
    }

    // This lane's rows, and their queries: lane (col, g) holds channels
    // 64 j + 16 g .. + 15.
    int lo[NQ], hi[NQ];
    f16x8 q[PARTS][NQ][KL][2];
    float qf[NQ];
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
        const int row = r.row0 + 16 * b + col;
        const RowPlace place = place_of(a, row < r.n_rows ? row : r.n_rows - 1);
        if (TREE)
            row_past(a, r, place.token, lo[b], hi[b]);
        else
            row_keys(a, r, place.token, lo[b], hi[b]);
        float x[KL][16];
        float amax = 0.0f;
        const int64_t at = (int64_t)(r.o0 + place.token) * a.q_token +
                           (kvh * a.ratio + place.member) * a.q_head + 16 * g;
#pragma unroll
        for (int j = 0; j < KL; ++j) {
            load_query<16>(a, at + 64 * j, x[j]);
#pragma unroll
            for (int e = 0; e < 16; ++e) amax = fmaxf(amax, fabsf(x[j][e]));
        }
        float up;
        query_factors(a, group_max(amax), up, qf[b]);
#pragma unroll
        for (int j = 0; j < KL; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float y = x[j][8 * h + i] * up;
                    q[0][b][j][h][i] = (_Float16)y;
                    if (PARTS > 1)
                        q[PARTS - 1][b][j][h][i] = (_Float16)(y - (float)q[0][b][j][h][i]);
                }
    }

    float m[NQ], l[NQ], vref = 0.0f;
    f32x4 o[NQ][ND];
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
        m[b] = -kInf;
        l[b] = 0.0f;
#pragma unroll
        for (int n = 0; n < ND; ++n) o[b][n] = f32x4{0, 0, 0, 0};
    }

    for (int tile = tb + wave; tile < te; tile += NW) {
        const int key0 = tile * kTileKeys;
        const int krun = key0 + 16 * (col >> 2), orun = key0 + 16 * g;
        const bool there = opage >= 0 && opage < a.cache.n_pages;
        const int64_t kb = kpage >= 0 && kpage < a.cache.n_pages ? kpage : 0;
        const int64_t ob = (int64_t)(there ? opage : 0) * H + kvh;
        const uint8_t *kc = a.cache.k_codes + (kb * H + kvh) * P * D +
                            ((krun & (P - 1)) + (col & 3)) * D + 16 * g;
        const uint8_t *vc = a.cache.v_codes + ob * P * D + (int64_t)(col * P + (orun & (P - 1)));
        u32x4v kw[4][KL], vw[ND];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < KL; ++j)
                kw[i][j] = *reinterpret_cast<const u32x4v *>(kc + 4 * i * D + 64 * j);
        const float ks = there ? a.cache.k_scales[ob] : 0.0f;
        const float vs = there ? a.cache.v_scales[ob] : 0.0f;
#pragma unroll
        for (int n = 0; n < ND; ++n)
            vw[n] = *reinterpret_cast<const u32x4v *>(vc + 16 * n * P);
        if (tile + NW < te) {
            kpage = page_of(krun + NW * kTileKeys);
            opage = page_of(orun + NW * kTileKeys);
        }

        // a lane's 16 keys: orun + 4 i + c
        float s[NQ][4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 acc[NQ];
#pragma unroll
            for (int b = 0; b < NQ; ++b) acc[b] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < KL; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f16x8 k = codes_f16<CODE>(kw[i][j][2 * h], kw[i][j][2 * h + 1]);
#pragma unroll
                    for (int b = 0; b < NQ; ++b)
#pragma unroll
                        for (int t = 0; t < PARTS; ++t)
                            acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[t][b][j][h],
                                                                            acc[b], 0, 0, 0);
                }
#pragma unroll
            for (int b = 0; b < NQ; ++b)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[b][i][c] = acc[b][c] * (ks * qf[b]);
        }
        // Keys a row does not see. The codes there may be left over from
        // another use of the page (not numbers, even), so scores are replaced
        // and value codes of keys outside every row's range are cleared. (A
        // tree's range ends with its step, whose rows are all written, also
        // those that no bit names.)
        if (key0 < lo_all || key0 + kTileKeys > hi_all || !__all(there)) {
#pragma unroll
            for (int b = 0; b < NQ; ++b) {
                uint32_t seen = 0;      // (TREE) a bit for each of the lane's keys
                if constexpr (TREE) {
                    const int row = r.row0 + 16 * b + col;
                    const int token = place_of(a, row < r.n_rows ? row : r.n_rows - 1).token;
                    seen = (uint32_t)(tree_keys(a, r, token, lo[b], hi[b], key0) >> (16 * g));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int key = orun + 4 * i + c;
                        const bool out = TREE ? !((seen >> (4 * i + c)) & 1)
                                              : key < lo[b] || key >= hi[b];
                        if (out || !there) s[b][i][c] = -kInf;
                    }
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t keep = 0;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int key = orun + 4 * w + c;
                    if (key >= lo_any && key < hi_any && there) keep |= 255u << (8 * c);
                }
#pragma unroll
                for (int n = 0; n < ND; ++n) vw[n][w] &= keep;
            }
        }
        // A weight carries its value scale, relative to vref, and so does the
        // maximum: m is the row's largest score + log2(vs / vref). The sum gets
        // the scale back.
        const float vmax = group_max(vs);
        if (__any(vmax > vref * kReferAgain)) {
#pragma unroll
            for (int b = 0; b < NQ; ++b) refer(vmax, vref, m[b], l[b]);
            vref = vmax;
        }
        const float back = scale_back(vs, vref), lback = __builtin_amdgcn_logf(back);
        f16x8 p[PARTS][NQ][2];
        float alpha[NQ];
#pragma unroll
        for (int b = 0; b < NQ; ++b) {
            float tmax = -kInf;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) tmax = fmaxf(tmax, s[b][i][c]);
            const float mn = fmaxf(m[b], group_max(tmax - lback));
            const float ms = mn == -kInf ? 0.0f : mn;
            alpha[b] = exp2_fast(m[b] - ms);
            m[b] = mn;
            const float sub = ms + lback - kWeightBits;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float w = exp2_fast(s[b][i][c] - sub);
                    sum += w;       // (before it is rounded: it may be below binary16)
                    const _Float16 first = (_Float16)w;
                    p[0][b][i >> 1][4 * (i & 1) + c] = first;
                    if (PARTS > 1)
                        p[PARTS - 1][b][i >> 1][4 * (i & 1) + c] = (_Float16)(w - (float)first);
                }
            l[b] = l[b] * alpha[b] + sum * back;
        }
#pragma unroll
        for (int n = 0; n < ND; ++n) {
            const f16x8 v0 = codes_f16<CODE>(vw[n][0], vw[n][1]);
            const f16x8 v1 = codes_f16<CODE>(vw[n][2], vw[n][3]);
#pragma unroll
            for (int b = 0; b < NQ; ++b) {
                f32x4 y = o[b][n] * alpha[b];
#pragma unroll
                for (int t = 0; t < PARTS; ++t) {
                    y = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[t][b][0], y, 0, 0, 0);
                    y = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[t][b][1], y, 0, 0, 0);
                }
                o[b][n] = y;
            }
        }
    }

    // Join the waves, 16 rows at a time: lane (col, g) holds channels
    // 16 n + 4 g + c of row col. A wave leaves its own mean (mean_factor), and
    // the means are joined by their shares of the sum.
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
        const float sum = group_sum(l[b]);
        if (b > 0) __syncthreads();
        if (col < rows_max) {
            if (g == 0) {
                lds_ml[(wave * rows_max + col) * 2] = m[b];
                lds_ml[(wave * rows_max + col) * 2 + 1] = sum;
            }
            float *dst = lds + (wave * rows_max + col) * (D + 4) + 4 * g;
            const float norm = mean_factor(vref, sum);
#pragma unroll
            for (int n = 0; n < ND; ++n)
                *reinterpret_cast<f32x4 *>(dst + 16 * n) = o[b][n] * kSumUnit * norm;
        }
        __syncthreads();
        // 4 channels a thread
        const int row0 = r.row0 + 16 * b;
        const int rows = r.n_rows - row0 < 16 ? r.n_rows - row0 : 16;
        for (int i = threadIdx.x; i < rows * (D / 4); i += 64 * NW) {
            const int orow = i / (D / 4), d = i % (D / 4) * 4;
            float mm = -kInf, ll = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) mm = fmaxf(mm, lds_ml[(w * rows_max + orow) * 2]);
            const float ms = mm == -kInf ? 0.0f : mm;
            float f[NW];
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const int at = w * rows_max + orow;
                f[w] = exp2_fast(lds_ml[at * 2] - ms) * lds_ml[at * 2 + 1];
                ll += f[w];
            }
            const float norm = ll == 0.0f ? 0.0f : 1.0f / ll;
            f32x4 y = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < NW; ++w)
                y += f[w] * norm *
                     *reinterpret_cast<const f32x4 *>(lds + (w * rows_max + orow) * (D + 4) + d);
            const RowPlace place = place_of(a, row0 + orow);
            const int64_t at = (int64_t)(r.o0 + place.token) * a.n_heads + kvh * a.ratio +
                               place.member;
            if (alone && a.n_splits > 1 && d == 0) a.part_ml[2 * at + 1] = kAlone;
            if (!alone) {
                const int64_t part = (int64_t)split * a.batch.n_tokens * a.n_heads + at;
                if (d == 0) {
                    a.part_ml[2 * part] = mm;
                    a.part_ml[2 * part + 1] = ll;
                }
                *reinterpret_cast<f32x4 *>(a.part_o + part * D + d) = y;
                continue;
            }
            if (a.out_bf16)
                *reinterpret_cast<u32x2v *>(static_cast<uint16_t *>(a.out) + at * D + d) =
                    u32x2v{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])};
            else
                *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + at * D + d) = y;
        }
    }
}

// Joins the key ranges of a row (token, head), each of which left its mean, its
// maximum and its sum: four waves a row, wave w takes ranges w, w + 4, .... Lane s
// holds range s's maximum and sum, so the factors cost one load. The ranges up to the
// last with a sum were all written; they are read four at a time, those past it as the
// last, times 0.
template <int D>
__global__ __launch_bounds__(256) void attend_join_kernel(Attend a)
{
    constexpr int N = D / 64, W = 4;
    __shared__ float lds[W][D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rows = a.batch.n_tokens * a.n_heads;
    const int64_t at = blockIdx.x;
    f32x2 ml = {-kInf, 0.0f};
    if (lane < a.n_splits)
        ml = *reinterpret_cast<const f32x2 *>(a.part_ml + 2 * (lane * rows + at));
    const int token = (int)((uint32_t)at / (uint32_t)a.n_heads);
    if (token < clamp_row(a.batch, 0) || token >= clamp_row(a.batch, (int)a.batch.n_seqs)) return;
    if (__shfl(ml[1], 0) == kAlone) return;     // written already
    float m = ml[0];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    float f = exp2_fast(ml[0] - (m == -kInf ? 0.0f : m)) * ml[1];
    float l = f;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
    f *= l == 0.0f ? 0.0f : 1.0f / l;
    const uint64_t has = __ballot(ml[1] != 0.0f);
    const int last = has ? 63 - __builtin_clzll(has) : -1;
    float y[N] = {};
    const float *src = a.part_o + at * D + lane * N;
    for (int s = wave; s <= last; s += 4 * W) {
        float x[4][N];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = s + i * W < last ? s + i * W : last;
#pragma unroll
            for (int d = 0; d < N; ++d) x[i][d] = src[r * rows * D + d];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float fs = s + i * W <= last ? __shfl(f, s + i * W) : 0.0f;
#pragma unroll
            for (int d = 0; d < N; ++d) y[d] += fs * x[i][d];
        }
    }
#pragma unroll
    for (int d = 0; d < N; ++d) lds[wave][lane * N + d] = y[d];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int w = 1; w < W; ++w) y[d] += lds[w][lane * N + d];
#pragma unroll
    for (int d = 0; d < N; ++d) {
        const int64_t i = at * D + lane * N + d;
        if (a.out_bf16)
            static_cast<uint16_t *>(a.out)[i] = (uint16_t)bf16_bits(y[d]);
        else
            static_cast<float *>(a.out)[i] = y[d];
    }
}

// The same for up to 8 ranges, 16 lanes a row, so that a wave has four rows' loads in
// flight: 34000 rows of 128 in two or three ranges each 6.5 us, 12.8 with a wave a row.
template <int D>
__global__ __launch_bounds__(256) void attend_join_few_kernel(Attend a)
{
    constexpr int N = D / 16;
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4 & 3;
    const int64_t rows = a.batch.n_tokens * a.n_heads;
    const int64_t at = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const bool inside = at < rows;
    f32x2 ml = {-kInf, 0.0f};
    if (inside && lane < a.n_splits)
        ml = *reinterpret_cast<const f32x2 *>(a.part_ml + 2 * (lane * rows + at));
    const int token = (int)((uint32_t)at / (uint32_t)a.n_heads);
    float m = ml[0];
#pragma unroll
    for (int d = 1; d < 16; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    float f = exp2_fast(ml[0] - (m == -kInf ? 0.0f : m)) * ml[1];
    float l = f;
#pragma unroll
    for (int d = 1; d < 16; d *= 2) l += __shfl_xor(l, d);
    f *= l == 0.0f ? 0.0f : 1.0f / l;
    const uint32_t has = (uint32_t)(__ballot(ml[1] != 0.0f) >> (16 * group)) & 0xFFFFu;
    const int last = has ? 31 - __builtin_clz(has) : -1;
    const bool written = __shfl(ml[1], 16 * group) == kAlone;
    if (!inside || written || token < clamp_row(a.batch, 0) ||
        token >= clamp_row(a.batch, (int)a.batch.n_seqs))
        return;
    f32x4 y[N / 4] = {};
    const float *src = a.part_o + at * D + lane * N;
    for (int s = 0; s <= last; s += 2) {
        f32x4 x[2][N / 4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = s + i < last ? s + i : last;
#pragma unroll
            for (int d = 0; d < N / 4; ++d)
                x[i][d] = *reinterpret_cast<const f32x4 *>(src + r * rows * D + 4 * d);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float fs = s + i <= last ? __shfl(f, 16 * group + s + i) : 0.0f;
#pragma unroll
            for (int d = 0; d < N / 4; ++d) y[d] += fs * x[i][d];
        }
    }
#pragma unroll
    for (int d = 0; d < N / 4; ++d) {
        const int64_t i = at * D + lane * N + 4 * d;
        if (a.out_bf16)
            *reinterpret_cast<u32x2v *>(static_cast<uint16_t *>(a.out) + i) =
                u32x2v{bf16_pair(y[d][0], y[d][1]), bf16_pair(y[d][2], y[d][3])};
        else
            *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + i) = y[d];
    }
}

template <int D, int CODE, int PARTS, bool TREE>
hipError_t few_parts(const Attend &a, const AttendPlan &p, hipStream_t stream)
{
    const dim3 grid((unsigned)attend_row_tiles(a.batch, a.ratio, p.tile), a.cache.n_kv_heads,
                    a.n_splits);
    // (two parts of heads of 256 pass the registers of a wave of eight)
    constexpr int MANY = D == 256 && PARTS > 1 ? 4 : many_waves(D);
    if (p.waves > 4)
        attend_kernel<D, CODE, MANY, 1, PARTS, TREE>
            <<<grid, 64 * MANY, few_lds(D, MANY, a.lds_rows), stream>>>(a);
    else if (p.tile == kWideTile)
        attend_kernel<D, CODE, 4, D <= 128 ? 2 : 1, PARTS, TREE>
            <<<grid, 256, few_lds(D, 4, a.lds_rows), stream>>>(a);
    else
        attend_kernel<D, CODE, 4, 1, PARTS, TREE>
            <<<grid, 256, few_lds(D, 4, a.lds_rows), stream>>>(a);
    return hipGetLastError();
}

template <int D, int CODE>
hipError_t few_code(const Attend &a, const AttendPlan &p, hipStream_t stream)
{
    if (a.seen)
        return a.out_bf16 ? few_parts<D, CODE, 1, true>(a, p, stream)
                          : few_parts<D, CODE, 2, true>(a, p, stream);
    return a.out_bf16 ? few_parts<D, CODE, 1, false>(a, p, stream)
                      : few_parts<D, CODE, 2, false>(a, p, stream);
}

template <int D>
hipError_t few_dim(const Attend &a, const AttendPlan &p, hipStream_t stream)
{
    return a.cache.code_type == RRQ_CODE_INT8 ? few_code<D, RRQ_CODE_INT8>(a, p, stream)
                                              : few_code<D, RRQ_CODE_FP8>(a, p, stream);
}

template <int D>
hipError_t join_dim(const Attend &a, hipStream_t stream)
{
    const unsigned rows = (unsigned)(a.batch.n_tokens * a.n_heads);
    if (a.n_splits > 8)
        attend_join_kernel<D><<<rows, 256, 0, stream>>>(a);
    else
        attend_join_few_kernel<D><<<(rows + 15) / 16, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

AttendPlan attend_plan(const rrq_cache &c, const rrq_batch &b, int n_heads, int64_t window,
                       bool tree)
{
    const int ratio = n_heads / c.n_kv_heads;
    AttendPlan p = {};
    const int64_t rows = b.n_tokens * ratio;
    // The form by the rows a sequence and kv head (mean): this one reads and
    // widens the codes once a row tile, the other once for 128 rows, but waits
    // at a barrier each tile of keys. Measured at 16 sequences of 300 to 9000
    // positions: 60 rows with heads of 64, 26.8 us here and 29.7 there; 40 rows
    // with heads of 128, 58 and 49; with heads of 256, 125 and 84. Where there are
    // few row tiles, time is latency and this form ahead: 160 rows on 900
    // positions, 8 kv heads of 128, 17.3 and 19.0; 84 rows of 4 sequences of 2000,
    // 2 kv heads of 64, 13.3 and 20.4; 240 rows on 3000, 2 of 256, 20.9 and 33.9
    // (but 120 rows on 30000, 2 of 256, 58 and 51).
    // Tiles of 32 rows halve the codes to widen (20 rows, heads of 128: 58 us;
    // 75 in tiles of 16), but hold two rows' queries and outputs a lane: with
    // heads of 256 that no longer fits the registers.
    p.tile = rows > 16 * b.n_seqs && c.head_dim <= 128 ? kWideTile : 16;
    p.rows_form = rows > (c.head_dim == 64 ? 64 : 32) * b.n_seqs &&
                  attend_row_tiles(b, ratio, p.tile) * c.n_kv_heads > kServeCus / 4;
    if (p.rows_form) p.tile = kRowsTile;
    // Drafted tokens of few sequences: as long as all pairs of a 16-row tile and a tile
    // of keys are few, time is the latency of a range, and shortest in 16-row tiles.
    // Heads of 128: 25 rows x 4 on 2000 positions (1700 pairs) 15.2 us in tiles of 16
    // and 17.7 in tiles of 32, 60 x 4 on 3000 (6000) 24.8 and 26.0, 25 x 4 on 8000
    // (7000) 31 and 27. Heads of 256, 9 to 17 x 4 of 6 sequences: in a window of 1024
    // (2000) 23.2 and in the many-row form 33.6, on 7000 (11900) 60 and 69; of 16
    // sequences (30000) 113 and 79. Heads of 64, 8 sequences of 12 x 12 on 5000 (10000)
    // 22.5 and 25.1.
    if (tree) {
        int64_t keys = b.max_pages * c.page_size;
        if (window > 0 && window < keys) keys = window;
        const int64_t pairs = attend_row_tiles(b, ratio, 16) * c.n_kv_heads *
                              ((keys + kTileKeys - 1) / kTileKeys);
        if (pairs <= (c.head_dim == 128 ? 6400 : 12800)) {
            p.tile = 16;
            p.rows_form = false;
        }
    }
    const int64_t units = attend_row_tiles(b, ratio, p.tile) * c.n_kv_heads;
    p.lds_rows = rows < 16 ? (int)rows : 16;
    p.waves = 4;
    p.splits = 1;
    // positions a row tile can reach over: the table's, or its window's (and one
    // tile, as windows start anywhere)
    int64_t reach = b.max_pages * c.page_size;
    if (window > 0 && window < reach) {
        const int64_t wide = window + p.tile / ratio + kTileKeys;
        reach = wide < reach ? wide : reach;
    }
    // Few short sequences: one workgroup of many waves, two tiles a wave at most
    // (one with heads of 256), saves the join's launch. One sequence: heads of
    // 128, 1000 positions 12.0 us, 14.6 in ranges of 512; 2000 positions 17.7
    // and 14.7; heads of 64, 2000 positions 11.7 and 13.5; heads of 256, 500
    // positions 12.9 and 14.3, 1000 positions 20.6 and 18.6.
    const int many = many_waves(c.head_dim);
    const int64_t few_keys = many * kTileKeys * (c.head_dim == 256 ? 1 : 2);
    if (p.tile == 16 && reach <= few_keys && units <= kServeCus &&
        few_lds(c.head_dim, many, p.lds_rows) <= 65536) {
        p.waves = many;
        return p;
    }
    // Workgroups to aim at and the shortest ranges.
    // 16-row tiles: three times what is resident, as lengths differ; 512 keys.
    // Three sequences of about 115000 positions: 143 us at 2048 workgroups, 154 at
    // 1024, 165 at 512; 32 sequences of 2000: 33 us in ranges of 512 keys, 35 of
    // 256, 53 of 1024.
    // 32-row tiles: what is resident (16 sequences of 300 to 9000 positions, heads
    // of 64: 23.3 us at 512, 25.7 at 768).
    // 128-row tiles, whose ranges cost a written and joined output of 128 rows:
    // 1.5 a compute unit of 256 keys at least where the row tiles alone do not
    // fill the card (a second round of workgroups would cost more than it
    // shares out), else 768 of 1024 keys. In us, the two rules in this order:
    // 300 rows x 4 on 2000 positions, heads of 128, 37.6 and 41.8; 40 x 4 on
    // 900, 18.9 and 30.4; 16 sequences of 300 to 9000 with 160 rows, 146 and
    // 160; five chunks of 174 to 900 tokens (over 256 row tiles), heads of 128,
    // 251 and 238, heads of 256 and a window of 1024, 111 and 107. Heads of 64, three
    // workgroups resident a compute unit, ranges of 512 keys: 4800 rows on 3000
    // positions 35, and 43 of 256 keys.
    const bool full = units > kServeCus + kServeCus / 4;
    // Trees without a window (packed, rrq_attention_rows.hip): about what is resident at
    // once, of 512 keys. Heads of 128, 16 trees of 40 to 65 rows on 300 to 9000, and one
    // of 130 on 20000: 180 and 83 us at 480, 181 and 86 at 448, 180 and 91 at 512; 4 of 20
    // to 33 on 500 to 4000: 29.7 in ranges of 512 keys, 36.5 of 320. Heads of 64, the first:
    // 119 at 768, 127 at 512; of 256, 16 trees of 9 to 17: 70 at 480, 91 at 768.
    if (p.rows_form && tree && window == 0) {
        p.target = c.head_dim == 64 ? 768 : 480;
        p.min_tiles = 8;
    } else if (p.rows_form) {
        p.target = c.head_dim == 64 ? 640 : (full ? 768 : 384);
        p.min_tiles = c.head_dim == 64 ? 8 : (full ? 16 : 4);
    } else {
        p.target = p.tile == kWideTile ? 512 : 2048;
        p.min_tiles = 8;
    }
    if (units >= (p.rows_form ? 4 * kServeCus : p.target)) return p;
    const int64_t least = p.min_tiles * kTileKeys;
    if (reach <= least + least / 2) return p;       // split_tiles would leave it whole (120 us)
    const int64_t most = (reach + least - 1) / least;
    int64_t n = 4 * p.target / units;
    n = n > most ? most : n;
    p.splits = n < 1 ? 1 : (n > 64 ? 64 : (int)n);
    return p;
}

hipError_t launch_attend(const Attend &a, const AttendPlan &p, hipStream_t stream)
{
    hipError_t e;
    if (p.rows_form)
        e = launch_attend_rows(a, stream);
    else if (a.cache.head_dim == 64)
        e = few_dim<64>(a, p, stream);
    else if (a.cache.head_dim == 128)
        e = few_dim<128>(a, p, stream);
    else
        e = few_dim<256>(a, p, stream);
    if (e != hipSuccess || a.n_splits == 1) return e;
    if (a.cache.head_dim == 64) return join_dim<64>(a, stream);
    if (a.cache.head_dim == 128) return join_dim<128>(a, stream);
    return join_dim<256>(a, stream);
}

}  // namespace rrq_detail
