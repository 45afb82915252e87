// Attention over the 8-bit cache for many query rows a sequence (prompt
// chunks): tiles of 128 rows, four waves of 32, that share each 64-key tile
// through LDS.
//
// With many rows the products bound the kernel, not the cache's bytes, so the
// codes are turned to binary16 once a workgroup, on their way into LDS, and
// every wave reads its operands from there. As in the few-row form the keys
// are the matrix rows (S^T = K Q^T, O^T = V^T P^T): a lane's 16 results of a
// 32 x 32 product are keys 8 (r / 4) + 4 (lane / 32) + r % 4 of one query row,
// and become the second product's operand as they are, because the values'
// 16-key runs are laid out in LDS in that order.
//
// Scales: a run of 16 keys lies in one page, so its key scale and value scale
// are wave-uniform. The weights carry the value scale through the exponent,
//   w = exp2(s c - m + lv),  c = key scale x query factor, lv = log2(vs / vref),
// and the sum of the softmax gets it back once a run: l += (vref / vs) sum w.
// vref is the largest value scale so far, so w <= 1 (times 2^8, below).
//
// The running maximum m moves only when a tile's exceeds it by 8 (weights
// then grow to 2^8 at most): most tiles skip the output's rescaling.
#include <type_traits>

#include "rrq_attention.h"

namespace rrq_detail {
namespace {

constexpr int kKeys = kTileKeys;
constexpr float kSlack = 8.0f;
// Weights carry a factor of 2^6: with the slack's 2^8 they reach 2^14 in
// binary16, and its normal range ends at 2^-20 of a row's largest weight.

typedef float f32x16 __attribute__((ext_vector_type(16)));

// Lane i's value in every lane.
__device__ __forceinline__ float lane_value(float x, int i)
{
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i));
}

template <int D, int CODE>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void attend_rows_kernel(Attend a)
{
    constexpr int KROW = D * 2 + 16;        // LDS bytes of a key row: 16 more than a
    constexpr int VROW = kKeys * 2 + 16;    // multiple of 128, so 8 rows span all banks
    constexpr int KB = kKeys * KROW, VB = D * VROW;
    constexpr int KT = kKeys * D / 16 / 256;    // 16-code pieces a thread stages
    constexpr int ND = D / 32, NK = D / 16;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * (KB + VB)];

    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int col = lane & 31, hb = lane >> 5;
    const int H = a.cache.n_kv_heads, P = a.cache.page_size;
    // heads are the fastest index: workgroups go to the 8 XCDs in turn, so a
    // head's workgroups share an L2 (at 8 heads); the last rows, which see the
    // most keys, come first
    const int kvh = blockIdx.x % H;
    RowTile r;
    if (!find_rows<kRowsTile>(a, gridDim.x / H - 1 - blockIdx.x / H, r)) return;

    const int64_t row = r.row0 + 32 * wave + col;
    const bool live = row < r.n_rows;
    const int64_t token = (live ? row : r.n_rows - 1) / a.ratio;
    const int head = kvh * a.ratio + (int)((live ? row : r.n_rows - 1) % a.ratio);
    int lo, hi, lo_any, hi_any, lo_all, hi_all;
    row_keys(a, r, token, lo, hi);
    tile_keys<kRowsTile>(a, r, lo_any, hi_any, lo_all, hi_all);
    int tb, te;
    split_tiles<kRowsTile>(a, lo_any, hi_any, blockIdx.y, tb, te);
    const int32_t *table = a.batch.page_table + r.seq * a.batch.table_stride;

    // queries: lane (col, hb) holds channels 16 j + 8 hb .. + 7 of its row
    f16x8 q[NK];
    float qf;
    {
        float x[NK][8];
        float amax = 0.0f;
        const int64_t at = (r.o0 + token) * a.q_token + head * a.q_head + 8 * hb;
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            load_query<8>(a, at + 16 * j, x[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[j][e]));
        }
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        float up;
        query_factors(a, amax, up, qf);
#pragma unroll
        for (int j = 0; j < NK; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) q[j][e] = (_Float16)(x[j][e] * up);
    }

    // Staging. Keys: thread t takes 16-code piece t % KP of key rows t / KP +
    // KSTEP i; a wave's rows lie in one run, so their page is wave-uniform.
    // Values: run t % 4 of channel t / 4 + 64 i. Lane % 4 is the run whose page
    // and scales a lane looks up.
    constexpr int KP = D / 16, KSTEP = 256 / KP;
    const int shift = __builtin_ctz(P);
    const int64_t head_bytes = (int64_t)P * D;
    const int krow = t / KP, vrun = t & 3;
    u32x4v kw[KT], vw[KT];
    int page = -1;                      // of the tile after the one in registers
    float ksr, vsr;                     // of the tile in registers: its scales (0: absent)
    bool absent;                        // and whether the lane's run is absent
    // Tiles past the last are the last again: staged, never used.
    auto find_page = [&](int tile) {
        const int key = (tile < te ? tile : te - 1) * kKeys + 16 * vrun;
        page = -1;
        if (key < hi_any && key + 16 > lo_any) page = table[key >> shift];
    };
    auto load_tile = [&](int tile) {
        const int key0 = (tile < te ? tile : te - 1) * kKeys;
        absent = (uint32_t)page >= (uint64_t)a.cache.n_pages;
        const int safe = absent ? 0 : page;
#pragma unroll
        for (int i = 0; i < KT; ++i) {
            const int row0 = KSTEP * i + 64 / KP * wave;        // wave's first row
            const int64_t p = __builtin_amdgcn_readlane(safe, row0 >> 4);
            const uint8_t *src = a.cache.k_codes + (p * H + kvh) * head_bytes;
            kw[i] = *reinterpret_cast<const u32x4v *>(
                src + (uint32_t)(((key0 + krow + KSTEP * i) & (P - 1)) * D + 16 * (t % KP)));
        }
        const int64_t block = (int64_t)safe * H + kvh;
        const uint8_t *src = a.cache.v_codes + block * head_bytes +
                             (uint32_t)((t / 4) * P + ((key0 + 16 * vrun) & (P - 1)));
#pragma unroll
        for (int i = 0; i < KT; ++i)
            vw[i] = *reinterpret_cast<const u32x4v *>(src + 64 * i * P);
        ksr = absent ? 0.0f : a.cache.k_scales[block];
        vsr = absent ? 0.0f : a.cache.v_scales[block];
    };
    // Values of keys that no row sees may be left over from another use of the
    // page (not numbers, even): cleared.
    auto clear_unseen = [&](int tile) {
        const int run = (tile < te ? tile : te - 1) * kKeys + 16 * vrun;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t keep = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int key = run + 4 * w + c;
                if (key >= lo_any && key < hi_any && !absent) keep |= 255u << (8 * c);
            }
#pragma unroll
            for (int i = 0; i < KT; ++i) vw[i][w] &= keep;
        }
    };
    auto store_tile = [&](uint8_t *buf) {
#pragma unroll
        for (int i = 0; i < KT; ++i) {
            uint8_t *at = buf + (krow + KSTEP * i) * KROW + 32 * (t % KP);
            *reinterpret_cast<f16x8 *>(at) = codes_f16<CODE>(kw[i][0], kw[i][1]);
            *reinterpret_cast<f16x8 *>(at + 16) = codes_f16<CODE>(kw[i][2], kw[i][3]);
        }
#pragma unroll
        for (int i = 0; i < KT; ++i) {
            uint8_t *at = buf + KB + (t / 4 + 64 * i) * VROW + 32 * vrun;
            *reinterpret_cast<f16x8 *>(at) = codes_f16<CODE>(vw[i][0], vw[i][2]);
            *reinterpret_cast<f16x8 *>(at + 16) = codes_f16<CODE>(vw[i][1], vw[i][3]);
        }
    };
    // tiles whose keys not every row sees
    auto at_edge = [&](int tile) {
        return tile * kKeys < lo_all || tile * kKeys + kKeys > hi_all;
    };

    float m = -kInf, l = 0.0f, vref = 0.0f;
    f32x16 o[ND];
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[n][e] = 0.0f;

    float kst = 0.0f, vst = 0.0f;       // scales of the tile in LDS
    uint32_t gone = 0;                  // its absent runs
    if (tb < te) {
        find_page(tb);
        load_tile(tb);
        find_page(tb + 1);
        clear_unseen(tb);
        store_tile(lds + (tb & 1) * (KB + VB));
        kst = ksr;
        vst = vsr;
        gone = (uint32_t)__ballot(absent) & 15u;
        load_tile(tb + 1);
        find_page(tb + 2);
        __syncthreads();
    }
    for (int tile = tb; tile < te; ++tile) {
        const uint8_t *buf = lds + (tile & 1) * (KB + VB);
        const uint32_t next_gone = (uint32_t)__ballot(absent) & 15u;
        if (at_edge(tile + 1) || next_gone) clear_unseen(tile + 1);

        f32x16 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[h][e] = 0.0f;
#pragma unroll
            for (int j = 0; j < NK; ++j) {
                const f16x8 k = *reinterpret_cast<const f16x8 *>(
                    buf + (32 * h + col) * KROW + 32 * j + 16 * hb);
                s[h] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[j], s[h], 0, 0, 0);
            }
        }
        store_tile(lds + ((tile + 1) & 1) * (KB + VB));
        const float next_ks = ksr, next_vs = vsr;
        load_tile(tile + 2);
        find_page(tile + 3);

        f16x8 p[4];
        // c: factor of a run's products; masked: -inf stands for a key the row
        // does not see
        auto softmax = [&](auto masked) {
            float tmax = -kInf, c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x = s[i >> 1][8 * (i & 1)];
#pragma unroll
                for (int e = 1; e < 8; ++e) x = fmaxf(x, s[i >> 1][8 * (i & 1) + e]);
                c[i] = lane_value(kst, i) * qf;
                // a run without a visible key: -inf stays, even times 0
                tmax = fmaxf(tmax, masked && x == -kInf ? -kInf : x * c[i]);
            }
            tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
            const float vmax = fmaxf(fmaxf(lane_value(vst, 0), lane_value(vst, 1)),
                                     fmaxf(lane_value(vst, 2), lane_value(vst, 3)));
            if (__any(tmax > m + kSlack) || vmax > vref) {
                const float mn = fmaxf(m, tmax);
                const float alpha = mn == -kInf ? 0.0f : exp2_fast(m - mn);
                m = mn;
                l *= alpha;
                const float vn = fmaxf(vref, vmax);
                const float oa = vn > 0.0f ? alpha * (vref / vn) : 0.0f;
                vref = vn;
#pragma unroll
                for (int n = 0; n < ND; ++n) o[n] *= oa;
            }
            const float ms = (m == -kInf ? 0.0f : m) - 6.0f;    // - 6: the weights' factor
            // vref / vs of the lane's run, and its log2. A block of zeros may
            // take any scale: vref's keeps w at the weight. Past 2^100 w is 0
            // in binary16 for any factor.
            const float backs =
                vst > 0.0f ? fminf(vref * __builtin_amdgcn_rcpf(vst), 0x1p100f) : 1.0f;
            const float lbacks = __builtin_amdgcn_logf(backs);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float back = lane_value(backs, i), sub = ms + lane_value(lbacks, i);
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = s[i >> 1][8 * (i & 1) + e];
                    float w = exp2_fast(__builtin_fmaf(x, c[i], -sub));
                    if (masked) w = x == -kInf ? 0.0f : w;
                    sum += w;
                    p[i][e] = (_Float16)w;
                }
                l += sum * back;
            }
        };
        if (at_edge(tile) || gone) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = tile * kKeys + 32 * h + 8 * (e >> 2) + 4 * hb + (e & 3);
                    if (key < lo || key >= hi || ((gone >> (2 * h + (e >> 3))) & 1))
                        s[h][e] = -kInf;
                }
            softmax(std::true_type{});
        } else {
            softmax(std::false_type{});
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < ND; ++n) {
                const f16x8 v = *reinterpret_cast<const f16x8 *>(
                    buf + KB + (32 * n + col) * VROW + 32 * i + 16 * hb);
                o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[i], o[n], 0, 0, 0);
            }
        kst = next_ks;
        vst = next_vs;
        gone = next_gone;
        __syncthreads();
    }

    // both l and o carry the weights' factor
    l += __shfl_xor(l, 32);
    if (!live) return;
    const int64_t at = (r.o0 + token) * a.n_heads + head;
    if (a.n_splits > 1) {
        const int64_t part = (int64_t)blockIdx.y * a.batch.n_tokens * a.n_heads + at;
        if (hb == 0) {
            a.part_ml[2 * part] = m;
            a.part_ml[2 * part + 1] = l;
        }
        if (te <= tb) return;
        float *dst = a.part_o + part * D + 4 * hb;
#pragma unroll
        for (int n = 0; n < ND; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4 *>(dst + 32 * n + 8 * g) =
                    f32x4{o[n][4 * g], o[n][4 * g + 1], o[n][4 * g + 2], o[n][4 * g + 3]} * vref;
        return;
    }
    const float norm = l == 0.0f ? 0.0f : vref / l;
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 y = f32x4{o[n][4 * g], o[n][4 * g + 1], o[n][4 * g + 2],
                                  o[n][4 * g + 3]} * norm;
            const int64_t d = at * D + 32 * n + 8 * g + 4 * hb;
            if (a.out_bf16)
                *reinterpret_cast<u32x2v *>(static_cast<uint16_t *>(a.out) + d) =
                    u32x2v{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])};
            else
                *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + d) = y;
        }
}

template <int D>
hipError_t rows_dim(const Attend &a, hipStream_t stream)
{
    const dim3 grid((unsigned)(attend_row_tiles(a.batch, a.ratio, kRowsTile) *
                               a.cache.n_kv_heads), a.n_splits);
    auto kernel = a.cache.code_type == RRQ_CODE_INT8 ? attend_rows_kernel<D, RRQ_CODE_INT8>
                                                     : attend_rows_kernel<D, RRQ_CODE_FP8>;
    kernel<<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_rows(const Attend &a, hipStream_t stream)
{
    if (a.cache.head_dim == 64) return rows_dim<64>(a, stream);
    if (a.cache.head_dim == 128) return rows_dim<128>(a, stream);
    return rows_dim<256>(a, stream);
}

}  // namespace rrq_detail
