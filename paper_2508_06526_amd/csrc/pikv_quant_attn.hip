// Routed attention over a cache held in 8 bits (pikv_sharded_attn's mathematics on the values code * scale) as a split
// flash-decode on the matrix cores:
//
//   quant_attn_partial : grid over (sequence, kv head and its rows, selected shard, split), 4 waves a block; one (max, sum,
//                        acc[D]) partial per row and block, in the layout of the merge that pikv_sharded_attn uses too.
//
// A code is exact in bf16, so the products are those of the codes, and the scales - one per 16 slots or more, the same for
// all lanes - multiply what comes out: a score by its K block's scale, a weight by its V block's before it meets the codes.
// Both are powers of two.
//
// Per wave and 32 entries, lane (c, r) = (lane % 16, lane / 16), the query rows padded to 16:
//   * S^T[entry][row] = K . Q^T.  The order of the contraction is free as long as both operands agree, so lane (c, r) takes
//     entry c's bytes as they come in 16-byte pieces; no trip through LDS.
//   * The lane's scores are those of entries 4r .. 4r+3 and 16+4r .. 16+4r+3 of query row c, and these, as weights, are the
//     operand P^T of the second product (three bf16 parts: all 24 bits).
//   * O^T[d][row] += V^T . P^T: lane (c, r) loads D / 16 bytes of those 8 entries' rows; output set i takes the i-th byte of
//     each.
#include "pikv_combine_dev.h"
#include "pikv_mfma_dev.h"
#include "pikv_quant_dev.h"

#include <math.h>

namespace pikv {
namespace {

constexpr int kWaves = 4;
constexpr int kRows = 16;               // query rows of a block
constexpr int kTile = 32;               // entries of a wave's pass

struct QuantAttnParams {
    const void *q;
    const void *const *K, *const *V;
    const float *K_scales, *V_scales;
    const int32_t *n_valid, *topk;
    float *part_acc, *part_ml, *scores;
    int64_t stride_h, stride_s;
    FastDiv by_nsplit, by_k, by_groups, by_row_blocks, by_draft;   // by_groups: row blocks of a sequence; by_row_blocks: of a kv head
    int Hq, Hkv, G, E, S, k, rr, tq, heads, rows;                  // heads: query heads of one draft query; rows: a block's, at most
    int nsplit, chunk, n_blocks, block_bits;
    uint32_t nsplit_rcp;
    float scale;
};

// Where the caller keeps query row `row` of kv head hk (rows of a kv head: draft query, head of the group).
__device__ __forceinline__ int64_t query_row(const QuantAttnParams &p, int b, int hk, int row) {
    if (p.tq <= 1) return (int64_t)b * p.Hq + hk * p.G + row;
    const int g = (int)p.by_draft.d;
    int t = (int)__umulhi((uint32_t)row, p.by_draft.rcp), gg = row - t * g;      // t: the quotient or one less
    if (gg >= g) ++t, gg -= g;
    return (int64_t)b * p.Hq + t * p.heads + hk * g + gg;
}

// 8 codes (two words, or byte i of eight words) as a bf16 operand.
template <int F>
__device__ __forceinline__ uint4 codes_operand(uint32_t lo, uint32_t hi) {
    if constexpr (F == PIKV_QUANT_INT8) {
        float f[8];
        decode4<F>(lo, f);
        decode4<F>(hi, f + 4);
        auto upper = [](float b, float a) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
        return make_uint4(upper(f[1], f[0]), upper(f[3], f[2]), upper(f[5], f[4]), upper(f[7], f[6]));
    } else {
        auto pair = [](uint32_t w, auto high) {
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, decltype(high)::value));
        };
        return make_uint4(pair(lo, std::false_type{}), pair(lo, std::true_type{}), pair(hi, std::false_type{}), pair(hi, std::true_type{}));
    }
}

template <int W, int F, int QP>
__global__ __launch_bounds__(kWaves *kWave) void quant_attn_partial(QuantAttnParams p) {
    constexpr int KB = W / 4 < 16 ? W / 4 : 16, KU = W / 4 / KB;       // bytes of a K piece, pieces of a lane
    constexpr int KS = W / 32, SETS = W / 16;                           // steps of a score; output sets
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, r = lane >> 4;
    int split, j, group, row_block;
    int id = fast_divide(p.by_nsplit, blockIdx.x, &split);
    id = fast_divide(p.by_k, id, &j);
    const int b = fast_divide(p.by_groups, id, &group);
    const int hk = fast_divide(p.by_row_blocks, group, &row_block);
    const int row0 = row_block * p.rows, rows = min(p.rows, p.G - row0), h0 = hk * p.G + row0;
    const int e = p.topk[(int64_t)(b * p.rr + (p.rr == 1 ? 0 : h0)) * p.k + j];
    const int64_t be = (int64_t)b * p.E + e;
    const int n = min(p.n_valid[be], p.S);
    int per = p.chunk;
    if (p.nsplit_rcp != 0) {                 // cut by what the shard holds
        constexpr int ROUND = kWaves * kTile;
        per = (int)__umulhi((uint32_t)(max(n, 0) + p.nsplit - 1), p.nsplit_rcp);
        per = min((max(per, 1) + ROUND - 1) / ROUND * ROUND, p.chunk);
    }
    const int first = split * per, last = min(n, first + per);
    const int64_t part_base = (((int64_t)b * p.Hq + h0) * p.k + j) * p.nsplit + split, part_row = (int64_t)p.k * p.nsplit;
    if (first >= last) {
        for (int idx = tid; idx < rows * (W / 4); idx += kWaves * kWave) {
            const int g = idx / (W / 4), d = (idx - g * (W / 4)) * 4;
            const int64_t at = part_base + g * part_row;
            *reinterpret_cast<float4 *>(p.part_acc + at * W + d) = make_float4(0.f, 0.f, 0.f, 0.f);
            if (d == 0) *reinterpret_cast<float2 *>(p.part_ml + at * 2) = make_float2(-INFINITY, 0.f);
        }
        return;
    }
    const char *Kb = static_cast<const char *>(p.K[be]) + hk * p.stride_h, *Vb = static_cast<const char *>(p.V[be]) + hk * p.stride_h;
    const int64_t scale_row = (be * p.Hkv + hk) * p.n_blocks;

    // Query operand of step s = 2 u + v: lane (c, r) holds values 4 KB u + KB r + 8 v + 0 .. 7 of row c.
    uint4 qop[KS][QP];
    {
        const int64_t at = query_row(p, b, hk, row0 + min(c, rows - 1)) * W;
        const bool aligned = (reinterpret_cast<uintptr_t>(p.q) & 15) == 0;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int d = 4 * KB * (s / (KB / 8)) + KB * r + 8 * (s % (KB / 8));
            if constexpr (QP == 1) {
                qop[s][0] = load_query<uint4>(static_cast<const bf16 *>(p.q) + at + d, aligned);
            } else {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = static_cast<const float *>(p.q)[at + d + i];
                split_bf16(f, qop[s]);
            }
        }
    }

    float m = -INFINITY, l = 0.0f;
    f32x4_t acc[SETS];
#pragma unroll
    for (int i = 0; i < SETS; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    for (int t0 = first + wave * kTile; t0 < last; t0 += kWaves * kTile) {
        float sv[8];
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
            const int slot = min(t0 + 16 * hb + c, last - 1);
            const char *row = Kb + (int64_t)slot * p.stride_s + KB * r;
            uint32_t w[KU][KB / 4];
#pragma unroll
            for (int u = 0; u < KU; ++u) load_words_stream<KB / 4>(w[u], row + 4 * KB * u);
            const float ks = p.K_scales[scale_row + (min(t0 + 16 * hb, last - 1) >> p.block_bits)];
            f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = QP - 1; k >= 0; --k)
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const int u = s / (KB / 8), v = s % (KB / 8);
                    sc = mfma_rows(codes_operand<F>(w[u][2 * v], w[u][2 * v + 1]), qop[s][k], sc);
                }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int at = t0 + 16 * hb + 4 * r + x;
                sv[4 * hb + x] = at < last ? sc[x] * ks * p.scale : -INFINITY;
            }
            if (p.scores != nullptr && c < rows) {
                float *to = p.scores + (((int64_t)b * p.Hq + h0 + c) * p.k + j) * p.S + t0 + 16 * hb + 4 * r;
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (t0 + 16 * hb + 4 * r + x < last) to[x] = sv[4 * hb + x];
            }
        }
        float tm = sv[0];
#pragma unroll
        for (int x = 1; x < 8; ++x) tm = fmaxf(tm, sv[x]);
        const float mn = fmaxf(m, group_max(tm)), corr = __expf(m - mn);
        m = mn;
        l *= corr;
#pragma unroll
        for (int i = 0; i < SETS; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) acc[i][x] *= corr;
        float tl = 0.0f;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            sv[x] = __expf(sv[x] - mn);
            tl += sv[x];
        }
        l += tl;
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
            const float vs = p.V_scales[scale_row + (min(t0 + 16 * hb, last - 1) >> p.block_bits)];
#pragma unroll
            for (int x = 0; x < 4; ++x) sv[4 * hb + x] *= vs;
        }
        uint4 pop[3];
        split_bf16(sv, pop);
        uint8_t vr[8][SETS];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const int slot = min(t0 + 16 * (t >> 2) + 4 * r + (t & 3), last - 1);
            const char *row = Vb + (int64_t)slot * p.stride_s + SETS * c;
#pragma unroll
            for (int i = 0; i < SETS; ++i) vr[t][i] = (uint8_t)row[i];
        }
#pragma unroll
        for (int i = 0; i < SETS; ++i) {
            uint32_t lo = 0, hi = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                lo |= (uint32_t)vr[t][i] << (8 * t);
                hi |= (uint32_t)vr[4 + t][i] << (8 * t);
            }
            const uint4 vop = codes_operand<F>(lo, hi);
            f32x4_t small = mfma_rows(vop, pop[2], f32x4_t{0.f, 0.f, 0.f, 0.f});
            small = mfma_rows(vop, pop[1], small);
            acc[i] += mfma_rows(vop, pop[0], f32x4_t{0.f, 0.f, 0.f, 0.f}) + small;
        }
    }

    // waves -> LDS -> the block's partial (rows padded by 4 floats: banks)
    constexpr int AP = W + 4;
    __shared__ __attribute__((aligned(16))) float sm_acc[kWaves][kRows][AP];
    __shared__ float sm_m[kWaves][kRows], sm_l[kWaves][kRows];
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (c < rows) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int i = 0; i < SETS; ++i) sm_acc[wave][c][SETS * (4 * r + x) + i] = acc[i][x];
    }
    if (r == 0) {
        sm_m[wave][c] = m;
        sm_l[wave][c] = l;
    }
    __syncthreads();
    for (int idx = tid; idx < rows * (W / 4); idx += kWaves * kWave) {
        const int g = idx / (W / 4), d = (idx - g * (W / 4)) * 4;
        float M = sm_m[0][g];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sm_m[w][g]);
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        float L = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = sm_m[w][g] == -INFINITY ? 0.0f : __expf(sm_m[w][g] - M);
            const float4 o = *reinterpret_cast<const float4 *>(&sm_acc[w][g][d]);
            a.x = fmaf(o.x, f, a.x);
            a.y = fmaf(o.y, f, a.y);
            a.z = fmaf(o.z, f, a.z);
            a.w = fmaf(o.w, f, a.w);
            L = fmaf(sm_l[w][g], f, L);
        }
        const int64_t at = part_base + g * part_row;
        *reinterpret_cast<float4 *>(p.part_acc + at * W + d) = a;
        if (d == 0) *reinterpret_cast<float2 *>(p.part_ml + at * 2) = make_float2(M, L);
    }
}

struct QuantPlan {
    int rows, row_blocks;      // query rows of a block; row blocks of a kv head
    int nsplit, chunk;
    size_t acc_bytes, ml_bytes;
};

int make_plan(const pikv_desc *d, int k, QuantPlan *plan) {
    const int rc = check_quant(d, PIKV_QUANT_INT8, 16);
    if (rc != PIKV_OK) return rc;
    if (k < 1 || k > d->E) return PIKV_ERR_INVALID;
    const int G = d->Hq / d->Hkv, tq = d->tq > 1 ? d->tq : 1;
    const bool per_head = d->route_rows_per_seq != 1;
    if (tq > 1 && (per_head || d->Hq % tq != 0 || G % tq != 0)) return PIKV_ERR_UNSUPPORTED;
    if (d->stride_s > (1 << 24)) return PIKV_ERR_UNSUPPORTED;
    plan->rows = per_head ? 1 : G < kRows ? G : kRows;
    plan->row_blocks = (G + plan->rows - 1) / plan->rows;
    const int64_t units = (int64_t)d->B * d->Hkv * plan->row_blocks * k;
    int64_t nsplit = units > 0 ? 256 * 3 / units : 1;
    const int64_t most = d->S / (kWaves * kTile);
    if (nsplit > most) nsplit = most;
    if (nsplit > kMaxPartialsPerHead / k) nsplit = kMaxPartialsPerHead / k;
    if (nsplit < 1) nsplit = 1;
    int64_t chunk = (d->S + nsplit - 1) / nsplit;
    chunk = (chunk + kTile - 1) / kTile * kTile;
    plan->chunk = (int)chunk;
    plan->nsplit = (int)((d->S + chunk - 1) / chunk);
    if (units * plan->nsplit >= (1 << 23)) return PIKV_ERR_UNSUPPORTED;
    const size_t partials = (size_t)d->B * d->Hq * k * plan->nsplit;
    plan->acc_bytes = (partials * d->D * sizeof(float) + 255) / 256 * 256;
    plan->ml_bytes = (partials * 2 * sizeof(float) + 255) / 256 * 256;
    return PIKV_OK;
}

size_t workspace_bytes(const QuantPlan &plan) { return plan.acc_bytes + plan.ml_bytes + 256; }

}  // namespace
}  // namespace pikv

using namespace pikv;

extern "C" size_t pikv_quant_attn_workspace_bytes(const pikv_desc *desc, int32_t k) {
    QuantPlan plan;
    return make_plan(desc, k, &plan) == PIKV_OK ? workspace_bytes(plan) : 0;
}

extern "C" int pikv_quant_attn(const pikv_desc *desc, int32_t format, int32_t block, const void *q, const void *const *K_shards,
                               const void *const *V_shards, const float *K_scales, const float *V_scales, const int32_t *n_valid,
                               const int32_t *topk_idx, const float *gates, int32_t k, int32_t combine, float scale, float *y,
                               float *row_max, float *row_norm, float *scores, float *slot_coef, void *workspace,
                               size_t workspace_bytes_given, void *stream) {
    int rc = check_quant(desc, format, block);
    if (rc != PIKV_OK) return rc;
    QuantPlan plan;
    rc = make_plan(desc, k, &plan);
    if (rc != PIKV_OK) return rc;
    if (!q || !K_shards || !V_shards || !K_scales || !V_scales || !n_valid || !topk_idx || !y) return PIKV_ERR_INVALID;
    if (combine != PIKV_COMBINE_LSE && combine != PIKV_COMBINE_LOCAL) return PIKV_ERR_INVALID;
    if (!(scale == scale)) return PIKV_ERR_INVALID;
    if (desc->B == 0) return PIKV_OK;
    if (!workspace || workspace_bytes_given < workspace_bytes(plan)) return PIKV_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return PIKV_ERR_INVALID;
    const int tq = desc->tq > 1 ? desc->tq : 1;
    QuantAttnParams p;
    p.q = q;
    p.K = K_shards;
    p.V = V_shards;
    p.K_scales = K_scales;
    p.V_scales = V_scales;
    p.n_valid = n_valid;
    p.topk = topk_idx;
    p.part_acc = static_cast<float *>(workspace);
    p.part_ml = p.part_acc + plan.acc_bytes / sizeof(float);
    p.scores = scores;
    p.stride_h = desc->stride_h;
    p.stride_s = desc->stride_s;
    p.Hq = desc->Hq;
    p.Hkv = desc->Hkv;
    p.G = desc->Hq / desc->Hkv;
    p.E = desc->E;
    p.S = desc->S;
    p.k = k;
    p.rr = desc->route_rows_per_seq;
    p.tq = tq;
    p.heads = desc->Hq / tq;
    p.rows = plan.rows;
    p.by_nsplit = fast_div(plan.nsplit);
    p.by_k = fast_div(k);
    p.by_groups = fast_div(desc->Hkv * plan.row_blocks);
    p.by_row_blocks = fast_div(plan.row_blocks);
    p.by_draft = fast_div(p.G / tq);
    p.nsplit = plan.nsplit;
    p.chunk = plan.chunk;
    p.n_blocks = (desc->S - 1) / block + 1;
    p.block_bits = __builtin_ctz(block);
    p.nsplit_rcp = plan.nsplit > 1 ? (uint32_t)(((uint64_t)1 << 32) / plan.nsplit + 1) : 0u;
    p.scale = scale > 0.0f ? scale : 1.0f / sqrtf((float)desc->D);
    CombineParams c;
    c.part_acc = p.part_acc;
    c.part_ml = p.part_ml;
    c.gates = gates;
    c.U_V = nullptr;
    c.y = y;
    c.row_max = row_max;
    c.row_norm = row_norm;
    c.slot_coef = slot_coef;
    c.Hq = desc->Hq;
    c.G = p.G;
    c.D = c.W = desc->D;
    c.k = k;
    c.rr = p.rr;
    c.rank = 0;
    c.nsplit = plan.nsplit;
    c.combine = combine;
    c.value_bias = 0;
    c.tq = tq;
    c.by_Hq = fast_div(c.Hq);
    c.by_G = fast_div(c.G);
    c.decoder_bytes = 0;
    const dim3 grid((unsigned)((int64_t)desc->B * desc->Hkv * plan.row_blocks * k * plan.nsplit)), threads(kWaves * kWave);
    hipStream_t st = as_stream(stream);
    auto launch = [&](auto width, auto fmt) {
        constexpr int W = decltype(width)::value, F = decltype(fmt)::value;
        if (desc->dtype == PIKV_F32) hipLaunchKernelGGL((quant_attn_partial<W, F, 3>), grid, threads, 0, st, p);
        else hipLaunchKernelGGL((quant_attn_partial<W, F, 1>), grid, threads, 0, st, p);
    };
    auto by_width = [&](auto fmt) {
        if (desc->D == 32) launch(std::integral_constant<int, 32>{}, fmt);
        else if (desc->D == 64) launch(std::integral_constant<int, 64>{}, fmt);
        else launch(std::integral_constant<int, 128>{}, fmt);
    };
    if (format == PIKV_QUANT_INT8) by_width(std::integral_constant<int, PIKV_QUANT_INT8>{});
    else by_width(std::integral_constant<int, PIKV_QUANT_E4M3>{});
    rc = launch_status();
    if (rc != PIKV_OK) return rc;
    return pikv_sharded_attn_merge(desc, &c, stream);
}
