// Routed attention over a cache held in 8 bits (pikv_sharded_attn's mathematics on the values code * scale) as a split
// flash-decode on the matrix cores:
//
//   quant_attn_partial : grid over (sequence, kv head and its rows, selected shard, split), 4 waves a block; one (max, sum,
//                        acc[D]) partial per row and block, in the layout of the merge that pikv_sharded_attn uses too.  Short calls:
//                        a block of 8 waves for all shards of its rows, merge included.
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
// A lane's piece of the next stage is requested as soon as this one's has been used: K behind the scores, V behind the output.
//
// Bound by memory from some 100 MB of codes on: 32 sequences x 32 kv heads x 2 shards of 2048 x 128 codes, 1.07 GB, in 173 us with the merge (6.2 TB/s; a
// pass that only reads 156).  Below by the trips and launches around it: 64 MB under 4 query heads, with 4 MB of scores, 16.6 us (median; the loads
// alone 14.2, a read-only pass 12.1) and a merge of 4.5.  Two stages ahead instead of one, or eight waves a block, changed
// nothing but the registers.
#include "pikv_combine_dev.h"
#include "pikv_mfma_dev.h"
#include "pikv_quant_dev.h"

#include <math.h>

namespace pikv {
namespace {

constexpr int kWaves = 4;
constexpr int kRows = 16;               // query rows of a matrix tile
constexpr int kMergedWaves = 8;         // of a block that takes all shards of its rows
constexpr int kTile = 32;               // entries of a stage of a wave
// Row tiles of a block, at most.  (Four fit a CU once, with their accumulators moved to and fro: 64 rows over 32K entries of each of 4
// kv heads 26.5 us, as two blocks of two, the second reading from the caches, 22.7, as four of one 25.9; 32 rows in blocks of two 23.7, of one 28.7.)
constexpr int kMostTiles = 2;
constexpr int kLongestBlock = 1024;     // rows of a block, while the merge holds the partials

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
    int shard_waves;                   // merged form: waves of a shard
    struct {
        const float *gates;
        float *y, *row_max, *row_norm, *slot_coef;
        int combine;
    } merge;
};

// Where the caller keeps query row `row` of kv head hk (rows of a kv head: draft query, head of the group).
__device__ __forceinline__ int64_t query_row(const QuantAttnParams &p, int b, int hk, int row) {
    if (p.tq <= 1) return (int64_t)b * p.Hq + hk * p.G + row;
    const int g = (int)p.by_draft.d;
    int t = (int)__umulhi((uint32_t)row, p.by_draft.rcp), gg = row - t * g;      // t: the quotient or one less
    if (gg >= g) ++t, gg -= g;
    return (int64_t)b * p.Hq + t * p.heads + hk * g + gg;
}

// 8 codes (two words) as a bf16 operand.
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

// Bytes 4 w + 0 .. 3 of four rows, transposed: out[i] holds byte i of each.
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&out)[4]) {
    const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u);
    const uint32_t ab2 = __builtin_amdgcn_perm(b, a, 0x07030602u), cd2 = __builtin_amdgcn_perm(d, c, 0x07030602u);
    out[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(cd2, ab2, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(cd2, ab2, 0x07060302u);
}

// Loads through a buffer descriptor: a request past its end reads zeros and costs no trip to memory, so that the last tile and
// the requests ahead of it need no clamps and no branches.  The whole offset goes into the lane's operand, which is what the
// end is compared with.  NT: non-temporal, for what no later request finds part of in the caches.
template <int BYTES, bool NT>
__device__ __forceinline__ void buffer_load(uint32_t (&dst)[BYTES < 4 ? 1 : BYTES / 4], __amdgpu_buffer_rsrc_t rsrc, uint32_t offset) {
    if constexpr (BYTES == 16) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b128(rsrc, offset, 0, NT ? 2 : 0);
        dst[0] = v[0], dst[1] = v[1], dst[2] = v[2], dst[3] = v[3];
    } else if constexpr (BYTES == 8) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(rsrc, offset, 0, NT ? 2 : 0);
        dst[0] = v[0], dst[1] = v[1];
    } else if constexpr (BYTES == 4) {
        dst[0] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, offset, 0, NT ? 2 : 0);
    } else {
        dst[0] = __builtin_amdgcn_raw_buffer_load_b16(rsrc, offset, 0, NT ? 2 : 0);
    }
}

// Blocks a CU holds at the least (registers).
constexpr int quant_blocks_per_cu(int row_tiles, int parts) { return row_tiles == 1 ? (parts == 1 ? 4 : 3) : 2; }

// The merge of a block that holds all selected shards of its rows: 8 lanes a row, lane w with wave w's (max, sum) pair.  A
// shard's waves are 8, 4, 2 or 1 neighbours: joined by an xor butterfly, then the shards with their gates (as head_weights, in
// both combine modes).  Leaves every wave's factor.
__device__ __forceinline__ void merge_rows(const QuantAttnParams &p, int b, int h0, int hk, int row0, int rows, float gate, const float (&m)[kMergedWaves][kRows],
                                           const float (&l)[kMergedWaves][kRows], float (&factor)[kMergedWaves][kRows]) {
    static_assert(kMergedWaves == 8, "a row is 8 lanes");
    const int g = threadIdx.x >> 3, w = threadIdx.x & 7, per = p.shard_waves, j = w / per;
    if (threadIdx.x >= kRows * 8) return;    // whole waves
    const bool used = g < rows && j < p.k;
    const float mw = used ? m[w][g] : -INFINITY, lw = used ? l[w][g] : 0.0f;
    float Mj = mw;
    for (int off = 1; off < per; off <<= 1) Mj = fmaxf(Mj, __shfl_xor(Mj, off, kWave));
    float Zj = mw == -INFINITY ? lw : lw * __expf(mw - Mj);                    // (a wave without rows: 0)
    for (int off = 1; off < per; off <<= 1) Zj += __shfl_xor(Zj, off, kWave);
    const bool live = Zj > 0.0f, lse = p.merge.combine == PIKV_COMBINE_LSE;
    float M = live ? Mj : -INFINITY;
    for (int off = per; off < 8; off <<= 1) M = fmaxf(M, __shfl_xor(M, off, kWave));
    const float e = __expf(Mj - M);
    float norm = live ? (lse ? gate * Zj * e : gate) : 0.0f;
    for (int off = per; off < 8; off <<= 1) norm += __shfl_xor(norm, off, kWave);
    if (!used) return;
    const float weight = !live ? 0.0f : lse ? gate * e / norm : gate / (norm * Zj);
    factor[w][g] = lw > 0.0f && live ? weight * __expf(mw - Mj) : 0.0f;
    if (w % per == 0 && p.merge.slot_coef) {
        float *to = p.merge.slot_coef + (((int64_t)b * p.Hq + h0 + g) * p.k + j) * 2;
        to[0] = !live ? 0.0f : lse ? M : Mj;
        to[1] = !live ? 0.0f : lse ? gate / norm : weight;
    }
    if (w == 0) {
        const int64_t row = query_row(p, b, hk, row0 + g);
        if (p.merge.row_max) p.merge.row_max[row] = M;
        if (p.merge.row_norm) p.merge.row_norm[row] = norm;
    }
}

// WAVES == kWaves: a split of a shard, partials for the merge.  WAVES == kMergedWaves: all selected shards of the rows by one
// block, some of its waves each, and the merge behind them: short calls in one launch.
template <int W, int F, int QP, int RT, bool SC, int WAVES>
__global__ __launch_bounds__(WAVES *kWave, WAVES == kWaves ? quant_blocks_per_cu(RT, QP) : 1) void quant_attn_partial(QuantAttnParams p) {
    constexpr bool MERGED = WAVES == kMergedWaves;
    constexpr int KB = W / 4 < 16 ? W / 4 : 16, KU = W / 4 / KB;       // bytes of a K piece, pieces of a lane
    constexpr int KS = W / 32, SETS = W / 16;                           // steps of a score; output sets, bytes of a V piece
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, r = lane >> 4;
    int split = 0, j, group, row_block, id = blockIdx.x;
    if constexpr (MERGED) {
        j = min(wave / p.shard_waves, p.k);              // (k: a wave that is left over)
    } else {
        id = fast_divide(p.by_nsplit, id, &split);
        id = fast_divide(p.by_k, id, &j);
    }
    const int b = fast_divide(p.by_groups, id, &group);
    const int hk = fast_divide(p.by_row_blocks, group, &row_block);
    const int row0 = row_block * p.rows, rows = min(p.rows, p.G - row0), h0 = hk * p.G + row0;
    // One trip to memory: lane e takes shard e's count and addresses beside the selection, which picks among them.
    const int64_t be_lane = (int64_t)b * p.E + min(lane, p.E - 1);
    const int n_lane = p.n_valid[be_lane];
    const uint64_t K_lane = reinterpret_cast<uint64_t>(p.K[be_lane]), V_lane = reinterpret_cast<uint64_t>(p.V[be_lane]);
    const int sel = __builtin_amdgcn_readfirstlane(p.topk[(int64_t)(b * p.rr + (p.rr == 1 ? 0 : h0)) * p.k + min(j, p.k - 1)]);
    const int e = min(max(sel, 0), p.E - 1);
    float gate = 1.0f;                       // (ahead of the rows: the merge has no trip of its own)
    if (MERGED && p.merge.gates) gate = p.merge.gates[(int64_t)(b * p.rr + (p.rr == 1 ? 0 : h0)) * p.k + min((lane & 7) / p.shard_waves, p.k - 1)];
    const int64_t be = (int64_t)b * p.E + e;
    const int n = sel == e ? min(__builtin_amdgcn_readlane(n_lane, e), p.S) : 0;      // (no such shard: empty)
    auto address = [&](uint64_t of_lane) {
        const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)of_lane, e), hi = __builtin_amdgcn_readlane((int)(uint32_t)(of_lane >> 32), e);
        return reinterpret_cast<char *>(((uint64_t)hi << 32) | lo) + hk * p.stride_h;
    };
    int per = p.chunk;
    if (!MERGED && p.nsplit_rcp != 0) {      // cut by what the shard holds
        constexpr int ROUND = kWaves * kTile;
        per = (int)__umulhi((uint32_t)(max(n, 0) + p.nsplit - 1), p.nsplit_rcp);
        per = min((max(per, 1) + ROUND - 1) / ROUND * ROUND, p.chunk);
    }
    // The wave's rows: stages of kTile rows at `start`, a round apart.
    const int first = split * per, last = MERGED && j == p.k ? 0 : min(n, first + per);
    const int start = first + (MERGED ? wave % p.shard_waves : wave) * kTile, round = (MERGED ? p.shard_waves : kWaves) * kTile;
    const int64_t part_base = (((int64_t)b * p.Hq + h0) * p.k + j) * p.nsplit + split, part_row = (int64_t)p.k * p.nsplit;
    if (!MERGED && first >= last) {
        for (int idx = tid; idx < rows * (W / 4); idx += kWaves * kWave) {
            const int g = idx / (W / 4), d = (idx - g * (W / 4)) * 4;
            const int64_t at = part_base + g * part_row;
            *reinterpret_cast<float4 *>(p.part_acc + at * W + d) = make_float4(0.f, 0.f, 0.f, 0.f);
            if (d == 0) *reinterpret_cast<float2 *>(p.part_ml + at * 2) = make_float2(-INFINITY, 0.f);
        }
        return;
    }
    char *Kb = address(K_lane), *Vb = address(V_lane);
    const uint32_t rb = (uint32_t)p.stride_s;
    const int64_t scale_row = (be * p.Hkv + hk) * p.n_blocks;
    const float *scales = ((lane & 2) ? p.V_scales : p.K_scales) + scale_row;

    // A stage: K rows, V rows and (lanes 0 .. 3: K of either half, V of either) the scales of 32 entries.
    uint32_t kr[2][KU][KB / 4], vr[8][SETS < 4 ? 1 : SETS / 4];
    float sr;
    const uint32_t k_lane = c * rb + KB * r, v_lane = 4 * r * rb + SETS * c;
    auto opaque = [](uint32_t v) {           // (else an offset per load is carried through the loop)
        asm volatile("" : "+v"(v));
        return v;
    };
    auto rsrc = [&](char *base, int t0) {    // rows t0 .. of the split: the last one ends after its W bytes
        const int at = min(t0, last);
        const uint32_t bytes = at < last ? (uint32_t)(min(last - at, kTile) - 1) * rb + W : 0u;
        return __builtin_amdgcn_make_buffer_rsrc(base + (int64_t)at * rb, 0, bytes, 0x00020000);
    };
    auto load_k = [&](int t0) {
        sr = scales[max(min(t0 + 16 * (lane & 1), last - 1), 0) >> p.block_bits];
        const auto from = rsrc(Kb, t0);
        const uint32_t at = opaque(k_lane);
#pragma unroll
        for (int hb = 0; hb < 2; ++hb)
#pragma unroll
            for (int u = 0; u < KU; ++u) buffer_load<KB, true>(kr[hb][u], from, at + 16 * hb * rb + 4 * KB * u);
    };
    auto load_v = [&](int t0) {
        const auto from = rsrc(Vb, t0);
        const uint32_t at = opaque(v_lane);
#pragma unroll
        for (int t = 0; t < 8; ++t) buffer_load<SETS, W == 128>(vr[t], from, at + (16 * (t >> 2) + (t & 3)) * rb);
    };

    // Query operand of row tile rt, step s = (KB / 8) u + v: lane (c, r) holds values 4 KB u + KB r + 8 v + 0 .. 7 of its row c.
    uint4 qop[RT][KS][QP];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int64_t at = query_row(p, b, hk, row0 + min(rt * kRows + c, rows - 1)) * W;
        const bool aligned = (reinterpret_cast<uintptr_t>(p.q) & 15) == 0;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int d = 4 * KB * (s / (KB / 8)) + KB * r + 8 * (s % (KB / 8));
            if constexpr (QP == 1) {
                qop[rt][s][0] = load_query<uint4>(static_cast<const bf16 *>(p.q) + at + d, aligned);
            } else {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = static_cast<const float *>(p.q)[at + d + i];
                split_bf16(f, qop[rt][s]);
            }
        }
    }
    load_k(start);
    load_v(start);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int k = 0; k < QP; ++k) hold_operand(qop[rt][s][k]);        // complete here, not behind loads in the loop

    float m[RT], l[RT];
    f32x4_t acc[RT][SETS];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.0f;
#pragma unroll
        for (int i = 0; i < SETS; ++i) acc[rt][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    for (int t0 = start; t0 < last; t0 += round) {
        // scores sv[rt][4 hb + x]: entry t0 + 16 hb + 4 r + x, row c of row tile rt
        float sv[RT][8];
        const int scale_bits = __float_as_int(sr);
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
            const float ks = __int_as_float(__builtin_amdgcn_readlane(scale_bits, hb));
            f32x4_t sc[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) sc[rt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const auto &w = kr[hb][s / (KB / 8)];
                const int v = s % (KB / 8);
                const uint4 kop = codes_operand<F>(w[2 * v], w[2 * v + 1]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int k = QP - 1; k >= 0; --k) sc[rt] = mfma_rows(kop, qop[rt][s][k], sc[rt]);
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int x = 0; x < 4; ++x) sv[rt][4 * hb + x] = sc[rt][x] * ks * p.scale;
        }
        const float vs0 = __int_as_float(__builtin_amdgcn_readlane(scale_bits, 2)), vs1 = __int_as_float(__builtin_amdgcn_readlane(scale_bits, 3));
        load_k(t0 + round);
        if (t0 + kTile > last) {             // (uniform)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    if (t0 + 16 * (x >> 2) + 4 * r + (x & 3) >= last) sv[rt][x] = -INFINITY;
        }
        if constexpr (SC) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                if (rt * kRows + c < rows) {
                    float *to = p.scores + (((int64_t)b * p.Hq + h0 + rt * kRows + c) * p.k + j) * p.S;
#pragma unroll
                    for (int hb = 0; hb < 2; ++hb) {
                        const int at = t0 + 16 * hb + 4 * r;
                        if (at + 4 <= last && (p.S & 3) == 0) {
                            store16(to + at, make_uint4(__float_as_uint(sv[rt][4 * hb]), __float_as_uint(sv[rt][4 * hb + 1]),
                                                        __float_as_uint(sv[rt][4 * hb + 2]), __float_as_uint(sv[rt][4 * hb + 3])));
                        } else {
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                if (at + x < last) to[at + x] = sv[rt][4 * hb + x];
                        }
                    }
                }
        }
        uint4 pop[RT][3];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float tm = sv[rt][0];
#pragma unroll
            for (int x = 1; x < 8; ++x) tm = fmaxf(tm, sv[rt][x]);
            const float mn = fmaxf(m[rt], group_max(tm));
            if (__any(mn > m[rt])) {         // else the factor is 1 in every lane
                const float corr = __expf(m[rt] - mn);
                m[rt] = mn;
                l[rt] *= corr;
#pragma unroll
                for (int i = 0; i < SETS; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x) acc[rt][i][x] *= corr;
            }
            float tl[2];
#pragma unroll
            for (int hb = 0; hb < 2; ++hb) {
#pragma unroll
                for (int x = 0; x < 4; ++x) sv[rt][4 * hb + x] = __expf(sv[rt][4 * hb + x] - mn);
                tl[hb] = (sv[rt][4 * hb] + sv[rt][4 * hb + 1]) + (sv[rt][4 * hb + 2] + sv[rt][4 * hb + 3]);
#pragma unroll
                for (int x = 0; x < 4; ++x) sv[rt][4 * hb + x] *= hb ? vs1 : vs0;
            }
            l[rt] += tl[0] + tl[1];
            split_bf16(sv[rt], pop[rt]);
        }
        // O^T += V^T P^T, output set i takes byte i of each of the lane's 8 V rows
#pragma unroll
        for (int w = 0; w < (SETS + 3) / 4; ++w) {
            uint32_t lo[4], hi[4];
            if constexpr (F == PIKV_QUANT_E4M3) {
                transpose4(vr[0][w], vr[1][w], vr[2][w], vr[3][w], lo);
                transpose4(vr[4][w], vr[5][w], vr[6][w], vr[7][w], hi);
            }
#pragma unroll
            for (int i = 0; i < (SETS < 4 ? SETS : 4); ++i) {
                uint4 vop;
                if constexpr (F == PIKV_QUANT_E4M3) {
                    vop = codes_operand<F>(lo[i], hi[i]);
                } else {                     // (a conversion takes its byte from any place)
                    auto pair = [&](int t) {
                        const float a = (float)(int8_t)(vr[t][w] >> (8 * i)), b = (float)(int8_t)(vr[t + 1][w] >> (8 * i));
                        return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
                    };
                    vop = make_uint4(pair(0), pair(2), pair(4), pair(6));
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int part = 2; part >= 0; --part) acc[rt][4 * w + i] = mfma_rows(vop, pop[rt][part], acc[rt][4 * w + i]);
            }
        }
        load_v(t0 + round);
    }

    // waves -> LDS -> the block's partial, row tile by row tile (rows padded by 4 floats: banks)
    constexpr int AP = W + 4;
    extern __shared__ __attribute__((aligned(16))) float sm_acc[];       // [wave][row][AP], rows of a tile
    __shared__ float sm_m[WAVES][kRows], sm_l[WAVES][kRows], sm_f[WAVES][kRows];
    const int tile_rows = min(kRows, p.rows);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (rt * kRows >= rows) break;
        const int rows_here = min(kRows, rows - rt * kRows);
        float ls = l[rt];
        ls += __shfl_xor(ls, 16, kWave);
        ls += __shfl_xor(ls, 32, kWave);
        if (rt > 0) __syncthreads();
        if (c < rows_here) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int i = 0; i < SETS; ++i) sm_acc[(wave * tile_rows + c) * AP + SETS * (4 * r + x) + i] = acc[rt][i][x];
        }
        if (r == 0) {
            sm_m[wave][c] = m[rt];
            sm_l[wave][c] = ls;
        }
        __syncthreads();
        if constexpr (MERGED) {
            merge_rows(p, b, h0, hk, row0, rows_here, gate, sm_m, sm_l, sm_f);
            __syncthreads();
        }
        for (int idx = tid; idx < rows_here * (W / 4); idx += WAVES * kWave) {
            const int g = idx / (W / 4), d = (idx - g * (W / 4)) * 4;
            float M = sm_m[0][g];
            if constexpr (!MERGED) {
#pragma unroll
                for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sm_m[w][g]);
            }
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
            float L = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                if (MERGED && w >= p.k * p.shard_waves) break;
                const float f = MERGED ? sm_f[w][g] : sm_m[w][g] == -INFINITY ? 0.0f : __expf(sm_m[w][g] - M);
                const float4 o = *reinterpret_cast<const float4 *>(sm_acc + (w * tile_rows + g) * AP + d);
                a.x = fmaf(o.x, f, a.x);
                a.y = fmaf(o.y, f, a.y);
                a.z = fmaf(o.z, f, a.z);
                a.w = fmaf(o.w, f, a.w);
                L = fmaf(sm_l[w][g], f, L);
            }
            if constexpr (MERGED) {
                float *to = p.merge.y + query_row(p, b, hk, row0 + g) * W + d;      // (y need not be 16-byte aligned)
                to[0] = a.x, to[1] = a.y, to[2] = a.z, to[3] = a.w;
            } else {
                const int64_t at = part_base + (rt * kRows + g) * part_row;
                *reinterpret_cast<float4 *>(p.part_acc + at * W + d) = a;
                if (d == 0) *reinterpret_cast<float2 *>(p.part_ml + at * 2) = make_float2(M, L);
            }
        }
    }
}

struct QuantPlan {
    int row_tiles, rows, row_blocks;      // matrix tiles and query rows of a block; row blocks of a kv head
    int nsplit, chunk;
    bool merged;               // one launch, no partials
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
    // row tiles of a block: what the group takes; fp32 queries, three operands each, one
    plan->row_tiles = per_head || G <= kRows || d->dtype == PIKV_F32 ? 1 : kMostTiles;
    plan->rows = per_head ? 1 : G < plan->row_tiles * kRows ? G : plan->row_tiles * kRows;
    plan->row_blocks = (G + plan->rows - 1) / plan->rows;
    const int64_t units = (int64_t)d->B * d->Hkv * plan->row_blocks * k;
    // The merged form, one launch and no partials.  Where a wave has one stage of 128 values, or two of fewer (1 x 8 kv heads x 2 shards of 128
    // entries of 128 values 7.5 -> 6.3 us, of 256 of 64 values 7.0 -> 6.2; two stages of 128 values 7.6 -> 8.5, four of 32 values 7.0 -> 7.8).
    // And where there are blocks for most CUs without splits: 24 x 8 x 2 of 256 entries 13.0 -> 9.6, of 1024 26.7 -> 23.1, of 2048 even, 8 shards of 512
    // even; 80 x 8 x 2 of 512 39.0 -> 35.9.  With 128 blocks the splits win from 512 entries on (12.4 against 13.4; of 1024 17.5 against 21.6).
    // (Above 640 blocks splits, for many short shards: 2048 blocks of 256 entries 32.2 against 35.5; 768 and 1280 blocks of 512 would gain, 45 -> 39 and
    // 71 -> 60.)
    const int64_t blocks = units / k, rows = (int64_t)k * d->S;
    const bool one_round = (int64_t)d->S * (d->D > 64 ? d->D : 64) <= (int64_t)128 * kTile * (kMergedWaves / k);
    plan->merged = plan->row_tiles == 1 && k <= kMergedWaves && blocks <= 640 && (one_round || (blocks >= 192 && rows <= 4096));
    // A block per CU, and blocks of at most 1024 rows, but none of fewer than a stage of each wave.
    int64_t nsplit = units > 0 ? 256 / units : 1;
    const int64_t finer = (d->S + kLongestBlock - 1) / kLongestBlock, most = (d->S + kWaves * kTile - 1) / (kWaves * kTile);
    if (nsplit < finer) nsplit = finer;
    if (plan->merged) nsplit = 1;
    if (nsplit > most) nsplit = most;
    if (nsplit > kMaxPartialsPerHead / k) nsplit = kMaxPartialsPerHead / k;
    if (nsplit < 1) nsplit = 1;
    int64_t chunk = (d->S + nsplit - 1) / nsplit;
    chunk = (chunk + kTile - 1) / kTile * kTile;
    plan->chunk = (int)chunk;
    plan->nsplit = (int)((d->S + chunk - 1) / chunk);
    if (units * plan->nsplit >= (1 << 23)) return PIKV_ERR_UNSUPPORTED;
    // A launch has fewer than 2^32 threads; the merge's have a block for every query row.
    if (!plan->merged && (int64_t)d->B * d->Hq * combine_threads(k * plan->nsplit) >= (int64_t)1 << 32) return PIKV_ERR_UNSUPPORTED;
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
    if (combine != PIKV_COMBINE_LSE && combine != PIKV_COMBINE_LOCAL) return PIKV_ERR_INVALID;
    if (!(scale == scale)) return PIKV_ERR_INVALID;
    if (desc->B == 0) return PIKV_OK;            // (tensors without elements have no address)
    if (!q || !K_shards || !V_shards || !K_scales || !V_scales || !n_valid || !topk_idx || !y) return PIKV_ERR_INVALID;
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
    p.shard_waves = kMergedWaves / k;
    p.merge = {gates, y, row_max, row_norm, slot_coef, combine};
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
    const int waves = plan.merged ? kMergedWaves : kWaves;
    const dim3 grid((unsigned)((int64_t)desc->B * desc->Hkv * plan.row_blocks * (plan.merged ? 1 : k * plan.nsplit))), threads(waves * kWave);
    const size_t lds = (size_t)waves * (plan.rows < kRows ? plan.rows : kRows) * (desc->D + 4) * sizeof(float);
    hipStream_t st = as_stream(stream);
    auto launch = [&](auto width, auto fmt) {
        constexpr int W = decltype(width)::value, F = decltype(fmt)::value;
        auto go = [&](auto parts, auto tiles) {
            constexpr int QP = decltype(parts)::value, RT = decltype(tiles)::value;
            auto scored = [&](auto with) {
                constexpr bool SC = decltype(with)::value;
                if constexpr (RT == 1) {
                    if (plan.merged) {
                        hipLaunchKernelGGL((quant_attn_partial<W, F, QP, RT, SC, kMergedWaves>), grid, threads, lds, st, p);
                        return;
                    }
                }
                hipLaunchKernelGGL((quant_attn_partial<W, F, QP, RT, SC, kWaves>), grid, threads, lds, st, p);
            };
            if (scores) scored(std::true_type{});
            else scored(std::false_type{});
        };
        const std::integral_constant<int, 1> one{};
        if (desc->dtype == PIKV_F32) go(std::integral_constant<int, 3>{}, one);
        else if (plan.row_tiles == 1) go(one, one);
        else go(one, std::integral_constant<int, kMostTiles>{});
    };
    auto by_width = [&](auto fmt) {
        if (desc->D == 32) launch(std::integral_constant<int, 32>{}, fmt);
        else if (desc->D == 64) launch(std::integral_constant<int, 64>{}, fmt);
        else launch(std::integral_constant<int, 128>{}, fmt);
    };
    if (format == PIKV_QUANT_INT8) by_width(std::integral_constant<int, PIKV_QUANT_INT8>{});
    else by_width(std::integral_constant<int, PIKV_QUANT_E4M3>{});
    rc = launch_status();
    if (rc != PIKV_OK || plan.merged) return rc;
    return pikv_sharded_attn_merge(desc, &c, stream);
}
