// Routed attention over a paged cache (pikv_sharded_attn's mathematics, with capped scores, a distance bias, a window and a prefix) as a
// split flash-decode on the matrix cores:
//
//   paged_attn_partial : grid over (sequence, kv head and its rows, selected shard, split), 4 waves a block; one (max, sum, acc[D])
//                        partial per row and block, in the layout of the merge that pikv_sharded_attn uses too.  Short calls: a block
//                        of 8 waves for all shards of its rows, merge included.
//
// Per wave and stage of 32 (bf16) or 16 (fp32) entries, lane (c, r) = (lane % 16, lane / 16), the query rows padded to 16:
//   * S^T[entry][row] = K . Q^T: the order of a contraction is free, so lane (c, r) takes entry c's row in the 16-byte pieces
//     4 u + r as they come from memory; no trip through LDS.
//   * The lane's scores are those of entries 4 r .. 4 r + 3 (bf16: and 16 + 4 r ..) of query row c, and these, as weights, are the operand P^T
//     of the second product (bf16: three parts, all 24 bits: the entries' own rounding is the only one).
//   * O^T[d][row] += V^T . P^T: lane (c, r) loads values D / 16 c .. of those entries' rows; output set i takes the i-th value of each.
// Every 16 entries lie in one page.  A lane holds one of the next 64 pages' numbers, so that the address of a request costs no trip of
// its own; requests go out a stage ahead through buffer descriptors that end with the last entry.
//
// Bound by the rows: 128 MiB (a sequence, 4 shards of 8192 slots, 32 heads over 8 of 128 bf16 values, raw scores written) 22.8 us, 5.9 TB/s, and the merge
// 4.5; 296 MB of 32 ragged sequences with capped scores and a distance bias 61 - 67 us in one launch, by the card, 4.4 - 4.9 TB/s.
#include "pikv_combine_dev.h"
#include "pikv_decode_dev.h"
#include "pikv_mfma_dev.h"
#include "pikv_paged_dev.h"
#include "pikv_scores_dev.h"

#include <math.h>

namespace pikv {
namespace {

constexpr int kWaves = 4;
constexpr int kMostTiles = 2;           // row tiles of a block
constexpr int kLongestBlock = 1024;     // rows of a block, while the merge holds the partials

template <typename T>
constexpr int stage_entries = sizeof(T) == 2 ? 32 : 16;

struct PagedAttnParams {
    const void *q;
    const char *K, *V;
    const int32_t *n_valid, *topk, *prefix, *entry_pos, *q_pos;
    const float *slopes;
    float *part_acc, *part_ml, *scores;
    PageGeometry pages;
    FastDiv by_nsplit, by_k, by_groups, by_row_blocks, by_draft;   // by_groups: row blocks of a sequence; by_row_blocks: of a kv head
    int Hq, Hkv, G, E, S, k, rr, tq, heads, rows;                  // heads: query heads of one draft query; rows: a block's, at most
    int nsplit, chunk, window;
    uint32_t nsplit_rcp;
    float scale, cap, cap_rcp;
    int shard_waves;                   // merged form: waves of a shard
    struct {
        const float *gates;
        float *y, *row_max, *row_norm, *slot_coef;
        int combine;
    } merge;
};

__device__ __forceinline__ f32x4_t mfma_value(float a, float b, f32x4_t acc) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, acc, 0, 0, 0); }

// WAVES == kWaves: a split of a shard, partials for the merge.  WAVES == kMergedWaves: all selected shards of the rows by one
// block, some of its waves each, and the merge behind them: short calls in one launch.  POS: scores or what is seen go by positions.
template <typename T, int W, int RT, bool SC, bool POS, int WAVES>
__global__ __launch_bounds__(WAVES *kWave, WAVES == kWaves ? (RT == 1 && !(POS && W == 128) ? 3 : 2) : 1) void paged_attn_partial(PagedAttnParams p) {
    constexpr bool MERGED = WAVES == kMergedWaves, BF = sizeof(T) == 2;
    constexpr int ES = sizeof(T), STAGE = stage_entries<T>, HB = STAGE / 16, NX = 4 * HB;      // NX: entries of a lane
    constexpr int KU = W * ES / 64;                                     // 16-byte K pieces of a lane
    constexpr int SETS = W / 16, VB = SETS * ES, VW = VB / 4;           // output sets; bytes and words of a lane's piece of a V row
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
    // One trip to memory: lane e takes shard e's count beside the selection, which picks among them.
    const int n_lane = p.n_valid[(int64_t)b * p.E + min(lane, p.E - 1)];
    const int sel = __builtin_amdgcn_readfirstlane(p.topk[(int64_t)(b * p.rr + (p.rr == 1 ? 0 : h0)) * p.k + min(j, p.k - 1)]);
    const int e = min(max(sel, 0), p.E - 1);
    float gate = 1.0f;                       // (ahead of the rows: the merge has no trip of its own)
    if (MERGED && p.merge.gates) gate = p.merge.gates[(int64_t)(b * p.rr + (p.rr == 1 ? 0 : h0)) * p.k + min((lane & 7) / p.shard_waves, p.k - 1)];
    const int64_t be = (int64_t)b * p.E + e;
    const int n = sel == e ? min(__builtin_amdgcn_readlane(n_lane, e), p.S) : 0;      // (no such shard: empty)
    int per = p.chunk;
    if (!MERGED && p.nsplit_rcp != 0) {      // cut by what the shard holds
        constexpr int ROUND = kWaves * STAGE;
        per = (int)__umulhi((uint32_t)(max(n, 0) + p.nsplit - 1), p.nsplit_rcp);
        per = min((max(per, 1) + ROUND - 1) / ROUND * ROUND, p.chunk);
    }
    // The wave's rows: stages at `start`, a round apart.
    const int first = split * per, last = MERGED && j == p.k ? 0 : min(n, first + per);
    const int start = first + (MERGED ? wave % p.shard_waves : wave) * STAGE, round = (MERGED ? p.shard_waves : kWaves) * STAGE;
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
    const uint32_t rb = (uint32_t)p.pages.stride_s;
    // (lanes' registers hold what only they read by: scalar ones are short)
    typedef const int32_t __attribute__((address_space(1))) *lane_ptr;
    auto of_lanes = [](const int32_t *at) {
        uint64_t v = reinterpret_cast<uint64_t>(at);
        asm volatile("" : "+v"(v));
        return (lane_ptr)v;
    };
    const lane_ptr table = of_lanes(p.pages.table + be * p.pages.per_shard);
    const lane_ptr positions = POS ? of_lanes(p.entry_pos + be * p.S) : nullptr;
    const char *Kh = p.K + hk * p.pages.stride_h, *Vh = p.V + hk * p.pages.stride_h;

    // Pages: the lane's is page_base + lane of the shard.
    int page_base = start >> p.pages.bits, page_lane = table[min(page_base + lane, p.pages.per_shard - 1)];
    asm volatile("" : "+v"(page_lane));      // here, once, and not behind the requests of the loop
    auto page_of = [&](int t0) {             // of entries t0 .. t0 + 15; -1: none
        const int at = min(t0, p.S - 1) >> p.pages.bits;
        if ((uint32_t)(at - page_base) >= (uint32_t)kWave) {
            page_base = at;
            page_lane = table[min(page_base + lane, p.pages.per_shard - 1)];
            asm volatile("" : "+v"(page_lane));
        }
        const int page = __builtin_amdgcn_readlane(page_lane, at - page_base);
        return page >= 0 && page < p.pages.n_pages ? page : -1;
    };
    // A stage: K rows, V rows and the positions of the lane's entries.
    uint32_t kr[HB][KU][4], vr[NX][VW];
    int pr[POS ? NX : 1], page[HB];
    const uint32_t k_lane = c * rb + 16 * r, v_lane = 4 * r * rb + VB * c;
    auto opaque = [](uint32_t v) {           // (else an offset per load is carried through the loop)
        asm volatile("" : "+v"(v));
        return v;
    };
    auto rsrc = [&](const char *base, int pg, int t) {      // entries t .. t + 15, the last one ending after its W values
        const int here = pg < 0 ? 0 : min(max(last - t, 0), 16);
        const char *at = base + (here > 0 ? pg * p.pages.stride_page + (int64_t)(t & ((1 << p.pages.bits) - 1)) * rb : 0);
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at), 0, here > 0 ? (uint32_t)(here - 1) * rb + W * ES : 0u, 0x00020000);
    };
    auto load_k = [&](int t0) {
        if constexpr (POS) {
#pragma unroll
            for (int x = 0; x < NX; ++x) pr[x] = positions[max(min(t0 + 16 * (x >> 2) + 4 * r + (x & 3), last - 1), 0)];
        }
        const uint32_t at = opaque(k_lane);
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) {
            page[hb] = page_of(t0 + 16 * hb);
            const auto from = rsrc(Kh, page[hb], t0 + 16 * hb);
#pragma unroll
            for (int u = 0; u < KU; ++u) buffer_load<16, true>(kr[hb][u], from, at + 64 * u);
        }
    };
    auto load_v = [&](int t0) {              // (behind load_k of the same stage: its pages)
        const uint32_t at = opaque(v_lane);
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) {
            const auto from = rsrc(Vh, page[hb], t0 + 16 * hb);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if constexpr (VB <= 16) {
                    buffer_load<VB, W * ES >= 256>(vr[4 * hb + x], from, at + x * rb);
                } else {
                    uint32_t half[4];
#pragma unroll
                    for (int u = 0; u < VB / 16; ++u) {
                        buffer_load<16, true>(half, from, at + x * rb + 16 * u);
#pragma unroll
                        for (int i = 0; i < 4; ++i) vr[4 * hb + x][4 * u + i] = half[i];
                    }
                }
            }
        }
    };

    // Query operand of row tile rt: lane (c, r) holds the pieces 4 u + r of its row c.
    uint4 qop[RT][KU];
    int my_pos[RT], low[RT];                 // the query's position; the first that it sees, and how many from there
    uint32_t reach[RT];
    float slope[RT];
    const uint32_t prefix = POS && p.prefix ? max(p.prefix[b], 0) : 0;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int64_t row = query_row(p, b, hk, row0 + min(rt * kRows + c, rows - 1));
        const bool aligned = (reinterpret_cast<uintptr_t>(p.q) & 15) == 0;
#pragma unroll
        for (int u = 0; u < KU; ++u) {
            const int64_t at = row * W + (16 / ES) * (4 * u + r);
            if constexpr (BF) {
                qop[rt][u] = load_query<uint4>(static_cast<const bf16 *>(p.q) + at, aligned);
            } else {
                const float *f = static_cast<const float *>(p.q) + at;
                qop[rt][u] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            }
        }
        my_pos[rt] = low[rt] = 0;
        reach[rt] = 0;
        slope[rt] = 0.0f;
        if constexpr (POS) {
            const int in_sequence = (int)(row - (int64_t)b * p.Hq), t = in_sequence / p.heads;
            my_pos[rt] = p.q_pos[(int64_t)b * p.tq + t];
            low[rt] = p.window > 0 ? max(my_pos[rt] - p.window + 1, 0) : 0;
            reach[rt] = my_pos[rt] >= 0 ? my_pos[rt] - low[rt] + 1 : 0;
            if (p.slopes) slope[rt] = p.slopes[in_sequence - t * p.heads];
        }
    }
    load_k(start);
    load_v(start);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int u = 0; u < KU; ++u) hold_operand(qop[rt][u]);        // complete here, not behind loads in the loop

    float m[RT], l[RT];
    f32x4_t acc[RT][SETS];
    uint32_t most[RT], least[RT];            // POS: the accumulators (4 i + x) that get an infinity at the end
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        most[rt] = least[rt] = 0u;
        m[rt] = -INFINITY;
        l[rt] = 0.0f;
#pragma unroll
        for (int i = 0; i < SETS; ++i) acc[rt][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    float *score_row[SC ? RT : 1] = {};
    if constexpr (SC) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            uint64_t at = reinterpret_cast<uint64_t>(p.scores + (((int64_t)b * p.Hq + h0 + rt * kRows + c) * p.k + j) * p.S);
            asm volatile("" : "+v"(at));
            score_row[rt] = reinterpret_cast<float *>(at);
        }
    }
    const bool score_quads = (p.S & 3) == 0;
    for (int t0 = start; t0 < last; t0 += round) {
        // scores sv[rt][4 hb + x]: entry t0 + 16 hb + 4 r + x, row c of row tile rt
        float sv[RT][NX];
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) {
            f32x4_t sc[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) sc[rt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < KU; ++u) {
                const uint32_t(&w)[4] = kr[hb][u];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    if constexpr (BF) {
                        sc[rt] = mfma_rows(make_uint4(w[0], w[1], w[2], w[3]), qop[rt][u], sc[rt]);
                    } else {
                        sc[rt] = mfma_value(__uint_as_float(w[0]), __uint_as_float(qop[rt][u].x), sc[rt]);
                        sc[rt] = mfma_value(__uint_as_float(w[1]), __uint_as_float(qop[rt][u].y), sc[rt]);
                        sc[rt] = mfma_value(__uint_as_float(w[2]), __uint_as_float(qop[rt][u].z), sc[rt]);
                        sc[rt] = mfma_value(__uint_as_float(w[3]), __uint_as_float(qop[rt][u].w), sc[rt]);
                    }
                }
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int x = 0; x < 4; ++x) sv[rt][4 * hb + x] = sc[rt][x];
        }
        int pos[POS ? NX : 1];
        if constexpr (POS) {
#pragma unroll
            for (int x = 0; x < NX; ++x) pos[x] = pr[x];
        }
        bool there[HB];
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) there[hb] = page[hb] >= 0;
        load_k(t0 + round);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (p.cap > 0.0f) {              // (uniform)
                cap_scores(sv[rt], p.scale, p.cap, p.cap_rcp);
            } else {
#pragma unroll
                for (int x = 0; x < NX; ++x) sv[rt][x] *= p.scale;
            }
        }
        bool whole = t0 + STAGE <= last;
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) whole = whole && there[hb];
        if (!whole) {                        // (uniform)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int x = 0; x < NX; ++x)
                    if (t0 + 16 * (x >> 2) + 4 * r + (x & 3) >= last || !there[x >> 2]) sv[rt][x] = -INFINITY;
        }
        uint32_t seen[RT];                   // of the lane's entries, by its row
        if constexpr (POS) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                seen[rt] = 0;
#pragma unroll
                for (int x = 0; x < NX; ++x) {
                    // (unsigned: a negative position lies beyond either)
                    const bool sees = ((uint32_t)pos[x] - (uint32_t)low[rt] < reach[rt]) | ((uint32_t)pos[x] < prefix);
                    const int far = (int)((uint32_t)my_pos[rt] - (uint32_t)pos[x]);
                    sv[rt][x] = sees ? fmaf(-slope[rt], fabsf((float)far), sv[rt][x]) : -INFINITY;
                    seen[rt] |= sees ? 1u << x : 0u;
                }
            }
        }
        if constexpr (SC) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                if (rt * kRows + c < rows) {
                    float *to = score_row[rt];
#pragma unroll
                    for (int hb = 0; hb < HB; ++hb) {
                        const int at = t0 + 16 * hb + 4 * r;
                        if (at + 4 <= last && score_quads) {
                            store_floats(to + at, make_float4(sv[rt][4 * hb], sv[rt][4 * hb + 1], sv[rt][4 * hb + 2], sv[rt][4 * hb + 3]));
                        } else {
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                if (at + x < last) *(float __attribute__((address_space(1))) *)(uintptr_t)(to + at + x) = sv[rt][4 * hb + x];
                        }
                    }
                }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float tm = sv[rt][0];
#pragma unroll
            for (int x = 1; x < NX; ++x) tm = fmaxf(tm, sv[rt][x]);
            const float mn = fmaxf(m[rt], group_max(tm)), base = mn == -INFINITY ? 0.0f : mn;      // (nothing seen yet: weights of zero)
            if (__any(mn > m[rt])) {         // else the factor is 1 in every lane
                const float corr = __expf(m[rt] - base);
                m[rt] = mn;
                l[rt] *= corr;
#pragma unroll
                for (int i = 0; i < SETS; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x) acc[rt][i][x] *= corr;
            }
            float tl[HB];
#pragma unroll
            for (int hb = 0; hb < HB; ++hb) {
#pragma unroll
                for (int x = 0; x < 4; ++x) sv[rt][4 * hb + x] = __expf(sv[rt][4 * hb + x] - base);
                tl[hb] = (sv[rt][4 * hb] + sv[rt][4 * hb + 1]) + (sv[rt][4 * hb + 2] + sv[rt][4 * hb + 3]);
            }
            l[rt] += HB == 2 ? tl[0] + tl[HB - 1] : tl[0];
        }
        auto operand = [&](int i, auto of) {     // bf16: value i of the lane's V rows, of(word): of two of them
            auto pair = [&](int t) { return of(__builtin_amdgcn_perm(vr[t + 1][i / 2], vr[t][i / 2], (i & 1) ? 0x07060302u : 0x05040100u)); };
            return make_uint4(pair(0), pair(2), pair(NX - 4), pair(NX - 2));
        };
        // A value that is no number stays out of the rows that do not see its entry (0 x NaN is NaN).  Rare: the rows that see one are
        // counted with a product of their own and get the infinities at the end - a NaN is both - and here it counts as zero.
        bool odd = false;
        if constexpr (POS) {
            bool hides = false, bad = false;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) hides |= seen[rt] != (1u << NX) - 1;
            if (__any(hides)) {
#pragma unroll
                for (int x = 0; x < NX; ++x)
#pragma unroll
                    for (int w = 0; w < VW; ++w) bad |= (vr[x][w] & 0x7f800000u) == 0x7f800000u || (BF && (vr[x][w] & 0x7f80u) == 0x7f80u);
            }
            odd = __any(bad);
            if (odd) {
                // 1 for +inf or a NaN as the bf16 value in the upper half; of -inf with the sign flipped.  (Without comparisons: their
                // results side by side take the scalar registers.)
                auto above = [](uint32_t v) {
                    const uint32_t special = (((v & 0x7f800000u) ^ 0x7f800000u) - 1u) >> 31, nan = (0u - (v & 0x7f0000u)) >> 31;
                    return special & (~v >> 31 | nan);
                };
                auto ones = [&](uint32_t v, uint32_t flip) { return above(v ^ flip) * 0x3f800000u | above((v << 16) ^ flip) * 0x3f80u; };
                const f32x4_t none = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < SETS; ++i)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        f32x4_t up = none, down = none;
                        if constexpr (BF) {
                            auto sees = [&](int x) { return ((seen[rt] >> x) & 1u) * 0x3f80u | ((seen[rt] >> (x + 1)) & 1u) * 0x3f800000u; };
                            const uint4 by = make_uint4(sees(0), sees(2), sees(NX - 4), sees(NX - 2));
                            up = mfma_rows(operand(i, [&](uint32_t v) { return ones(v, 0u); }), by, none);
                            down = mfma_rows(operand(i, [&](uint32_t v) { return ones(v, 0x80000000u); }), by, none);
                        } else {
#pragma unroll
                            for (int x = 0; x < NX; ++x) {
                                const float v = __uint_as_float(vr[x][i % VW]), sees = (seen[rt] >> x) & 1u ? 1.0f : 0.0f;
                                up = mfma_value(v == INFINITY || v != v ? 1.0f : 0.0f, sees, up);
                                down = mfma_value(v == -INFINITY || v != v ? 1.0f : 0.0f, sees, down);
                            }
                        }
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            most[rt] |= up[x] > 0.0f ? 1u << (4 * i + x) : 0u;
                            least[rt] |= down[x] > 0.0f ? 1u << (4 * i + x) : 0u;
                        }
                        __builtin_amdgcn_sched_barrier(0);       // (side by side the sets' counts cost registers of the whole loop)
                    }
            }
        }
        // O^T += V^T P^T, output set i takes value i of each of the lane's V rows
        if constexpr (BF) {
            uint4 pop[RT][3];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) split_bf16(sv[rt], pop[rt]);
#pragma unroll
            for (int i = 0; i < SETS; ++i) {
                uint4 vop = operand(i, [](uint32_t v) { return v; });
                if (POS && odd)
                    vop = operand(i, [](uint32_t v) {
                        return ((v & 0x7f800000u) == 0x7f800000u ? 0u : v & 0xffff0000u) | ((v & 0x7f80u) == 0x7f80u ? 0u : v & 0xffffu);
                    });
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int part = 2; part >= 0; --part) acc[rt][i] = mfma_rows(vop, pop[rt][part], acc[rt][i]);
            }
        } else {
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int i = 0; i < SETS; ++i) {
                    float v = __uint_as_float(vr[x][i % VW]);
                    if (POS && odd) v = v - v == 0.0f ? v : 0.0f;
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) acc[rt][i] = mfma_value(v, sv[rt][x], acc[rt][i]);
                }
        }
        load_v(t0 + round);
    }

    // The arguments from here on are read again: held through the loop they take more scalar registers than there are.
    auto late = (const PagedAttnParams __attribute__((address_space(4))) *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(late));
    const auto &pe = *late;
    // waves -> LDS -> the block's partial, row tile by row tile (rows padded by 4 floats: banks)
    constexpr int AP = W + 4;
    extern __shared__ __attribute__((aligned(16))) float sm_acc[];       // [wave][row][AP], rows of a tile
    __shared__ float sm_m[WAVES][kRows], sm_l[WAVES][kRows], sm_f[WAVES][kRows];
    const int tile_rows = min(kRows, pe.rows);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (rt * kRows >= rows) break;
        const int rows_here = min(kRows, rows - rt * kRows);
        float ls = l[rt];
        ls += __shfl_xor(ls, 16, kWave);
        ls += __shfl_xor(ls, 32, kWave);
        if (rt > 0) __syncthreads();
        if (POS && __any((most[rt] | least[rt]) != 0u)) {
#pragma unroll
            for (int i = 0; i < SETS; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if (most[rt] >> (4 * i + x) & 1u) acc[rt][i][x] += INFINITY;
                    if (least[rt] >> (4 * i + x) & 1u) acc[rt][i][x] -= INFINITY;
                }
        }
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
            merge_rows(pe, b, h0, hk, row0, rows_here, gate, sm_m, sm_l, sm_f);
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
                if (MERGED && w >= pe.k * pe.shard_waves) break;
                const float f = MERGED ? sm_f[w][g] : sm_m[w][g] == -INFINITY ? 0.0f : __expf(sm_m[w][g] - M);
                const float4 o = *reinterpret_cast<const float4 *>(sm_acc + (w * tile_rows + g) * AP + d);
                a.x = fmaf(o.x, f, a.x);
                a.y = fmaf(o.y, f, a.y);
                a.z = fmaf(o.z, f, a.z);
                a.w = fmaf(o.w, f, a.w);
                L = fmaf(sm_l[w][g], f, L);
            }
            if constexpr (MERGED) {
                float *to = pe.merge.y + query_row(pe, b, hk, row0 + g) * W + d;      // (y need not be 16-byte aligned)
                to[0] = a.x, to[1] = a.y, to[2] = a.z, to[3] = a.w;
            } else {
                const int64_t at = part_base + (rt * kRows + g) * part_row;
                *reinterpret_cast<float4 *>(pe.part_acc + at * W + d) = a;
                if (d == 0) *reinterpret_cast<float2 *>(pe.part_ml + at * 2) = make_float2(M, L);
            }
        }
    }
}

struct PagedPlan {
    int row_tiles, rows, row_blocks;      // matrix tiles and query rows of a block; row blocks of a kv head
    int nsplit, chunk;
    bool merged;               // one launch, no partials
    size_t acc_bytes, ml_bytes;
};

int make_plan(const pikv_desc *d, int k, bool positions, PagedPlan *plan) {
    const pikv_pages any = {1, 16, (int64_t)1 << 40, (int64_t)16 * (d ? d->D : 0), d ? d->D : 0};
    const int rc = check_paged(d, &any);
    if (rc != PIKV_OK) return rc;
    if (k < 1 || k > d->E) return PIKV_ERR_INVALID;
    const int G = d->Hq / d->Hkv, tq = d->tq > 1 ? d->tq : 1;
    const bool per_head = d->route_rows_per_seq != 1;
    if (tq > 1 && (per_head || d->Hq % tq != 0 || G % tq != 0)) return PIKV_ERR_UNSUPPORTED;
    const int stage = d->dtype == PIKV_F32 ? stage_entries<float> : stage_entries<bf16>;
    // (fp32 rows, and those of 128 values whose entries have positions, leave no registers for a second tile)
    plan->row_tiles = per_head || G <= kRows || d->dtype == PIKV_F32 || (positions && d->D == 128) ? 1 : kMostTiles;
    plan->rows = per_head ? 1 : G < plan->row_tiles * kRows ? G : plan->row_tiles * kRows;
    plan->row_blocks = (G + plan->rows - 1) / plan->rows;
    const int64_t units = (int64_t)d->B * d->Hkv * plan->row_blocks * k;
    // One launch or two.  One: where a block's waves get a stage each, and where its blocks, one on a CU, fill the CUs' rounds - 9 of 10 of
    // them, or 3 of 4 of a single one - with up to 4096 (1024) rows each; then the second launch and the partials cost more than blocks
    // of unequal length.  us, in one launch and in two, 8 kv heads of 4 rows, bf16, 2 shards of S full slots:
    //   128 values, S = 64 / 128:               8 blocks 6.3 : 7.4,  7.4 : 7.9;     192 blocks 6.6 : 9.6,  8.5 : 11.3
    //   128 values, S = 512 / 1024 / 2048:      192 blocks 22 : 26,  40 : 44,  75 : 68;     256 blocks 24 : 28,  44 : 46,  85 : 90;
    //                                           320 blocks 41 : 37,  74 : 62,  142 : 113;   640 blocks 67 : 64,  123 : 113,  235 : 221;
    //                                           1024 blocks 98 : 96,  173 : 179,  336 : 356
    //   shards of 0 .. S slots, 256 blocks:     19 : 22,  35 : 39,  66 : 66;   S = 4096: 114 : 99
    //   4 shards, with positions, 192 blocks:   S = 256  24 : 24,  512  44 : 39;   fp32, 640 blocks: S = 256  81 : 70
    const int64_t blocks = units / k, rows = (int64_t)k * d->S, places = (blocks + 255) / 256 * 256;
    const bool one_round = blocks <= 640 && (int64_t)d->S * (d->D > 64 ? d->D : 64) <= (int64_t)128 * stage * (kMergedWaves / k);
    const bool filled = blocks <= 1024 && ((10 * blocks >= 9 * places && rows <= 4096) || (blocks >= 192 && blocks <= 256 && rows <= 1024));
    plan->merged = plan->row_tiles == 1 && k <= kMergedWaves && (one_round || filled);
    // A block per CU, and blocks of at most 1024 rows, but none of fewer than a stage of each wave.
    int64_t nsplit = units > 0 ? 256 / units : 1;
    const int64_t finer = (d->S + kLongestBlock - 1) / kLongestBlock, most = (d->S + kWaves * stage - 1) / (kWaves * stage);
    if (nsplit < finer) nsplit = finer;
    if (plan->merged) nsplit = 1;
    if (nsplit > most) nsplit = most;
    if (nsplit > kMaxPartialsPerHead / k) nsplit = kMaxPartialsPerHead / k;
    if (nsplit < 1) nsplit = 1;
    int64_t chunk = (d->S + nsplit - 1) / nsplit;
    chunk = (chunk + stage - 1) / stage * stage;
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

size_t workspace_bytes(const PagedPlan &plan) { return plan.acc_bytes + plan.ml_bytes + 256; }

}  // namespace
}  // namespace pikv

using namespace pikv;

extern "C" size_t pikv_paged_attn_workspace_bytes(const pikv_desc *desc, int32_t k) {
    PagedPlan plan, positioned;
    if (make_plan(desc, k, false, &plan) != PIKV_OK || make_plan(desc, k, true, &positioned) != PIKV_OK) return 0;
    return workspace_bytes(plan) > workspace_bytes(positioned) ? workspace_bytes(plan) : workspace_bytes(positioned);
}

extern "C" int pikv_paged_attn(const pikv_desc *desc, const pikv_pages *pages, const void *q, const void *K_pool, const void *V_pool,
                               const int32_t *page_table, const int32_t *n_valid, const int32_t *topk_idx, const float *gates, int32_t k,
                               int32_t combine, float scale, float cap, const float *slopes, int32_t window, const int32_t *prefix,
                               const int32_t *entry_pos, const int32_t *q_pos, float *y, float *row_max, float *row_norm, float *scores,
                               float *slot_coef, void *workspace, size_t workspace_bytes_given, void *stream) {
    int rc = check_paged(desc, pages);
    if (rc != PIKV_OK) return rc;
    PagedPlan plan;
    rc = make_plan(desc, k, entry_pos != nullptr, &plan);
    if (rc != PIKV_OK) return rc;
    if (combine != PIKV_COMBINE_LSE && combine != PIKV_COMBINE_LOCAL) return PIKV_ERR_INVALID;
    if (!(scale - scale == 0.0f) || !(cap >= 0.0f) || !(cap - cap == 0.0f)) return PIKV_ERR_INVALID;
    if (!score_factors_finite(scale, desc->D, cap)) return PIKV_ERR_UNSUPPORTED;
    if ((entry_pos != nullptr) != (q_pos != nullptr) || ((slopes || window > 0 || prefix) && !entry_pos && desc->B > 0)) return PIKV_ERR_INVALID;
    if (desc->B == 0) return PIKV_OK;            // (tensors without elements have no address)
    if (!q || !K_pool || !V_pool || !page_table || !n_valid || !topk_idx || !y) return PIKV_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(K_pool) % 16 != 0 || reinterpret_cast<uintptr_t>(V_pool) % 16 != 0) return PIKV_ERR_INVALID;
    if (!workspace || workspace_bytes_given < workspace_bytes(plan)) return PIKV_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return PIKV_ERR_INVALID;
    const int tq = desc->tq > 1 ? desc->tq : 1;
    PagedAttnParams p;
    p.q = q;
    p.K = static_cast<const char *>(K_pool);
    p.V = static_cast<const char *>(V_pool);
    p.n_valid = n_valid;
    p.topk = topk_idx;
    p.prefix = prefix;
    p.entry_pos = entry_pos;
    p.q_pos = q_pos;
    p.slopes = slopes;
    p.part_acc = static_cast<float *>(workspace);
    p.part_ml = p.part_acc + plan.acc_bytes / sizeof(float);
    p.scores = scores;
    p.pages = page_geometry(desc, pages, page_table);
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
    p.window = window;
    p.nsplit_rcp = plan.nsplit > 1 ? (uint32_t)(((uint64_t)1 << 32) / plan.nsplit + 1) : 0u;
    p.scale = score_scale(scale, desc->D);
    p.cap = cap;
    p.cap_rcp = cap > 0.0f ? 1.0f / cap : 0.0f;
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
    auto launch = [&](auto type, auto width, auto tiles) {
        typedef decltype(type) T;
        constexpr int W = decltype(width)::value, RT = decltype(tiles)::value;
        auto go = [&](auto with, auto by_position) {
            constexpr bool SC = decltype(with)::value, POS = decltype(by_position)::value;
            if constexpr (RT == 1) {
                if (plan.merged) {
                    hipLaunchKernelGGL((paged_attn_partial<T, W, RT, SC, POS, kMergedWaves>), grid, threads, lds, st, p);
                    return;
                }
            }
            if constexpr (RT == 1 || !POS || W != 128) hipLaunchKernelGGL((paged_attn_partial<T, W, RT, SC, POS, kWaves>), grid, threads, lds, st, p);
        };
        auto positioned = [&](auto with) {
            if (entry_pos) go(with, std::true_type{});
            else go(with, std::false_type{});
        };
        if (scores) positioned(std::true_type{});
        else positioned(std::false_type{});
    };
    auto by_width = [&](auto type, auto tiles) {
        if (desc->D == 32) launch(type, std::integral_constant<int, 32>{}, tiles);
        else if (desc->D == 64) launch(type, std::integral_constant<int, 64>{}, tiles);
        else launch(type, std::integral_constant<int, 128>{}, tiles);
    };
    const std::integral_constant<int, 1> one{};
    if (desc->dtype == PIKV_F32) by_width(float{}, one);
    else if (plan.row_tiles == 1) by_width(bf16{}, one);
    else by_width(bf16{}, std::integral_constant<int, kMostTiles>{});
    rc = launch_status();
    if (rc != PIKV_OK || plan.merged) return rc;
    // (the merge's checks go by a descriptor of whole shards)
    pikv_desc whole = *desc;
    whole.stride_s = desc->D;
    whole.stride_h = (int64_t)desc->S * desc->D;
    return pikv_sharded_attn_merge(&whole, &c, stream);
}
