// Pieces of the split decode kernels over 8-bit and paged shards: requests, query rows, the merge inside a block.
#pragma once

#include "pikv_common.h"

#include <math.h>

namespace pikv {

constexpr int kRows = 16;               // query rows of a matrix tile
constexpr int kMergedWaves = 8;         // of a block that takes all shards of its rows

// Where the caller keeps query row `row` of kv head hk (rows of a kv head: draft query, head of the group).
template <typename PARAMS>
__device__ __forceinline__ int64_t query_row(const PARAMS &p, int b, int hk, int row) {
    if (p.tq <= 1) return (int64_t)b * p.Hq + hk * p.G + row;
    const int g = (int)p.by_draft.d;
    int t = (int)__umulhi((uint32_t)row, p.by_draft.rcp), gg = row - t * g;      // t: the quotient or one less
    if (gg >= g) ++t, gg -= g;
    return (int64_t)b * p.Hq + t * p.heads + hk * g + gg;
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

// The merge of a block that holds all selected shards of its rows: 8 lanes a row, lane w with wave w's (max, sum) pair.  A
// shard's waves are 8, 4, 2 or 1 neighbours: joined by an xor butterfly, then the shards with their gates (as head_weights, in
// both combine modes).  Leaves every wave's factor.
template <typename PARAMS>
__device__ __forceinline__ void merge_rows(const PARAMS &p, int b, int h0, int hk, int row0, int rows, float gate, const float (&m)[kMergedWaves][kRows],
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

}  // namespace pikv
