// What the calls on packed prompts share: arguments, masks, changed scores.
#pragma once

#include "pikv_mfma_dev.h"
#include "pikv_scores_dev.h"

#include <math.h>

namespace pikv {

struct PromptParams {
    const void *q, *k, *v;
    const int32_t *cu, *prefix;
    const float *slopes;
    void *out;
    float *row_max, *row_norm;          // pikv_prompt_mass: inputs
    float *mass, *parts;
    int64_t q_stride, k_stride, v_stride;
    FastDiv by_head, by_tile, by_split;
    uint32_t G_rcp;                     // 2^32 / G, rounded up: a row of a kv head's queries / G
    int tokens, max_len, Hq, Hkv, G, B, window, tiles, nsplit;
    float scale, cap, cap_rcp;
    float unit, unit_log2, margin;      // pikv_prompt_attn: of the scores as they are kept
};

// row / G for 0 <= row < 2^31: rows of a kv head are (token, head of the group).  (G_rcp is at most 2^32 / G + 1: for such rows the product is the
// quotient or one more.)
__device__ __forceinline__ int row_token(const PromptParams &p, int row) {
    if (p.G == 1) return row;
    int t = (int)__umulhi((uint32_t)row, p.G_rcp);
    if (t * p.G > row) --t;              // (the reciprocal is rounded up)
    return t;
}

// What block `id` takes: its tile (0 .. tiles - 1; counted down for `last_first`), kv head and sequence.  Blocks go to the XCDs in turn, so
// that the heads of a sequence stay on one where there are 8; the sequences are turned by one from tile to tile, or where there are fewer
// heads an XCD would get all blocks of a long one (4 ragged prompts of up to 4001 tokens, 4 kv heads: 275 us
// without turning them, 183 with).
__device__ __forceinline__ int prompt_block(const PromptParams &p, int id, bool last_first, int *hk, int *b) {
    id = fast_divide(p.by_head, id, hk);
    int tile = fast_divide(p.by_tile, id, b), turn;              // (by_tile: sequences)
    if (last_first) tile = p.tiles - 1 - tile;
    fast_divide(p.by_tile, tile, &turn);
    *b += turn;
    if (*b >= p.B) *b -= p.B;
    return tile;
}

struct Span {
    int first, n;                        // the sequence's rows; n: those below max_len
};
__device__ __forceinline__ Span prompt_span(const PromptParams &p, int b) {
    const int lo = min(max(p.cu[b], 0), p.tokens), hi = min(max(p.cu[b + 1], lo), p.tokens);
    return {__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(min(hi - lo, p.max_len))};
}

typedef float f32x16_t __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16_t mfma32(uint4 a, uint4 b, f32x16_t acc) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mfma32(float a, float b, f32x16_t acc) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, acc, 0, 0, 0); }

// Max and sum over the lanes c and c + 32, in both.
__device__ __forceinline__ float halves_max(float x) {
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}

// Checks common to the calls on prompts; `values`: v and out are there too.
inline int check_prompt(const void *q, const void *k, const void *v, bool values, int tokens, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                        int Hq, int Hkv, int D, int dtype, int B, int max_len, float scale, float cap) {
    if (tokens < 0 || B < 0 || max_len < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return PIKV_ERR_INVALID;
    if (dtype != PIKV_F32 && dtype != PIKV_BF16) return PIKV_ERR_INVALID;
    if (!(scale - scale == 0.0f) || !(cap >= 0.0f) || !(cap - cap == 0.0f)) return PIKV_ERR_INVALID;
    if ((D != 32 && D != 64 && D != 128) || Hq > 256 || tokens > (1 << 23)) return PIKV_ERR_UNSUPPORTED;
    if (!score_factors_finite(scale, D, cap)) return PIKV_ERR_UNSUPPORTED;
    const int es = elem_bytes(dtype);
    auto rows = [&](const void *p, int64_t stride, int heads) {
        return stride >= (int64_t)heads * D && stride * es % 16 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0;
    };
    // (64 rows are addressed with 32 bits)
    const int64_t most = (1 << 25) / es;
    if (q_stride > most || k_stride > most || (values && v_stride > most)) return PIKV_ERR_UNSUPPORTED;
    if (!rows(q, q_stride, Hq) || !rows(k, k_stride, Hkv) || (values && !rows(v, v_stride, Hkv))) return PIKV_ERR_INVALID;
    return PIKV_OK;
}

inline PromptParams prompt_params(const void *q, const void *k, int tokens, int64_t q_stride, int64_t k_stride, int Hq, int Hkv, int D,
                                  const int32_t *cu, int B, int max_len, const int32_t *prefix, float scale, float cap, const float *slopes,
                                  int window) {
    PromptParams p{};
    p.q = q;
    p.k = k;
    p.cu = cu;
    p.prefix = prefix;
    p.slopes = slopes;
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.G = Hq / Hkv;
    p.G_rcp = p.G > 1 ? (uint32_t)(((uint64_t)1 << 32) / p.G + 1) : 0u;
    p.tokens = tokens;
    p.max_len = max_len;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.B = B;
    p.window = window;
    p.scale = score_scale(scale, D);
    p.cap = cap;
    p.cap_rcp = cap > 0.0f ? 1.0f / cap : 0.0f;
    return p;
}

constexpr int kPromptTile = 128;         // rows (or entries) of a block
inline int64_t prompt_tiles(int64_t rows) { return (rows + kPromptTile - 1) / kPromptTile; }

}  // namespace pikv
