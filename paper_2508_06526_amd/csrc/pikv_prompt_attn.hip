// Attention of packed prompts among themselves, on the matrix cores.
//
// The queries of a kv head are rows (token, head of its group); a block takes 128 of them, 32 a wave, and walks the tiles of
// entries that any of them sees, K and V of a tile in LDS, the next tile on its way in registers.  Per wave and tile, lane (c, h) =
// (lane % 32, lane / 32):
//   * S^T[entry][row] = K . Q^T: the lane gets the scores of row c at entries 8 (i / 4) + 4 h + i % 4 of each 32, i = 0 .. 15, so that a
//     row's maximum and sum are the lane's own but for one exchange between the halves.
//   * Its weights are the operand P^T of the second product as they lie: the order of a contraction is free, and V^T's operand takes the
//     entries in the same order (bf16: transposing reads of 4 entries from LDS).
//   * O^T[d][row] += V^T . P^T.
// One pass with the running maximum and sum of the softmax (fp32).  bf16: a weight is rounded once, to bf16, on its way into the second
// product - half a step of 2^-8 of each, as the output's own rounding - the sum is of the unrounded ones.
#include "pikv_prompt_dev.h"

namespace pikv {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave, kRows = 32;      // rows of a wave

// LDS tiles of KEYS entries x D values, in 16-byte chunks, a row's chunks exchanged by an xor so that the reads of a wave spread over
// the banks: K is read as one chunk of 32 entries each, V (bf16) as 64 bytes of 4 neighbouring entries each.
template <typename T, int D>
struct Tile {
    static constexpr int KEYS = sizeof(T) == 2 ? 64 : 32;
    static constexpr int CHUNKS = D * (int)sizeof(T) / 16;            // of a row
    static constexpr int PER_THREAD = KEYS * CHUNKS / kThreads;       // of a tile
    static constexpr int PER_LINE = CHUNKS >= 16 ? 1 : 16 / CHUNKS;   // rows of 256 bytes
    static __device__ __forceinline__ int k_chunk(int key, int c) { return key * CHUNKS + (c ^ ((key / PER_LINE) & (CHUNKS < 16 ? CHUNKS - 1 : 15))); }
    static __device__ __forceinline__ int v_chunk(int key, int c) {
        if constexpr (sizeof(T) == 2) return key * CHUNKS + (c ^ (((key / PER_LINE) & (CHUNKS / 4 - 1)) << 2));
        else return key * CHUNKS + c;
    }
};

typedef short s16x4_lds __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 read_transposed(const void *at) {
    typedef __attribute__((address_space(3))) s16x4_lds *lds_ptr;
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)at));
}

__device__ __forceinline__ bool not_finite(float x) { return !(x - x == 0.0f); }

template <typename T, int D, bool CHANGED>
__global__ __launch_bounds__(kThreads, 2) void prompt_attn(PromptParams p) {
    typedef Tile<T, D> L;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int KEYS = L::KEYS, KB = KEYS / 32, DT = D / 32, BUFFERS = 2;
    constexpr int QN = D * (int)sizeof(T) / 32;                       // 16-byte pieces of a lane's query
    constexpr float kLog2e = 1.44269504088896340736f;
    __shared__ __attribute__((aligned(16))) uint4 Ks[BUFFERS][KEYS * L::CHUNKS], Vs[BUFFERS][KEYS * L::CHUNKS];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 31, h = lane >> 5;
    // the blocks with the most entries first
    int hk, b;
    const int rest = fast_divide(p.by_head, blockIdx.x, &hk);
    int at_tile = fast_divide(p.by_tile, rest, &b);                   // (by_tile: sequences)
    at_tile = p.tiles - 1 - at_tile;
    const Span span = prompt_span(p, b);
    const int n = span.n, rows = n * p.G, row0 = at_tile * kPromptTile;
    if (row0 >= rows) return;
    const int prefix = p.prefix ? __builtin_amdgcn_readfirstlane(min(max(p.prefix[b], 0), n)) : 0;
    const int last_token = row_token(p, min(row0 + kPromptTile, rows) - 1), first_token = row_token(p, row0);
    // tiles 0 .. prefix_tiles - 1, then window_tile .. last_tile
    const int prefix_tiles = (prefix + KEYS - 1) / KEYS;
    const int window_tile = max(prefix_tiles, p.window > 0 ? max(first_token - p.window + 1, 0) / KEYS : 0);
    const int last_tile = max(prefix_tiles - 1, last_token / KEYS);
    auto after = [&](int t) { return t + 1 < prefix_tiles ? t + 1 : max(t + 1, window_tile); };

    // the wave's rows
    const int wave_row = row0 + wave * kRows;
    const int row = min(wave_row + c, rows - 1), token = row_token(p, row), head = hk * p.G + row - token * p.G;
    const int wave_first = row_token(p, min(wave_row, rows - 1)), wave_last = row_token(p, min(wave_row + kRows, rows) - 1);
    const float slope = CHANGED && p.slopes ? p.slopes[head] : 0.0f;

    const char *Kb = static_cast<const char *>(p.k) + ((int64_t)span.first * p.k_stride + hk * D) * sizeof(T);
    const char *Vb = static_cast<const char *>(p.v) + ((int64_t)span.first * p.v_stride + hk * D) * sizeof(T);
    uint4 kr[L::PER_THREAD], vr[L::PER_THREAD];
    auto request = [&](int t) {
#pragma unroll
        for (int u = 0; u < L::PER_THREAD; ++u) {
            const int at = tid + u * kThreads, key = min(t * KEYS + at / L::CHUNKS, n - 1), chunk = at % L::CHUNKS;      // (past the end: the last entry again)
            kr[u] = load16(Kb + (int64_t)key * p.k_stride * sizeof(T) + chunk * 16);
            vr[u] = load16(Vb + (int64_t)key * p.v_stride * sizeof(T) + chunk * 16);
        }
    };
    auto place = [&](int buffer) {
#pragma unroll
        for (int u = 0; u < L::PER_THREAD; ++u) {
            const int at = tid + u * kThreads, key = at / L::CHUNKS, chunk = at % L::CHUNKS;
            Ks[buffer][L::k_chunk(key, chunk)] = kr[u];
            Vs[buffer][L::v_chunk(key, chunk)] = vr[u];
        }
    };
    int tile = prefix_tiles > 0 ? 0 : window_tile;
    request(tile);
    // the query operand: 16-byte pieces 2 s + h of row c
    uint4 q[QN];
    {
        const char *from = static_cast<const char *>(p.q) + ((int64_t)(span.first + token) * p.q_stride + (int64_t)head * D) * sizeof(T);
#pragma unroll
        for (int s = 0; s < QN; ++s) q[s] = load16(from + (2 * s + h) * 16);
    }
    f32x16_t acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
    float m = -INFINITY, l = 0.0f;       // of the products (CHANGED: of the scores)
    const float to_log2 = CHANGED ? kLog2e : p.scale * kLog2e;
    place(0);
    __syncthreads();
    int buffer = 0;
    for (; tile <= last_tile; buffer ^= 1) {
        const int next = after(tile), key0 = tile * KEYS;
        if (next <= last_tile) request(next);
        const bool in_prefix = key0 < prefix;
        const bool any = in_prefix || (key0 <= wave_last && (p.window <= 0 || wave_first - (key0 + KEYS - 1) < p.window));
        if (any) {
            float s[KB][16];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                f32x16_t sc;
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
#pragma unroll
                for (int u = 0; u < QN; ++u) {
                    const uint4 kop = Ks[buffer][L::k_chunk(kb * 32 + c, 2 * u + h)];
                    if constexpr (BF) {
                        sc = mfma32(kop, q[u], sc);
                    } else {
                        sc = mfma32(__uint_as_float(kop.x), __uint_as_float(q[u].x), sc);
                        sc = mfma32(__uint_as_float(kop.y), __uint_as_float(q[u].y), sc);
                        sc = mfma32(__uint_as_float(kop.z), __uint_as_float(q[u].z), sc);
                        sc = mfma32(__uint_as_float(kop.w), __uint_as_float(q[u].w), sc);
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kb][i] = sc[i];
                if constexpr (CHANGED) {
                    if (p.cap > 0.0f) cap_scores(s[kb], p.scale, p.cap, p.cap_rcp);
                    const float unit = p.cap > 0.0f ? 1.0f : p.scale;
                    const int first = key0 + kb * 32 + 4 * h - token;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[kb][i] = fmaf(-slope, fabsf((float)(first + 8 * (i >> 2) + (i & 3))), s[kb][i] * unit);
                }
            }
            // seen whole by all rows of the wave, or not
            const bool masked = !(key0 + KEYS <= n && (key0 + KEYS <= prefix || (key0 + KEYS - 1 <= wave_first &&
                                                                                (p.window <= 0 || wave_last - key0 < p.window))));
            auto seen = [&](int key) {
                return key < n && (key < prefix || (key <= token && (p.window <= 0 || token - key < p.window)));
            };
            if (masked) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (!seen(key0 + kb * 32 + 8 * (i >> 2) + 4 * h + (i & 3))) s[kb][i] = -INFINITY;
            }
            float most = s[0][0];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) most = fmaxf(most, s[kb][i]);
            const float now = fmaxf(m, halves_max(most));
            const float base = now == -INFINITY ? 0.0f : now;        // (nothing seen yet: weights of zero)
            if (__any(now > m)) {
                const float corr = __builtin_amdgcn_exp2f((m - base) * to_log2);
                m = now;
                l *= corr;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[d][i] *= corr;
            }
            float sum = 0.0f;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[kb][i] = __builtin_amdgcn_exp2f((s[kb][i] - base) * to_log2);
                    sum += s[kb][i];
                }
            l += sum;
            // A value that is no number stays out of the rows that do not see its entry: 0 x NaN is NaN.  (Rare; found per tile.)
            bool odd = false;
            if (masked) {
                uint32_t most_exponent = 0;
                const uint32_t *words = reinterpret_cast<const uint32_t *>(Vs[buffer]);
                for (int i = lane; i < KEYS * L::CHUNKS * 4; i += kWave) {
                    const uint32_t w = words[i] & 0x7fffffffu;
                    most_exponent = max(most_exponent, BF ? max(w >> 16, w & 0x7fffu) : w);
                }
                odd = __any(most_exponent >= (BF ? 0x7f80u : 0x7f800000u));
            }
            auto finite = [&](uint32_t w) {      // bf16: two values; those that are no numbers become zero
                if constexpr (BF) return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
                else return (w & 0x7f800000u) == 0x7f800000u ? 0u : w;
            };
            if constexpr (BF) {
                const char *Vt = reinterpret_cast<const char *>(Vs[buffer]);
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int st = 0; st < 2; ++st) {
                        uint4 pop[1];
                        split_bf16(&s[kb][8 * st], pop);
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            // 16 lanes read 4 entries x 16 values: lane g of them entry g / 4, values 4 (g % 4) ..
                            const int g = lane & 15, key = kb * 32 + 16 * st + 4 * h + (g >> 2), value = d * 32 + (lane & 16) + 4 * (g & 3);
                            uint2 lo = read_transposed(Vt + L::v_chunk(key, value >> 3) * 16 + (value & 7) * 2);
                            uint2 hi = read_transposed(Vt + L::v_chunk(key + 8, value >> 3) * 16 + (value & 7) * 2);
                            if (odd) lo = make_uint2(finite(lo.x), finite(lo.y)), hi = make_uint2(finite(hi.x), finite(hi.y));
                            acc[d] = mfma32(make_uint4(lo.x, lo.y, hi.x, hi.y), pop[0], acc[d]);
                        }
                    }
            } else {
                const float *Vt = reinterpret_cast<const float *>(Vs[buffer]);
#pragma unroll
                for (int i = 0; i < 16; ++i)
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        float v = Vt[(8 * (i >> 2) + 4 * h + (i & 3)) * D + d * 32 + c];
                        if (odd) v = __uint_as_float(finite(__float_as_uint(v)));
                        acc[d] = mfma32(v, s[0][i], acc[d]);
                    }
            }
            if (odd) {
                for (int key = 0; key < KEYS; ++key) {
                    if (!seen(key0 + key)) continue;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int value = d * 32 + 8 * (i >> 2) + 4 * h + (i & 3), per = 16 / (int)sizeof(T);
                            const T *chunk = reinterpret_cast<const T *>(&Vs[buffer][L::v_chunk(key, value / per)]);
                            const float v = load_scalar<T>(chunk, value % per);
                            if (not_finite(v)) acc[d][i] += v;
                        }
                }
            }
        }
        if (next <= last_tile) place(buffer ^ 1);
        __syncthreads();
        tile = next;
    }
    l = halves_sum(l);
    if (wave_row + c >= rows) return;
    const int64_t to = (int64_t)(span.first + token) * p.Hq + head;
    if (p.row_max && h == 0) {
        p.row_max[to] = CHANGED ? m : m * p.scale;
        p.row_norm[to] = l;
    }
    const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;    // (a NaN stays one)
    T *out = static_cast<T *>(p.out) + to * D;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = acc[d][4 * u + x] * inv;
            T *at = out + d * 32 + 8 * u + 4 * h;
            if constexpr (BF) {
                uint2 packed[1];
                split_bf16(v, packed);
                *reinterpret_cast<uint2 *>(at) = packed[0];
            } else {
                *reinterpret_cast<float4 *>(at) = make_float4(v[0], v[1], v[2], v[3]);
            }
        }
}

}  // namespace
}  // namespace pikv

using namespace pikv;

extern "C" int pikv_prompt_attn(const void *q, const void *k, const void *v, int32_t tokens, int64_t q_stride, int64_t k_stride,
                                int64_t v_stride, int32_t Hq, int32_t Hkv, int32_t D, int32_t dtype, const int32_t *cu_seqlens,
                                int32_t B, int32_t max_len, const int32_t *prefix, float scale, float cap, const float *slopes,
                                int32_t window, void *out, float *row_max, float *row_norm, void *stream) {
    const int rc = check_prompt(q, k, v, true, tokens, q_stride, k_stride, v_stride, Hq, Hkv, D, dtype, B, max_len, scale, cap);
    if (rc != PIKV_OK) return rc;
    if ((row_max != nullptr) != (row_norm != nullptr)) return PIKV_ERR_INVALID;
    if (max_len > tokens) max_len = tokens;
    const int G = Hq / Hkv;
    const int64_t tiles = prompt_tiles((int64_t)max_len * G);
    if ((int64_t)B * Hkv * tiles >= (1 << 23)) return PIKV_ERR_UNSUPPORTED;
    if (tokens == 0 || B == 0 || max_len == 0) return PIKV_OK;       // (tensors without elements have no address)
    if (!q || !k || !v || !cu_seqlens || !out || reinterpret_cast<uintptr_t>(out) % 16 != 0) return PIKV_ERR_INVALID;
    PromptParams p = prompt_params(q, k, tokens, q_stride, k_stride, Hq, Hkv, D, cu_seqlens, B, max_len, prefix, scale, cap, slopes, window);
    p.v = v;
    p.v_stride = v_stride;
    p.out = out;
    p.row_max = row_max;
    p.row_norm = row_norm;
    p.by_head = fast_div(Hkv);
    p.by_tile = fast_div(B);
    p.tiles = (int)tiles;
    const dim3 grid((unsigned)(B * Hkv * tiles)), threads(kThreads);
    hipStream_t st = as_stream(stream);
    auto launch = [&](auto type, auto width) {
        typedef decltype(type) T;
        constexpr int W = decltype(width)::value;
        if (cap > 0.0f || slopes) hipLaunchKernelGGL((prompt_attn<T, W, true>), grid, threads, 0, st, p);
        else hipLaunchKernelGGL((prompt_attn<T, W, false>), grid, threads, 0, st, p);
    };
    auto by_width = [&](auto type) {
        if (D == 32) launch(type, std::integral_constant<int, 32>{});
        else if (D == 64) launch(type, std::integral_constant<int, 64>{});
        else launch(type, std::integral_constant<int, 128>{});
    };
    if (dtype == PIKV_F32) by_width(float{});
    else by_width(bf16{});
    return launch_status();
}
