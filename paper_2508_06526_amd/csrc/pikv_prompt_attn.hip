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
// product - half a step of 2^-8 of each, as the output's own rounding - the sum is of the unrounded ones.  (Two parts instead, 16 bits: error
// against 64 bits 0.0021 -> 0.0016 of the values, which is the output's rounding alone, and half as many products again: 16384 tokens 2250 -> 2970 us, in a
// window 147 -> 168.)
//
// 16384 tokens, 32 heads over 8 of 128 bf16 values: 2240 - 2450 us by the card, 900 - 980 TFLOP/s; the matrix pipe is busy 44 % of the cycles, the softmax's instructions most of the
// others, and two waves a SIMD (registers) overlap the two as they come.  In a window of 1024 with capped scores (4 prompts of up to 4001, 16 heads over 4)
// 147 us; 57 tokens 7.3 us, fp32 documents of up to 403 tokens 20.7 (capped scores, each in the form for its size: 143 and 18.7 with one form for a wave).  32 rows a wave and 64 entries a tile are what 256 registers hold at 128
// values: tiles of 32 entries take 2630 us, 64 rows a wave (512 registers) 3930.
#include "pikv_decode_dev.h"
#include "pikv_prompt_dev.h"

namespace pikv {
namespace {

constexpr int kWaveRows = 32;            // rows of a wave
// Waves of a block of many rows.  (8 waves halve the way of a tile into LDS for each row, and wait for each other: 16384 tokens of 128 values 2269 us
// against 2325, of 64 values 1681 against 1363, 16 x 1024 tokens 240 against 219, ragged prompts in a window 167 against 153.)
constexpr int kWaves = 4;
constexpr int kMostWaves = 8;            // of a block that splits the tiles of its rows

// LDS tiles of KEYS entries x D values, in 16-byte chunks, a row's chunks exchanged by an xor so that the reads of a wave spread over
// the banks: K is read as one chunk of 32 entries each, V (bf16) as 64 bytes of 4 neighbouring entries each.
template <typename T, int D, int SPLIT>
struct Tile {
    static constexpr int KEYS = sizeof(T) == 2 && !SPLIT ? 64 : 32;
    static constexpr int THREADS = SPLIT ? kWave : kWaves * kWave;    // that bring a tile
    static constexpr int CHUNKS = D * (int)sizeof(T) / 16;            // of a row
    static constexpr int PER_THREAD = KEYS * CHUNKS / THREADS;        // of a tile
    static constexpr int PER_LINE = CHUNKS >= 16 ? 1 : 16 / CHUNKS;   // rows of 256 bytes
    static constexpr __device__ __forceinline__ int k_exchange(int key) { return (key / PER_LINE) & (CHUNKS < 16 ? CHUNKS - 1 : 15); }
    static constexpr __device__ __forceinline__ int v_exchange(int key) { return sizeof(T) == 2 ? ((key / PER_LINE) & (CHUNKS / 4 - 1)) << 2 : 0; }
    static __device__ __forceinline__ int k_chunk(int key, int c) { return key * CHUNKS + (c ^ k_exchange(key)); }
    static __device__ __forceinline__ int v_chunk(int key, int c) { return key * CHUNKS + (c ^ v_exchange(key)); }
};

typedef short s16x4_lds __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 read_transposed(const void *at) {
    typedef __attribute__((address_space(3))) s16x4_lds *lds_ptr;
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)at));
}

// CAP: scores capped by a tanh; BIAS: with a distance term.  SPLIT: for few rows, a block takes 32 of them and its waves every SPLIT-th tile each, by
// themselves; their results are joined at the end.
template <typename T, int D, bool CAP, bool BIAS, int SPLIT>
__global__ __launch_bounds__((SPLIT ? SPLIT : kWaves) * kWave, (SPLIT == kWaves && D == 128 ? 1 : 2)) void prompt_attn(PromptParams p) {
    typedef Tile<T, D, SPLIT> L;
    constexpr int WAVES = SPLIT ? SPLIT : kWaves, ROWS = SPLIT ? kWaveRows : WAVES * kWaveRows, THREADS = L::THREADS;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int KEYS = L::KEYS, KB = KEYS / 32, DT = D / 32, BUFFERS = SPLIT ? WAVES : 2, STEP = SPLIT ? WAVES : 1;
    constexpr int QN = D * (int)sizeof(T) / 32;                       // 16-byte pieces of a lane's query
    __shared__ __attribute__((aligned(16))) uint4 Ks[BUFFERS][KEYS * L::CHUNKS], Vs[BUFFERS][KEYS * L::CHUNKS];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 31, h = lane >> 5;
    int hk, b;
    const int at_tile = prompt_block(p, blockIdx.x, true, &hk, &b);      // (the blocks with the most entries first)
    const Span span = prompt_span(p, b);
    const int n = span.n, rows = n * p.G, row0 = at_tile * ROWS;
    if (row0 >= rows) return;
    const int prefix = p.prefix ? __builtin_amdgcn_readfirstlane(min(max(p.prefix[b], 0), n)) : 0;
    const int last_token = row_token(p, min(row0 + ROWS, rows) - 1), first_token = row_token(p, row0);
    // tiles 0 .. prefix_tiles - 1, then window_tile .. last_tile
    const int prefix_tiles = (prefix + KEYS - 1) / KEYS;
    const int window_tile = max(prefix_tiles, p.window > 0 ? max(first_token - p.window + 1, 0) / KEYS : 0);
    const int last_tile = max(prefix_tiles - 1, last_token / KEYS), count = prefix_tiles + max(last_tile - window_tile + 1, 0);
    auto tile_at = [&](int i) { return i < prefix_tiles ? i : i - prefix_tiles + window_tile; };

    // the wave's rows
    const int wave_row = row0 + (SPLIT ? 0 : wave) * kWaveRows;
    const int row = min(wave_row + c, rows - 1), token = row_token(p, row), head = hk * p.G + row - token * p.G;
    const int wave_first = row_token(p, min(wave_row, rows - 1)), wave_last = row_token(p, min(wave_row + kWaveRows, rows) - 1);
    // Scores are kept as they come: products (capped: parts of the cap) that p.unit makes scores of, or with a distance term scores.
    const float to_log2 = p.unit_log2, slope = BIAS ? p.slopes[head] : 0.0f;

    const int64_t k_bytes = p.k_stride * (int64_t)sizeof(T), v_bytes = p.v_stride * (int64_t)sizeof(T);
    const char *Kb = static_cast<const char *>(p.k) + span.first * k_bytes + hk * D * (int)sizeof(T);
    const char *Vb = static_cast<const char *>(p.v) + span.first * v_bytes + hk * D * (int)sizeof(T);
    auto opaque = [](uint32_t v) {           // (else an address per read is carried through the loop)
        asm volatile("" : "+v"(v));
        return v;
    };
    uint32_t kr[L::PER_THREAD][4], vr[L::PER_THREAD][4];
    // A tile's rows; those past the end read as zeros.
    auto request = [&](uint32_t (&to)[L::PER_THREAD][4], const char *base, int64_t stride, int t) {
        const int here = min(n - t * KEYS, KEYS);
        const auto from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base + t * KEYS * stride), 0, (uint32_t)(here - 1) * (uint32_t)stride + D * (int)sizeof(T), 0x00020000);
        const int tid = (int)opaque(threadIdx.x) & (THREADS - 1);
        const uint32_t at = (tid / L::CHUNKS) * (uint32_t)stride + (tid % L::CHUNKS) * 16;
#pragma unroll
        for (int u = 0; u < L::PER_THREAD; ++u) buffer_load<16, false>(to[u], from, at + u * (THREADS / L::CHUNKS) * (uint32_t)stride);
    };
    // Whether rows first .. last of tokens see all entries of a tile.
    auto seen_whole = [&](int t, int first, int last) {
        const int key0 = t * KEYS;
        return key0 + KEYS <= n && (key0 + KEYS <= prefix || (key0 + KEYS - 1 <= first && (p.window <= 0 || last - key0 < p.window)));
    };
    // A value that is no number stays out of the rows that do not see its entry: 0 x NaN is NaN.  Where a tile is not seen whole such
    // values go to LDS as zeros, and the block is told (rare).
    auto place = [&](int t, int buffer) {
        auto special = [](uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; };
        bool bad = false;
        if (!seen_whole(t, first_token, last_token)) {
#pragma unroll
            for (int u = 0; u < L::PER_THREAD; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t w = opaque(vr[u][i]);     // (else its masking, which the branch below has too, is done for every tile)
                    bad |= special(w) || (BF && special(w << 16));
                }
        }
        // pieces tid, tid + THREADS, ..: the exchange of rows tid / CHUNKS + u LINES is that of either
        constexpr int LINES = THREADS / L::CHUNKS;
        const int tid = (int)opaque(threadIdx.x) & (THREADS - 1);
        const uint32_t to_k = L::k_chunk(tid / L::CHUNKS, tid % L::CHUNKS) * 16 + buffer * (int)sizeof(Ks[0]);
        const uint32_t to_v = L::v_chunk(tid / L::CHUNKS, tid % L::CHUNKS) * 16 + buffer * (int)sizeof(Vs[0]);
        auto write_v = [&](auto of) {
#pragma unroll
            for (int u = 0; u < L::PER_THREAD; ++u)
                *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(Vs) + ((to_v ^ (L::v_exchange(u * LINES) * 16)) + u * THREADS * 16)) =
                    make_uint4(of(vr[u][0]), of(vr[u][1]), of(vr[u][2]), of(vr[u][3]));
        };
#pragma unroll
        for (int u = 0; u < L::PER_THREAD; ++u)
            *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(Ks) + ((to_k ^ (L::k_exchange(u * LINES) * 16)) + u * THREADS * 16)) =
                make_uint4(kr[u][0], kr[u][1], kr[u][2], kr[u][3]);
        if (__any(bad))
            write_v([&](uint32_t w) { return (special(w) ? 0u : w & (BF ? 0xffff0000u : 0xffffffffu)) | (BF && !special(w << 16) ? w & 0xffffu : 0u); });
        else
            write_v([](uint32_t w) { return w; });
        return bad;
    };
    auto placed = [&](int t, bool bad) {         // the barrier behind it: whether the tile held any
        if constexpr (SPLIT) {
            wave_lds_order();
            return __any(bad) != 0;
        } else {
            if (!seen_whole(t, first_token, last_token)) return __syncthreads_or(bad) != 0;
            __syncthreads();
            return false;
        }
    };
    int at = SPLIT ? wave : 0, buffer = SPLIT ? wave : 0;
    if (!SPLIT || at < count) {
        request(kr, Kb, k_bytes, tile_at(at));
        request(vr, Vb, v_bytes, tile_at(at));
    }
    // the query operand: 16-byte pieces 2 s + h of row c
    uint4 q[QN];
    {
        const char *from = static_cast<const char *>(p.q) + ((int64_t)(span.first + token) * p.q_stride + (int64_t)head * D) * sizeof(T);
#pragma unroll
        for (int s = 0; s < QN; ++s) q[s] = load16(from + (2 * s + h) * 16);
    }
#pragma unroll
    for (int s = 0; s < QN; ++s) hold_operand(q[s]);         // complete here, not behind requests in the loop
    f32x16_t acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
    // The maximum of the lane's scores so far; what they are taken relative to, which follows it only when a weight would pass 2^8:
    // most tiles then leave the accumulators alone.
    float top = -INFINITY, base = -INFINITY, shift = 0.0f, l = 0.0f;        // shift: base, 0 while nothing has been seen
    // accumulators that get an infinity at the end (a NaN: both), 32 to a word
    constexpr int WORDS = (DT * 16 + 31) / 32;
    uint32_t most_inf[WORDS] = {}, least_inf[WORDS] = {};
    bool odd = (!SPLIT || at < count) && placed(tile_at(at), place(tile_at(at), buffer));
    for (; at < count; at += STEP) {
        const int tile = tile_at(at), next = tile_at(at + STEP), key0 = tile * KEYS;
        const bool more = at + STEP < count;
        const int lane = (int)opaque(tid) & (kWave - 1), c = lane & 31, h = lane >> 5;      // (derived again in every round: registers)
        if (more) request(kr, Kb, k_bytes, next);
        const bool in_prefix = key0 < prefix;
        const bool any = in_prefix || (key0 <= wave_last && (p.window <= 0 || wave_first - (key0 + KEYS - 1) < p.window));
        if (any) {
            float s[KB][16];
            // chunk 2 u + h of entry c, exchanged: the exchange of chunk h with 2 u's bits on top
            const uint32_t k_at = opaque(L::k_chunk(c, h) * 16 + buffer * (int)sizeof(Ks[0]));
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                f32x16_t sc;
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
#pragma unroll
                for (int u = 0; u < QN; ++u) {
                    const uint4 kop = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(Ks) + ((k_at ^ (u * 32)) + kb * 32 * L::CHUNKS * 16));
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
                if constexpr (CAP) cap_parts(s[kb], p.scale * p.cap_rcp);
                if constexpr (BIAS) {
                    const int first = key0 + kb * 32 + 4 * h - token;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[kb][i] = fmaf(-slope, fabsf((float)(first + 8 * (i >> 2) + (i & 3))), s[kb][i] * (CAP ? p.cap : p.scale));
                }
            }
            if (more) request(vr, Vb, v_bytes, next);       // (behind the first product: its registers)
            const bool masked = !seen_whole(tile, wave_first, wave_last);
            // the lane's row sees entries low .. token and those below the prefix
            const int low = p.window > 0 ? max(token - p.window + 1, 0) : 0;
            auto seen = [&](int key) { return ((uint32_t)(key - low) <= (uint32_t)(token - low)) | (key < prefix); };
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
            top = fmaxf(top, most);
            if (__any(most > base + p.margin)) {
                // (rows of which this holds: the others keep theirs, so that no row's roundings hang on those beside it)
                const float highest = halves_max(fmaxf(top, base)), now = highest > base + p.margin ? highest : base;
                const float next_shift = now == -INFINITY ? 0.0f : now;
                const float corr = __builtin_amdgcn_exp2f((base - next_shift) * to_log2);
                base = now;
                shift = next_shift;
                l *= corr;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[d][i] *= corr;
            }
            float sum = 0.0f;
            const float shift_log2 = -shift * to_log2;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    // (bf16: one rounding less to spare, one operation less)
                    s[kb][i] = __builtin_amdgcn_exp2f(BF ? fmaf(s[kb][i], to_log2, shift_log2) : (s[kb][i] - shift) * to_log2);
                    sum += s[kb][i];
                }
            l += sum;
            if constexpr (BF) {
                // 16 lanes read 4 entries x 16 values: lane g of them entry g / 4, values 4 (g % 4) .. of the 16 (lane & 16 ..)
                const int g = lane & 15, value = (lane & 16) + 4 * (g & 3);
                const uint32_t v_at = opaque(L::v_chunk(4 * h + (g >> 2), value >> 3) * 16 + (value & 7) * 2 + buffer * (int)sizeof(Vs[0]));
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int st = 0; st < 2; ++st) {
                        uint4 pop[1];
                        split_bf16(&s[kb][8 * st], pop);
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const char *at = reinterpret_cast<const char *>(Vs) + ((v_at ^ (d * 64)) + (kb * 32 + 16 * st) * L::CHUNKS * 16);
                            const uint2 lo = read_transposed(at), hi = read_transposed(at + 8 * L::CHUNKS * 16);
                            acc[d] = mfma32(make_uint4(lo.x, lo.y, hi.x, hi.y), pop[0], acc[d]);
                        }
                    }
            } else {
                const float *Vt = reinterpret_cast<const float *>(Vs[buffer]);
#pragma unroll
                for (int i = 0; i < 16; ++i)
#pragma unroll
                    for (int d = 0; d < DT; ++d) acc[d] = mfma32(Vt[(8 * (i >> 2) + 4 * h + (i & 3)) * D + d * 32 + c], s[0][i], acc[d]);
            }
            if (odd) {
                for (int key = key0; key < min(key0 + KEYS, n); ++key) {
                    if (!seen(key)) continue;
                    const T *row = reinterpret_cast<const T *>(Vb + key * v_bytes);
#pragma unroll
                    for (int j = 0; j < DT * 16; ++j) {
                        const float v = load_scalar<T>(row, (j >> 4) * 32 + 8 * (j >> 2 & 3) + 4 * h + (j & 3));
                        most_inf[j / 32] |= v == INFINITY || v != v ? 1u << (j & 31) : 0u;
                        least_inf[j / 32] |= v == -INFINITY || v != v ? 1u << (j & 31) : 0u;
                        if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);       // (all at once they cost registers of the whole loop)
                    }
                }
            }
        }
        if (!any && more) request(vr, Vb, v_bytes, next);
        if constexpr (SPLIT) wave_lds_order();       // (the tile's reads before the next one's writes)
        else buffer ^= 1;
        odd = more && placed(next, place(next, buffer));
    }
    bool any_inf = false;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) any_inf |= (most_inf[w] | least_inf[w]) != 0u;
    if (__any(any_inf)) {
#pragma unroll
        for (int j = 0; j < DT * 16; ++j) {
            if (most_inf[j / 32] >> (j & 31) & 1u) acc[j >> 4][j & 15] += INFINITY;
            if (least_inf[j / 32] >> (j & 31) & 1u) acc[j >> 4][j & 15] -= INFINITY;
        }
    }
    l = halves_sum(l);
    top = halves_max(top);
    // (found again: not carried through the loop)
    const int my_lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), my_c = my_lane & 31, my_h = my_lane >> 5;
    const int my_row = wave_row + my_c, my_token = row_token(p, my_row);
    const int64_t to = (int64_t)(span.first + my_token) * p.Hq + hk * p.G + my_row - my_token * p.G;
    auto write_stats = [&] {
        if (p.row_max && my_h == 0) {
            p.row_max[to] = top * p.unit;
            p.row_norm[to] = l * __builtin_amdgcn_exp2f((shift - (top == -INFINITY ? 0.0f : top)) * to_log2);
        }
    };
    auto inverse = [&] { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; };       // (a NaN stays one)
    auto write4 = [&](int j, const float (&v)[4]) {          // accumulators j .. j + 3
        T *at = static_cast<T *>(p.out) + to * D + (j >> 4) * 32 + 8 * (j >> 2 & 3) + 4 * my_h;
        if constexpr (BF) {
            uint2 packed[1];
            split_bf16(v, packed);
            *reinterpret_cast<uint2 *>(at) = packed[0];
        } else {
            *reinterpret_cast<float4 *>(at) = make_float4(v[0], v[1], v[2], v[3]);
        }
    };
    if constexpr (SPLIT) {
        // the waves' accumulators over their tiles in LDS; each wave joins its part of them
        constexpr int N = DT * 16, MINE = N / WAVES;
        static_assert(WAVES * N * kWave * 4 <= (int)(sizeof(Ks) + sizeof(Vs)) && N % WAVES == 0, "joined where the tiles were");
        __shared__ float base_s[WAVES][kWaveRows], l_s[WAVES][kWaveRows], top_s[WAVES][kWaveRows];
        __syncthreads();
        float *mine = reinterpret_cast<float *>(wave < WAVES / 2 ? &Ks[0][0] : &Vs[0][0]) + (wave % (WAVES / 2)) * N * kWave;
#pragma unroll
        for (int j = 0; j < N; ++j) mine[j * kWave + my_lane] = acc[j >> 4][j & 15];
        if (my_h == 0) {
            base_s[wave][my_c] = base;
            l_s[wave][my_c] = l;
            top_s[wave][my_c] = top;
        }
        __syncthreads();
        base = top = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            base = fmaxf(base, base_s[w][my_c]);
            top = fmaxf(top, top_s[w][my_c]);
        }
        shift = base == -INFINITY ? 0.0f : base;
        l = 0.0f;
        float v[MINE] = {};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float factor = __builtin_amdgcn_exp2f((base_s[w][my_c] - shift) * to_log2);
            l = fmaf(l_s[w][my_c], factor, l);
            const float *from = reinterpret_cast<const float *>(w < WAVES / 2 ? &Ks[0][0] : &Vs[0][0]) + ((w % (WAVES / 2)) * N + wave * MINE) * kWave;
#pragma unroll
            for (int j = 0; j < MINE; ++j) v[j] = fmaf(from[j * kWave + my_lane], factor, v[j]);
        }
        if (my_row >= rows) return;
        if (wave == 0) write_stats();
        const float inv = inverse();
#pragma unroll
        for (int j = 0; j < MINE; j += 4) {
            const float four[4] = {v[j] * inv, v[j + 1] * inv, v[j + 2] * inv, v[j + 3] * inv};
            write4(wave * MINE + j, four);
        }
    } else {
        if (my_row >= rows) return;
        write_stats();
        const float inv = inverse();
#pragma unroll
        for (int j = 0; j < DT * 16; j += 4) {
            const float four[4] = {acc[j >> 4][j & 15] * inv, acc[j >> 4][(j & 15) + 1] * inv, acc[j >> 4][(j & 15) + 2] * inv, acc[j >> 4][(j & 15) + 3] * inv};
            write4(j, four);
        }
    }
}

// Few rows leave the chip empty: up to so many blocks of whole rows they are split instead, if there is more than a tile of 32 entries to split; of
// prompts of up to 128 tokens, which have little to split, up to a third of that.  us, whole and split, at a number of blocks (prompts) -
// bf16, 128 values: 128 (2048) 59.5 and 38.3, 160 (400) 16.6 and 15.2, 192 (1000) 34.6 and 38.6, 48 (100) 9.9 and 8.1, 96 (100) 10.1 and 14.1;
// 64 values: 256 (1024) 26.4 and 19.6, 512 (1000) 28.3 and 30.6, 128 (100) 7.7 and 6.9, 256 (100) 8.3 and 10.0; 32 values: 512 (1000) 22.2 and 19.8,
// 512 (500) 13.3 and 14.1.  fp32, 128 values: 256 (1024) 156 and 118, 512 (2048) 395 and 394, 256 (100) 24.9 and 44.4; 64 values: 520 (400) 51.0 and 33.1,
// 1024 (1000) 162 and 181, 256 (100) 15.1 and 18.8; 32 values: 1024 (1000) 96.9 and 88.0.
bool splits(int dtype, int D, int max_len, int64_t blocks) {
    const int64_t most = dtype == PIKV_F32 ? (D == 128 ? 300 : D == 64 ? 640 : 1024) : (D == 128 ? 176 : D == 64 ? 400 : 560);
    return max_len > 32 && blocks <= (max_len > 128 ? most : most / 3);
}

// Waves of such a block: 8 (and their tiles) take a CU of their own, which up to 256 blocks have.  us, 4 waves and 8, one prompt of 200 / 400 / 1000 /
// 2500 tokens in some 250 blocks - bf16, 128 values 9.4 : 9.4 (140 blocks), 11.5 : 10.2 (130), 18.3 : 15.0, 34.1 : 25.0; 64 values 6.6 : 6.7, 8.0 : 7.4, 12.3 :
// 10.4, 23.0 : 17.2; fp32, 64 values 10.9 : 11.3, 16.0 : 15.5, 28.1 : 26.3, 60.6 : 54.1; in 416 blocks bf16, 64 values 8.7 : 11.6, 13.1 : 14.2 (400, 1000).  fp32 tiles of 128
// values are too large for 8, of 32 values there are too few accumulators to join.
int split_waves(int dtype, int D, int max_len, int64_t blocks) {
    return blocks <= 256 && max_len > 256 && D >= 64 && D * elem_bytes(dtype) <= 256 ? kMostWaves : kWaves;
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
    const float unit = slopes ? 1.0f : cap > 0.0f ? cap : score_scale(scale, D), unit_log2 = unit * 1.44269504088896340736f;
    if (!(unit_log2 - unit_log2 == 0.0f)) return PIKV_ERR_UNSUPPORTED;
    if (max_len > tokens) max_len = tokens;
    const int G = Hq / Hkv;
    auto tiles_of = [&](int block_rows) { return ((int64_t)max_len * G + block_rows - 1) / block_rows; };
    const bool split = splits(dtype, D, max_len, (int64_t)B * Hkv * tiles_of(kWaves * kWaveRows));
    const int64_t tiles = tiles_of(split ? kWaveRows : kWaves * kWaveRows);
    if ((int64_t)B * Hkv * tiles >= (1 << 23)) return PIKV_ERR_UNSUPPORTED;
    const int waves = !split ? 0 : split_waves(dtype, D, max_len, (int64_t)B * Hkv * tiles);
    if (tokens == 0 || B == 0 || max_len == 0) return PIKV_OK;       // (tensors without elements have no address)
    if (!q || !k || !v || !cu_seqlens || !out || reinterpret_cast<uintptr_t>(out) % 16 != 0) return PIKV_ERR_INVALID;
    PromptParams p = prompt_params(q, k, tokens, q_stride, k_stride, Hq, Hkv, D, cu_seqlens, B, max_len, prefix, scale, cap, slopes, window);
    p.v = v;
    p.v_stride = v_stride;
    p.unit = unit;
    p.unit_log2 = unit_log2;
    p.margin = fminf(8.0f / p.unit_log2, 1e30f);     // (finite: the first maximum passes it)
    p.out = out;
    p.row_max = row_max;
    p.row_norm = row_norm;
    p.by_head = fast_div(Hkv);
    p.by_tile = fast_div(B);
    p.tiles = (int)tiles;
    const dim3 grid((unsigned)(B * Hkv * tiles)), threads((waves > 0 ? waves : kWaves) * kWave);
    hipStream_t st = as_stream(stream);
    auto launch = [&](auto type, auto width) {
        typedef decltype(type) T;
        constexpr int W = decltype(width)::value;
        auto go = [&](auto capped, auto biased) {
            constexpr bool CAP = decltype(capped)::value, BIAS = decltype(biased)::value;
            if constexpr (W >= 64 && W * sizeof(T) <= 256) {
                if (waves == kMostWaves) {
                    hipLaunchKernelGGL((prompt_attn<T, W, CAP, BIAS, kMostWaves>), grid, threads, 0, st, p);
                    return;
                }
            }
            if (waves > 0) hipLaunchKernelGGL((prompt_attn<T, W, CAP, BIAS, kWaves>), grid, threads, 0, st, p);
            else hipLaunchKernelGGL((prompt_attn<T, W, CAP, BIAS, 0>), grid, threads, 0, st, p);
        };
        const std::true_type yes{};
        const std::false_type no{};
        if (cap > 0.0f) {
            if (slopes) go(yes, yes);
            else go(yes, no);
        } else {
            if (slopes) go(no, yes);
            else go(no, no);
        }
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
