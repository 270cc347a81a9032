// The attention that each entry of a prompt got, over all of its tokens and query heads (Table 3 row H2O): column sums of the softmax, from
// the rows' maxima and sums that the attention left.
//
//   mass_partial : a block takes 256 entries of a kv head, 64 a wave, their keys in registers, and walks the rows (token, head of
//                  the group) that see any of them, 64 at a time through LDS.  S[row][entry] = Q . K^T puts an entry in a
//                  lane: lane (c, h) = (lane % 32, lane / 32) gets the scores of entries c and 32 + c at rows 8 (i / 4) + 4 h + i % 4 of each 32,
//                  and sums exp(s - row_max) / row_norm in its own registers, 32 rows at a time and then over them.
//   mass_join    : the kv heads' sums (and those of the runs that few blocks' rows were cut into), in a fixed order.
//
// 8192 tokens, 32 heads over 8 of 128 bf16 values: 334 - 353 us by the card, 780 - 823 TFLOP/s, the matrix pipe busy 36 - 39 % of the cycles: an exponential and three more vector
// operations for each score.  (32 entries a wave, which read a row's tile from LDS twice as often, in blocks of uneven length: 990 us; an address of its own
// for each piece of a tile, 64 bits wide: 381.)
#include "pikv_prompt_dev.h"

namespace pikv {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
// Entries of a wave, in 32 (fp32 keys of 64 would take all registers).
template <typename T>
constexpr int sets_of = sizeof(T) == 2 ? 2 : 1;
constexpr int kMostEntries = kWaves * 32 * 2;        // of a block

template <typename T, int D>
struct QTile {
    static constexpr int ROWS = 64;
    static constexpr int CHUNKS = D * (int)sizeof(T) / 16, PER_THREAD = ROWS * CHUNKS / kThreads;
    static constexpr int PER_LINE = CHUNKS >= 16 ? 1 : 16 / CHUNKS;
    static constexpr __device__ __forceinline__ int exchange(int row) { return (row / PER_LINE) & (CHUNKS < 16 ? CHUNKS - 1 : 15); }
    static __device__ __forceinline__ int chunk(int row, int c) { return row * CHUNKS + (c ^ exchange(row)); }
};

// CAP: scores capped by a tanh; BIAS: with a distance term.
template <typename T, int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(kThreads, 2) void mass_partial(PromptParams p) {
    typedef QTile<T, D> L;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int ROWS = L::ROWS, KN = D * (int)sizeof(T) / 32, SETS = sets_of<T>, ENTRIES = 32 * SETS;
    constexpr float kLog2e = 1.44269504088896340736f;
    __shared__ __attribute__((aligned(16))) uint4 Qs[2][ROWS * L::CHUNKS];
    // of a tile's rows: maximum, 1 / sum (0: gives nothing), token, slope
    __shared__ __attribute__((aligned(16))) float row_max_s[2][ROWS], weight_s[2][ROWS], slope_s[2][BIAS ? ROWS : 4];
    __shared__ __attribute__((aligned(16))) int token_s[2][ROWS];
    __shared__ int none_s[2];            // a row of the tile gives nothing
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 31, h = lane >> 5;
    int hk, b, split;
    const int id = fast_divide(p.by_split, blockIdx.x, &split);      // (a block's runs: on one XCD after the other)
    const int at_tile = prompt_block(p, id, false, &hk, &b);         // the entries with the most rows first
    const Span span = prompt_span(p, b);
    const int n = span.n, entry0 = at_tile * kWaves * ENTRIES;
    if (entry0 >= n) return;
    const int prefix = p.prefix ? __builtin_amdgcn_readfirstlane(min(max(p.prefix[b], 0), n)) : 0;
    const int entries_end = min(entry0 + kWaves * ENTRIES, n);
    // the rows that see any of the block's entries, and this block's run of them
    const bool all = entry0 < prefix;
    const int64_t seen_to = all || p.window <= 0 ? n : min((int64_t)n, (int64_t)entries_end - 1 + p.window);
    const int row_lo = (all ? 0 : entry0) * p.G, row_hi = (int)seen_to * p.G;
    const int per = ((row_hi - row_lo + p.nsplit - 1) / p.nsplit + ROWS - 1) / ROWS * ROWS;
    const int from = row_lo + split * per, to = min(row_hi, from + per);

    const int wave_entry = entry0 + wave * ENTRIES;
    uint4 kop[SETS][KN];
#pragma unroll
    for (int set = 0; set < SETS; ++set) {
        const char *K = static_cast<const char *>(p.k) + ((int64_t)(span.first + min(wave_entry + 32 * set + c, n - 1)) * p.k_stride + (int64_t)hk * D) * sizeof(T);
#pragma unroll
        for (int s = 0; s < KN; ++s) kop[set][s] = load16(K + (2 * s + h) * 16);
    }
    auto opaque = [](uint32_t v) {           // (else an address per read is carried through the loop)
        asm volatile("" : "+v"(v));
        return v;
    };
    uint4 qr[L::PER_THREAD];
    float max_r = 0.0f, norm_r = 0.0f, slope_r = 0.0f;
    int token_r = 0;
    // Rows row0 .. of the block's run, as they lie from the first one's token on: 32-bit offsets, and quotients of small numbers, for which the
    // reciprocal is exact.
    const uint32_t q_bytes = (uint32_t)p.q_stride * (uint32_t)sizeof(T), turn_bytes = q_bytes - p.G * D * (uint32_t)sizeof(T);
    auto request = [&](int row0) {
        const int tid = (int)opaque(threadIdx.x);
        const int token0 = row_token(p, row0), phase = row0 - token0 * p.G, last = min(ROWS, to - row0) - 1;
        const char *base = static_cast<const char *>(p.q) + ((int64_t)(span.first + token0) * p.q_stride + (int64_t)hk * p.G * D) * (int64_t)sizeof(T);
        auto token_of = [&](uint32_t row) { return p.G == 1 ? row : __umulhi(row, p.G_rcp); };
#pragma unroll
        for (int u = 0; u < L::PER_THREAD; ++u) {
            const uint32_t row = min(tid / L::CHUNKS + u * (kThreads / L::CHUNKS), last) + phase;
            qr[u] = load16(base + (token_of(row) * turn_bytes + row * (D * (uint32_t)sizeof(T)) + tid % L::CHUNKS * 16u));
        }
        if (tid < ROWS) {
            const uint32_t row = min(tid, last) + phase, token = token_of(row), head = row - token * p.G;
            const int64_t first = (int64_t)(span.first + token0) * p.Hq + hk * p.G;
            const uint32_t at = token * p.Hq + head;
            token_r = token0 + token;
            max_r = p.row_max[first + at];
            norm_r = tid <= last ? p.row_norm[first + at] : 0.0f;
            if constexpr (BIAS) slope_r = p.slopes[hk * p.G + head];
        }
    };
    auto place = [&](int buffer) {
        const int tid = (int)opaque(threadIdx.x);
        // (rows tid / CHUNKS + u LINES: their exchange is that of either)
        constexpr int LINES = kThreads / L::CHUNKS;
        const uint32_t at = L::chunk(tid / L::CHUNKS, tid % L::CHUNKS) * 16 + buffer * (int)sizeof(Qs[0]);
#pragma unroll
        for (int u = 0; u < L::PER_THREAD; ++u)
            *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(Qs) + ((at ^ (L::exchange(u * LINES) * 16)) + u * kThreads * 16)) = qr[u];
        if (tid < ROWS) {
            row_max_s[buffer][tid] = norm_r == 0.0f ? INFINITY : max_r;
            weight_s[buffer][tid] = norm_r == 0.0f ? 0.0f : 1.0f / norm_r;
            token_s[buffer][tid] = token_r;
            const bool none = __any(norm_r == 0.0f) != 0;        // (one wave)
            if (tid == 0) none_s[buffer] = none;
            if constexpr (BIAS) slope_s[buffer][tid] = slope_r;
        }
    };
    float total[SETS] = {};
#pragma unroll
    for (int set = 0; set < SETS; ++set)
#pragma unroll
        for (int s = 0; s < KN; ++s) hold_operand(kop[set][s]);      // complete here, not behind requests in the loop
    if (from < to) {                             // (uniform)
        request(from);
        place(0);
        __syncthreads();
        int buffer = 0;
        for (int row0 = from; row0 < to; row0 += ROWS, buffer ^= 1) {
            const int lane = (int)opaque(threadIdx.x) & (kWave - 1), c = lane & 31, h = lane >> 5;      // (derived again in every round: registers)
            if (row0 + ROWS < to) request(row0 + ROWS);
            const int first_token = row_token(p, row0), last_token = row_token(p, min(row0 + ROWS, to) - 1);
            const bool any = wave_entry < n && (wave_entry < prefix || (wave_entry <= last_token && (p.window <= 0 || first_token - (wave_entry + ENTRIES - 1) < p.window)));
            if (any) {
                // (a row that gives nothing may hold anything, scores that are no numbers among them: it is masked)
                const bool masked = __builtin_amdgcn_readfirstlane(none_s[buffer]) != 0 || !(wave_entry + ENTRIES <= prefix || (wave_entry + ENTRIES - 1 <= first_token &&
                                                                          (p.window <= 0 || last_token - wave_entry < p.window))) || row0 + ROWS > to;
                const uint32_t q_at = opaque(L::chunk(c, h) * 16 + buffer * (int)sizeof(Qs[0]));
                const uint32_t reach = p.window > 0 ? p.window : 0x80000000u;
                auto rows_of = [&](auto with_mask) {
                    constexpr bool MASKED = decltype(with_mask)::value;
#pragma unroll
                    for (int rb = 0; rb < ROWS / 32; ++rb) {
                        f32x16_t sc[SETS];
#pragma unroll
                        for (int set = 0; set < SETS; ++set)
#pragma unroll
                            for (int i = 0; i < 16; ++i) sc[set][i] = 0.0f;
#pragma unroll
                        for (int u = 0; u < KN; ++u) {
                            // (chunk 2 u + h of row c, exchanged: the exchange of chunk h with 2 u's bits on top)
                            const uint4 qop = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(Qs) + ((q_at ^ (u * 32)) + rb * 32 * L::CHUNKS * 16));
#pragma unroll
                            for (int set = 0; set < SETS; ++set) {
                                const uint4 k = kop[set][u];
                                if constexpr (BF) {
                                    sc[set] = mfma32(qop, k, sc[set]);
                                } else {
                                    sc[set] = mfma32(__uint_as_float(qop.x), __uint_as_float(k.x), sc[set]);
                                    sc[set] = mfma32(__uint_as_float(qop.y), __uint_as_float(k.y), sc[set]);
                                    sc[set] = mfma32(__uint_as_float(qop.z), __uint_as_float(k.z), sc[set]);
                                    sc[set] = mfma32(__uint_as_float(qop.w), __uint_as_float(k.w), sc[set]);
                                }
                            }
                        }
                        float s[SETS][16];
#pragma unroll
                        for (int set = 0; set < SETS; ++set) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[set][i] = sc[set][i];
                            if constexpr (CAP) {
                                if constexpr (BIAS) __builtin_amdgcn_sched_barrier(0);
                                cap_parts(s[set], p.scale * p.cap_rcp);
                                if constexpr (BIAS) __builtin_amdgcn_sched_barrier(0);
                            }
                        }
                        const float unit = CAP ? p.cap : p.scale;
                        float sum[SETS] = {};
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int r = rb * 32 + 8 * u + 4 * h;
                            const float4 top = *reinterpret_cast<const float4 *>(&row_max_s[buffer][r]), w = *reinterpret_cast<const float4 *>(&weight_s[buffer][r]);
                            const float tops[4] = {top.x, top.y, top.z, top.w}, ws[4] = {w.x, w.y, w.z, w.w};
                            int tokens[4] = {};
                            float slopes[4] = {};
                            if constexpr (BIAS || MASKED) {
                                const int4 t = *reinterpret_cast<const int4 *>(&token_s[buffer][r]);
                                tokens[0] = t.x, tokens[1] = t.y, tokens[2] = t.z, tokens[3] = t.w;
                            }
                            if constexpr (BIAS) {
                                const float4 f = *reinterpret_cast<const float4 *>(&slope_s[buffer][r]);
                                slopes[0] = f.x, slopes[1] = f.y, slopes[2] = f.z, slopes[3] = f.w;
                            }
#pragma unroll
                            for (int x = 0; x < 4; ++x)
#pragma unroll
                                for (int set = 0; set < SETS; ++set) {
                                    const int entry = wave_entry + 32 * set + c;
                                    float v = s[set][4 * u + x];
                                    if constexpr (BIAS) v = fmaf(-slopes[x], fabsf((float)(tokens[x] - entry)), v * unit) - tops[x];
                                    else v = fmaf(v, unit, -tops[x]);
                                    float e = __builtin_amdgcn_exp2f(v * kLog2e), weight = ws[x];        // (0: top is infinite)
                                    if constexpr (MASKED) {      // (both: what is not seen may hold anything)
                                        // (no short circuits: they become branches)
                                        const bool seen = (((uint32_t)(tokens[x] - entry) < reach) | (entry < prefix)) & (ws[x] != 0.0f);
                                        e = seen ? e : 0.0f;
                                        weight = seen ? weight : 0.0f;
                                    }
                                    sum[set] = fmaf(e, weight, sum[set]);
                                }
                            if constexpr (BIAS || MASKED) __builtin_amdgcn_sched_barrier(0);     // (all rows' values at once cost registers)
                        }
#pragma unroll
                        for (int set = 0; set < SETS; ++set) total[set] += sum[set];
                    }
                };
                if constexpr (BIAS) {            // (one form: two cost registers)
                    rows_of(std::true_type{});
                } else {
                    if (masked) rows_of(std::true_type{});
                    else rows_of(std::false_type{});
                }
            }
            if (row0 + ROWS < to) place(buffer ^ 1);
            __syncthreads();
        }
    }
#pragma unroll
    for (int set = 0; set < SETS; ++set) {
        const float sum = halves_sum(total[set]);
        const int entry = wave_entry + 32 * set + c;
        if (h == 0 && entry < n) {
            float *out = p.nsplit * p.Hkv == 1 ? p.mass : p.parts + (int64_t)(split * p.Hkv + hk) * p.tokens;
            out[span.first + entry] = sum;
        }
    }
}

// A wave takes the parts wave, wave + 8, ..; then the waves' sums.
constexpr int kJoinWaves = 8, kJoinThreads = kJoinWaves * kWave;

__global__ __launch_bounds__(kJoinThreads) void mass_join(PromptParams p) {
    __shared__ float sums[kJoinWaves][kWave];
    int b;
    const int at_tile = fast_divide(p.by_tile, blockIdx.x, &b);
    const Span span = prompt_span(p, b);
    if (at_tile * kWave >= span.n) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, entry = at_tile * kWave + lane;
    const float *from = p.parts + span.first + min(entry, span.n - 1);
    const int parts = p.nsplit * p.Hkv;
    float sum = 0.0f;
    for (int i = wave; i < parts; i += 4 * kJoinWaves) {
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = i + u * kJoinWaves < parts ? from[(int64_t)(i + u * kJoinWaves) * p.tokens] : 0.0f;
#pragma unroll
        for (int u = 0; u < 4; ++u) sum += v[u];
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || entry >= span.n) return;
#pragma unroll
    for (int w = 1; w < kJoinWaves; ++w) sum += sums[w][lane];
    p.mass[span.first + entry] = sum;
}

int64_t entry_tiles(int64_t entries, int per) { return (entries + per - 1) / per; }

// Runs that the rows of a block's entries are cut into.  The first entries have many rows, the last few: some eight blocks a CU even that out.
// At most 16, of 64 tokens at the least.
int runs_of(int B, int Hkv, int max_len) {
    const int64_t blocks = (int64_t)B * Hkv * entry_tiles(max_len, kMostEntries), most = ((int64_t)max_len + 63) / 64;
    int64_t runs = blocks > 0 ? 2048 / blocks : 1;
    if (runs > most) runs = most;
    return (int)(runs < 1 ? 1 : runs > 16 ? 16 : runs);
}

}  // namespace
}  // namespace pikv

using namespace pikv;

extern "C" size_t pikv_prompt_mass_workspace_bytes(int32_t tokens, int32_t Hkv, int32_t B, int32_t max_len) {
    if (tokens < 0 || Hkv < 1 || Hkv > 256 || B < 0 || max_len < 0 || tokens > (1 << 23)) return 0;
    if (max_len > tokens) max_len = tokens;
    return ((size_t)runs_of(B, Hkv, max_len) * Hkv * tokens * sizeof(float) + 255) / 256 * 256 + 256;
}

extern "C" int pikv_prompt_mass(const void *q, const void *k, int32_t tokens, int64_t q_stride, int64_t k_stride, int32_t Hq,
                                int32_t Hkv, int32_t D, int32_t dtype, const int32_t *cu_seqlens, int32_t B, int32_t max_len,
                                const int32_t *prefix, float scale, float cap, const float *slopes, int32_t window,
                                const float *row_max, const float *row_norm, float *mass, void *workspace, size_t workspace_bytes,
                                void *stream) {
    const int rc = check_prompt(q, k, nullptr, false, tokens, q_stride, k_stride, 0, Hq, Hkv, D, dtype, B, max_len, scale, cap);
    if (rc != PIKV_OK) return rc;
    if (max_len > tokens) max_len = tokens;
    const int64_t tiles = entry_tiles(max_len, kWaves * 32 * (dtype == PIKV_F32 ? sets_of<float> : sets_of<bf16>)), blocks = (int64_t)B * Hkv * tiles;
    const int runs = runs_of(B, Hkv, max_len);
    if ((int64_t)B * Hkv * prompt_tiles((int64_t)max_len * (Hq / Hkv)) >= (1 << 23) || blocks * runs >= (1 << 23)) return PIKV_ERR_UNSUPPORTED;
    const int64_t joins = B * entry_tiles(max_len, kWave);
    if (joins * kJoinThreads >= (int64_t)1 << 32) return PIKV_ERR_UNSUPPORTED;       // (threads of a launch)
    if (tokens == 0 || B == 0 || max_len == 0) return PIKV_OK;
    if (!q || !k || !cu_seqlens || !row_max || !row_norm || !mass) return PIKV_ERR_INVALID;
    if (!workspace || workspace_bytes < pikv_prompt_mass_workspace_bytes(tokens, Hkv, B, max_len)) return PIKV_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return PIKV_ERR_INVALID;
    PromptParams p = prompt_params(q, k, tokens, q_stride, k_stride, Hq, Hkv, D, cu_seqlens, B, max_len, prefix, scale, cap, slopes, window);
    p.row_max = const_cast<float *>(row_max);
    p.row_norm = const_cast<float *>(row_norm);
    p.mass = mass;
    p.parts = static_cast<float *>(workspace);
    p.nsplit = runs;
    p.by_head = fast_div(Hkv);
    p.by_split = fast_div(runs);
    p.by_tile = fast_div(B);
    p.tiles = (int)tiles;
    const dim3 grid((unsigned)(blocks * runs)), threads(kThreads);
    hipStream_t st = as_stream(stream);
    auto launch = [&](auto type, auto width) {
        typedef decltype(type) T;
        constexpr int W = decltype(width)::value;
        if (cap > 0.0f) {
            if (slopes) hipLaunchKernelGGL((mass_partial<T, W, true, true>), grid, threads, 0, st, p);
            else hipLaunchKernelGGL((mass_partial<T, W, true, false>), grid, threads, 0, st, p);
        } else {
            if (slopes) hipLaunchKernelGGL((mass_partial<T, W, false, true>), grid, threads, 0, st, p);
            else hipLaunchKernelGGL((mass_partial<T, W, false, false>), grid, threads, 0, st, p);
        }
    };
    auto by_width = [&](auto type) {
        if (D == 32) launch(type, std::integral_constant<int, 32>{});
        else if (D == 64) launch(type, std::integral_constant<int, 64>{});
        else launch(type, std::integral_constant<int, 128>{});
    };
    if (dtype == PIKV_F32) by_width(float{});
    else by_width(bf16{});
    int done = launch_status();
    if (done != PIKV_OK || runs * Hkv == 1) return done;
    hipLaunchKernelGGL(mass_join, dim3((unsigned)joins), dim3(kJoinThreads), 0, st, p);
    return launch_status();
}
