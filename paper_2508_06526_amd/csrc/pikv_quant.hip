// The cache held in 8 bits: written from dense shards, by a step's new entries, and read back.
//
//   quant_pack   : one block per 64 slots (128 with scale blocks of 128) of one (sequence, expert, kv head, K or V).  A wave
//                  takes 16 slots, holds them in registers, forms their largest magnitude on the bit patterns (a NaN is
//                  then the largest), joins it with the waves of the same scale block and writes codes and scale: one pass
//                  over the dense rows.
//   quant_read   : the same tiles the other way, value = code * scale.
//   Both are bound by memory.  Dense rows, read or written once, go past the caches (non-temporal), codes, which the next call
//   reads, do not: written and read back, 2.7 GB in fp32 in 396 us (6.8 TB/s; all through the caches 495, codes past them too 425 -
//   448), 1.6 GB in bf16 in 236 us (292; 237 - 257).  16-byte pieces of neighbouring lanes: with 8 fp32 values
//   a lane, two pieces, half of every line was written at a time (127 MB 38 -> 26.7 us).
//   quant_append : one block per (sequence, selected expert): slot rule and count of append_rows; a row of D values by D / 8
//                  lanes, which also move the codes of the block's other live slots where its scale does.
#include "pikv_mfma_dev.h"
#include "pikv_quant_dev.h"

namespace pikv {
namespace {

constexpr int kTileSlots = 64;          // slots of a block of 4 waves
constexpr int kWaveSlots = 16;

// 8 values of a lane: one 16-byte piece of a bf16 row, two of an fp32 one.
template <typename T>
struct Eight {
    static constexpr int N = sizeof(T) / 2;
    uint4 v[N];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = load16_stream(reinterpret_cast<const char *>(p) + 16 * i);
    }
    __device__ __forceinline__ void widen(float *f) const {
#pragma unroll
        for (int i = 0; i < N; ++i) Pack16<T>::widen(v[i], f + i * Pack16<T>::N);
    }
};
template <int N>
__device__ __forceinline__ uint32_t magnitude(const float (&f)[N]) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) most = max(most, __float_as_uint(f[i]) & 0x7fffffffu);
    return most;
}
// The largest of COUNT (a power of two) adjacent lanes' values, in all of them.
template <int COUNT>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
#pragma unroll
    for (int off = 1; off < COUNT; off <<= 1) x = max(x, (uint32_t)__shfl_xor((int)x, off, kWave));
    return x;
}

struct QuantParams {
    const void *const *K_dense, *const *V_dense;
    void *const *K, *const *V;
    float *K_scales, *V_scales;
    const int32_t *n_valid;
    int64_t dense_h, dense_s, code_h, code_s;     // strides, elements and bytes
    FastDiv by_tiles, by_Hkv;                     // tiles of a shard's kv head; kv heads
    int Hkv, S, n_blocks, block_bits;
};

// Tile `blockIdx.x`: K or V, tile, kv head, shard.  False: nothing valid in it.
struct Tile {
    int be, h, first, n, v;
};
__device__ __forceinline__ bool find_tile(const QuantParams &p, int slots, Tile *t) {
    int tile;
    t->v = blockIdx.x & 1;
    const int rest = fast_divide(p.by_tiles, blockIdx.x >> 1, &tile);
    t->be = fast_divide(p.by_Hkv, rest, &t->h);
    t->first = tile * slots;
    t->n = min(p.n_valid[t->be], p.S);
    return t->first < t->n;
}

// A lane's values are one 16-byte load: 8 of bf16, 4 of fp32.
template <typename T, int D, int F, int WAVES>
__global__ __launch_bounds__(WAVES *kWave) void quant_pack(QuantParams p) {
    constexpr int VPL = Pack16<T>::N, LPR = D / VPL, RPL = kWave / LPR, NL = kWaveSlots / RPL;     // values of a lane, lanes of a row, rows of a load, loads
    __shared__ uint32_t wave_most[WAVES];
    Tile t;
    if (!find_tile(p, WAVES * kWaveSlots, &t)) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    const int c = lane & (LPR - 1), r = lane / LPR;
    const int s0 = t.first + wave * kWaveSlots;
    const T *rows = static_cast<const T *>(t.v ? p.V_dense[t.be] : p.K_dense[t.be]) + t.h * p.dense_h + VPL * c;
    char *codes = static_cast<char *>(t.v ? p.V[t.be] : p.K[t.be]) + t.h * p.code_h + VPL * c;
    uint4 x[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) x[i] = load16_stream(rows + (int64_t)min(s0 + i * RPL + r, t.n - 1) * p.dense_s);    // (past the end: the last valid row)
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        float f[VPL];
        Pack16<T>::widen(x[i], f);
        if (s0 + i * RPL + r < t.n) most = max(most, magnitude(f));
    }
    const int together = 1 << (p.block_bits - 4), first = wave & ~(together - 1);            // waves of a scale block: 1 .. 8
    auto of_scale_block = [&](uint32_t mine) {
        mine = lanes_max<kWave>(mine);
        if (lane == 0) wave_most[wave] = mine;
        __syncthreads();
        for (int w = 0; w < together; ++w) mine = max(mine, wave_most[first + w]);
        return mine;
    };
    most = of_scale_block(most);
    // A row with a NaN or an infinity has no codes, and no part in the scale.
    const bool poisoned = most >= 0x7f800000u;
    auto bad_row = [&](const float (&f)[VPL]) { return lanes_max<LPR>(magnitude(f)) >= 0x7f800000u; };
    uint32_t of_block = 0;
    for (int w = 0; w < WAVES; ++w) of_block = max(of_block, wave_most[w]);
    if (of_block >= 0x7f800000u) {
        __syncthreads();
        uint32_t rest = 0;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            float f[VPL];
            Pack16<T>::widen(x[i], f);
            if (!bad_row(f) && s0 + i * RPL + r < t.n) rest = max(rest, magnitude(f));
        }
        most = of_scale_block(rest);
    }
    if (s0 >= t.n) return;
    const uint32_t scale = needed_scale<F>(most);
    const float inv = inverse_scale(scale);
    if (lane == 0 && wave == first)
        (t.v ? p.V_scales : p.K_scales)[((int64_t)t.be * p.Hkv + t.h) * p.n_blocks + (s0 >> p.block_bits)] =
            __uint_as_float(poisoned ? poisoned_scale(scale) : scale);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int slot = s0 + i * RPL + r;
        float f[VPL];
        Pack16<T>::widen(x[i], f);
        uint32_t w[VPL / 4];
#pragma unroll
        for (int u = 0; u < VPL / 4; ++u) w[u] = encode4<F>(f + 4 * u, inv);
        if (poisoned && bad_row(f)) {
#pragma unroll
            for (int u = 0; u < VPL / 4; ++u) w[u] = no_codes<F>();
        }
        char *to = codes + (int64_t)slot * p.code_s;
        if (slot < t.n) {
            if constexpr (VPL == 4) *reinterpret_cast<uint32_t *>(to) = w[0];
            else *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
        }
    }
}

template <typename T, int D, int F>
__global__ __launch_bounds__(256) void quant_read(QuantParams p) {
    constexpr int VPL = Pack16<T>::N, LPR = D / VPL, RPL = kWave / LPR, NL = kWaveSlots / RPL;
    Tile t;
    if (!find_tile(p, kTileSlots, &t)) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    const int c = lane & (LPR - 1), r = lane / LPR;
    const int s0 = t.first + wave * kWaveSlots;
    if (s0 >= t.n) return;
    T *rows = static_cast<T *>(const_cast<void *>(t.v ? p.V_dense[t.be] : p.K_dense[t.be])) + t.h * p.dense_h + VPL * c;
    const char *codes = static_cast<const char *>(t.v ? p.V[t.be] : p.K[t.be]) + t.h * p.code_h + VPL * c;
    const float scale = (t.v ? p.V_scales : p.K_scales)[((int64_t)t.be * p.Hkv + t.h) * p.n_blocks + (s0 >> p.block_bits)];
    typedef uint32_t Codes __attribute__((ext_vector_type(VPL / 4)));
    Codes w[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i)
        w[i] = *reinterpret_cast<const Codes *>(codes + (int64_t)min(s0 + i * RPL + r, t.n - 1) * p.code_s);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int slot = s0 + i * RPL + r;
        float f[VPL];
#pragma unroll
        for (int u = 0; u < VPL / 4; ++u) decode4<F>(w[i][u], f + 4 * u);
#pragma unroll
        for (int u = 0; u < VPL; ++u) f[u] *= scale;
        uint4 out[1];
        if constexpr (VPL == 4) out[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        else split_bf16(f, out);
        if (slot < t.n) store16_stream(rows + (int64_t)slot * p.dense_s, out[0]);
    }
}

struct QuantAppendParams {
    const void *K_new, *V_new;
    const int32_t *topk, *reuse_idx, *reuse_cnt;
    void *const *K, *const *V;
    float *K_scales, *V_scales, *utility;
    int32_t *n_valid;
    int64_t code_h, code_s;
    FastDiv by_k;
    int E, S, Hkv, k, max_evict, n_blocks, block_bits;
};

// A scale that stands this far (exponents) above what its block needs comes down: at most four times the need is kept, six bits of
// int8 at the least.  From eight times on, because the block's codes are read to find out and written again - the next entries
// would mostly raise a closer scale again.
constexpr uint32_t kMostSlack = 3u << 23, kOne = 127u << 23, kLeastScale = 1u << 23;

// Two trips to memory, as append_rows: lane e takes shard e's count, freed slot and addresses beside the selection, which picks
// among them, and the new rows come with those; then the block's old scale and the codes of the entry that leaves - and a third for
// the block's codes, eight slots at a time, where the scale grows, or where the entry that leaves reaches within an eighth of it (else another
// holds it up) and the new one does not.
template <typename T, int D, int F>
__global__ __launch_bounds__(1024) void quant_append(QuantAppendParams p) {
    constexpr int LPR = D / 8;
    int j;
    const int b = fast_divide(p.by_k, blockIdx.x, &j);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), c = tid & (LPR - 1);
    const int64_t be0 = (int64_t)b * p.E, be_lane = be0 + min(lane, p.E - 1);
    const int sel = p.topk[(int64_t)b * p.k + min(lane, p.k - 1)];
    const int n_lane = p.n_valid[be_lane];
    const uint64_t K_lane = reinterpret_cast<uint64_t>(p.K[be_lane]), V_lane = reinterpret_cast<uint64_t>(p.V[be_lane]);
    int cnt_lane = 0, idx_lane = 0;
    if (p.reuse_cnt) {                       // block-uniform
        cnt_lane = p.reuse_cnt[be_lane];
        idx_lane = p.reuse_idx[be_lane * p.max_evict];
    }
    const int row_step = blockDim.x / LPR, rows = 2 * p.Hkv;           // a row: (kv head, K or V), by D / 8 lanes of one wave
    auto new_row = [&](int row) {
        Eight<T> x;
        x.load(static_cast<const T *>((row & 1) ? p.V_new : p.K_new) + ((int64_t)b * p.Hkv + (row >> 1)) * D + 8 * c);
        return x;
    };
    Eight<T> x = new_row(min(tid / LPR, rows - 1));
    const int e = __builtin_amdgcn_readlane(sel, j), n = __builtin_amdgcn_readlane(n_lane, e), cnt = __builtin_amdgcn_readlane(cnt_lane, e);
    const int slot = cnt > 0 ? __builtin_amdgcn_readlane(idx_lane, e) : n;
    __syncthreads();                         // every thread has read n before it changes
    if (n >= p.S || slot < 0 || slot >= p.S) return;   // full shard: the entry is dropped
    // A shard listed twice takes the entry once: two blocks rounding one block's codes would round them twice.
    if (e < 0 || e >= p.E || __ballot(sel == e && lane < j) != 0) return;
    const int64_t be = be0 + e;
    const int blk = slot >> p.block_bits, lo = blk << p.block_bits;
    const int live = min(p.S, n + max(cnt, 1)), hi = min(lo + (1 << p.block_bits), live);      // live slots of the block: lo .. hi - 1
    const bool others = hi - lo > (slot < hi ? 1 : 0);
    auto address = [&](uint64_t of_lane) {
        const uint32_t low = __builtin_amdgcn_readlane((int)(uint32_t)of_lane, e), high = __builtin_amdgcn_readlane((int)(uint32_t)(of_lane >> 32), e);
        return reinterpret_cast<char *>(((uint64_t)high << 32) | low);
    };
    char *Ks = address(K_lane), *Vs = address(V_lane);
    for (int row = tid / LPR; row < rows; row += row_step) {
        const int h = row >> 1, v = row & 1;
        if (row >= row_step) x = new_row(row);
        float *at = (v ? p.V_scales : p.K_scales) + (be * p.Hkv + h) * p.n_blocks + blk;
        const uint32_t word = __float_as_uint(*at) & 0x7fffffffu;
        const bool poisoned = word >= 0x7f800000u;
        const uint32_t old = poisoned ? kept_scale(word) : word;
        char *codes = (v ? Vs : Ks) + h * p.code_h + 8 * c;
        uint2 leaves = make_uint2(0u, 0u);               // the lane's codes of the entry whose slot this is
        if (cnt > 0) leaves = *reinterpret_cast<const uint2 *>(codes + (int64_t)slot * p.code_s);
        float f[8];
        x.widen(f);
        const uint32_t need = needed_scale<F>(lanes_max<LPR>(magnitude(f)));
        const bool bad = need >= 0x7f800000u;
        // `use` with the lane's codes of each of the block's other live slots, eight requests together
        auto for_others = [&](auto use) {
            constexpr int kAtOnce = 8;
            for (int s0 = lo; s0 < hi; s0 += kAtOnce) {
                uint2 w[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) w[u] = *reinterpret_cast<const uint2 *>(codes + (int64_t)min(s0 + u, hi - 1) * p.code_s);
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    if (s0 + u < hi && s0 + u != slot) use(s0 + u, w[u]);
            }
        };
        auto largest = [&](uint2 w) {
            float g[8];
            decode4<F>(w.x, g);
            decode4<F>(w.y, g + 4);
            return magnitude(g);
        };
        uint32_t scale;
        bool marked = bad;                   // an entry of the block has no codes
        if (!others) {
            scale = need;
        } else if (cnt <= 0 && (poisoned ? old == 0 : bad)) {
            scale = kNanScale;               // without a freed slot: no codes are kept
            if (!poisoned) for_others([&](int s, uint2) { *reinterpret_cast<uint2 *>(codes + (int64_t)s * p.code_s) = make_uint2(0u, 0u); });
        } else if (poisoned && old == 0) {   // nothing was kept of the others: each is without codes until its slot is written
            scale = bad ? kLeastScale : need;
            marked = true;
            for_others([&](int s, uint2) { *reinterpret_cast<uint2 *>(codes + (int64_t)s * p.code_s) = make_uint2(no_codes<F>(), no_codes<F>()); });
        } else {
            scale = bad ? max(old, kLeastScale) : max(need, old);
            if (!bad && (poisoned || (need + kMostSlack <= old && needed_scale<F>(lanes_max<LPR>(largest(leaves))) + kMostSlack > kOne))) {
                // The entry that leaves may be what kept the scale up, and the new one needs far less: does what stays?  Or it may have been
                // the last one without codes.
                uint32_t most = 0;
                for_others([&](int, uint2 w) {
                    if (poisoned && has_no_codes<F>(w.x)) marked = true;
                    else most = max(most, largest(w));
                });
                most = lanes_max<LPR>(most);
                const int stays = most == 0 ? 0 : (int)(old >> 23) + (int)(needed_scale<F>(most) >> 23) - 127;     // biased exponent, may lie below the smallest
                const uint32_t enough = max(need, (uint32_t)max(stays, 1) << 23);
                if (cnt > 0 && enough + kMostSlack <= scale) scale = enough;
            }
            if (scale != old) {
                // old / scale: at most 1/2, 0 from where it underflows, and codes with it (so an old scale of 0, whose codes stand for
                // zeros); or, of a scale that comes down, so large that no code saturates
                const int shift = min((int)(old >> 23) - (int)(scale >> 23), 126);
                const float ratio = old == 0 || shift < -126 ? 0.0f : __uint_as_float((uint32_t)(127 + shift) << 23);
                for_others([&](int s, uint2 w) {
                    if (poisoned && has_no_codes<F>(w.x)) return;
                    float g[8];
                    decode4<F>(w.x, g);
                    decode4<F>(w.y, g + 4);
                    *reinterpret_cast<uint2 *>(codes + (int64_t)s * p.code_s) = make_uint2(encode4<F>(g, ratio), encode4<F>(g + 4, ratio));
                });
            }
        }
        uint2 to = make_uint2(0u, 0u);
        if (scale < 0x7f800000u) {
            const float inv = inverse_scale(scale);
            to = bad ? make_uint2(no_codes<F>(), no_codes<F>()) : make_uint2(encode4<F>(f, inv), encode4<F>(f + 4, inv));
        }
        *reinterpret_cast<uint2 *>(codes + (int64_t)slot * p.code_s) = to;
        if (c == 0) *at = __uint_as_float(scale < 0x7f800000u && marked ? poisoned_scale(scale) : scale);
    }
    if (tid == 0) {
        p.utility[be * p.S + slot] = 0.0f;
        p.n_valid[be] = n + 1;
    }
}

// The kernel for a dense type, row width and format.
template <class L>
void by_shape(const pikv_desc *d, int format, L launch) {
    auto by_format = [&](auto type, auto width) {
        if (format == PIKV_QUANT_INT8) launch(type, width, std::integral_constant<int, PIKV_QUANT_INT8>{});
        else launch(type, width, std::integral_constant<int, PIKV_QUANT_E4M3>{});
    };
    auto by_width = [&](auto type) {
        if (d->D == 32) by_format(type, std::integral_constant<int, 32>{});
        else if (d->D == 64) by_format(type, std::integral_constant<int, 64>{});
        else by_format(type, std::integral_constant<int, 128>{});
    };
    if (d->dtype == PIKV_F32) by_width(float{});
    else by_width(bf16{});
}

int quant_tiles(const pikv_desc *desc, int format, int block, int slots, const void *const *K_dense, const void *const *V_dense,
                int64_t dense_h, int64_t dense_s, const int32_t *n_valid, void *const *K, void *const *V, float *K_scales,
                float *V_scales, QuantParams *p, unsigned *grid) {
    const int rc = check_quant(desc, format, block);
    if (rc != PIKV_OK) return rc;
    const int eb = elem_bytes(desc->dtype);
    if (dense_s < desc->D || (dense_s * eb) % 16 != 0 || dense_h < 0 || (dense_h * eb) % 16 != 0) return PIKV_ERR_INVALID;
    if (desc->Hkv > 1 && dense_h < (int64_t)(desc->S - 1) * dense_s + desc->D) return PIKV_ERR_INVALID;
    const int tiles = (desc->S - 1) / slots + 1;
    // (a launch has fewer than 2^32 threads)
    const int64_t per_sequence = (int64_t)desc->E * desc->Hkv * 2 * tiles, most = ((int64_t)1 << 23) - 1;
    if (desc->B > 0 && per_sequence > most / desc->B) return PIKV_ERR_UNSUPPORTED;
    *grid = (unsigned)(desc->B * per_sequence);
    if (*grid == 0) return PIKV_OK;              // (tensors without elements have no address)
    if (!K_dense || !V_dense || !n_valid || !K || !V || !K_scales || !V_scales) return PIKV_ERR_INVALID;
    p->K_dense = K_dense;
    p->V_dense = V_dense;
    p->K = K;
    p->V = V;
    p->K_scales = K_scales;
    p->V_scales = V_scales;
    p->n_valid = n_valid;
    p->dense_h = dense_h;
    p->dense_s = dense_s;
    p->code_h = desc->stride_h;
    p->code_s = desc->stride_s;
    p->by_tiles = fast_div(tiles);
    p->by_Hkv = fast_div(desc->Hkv);
    p->Hkv = desc->Hkv;
    p->S = desc->S;
    p->n_blocks = (desc->S - 1) / block + 1;
    p->block_bits = __builtin_ctz(block);
    return PIKV_OK;
}

}  // namespace
}  // namespace pikv

using namespace pikv;

extern "C" int pikv_quant_pack(const pikv_desc *desc, int32_t format, int32_t block, const void *const *K_dense,
                               const void *const *V_dense, int64_t dense_stride_h, int64_t dense_stride_s,
                               const int32_t *n_valid, void *const *K_shards, void *const *V_shards, float *K_scales,
                               float *V_scales, void *stream) {
    QuantParams p;
    unsigned grid = 0;
    const int rc = quant_tiles(desc, format, block, block > kTileSlots ? block : kTileSlots, K_dense, V_dense, dense_stride_h,
                               dense_stride_s, n_valid, K_shards, V_shards, K_scales, V_scales, &p, &grid);
    if (rc != PIKV_OK || grid == 0) return rc;
    by_shape(desc, format, [&](auto type, auto width, auto fmt) {
        typedef decltype(type) T;
        constexpr int D = decltype(width)::value, F = decltype(fmt)::value;
        if (block > kTileSlots) hipLaunchKernelGGL((quant_pack<T, D, F, 8>), dim3(grid), dim3(512), 0, as_stream(stream), p);
        else hipLaunchKernelGGL((quant_pack<T, D, F, 4>), dim3(grid), dim3(256), 0, as_stream(stream), p);
    });
    return launch_status();
}

extern "C" int pikv_quant_read(const pikv_desc *desc, int32_t format, int32_t block, const void *const *K_shards,
                               const void *const *V_shards, const float *K_scales, const float *V_scales,
                               const int32_t *n_valid, void *const *K_dense, void *const *V_dense, int64_t dense_stride_h,
                               int64_t dense_stride_s, void *stream) {
    QuantParams p;
    unsigned grid = 0;
    const int rc = quant_tiles(desc, format, block, kTileSlots, K_dense, V_dense, dense_stride_h, dense_stride_s, n_valid,
                               const_cast<void *const *>(K_shards),
                               const_cast<void *const *>(V_shards),
                               const_cast<float *>(K_scales), const_cast<float *>(V_scales), &p, &grid);
    if (rc != PIKV_OK || grid == 0) return rc;
    by_shape(desc, format, [&](auto type, auto width, auto fmt) {
        hipLaunchKernelGGL((quant_read<decltype(type), decltype(width)::value, decltype(fmt)::value>), dim3(grid), dim3(256), 0,
                           as_stream(stream), p);
    });
    return launch_status();
}

extern "C" int pikv_quant_append(const pikv_desc *desc, int32_t format, int32_t block, const void *K_new, const void *V_new,
                                 const int32_t *topk_idx, int32_t k, const int32_t *reuse_idx, const int32_t *reuse_cnt,
                                 int32_t max_evict, void *const *K_shards, void *const *V_shards, float *K_scales,
                                 float *V_scales, float *utility, int32_t *n_valid, void *stream) {
    const int rc = check_quant(desc, format, block);
    if (rc != PIKV_OK) return rc;
    if (k < 1 || k > desc->E) return PIKV_ERR_INVALID;
    if (desc->B != 0) {                          // (tensors without elements have no address)
        if (!K_new || !V_new || !topk_idx || !K_shards || !V_shards || !K_scales || !V_scales || !utility || !n_valid)
            return PIKV_ERR_INVALID;
        if ((reuse_idx == nullptr) != (reuse_cnt == nullptr)) return PIKV_ERR_INVALID;
    }
    if (reuse_idx && max_evict < 1) return PIKV_ERR_INVALID;
    if (desc->route_rows_per_seq != 1) return PIKV_ERR_UNSUPPORTED;   // one insert per sequence
    if ((int64_t)desc->B * k > (1 << 21)) return PIKV_ERR_UNSUPPORTED;
    if (desc->B == 0) return PIKV_OK;
    QuantAppendParams p;
    p.K_new = K_new;
    p.V_new = V_new;
    p.topk = topk_idx;
    p.reuse_idx = reuse_idx;
    p.reuse_cnt = reuse_cnt;
    p.K = K_shards;
    p.V = V_shards;
    p.K_scales = K_scales;
    p.V_scales = V_scales;
    p.utility = utility;
    p.n_valid = n_valid;
    p.code_h = desc->stride_h;
    p.code_s = desc->stride_s;
    p.by_k = fast_div(k);
    p.E = desc->E;
    p.S = desc->S;
    p.Hkv = desc->Hkv;
    p.k = k;
    p.max_evict = max_evict;
    p.n_blocks = (desc->S - 1) / block + 1;
    p.block_bits = __builtin_ctz(block);
    const int lanes = 2 * desc->Hkv * (desc->D / 8);
    const int threads = lanes >= 1024 ? 1024 : (lanes + kWave - 1) / kWave * kWave;
    by_shape(desc, format, [&](auto type, auto width, auto fmt) {
        hipLaunchKernelGGL((quant_append<decltype(type), decltype(width)::value, decltype(fmt)::value>), dim3(desc->B * k), dim3(threads),
                           0, as_stream(stream), p);
    });
    return launch_status();
}
