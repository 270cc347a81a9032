// The cache held in 8 bits: written from dense shards, by a step's new entries, and read back.
//
//   quant_pack   : one block per 64 slots (128 with scale blocks of 128) of one (sequence, expert, kv head, K or V).  A wave
//                  takes 16 slots, holds them in registers, forms their largest magnitude on the bit patterns (a NaN is
//                  then the largest), joins it with the waves of the same scale block and writes codes and scale: one pass
//                  over the dense rows.
//   quant_read   : the same tiles the other way, value = code * scale.
//   quant_append : one block per (sequence, selected expert): slot rule and count of append_rows; a row of D values by D / 8
//                  lanes, which also round the codes of the block's other live slots where its scale grows.
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
template <typename T>
__device__ __forceinline__ void store8(T *p, const float *f) {
    if constexpr (sizeof(T) == 4) {
        store16(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
        store16(p + 4, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
    } else {
        uint4 out[1];
        split_bf16(f, out);
        store16(p, out[0]);
    }
}
__device__ __forceinline__ uint32_t magnitude(const float *f) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(f[i]) & 0x7fffffffu);
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

template <typename T, int D, int F, int WAVES>
__global__ __launch_bounds__(WAVES *kWave) void quant_pack(QuantParams p) {
    constexpr int LPR = D / 8, RPL = kWave / LPR, NL = kWaveSlots / RPL;     // lanes of a row, rows of a load, loads
    __shared__ uint32_t wave_most[WAVES];
    Tile t;
    if (!find_tile(p, WAVES * kWaveSlots, &t)) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    const int c = lane & (LPR - 1), r = lane / LPR;
    const int s0 = t.first + wave * kWaveSlots;
    const T *rows = static_cast<const T *>(t.v ? p.V_dense[t.be] : p.K_dense[t.be]) + t.h * p.dense_h + 8 * c;
    char *codes = static_cast<char *>(t.v ? p.V[t.be] : p.K[t.be]) + t.h * p.code_h + 8 * c;
    Eight<T> x[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) x[i].load(rows + (int64_t)min(s0 + i * RPL + r, t.n - 1) * p.dense_s);    // (past the end: the last valid row)
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        float f[8];
        x[i].widen(f);
        if (s0 + i * RPL + r < t.n) most = max(most, magnitude(f));
    }
    most = lanes_max<kWave>(most);
    if (lane == 0) wave_most[wave] = most;
    __syncthreads();
    const int together = 1 << (p.block_bits - 4);            // waves of a scale block: 1 .. 8
    const int first = wave & ~(together - 1);
    for (int w = 0; w < together; ++w) most = max(most, wave_most[first + w]);
    if (s0 >= t.n) return;
    const uint32_t scale = needed_scale<F>(most);
    const float inv = inverse_scale(scale);
    if (lane == 0 && wave == first)
        (t.v ? p.V_scales : p.K_scales)[((int64_t)t.be * p.Hkv + t.h) * p.n_blocks + (s0 >> p.block_bits)] = __uint_as_float(scale);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int slot = s0 + i * RPL + r;
        float f[8];
        x[i].widen(f);
        const uint2 w = make_uint2(encode4<F>(f, inv), encode4<F>(f + 4, inv));
        if (slot < t.n) *reinterpret_cast<uint2 *>(codes + (int64_t)slot * p.code_s) = w;
    }
}

template <typename T, int D, int F>
__global__ __launch_bounds__(256) void quant_read(QuantParams p) {
    constexpr int LPR = D / 8, RPL = kWave / LPR, NL = kWaveSlots / RPL;
    Tile t;
    if (!find_tile(p, kTileSlots, &t)) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    const int c = lane & (LPR - 1), r = lane / LPR;
    const int s0 = t.first + wave * kWaveSlots;
    if (s0 >= t.n) return;
    T *rows = static_cast<T *>(const_cast<void *>(t.v ? p.V_dense[t.be] : p.K_dense[t.be])) + t.h * p.dense_h + 8 * c;
    const char *codes = static_cast<const char *>(t.v ? p.V[t.be] : p.K[t.be]) + t.h * p.code_h + 8 * c;
    const float scale = (t.v ? p.V_scales : p.K_scales)[((int64_t)t.be * p.Hkv + t.h) * p.n_blocks + (s0 >> p.block_bits)];
    uint2 w[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i)
        w[i] = *reinterpret_cast<const uint2 *>(codes + (int64_t)min(s0 + i * RPL + r, t.n - 1) * p.code_s);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int slot = s0 + i * RPL + r;
        float f[8];
        decode4<F>(w[i].x, f);
        decode4<F>(w[i].y, f + 4);
#pragma unroll
        for (int u = 0; u < 8; ++u) f[u] *= scale;
        if (slot < t.n) store8(rows + (int64_t)slot * p.dense_s, f);
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

template <typename T, int D, int F>
__global__ __launch_bounds__(1024) void quant_append(QuantAppendParams p) {
    constexpr int LPR = D / 8;
    int j;
    const int b = fast_divide(p.by_k, blockIdx.x, &j);
    const int tid = threadIdx.x, c = tid & (LPR - 1);
    const int e = p.topk[(int64_t)b * p.k + j];
    const int64_t be = (int64_t)b * p.E + e;
    const int n = p.n_valid[be];
    const int cnt = p.reuse_cnt ? p.reuse_cnt[be] : 0;
    const int slot = cnt > 0 ? p.reuse_idx[be * p.max_evict] : n;
    __syncthreads();                         // every thread has read n before it changes
    if (n >= p.S || slot < 0 || slot >= p.S) return;   // full shard: the entry is dropped
    const int blk = slot >> p.block_bits, lo = blk << p.block_bits;
    const int live = min(p.S, n + max(cnt, 1)), hi = min(lo + (1 << p.block_bits), live);      // live slots of the block: lo .. hi - 1
    const bool others = hi - lo > (slot < hi ? 1 : 0);
    const int row_step = blockDim.x / LPR;
    for (int row = tid / LPR; row < 2 * p.Hkv; row += row_step) {      // (kv head, K or V); D / 8 lanes of one wave
        const int h = row >> 1, v = row & 1;
        Eight<T> x;
        x.load(static_cast<const T *>(v ? p.V_new : p.K_new) + ((int64_t)b * p.Hkv + h) * D + 8 * c);
        float *at = (v ? p.V_scales : p.K_scales) + (be * p.Hkv + h) * p.n_blocks + blk;
        const uint32_t old = __float_as_uint(*at);
        char *codes = static_cast<char *>(v ? p.V[be] : p.K[be]) + h * p.code_h + 8 * c;
        float f[8];
        x.widen(f);
        uint32_t scale = needed_scale<F>(lanes_max<LPR>(magnitude(f)));
        if (others) scale = max(scale, old & 0x7fffffffu);
        const float inv = inverse_scale(scale);
        if (others && scale != (old & 0x7fffffffu)) {
            // old / scale, at most 1/2; 0 from where it underflows, and codes with it (NaN scale: 0)
            const int shift = (int)(scale >> 23) - (int)(old >> 23);
            const float ratio = scale >= 0x7f800000u || shift > 126 ? 0.0f : __uint_as_float((uint32_t)(127 - shift) << 23);
            for (int s = lo; s < hi; ++s) {
                if (s == slot) continue;
                uint2 *held = reinterpret_cast<uint2 *>(codes + (int64_t)s * p.code_s);
                const uint2 w = *held;
                float g[8];
                decode4<F>(w.x, g);
                decode4<F>(w.y, g + 4);
                *held = make_uint2(encode4<F>(g, ratio), encode4<F>(g + 4, ratio));
            }
        }
        *reinterpret_cast<uint2 *>(codes + (int64_t)slot * p.code_s) = make_uint2(encode4<F>(f, inv), encode4<F>(f + 4, inv));
        if (c == 0) *at = __uint_as_float(scale);
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
    if (!K_dense || !V_dense || !n_valid || !K || !V || !K_scales || !V_scales) return PIKV_ERR_INVALID;
    const int eb = elem_bytes(desc->dtype);
    if (dense_s < desc->D || (dense_s * eb) % 16 != 0 || dense_h < 0 || (dense_h * eb) % 16 != 0) return PIKV_ERR_INVALID;
    if (desc->Hkv > 1 && dense_h < (int64_t)(desc->S - 1) * dense_s + desc->D) return PIKV_ERR_INVALID;
    const int tiles = (desc->S - 1) / slots + 1;
    // (a launch has fewer than 2^32 threads)
    const int64_t per_sequence = (int64_t)desc->E * desc->Hkv * 2 * tiles, most = ((int64_t)1 << 23) - 1;
    if (desc->B > 0 && per_sequence > most / desc->B) return PIKV_ERR_UNSUPPORTED;
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
    *grid = (unsigned)(desc->B * per_sequence);
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
    if (!K_new || !V_new || !topk_idx || !K_shards || !V_shards || !K_scales || !V_scales || !utility || !n_valid)
        return PIKV_ERR_INVALID;
    if (k < 1 || k > desc->E) return PIKV_ERR_INVALID;
    if ((reuse_idx == nullptr) != (reuse_cnt == nullptr)) return PIKV_ERR_INVALID;
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
