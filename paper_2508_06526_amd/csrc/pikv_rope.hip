// Norms of queries and keys for each head and the position rotation, out of a fused projection.
//
//   norm_rope : a block takes heads of one token, a 16-byte piece of a head per lane.
//               The sum of squares is joined by a butterfly over the head's lanes; the partner of a value in the rotation sits
//               rotary_dim / 2 values, whole lanes, away (or in the same lane, interleaved).  The angles of a token are the same for all of its
//               heads: cosines and sines are formed once per block, behind the first request for rows, and kept in LDS.
//
// Bound by memory: 16384 tokens x 48 heads of 128 bf16 values, 403 MB, in 71 us (5.7 TB/s; a plain copy here 5.1), 59 where the
// projection's rows are still in the Infinity Cache; a token in 2.5 us of the GPU's time, the launch and two trips to memory.
// Rows come through the caches, outputs go past them (with ordinary stores 75 us; rows past the caches as well 70, but 1024 tokens
// that are in them 8.1 instead of 6.9).
//
// Angle = position * inv_freq: in fp32 the product of a far position is off by its own rounding (position 10^6: 0.03
// radians), so it is formed in 64 bits, in revolutions; what is left after whole ones goes into cosine and sine as an fp32
// value and its remainder.
#include "pikv_mfma_dev.h"

#include <math.h>

namespace pikv {
namespace {

struct RopeParams {
    const void *x, *w_q, *w_k;
    const int32_t *positions;
    const float *inv_freq;
    void *q_out, *k_out, *v_out;
    int64_t token_stride;
    FastDiv by_parts;
    int Hq, Hkv, rotary, interleaved, heads, per_block;    // heads: of a token, in all; per_block: of them a block takes
    float eps;
};

constexpr int kRopeThreads = 256;

template <typename T, int D>
__global__ __launch_bounds__(kRopeThreads) void norm_rope(RopeParams p) {
    constexpr int VPL = Pack16<T>::N, LPR = D / VPL, STEP = kRopeThreads / LPR;      // values of a lane, lanes of a head, heads at once
    __shared__ float cos_s[64], sin_s[64];
    int part;
    const int token = fast_divide(p.by_parts, blockIdx.x, &part);
    const int tid = threadIdx.x, c = tid & (LPR - 1);
    const int first = part * p.per_block + tid / LPR, last = min(p.heads, (part + 1) * p.per_block);
    const int half = p.rotary >> 1;
    const T *row = static_cast<const T *>(p.x) + token * p.token_stride + VPL * c;
    auto load = [&](int head) { return load16(row + (int64_t)min(head, last - 1) * D); };      // (past the end: the last head once more)
    uint4 next = load(first);                // ahead of the angles
    if (tid < half) {
        const double turns = (double)p.positions[token] * (double)p.inv_freq[tid] * 0.15915494309189533577;      // 1 / (2 pi)
        const double half_turns = 2.0 * (turns - rint(turns));
        const float near = (float)half_turns, rest = (float)((half_turns - near) * M_PI);
        float sn, cs;
        sincospif(near, &sn, &cs);
        sin_s[tid] = fmaf(rest, cs, sn);         // what the rounding of the angle left, to first order (its square: 2^-47)
        cos_s[tid] = fmaf(-rest, sn, cs);
    }
    __syncthreads();
    for (int head = first; head < last; head += STEP) {
        const uint4 raw = next;
        if (head + STEP < last) next = load(head + STEP);
        const bool key = head >= p.Hq && head < p.Hq + p.Hkv, value = head >= p.Hq + p.Hkv;
        T *out;
        if (value) out = static_cast<T *>(p.v_out) + ((int64_t)token * p.Hkv + head - p.Hq - p.Hkv) * D;
        else if (key) out = static_cast<T *>(p.k_out) + ((int64_t)token * p.Hkv + head - p.Hq) * D;
        else out = static_cast<T *>(p.q_out) + ((int64_t)token * p.Hq + head) * D;
        out += VPL * c;
        if (value) {                                  // copied as they are
            store16_stream(out, raw);
            continue;
        }
        float z[VPL];
        Pack16<T>::widen(raw, z);
        const T *w = static_cast<const T *>(key ? p.w_k : p.w_q);
        if (w != nullptr) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) sum = fmaf(z[i], z[i], sum);
#pragma unroll
            for (int off = 1; off < LPR; off <<= 1) sum += __shfl_xor(sum, off, kWave);
            // r + rest = 1 / sqrt(v): r is off by the roundings of root and division, and rest is what they took (a step of Newton's,
            // r (1 - v r^2) / 2), so that the product is the only rounding of x / sqrt(v)
            const float v = sum * (1.0f / D) + p.eps, r = 1.0f / sqrtf(v);
            const float vr = v * r, vr_low = fmaf(v, r, -vr), left = fmaf(-vr, r, 1.0f) - vr_low * r;
            const float rest = r > 0.0f && r < INFINITY ? 0.5f * left * r : 0.0f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) z[i] = fmaf(z[i], r, z[i] * rest) * load_scalar<T>(w, VPL * c + i);
        }
        if (VPL * c < p.rotary) {                       // (rotary: a multiple of 16; a head's rotated lanes are whole pairs)
            if (p.interleaved) {
#pragma unroll
                for (int i = 0; i < VPL; i += 2) {
                    const float cs = cos_s[(VPL * c + i) / 2], sn = sin_s[(VPL * c + i) / 2], a = z[i], b = z[i + 1];
                    z[i] = a * cs - b * sn;
                    z[i + 1] = b * cs + a * sn;
                }
            } else {
                const bool second = VPL * c >= half;
                const int lane = tid & (kWave - 1), other = second ? lane - half / VPL : lane + half / VPL, i0 = second ? VPL * c - half : VPL * c;
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    const float with = __shfl(z[i], other, kWave), cs = cos_s[i0 + i], sn = sin_s[i0 + i];
                    z[i] = second ? z[i] * cs + with * sn : z[i] * cs - with * sn;
                }
            }
        }
        uint4 packed[1];
        if constexpr (VPL == 4) packed[0] = make_uint4(__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3]));
        else split_bf16(z, packed);
        store16_stream(out, packed[0]);
    }
}

}  // namespace
}  // namespace pikv

using namespace pikv;

extern "C" int pikv_norm_rope(const void *x, int32_t tokens, int64_t token_stride, int32_t Hq, int32_t Hkv, int32_t D,
                              int32_t dtype, const void *w_q, const void *w_k, float eps, const int32_t *positions,
                              const float *inv_freq, int32_t rotary_dim, int32_t interleaved, void *q_out, void *k_out,
                              void *v_out, void *stream) {
    if (tokens < 0 || Hq < 0 || Hkv < 0 || (Hq == 0 && Hkv == 0)) return PIKV_ERR_INVALID;
    if (dtype != PIKV_F32 && dtype != PIKV_BF16) return PIKV_ERR_INVALID;
    if (D != 16 && D != 32 && D != 64 && D != 128) return PIKV_ERR_UNSUPPORTED;
    if (rotary_dim < 0 || rotary_dim > D || rotary_dim % 16 != 0) return PIKV_ERR_INVALID;
    if (!(eps >= 0.0f) || eps > 3.0e38f) return PIKV_ERR_INVALID;
    const int64_t heads = (int64_t)Hq + (int64_t)Hkv * (v_out ? 2 : 1);
    if (heads > (1 << 20)) return PIKV_ERR_UNSUPPORTED;
    if (token_stride < heads * D || (token_stride * elem_bytes(dtype)) % 16 != 0) return PIKV_ERR_INVALID;
    if (tokens == 0) return PIKV_OK;             // (tensors without elements have no address)
    if (!x || (Hq > 0 && !q_out) || (Hkv > 0 && !k_out) || (rotary_dim > 0 && (!positions || !inv_freq))) return PIKV_ERR_INVALID;
    auto aligned = [](const void *ptr) { return reinterpret_cast<uintptr_t>(ptr) % 16 == 0; };
    if (!aligned(x) || !aligned(w_q) || !aligned(w_k) || !aligned(q_out) || !aligned(k_out) || !aligned(v_out)) return PIKV_ERR_INVALID;
    RopeParams p;
    p.x = x;
    p.w_q = w_q;
    p.w_k = w_k;
    p.positions = positions;
    p.inv_freq = inv_freq;
    p.q_out = q_out;
    p.k_out = k_out;
    p.v_out = v_out;
    p.token_stride = token_stride;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.rotary = rotary_dim;
    p.interleaved = interleaved ? 1 : 0;
    p.eps = eps;
    p.heads = (int)heads;
    const int at_once = kRopeThreads * 16 / (D * elem_bytes(dtype)), passes = (p.heads + at_once - 1) / at_once;
    // Few tokens: a block for each pass over heads, so that the passes run side by side (512 tokens x 80 heads of 128 values 6.7 against
    // 8.3 us).  Many: one block for all of a token's heads, its angles formed once (4096 tokens 36.7 -> 30.4).
    const int parts = (int64_t)tokens * passes <= 4096 ? passes : 1;
    p.per_block = parts > 1 ? at_once : p.heads;
    p.by_parts = fast_div(parts);
    if ((int64_t)tokens * parts > (1 << 23)) return PIKV_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)(tokens * parts));
    auto launch = [&](auto type) {
        typedef decltype(type) T;
        hipStream_t st = as_stream(stream);
        switch (D) {
            case 16: hipLaunchKernelGGL((norm_rope<T, 16>), grid, dim3(kRopeThreads), 0, st, p); break;
            case 32: hipLaunchKernelGGL((norm_rope<T, 32>), grid, dim3(kRopeThreads), 0, st, p); break;
            case 64: hipLaunchKernelGGL((norm_rope<T, 64>), grid, dim3(kRopeThreads), 0, st, p); break;
            default: hipLaunchKernelGGL((norm_rope<T, 128>), grid, dim3(kRopeThreads), 0, st, p); break;
        }
    };
    if (dtype == PIKV_F32) launch(float{});
    else launch(bf16{});
    return launch_status();
}
