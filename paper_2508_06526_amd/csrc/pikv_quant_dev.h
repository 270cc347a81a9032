// The 8-bit formats of the quantised cache: scales, codes and the values they stand for.
//
// A block's scale is a power of two, so x / scale is exact and a code as it is written is ONE rounding of x: kernels, tests and any
// other machine agree to the bit, a value code * scale has at most 8 significant bits and is exact in bf16, and a block whose
// scale grows rounds its codes (a second time) by a shift of the exponent.  (With scale = max / 127 the midpoint max / 2 falls on a tie
// that fp32 decides by the error of its division; what a power of two costs is up to one bit of int8, none of e4m3.)
#pragma once

#include "pikv_common.h"

namespace pikv {

// Host-side checks common to the calls on 8-bit shards.
inline int check_quant(const pikv_desc *d, int format, int block) {
    const int rc = check_desc(d, true);
    if (rc != PIKV_OK) return rc;
    if (format != PIKV_QUANT_INT8 && format != PIKV_QUANT_E4M3) return PIKV_ERR_INVALID;
    if (block != 16 && block != 32 && block != 64 && block != 128) return PIKV_ERR_INVALID;
    if (d->rank != 0 || d->D < 32 || d->S > (1 << 30)) return PIKV_ERR_UNSUPPORTED;
    if (d->stride_s % 16 != 0 || d->stride_h % 16 != 0) return PIKV_ERR_INVALID;     // bytes
    return PIKV_OK;
}

// Scales are kept as the bits of the fp32 power of two while they are compared: their unsigned order is
// that of the scales, a NaN above all.
constexpr uint32_t kNanScale = 0x7fc00000u;

// A block with an entry that holds a NaN or an infinity has a NaN for a scale, whose low eight bits are the exponent of the scale
// that the other entries' codes have, and that entry, in place of codes, a byte that no finite value gets: all read as
// NaN until such entries are gone, the others as before from then on.  Exponent 0: no codes were kept.
__device__ __forceinline__ uint32_t poisoned_scale(uint32_t scale) { return kNanScale | scale >> 23; }
__device__ __forceinline__ uint32_t kept_scale(uint32_t word) { return (word & ~0xffu) == kNanScale ? (word & 0xffu) << 23 : 0u; }
template <int F>
__device__ __forceinline__ uint32_t no_codes() {
    return F == PIKV_QUANT_INT8 ? 0x80808080u : 0x7f7f7f7fu;
}
template <int F>
__device__ __forceinline__ bool has_no_codes(uint32_t codes) {
    return F == PIKV_QUANT_INT8 ? (codes & 0xffu) == 0x80u : (codes & 0x7fu) == 0x7fu;
}

// The scale needed by magnitudes of up to `most` (bits of a non-negative fp32): the smallest power of two, 2^-126 at
// the least, with most <= limit * scale, limit = 127 = 1.984375 * 2^6 or 448 = 1.75 * 2^8.
template <int F>
__device__ __forceinline__ uint32_t needed_scale(uint32_t most) {
    constexpr uint32_t kMantissa = F == PIKV_QUANT_INT8 ? 0x7e0000u : 0x600000u;       // of the limit
    constexpr int kExponent = F == PIKV_QUANT_INT8 ? 6 : 8;
    if (most >= 0x7f800000u) return kNanScale;
    const int e = (int)((most + (0x7fffffu - kMantissa)) >> 23) - kExponent;           // biased; one more past the limit's mantissa
    return (uint32_t)max(e, 1) << 23;
}

// 1 / scale; 0 for a NaN scale, whose codes are then 0.
__device__ __forceinline__ float inverse_scale(uint32_t scale) {
    return scale >= 0x7f800000u ? 0.0f : __uint_as_float((254u << 23) - scale);
}

// Four codes of x * inv, nearest, ties to even (inv a power of two: the products are exact).  |x * inv| is at most the
// largest code, so that nothing saturates.
template <int F>
__device__ __forceinline__ uint32_t encode4(const float *x, float inv) {
    if constexpr (F == PIKV_QUANT_INT8) {
        // the low byte of 1.5 * 2^23 + v is v in two's complement, rounded by that one addition
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(fmaf(x[i], inv, 12582912.0f));
        const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(w[3], w[2], 0x04000c0cu);
        return lo | hi;
    } else {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
        return (uint32_t)w;
    }
}

template <int F>
__device__ __forceinline__ void decode4(uint32_t codes, float *x) {
    if constexpr (F == PIKV_QUANT_INT8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(codes >> (8 * i));
    } else {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
        x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
    }
}

}  // namespace pikv
