// Pieces of the matrix-core attention kernels: values as sums of bf16 operands, operands from memory, joins of lane groups.
#pragma once

#include "pikv_common.h"

namespace pikv {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// max over the four lanes c, c + 16, c + 32, c + 48, in all of them, without LDS: the swaps leave
// the two halves (then the two rows of each half) side by side in two registers.
__device__ __forceinline__ float group_max(float x) {
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
    const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// fp32 values (8 for uint4, 4 for uint2) as PARTS bf16 operands whose sum they are: each part
// rounds what the parts before it left (2 parts carry 16 bits of a value, 3 parts all 24).
template <int PARTS, typename OP>
__device__ __forceinline__ void split_bf16(const float *v, OP (&out)[PARTS]) {
    constexpr int NW = sizeof(OP) / 4;
    struct Words {
        uint32_t w[NW];
    } words[PARTS];
#pragma unroll
    for (int u = 0; u < NW; ++u) {
        f32x2_t rest = {v[2 * u], v[2 * u + 1]};
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
            const bf16x2_t part = __builtin_convertvector(rest, bf16x2_t);
            words[k].w[u] = __builtin_bit_cast(uint32_t, part);
            if (k + 1 < PARTS) rest = rest - f32x2_t{(float)part[0], (float)part[1]};
        }
    }
#pragma unroll
    for (int k = 0; k < PARTS; ++k) out[k] = __builtin_bit_cast(OP, words[k]);
}

// Consecutive bf16 query values as an operand; a caller's q need not be 16-byte aligned.
template <typename OP>
__device__ __forceinline__ OP load_query(const bf16 *q, bool aligned) {
    if (aligned) return *reinterpret_cast<const OP *>(q);
    struct {
        uint16_t v[sizeof(OP) / 2];
    } parts;
#pragma unroll
    for (unsigned i = 0; i < sizeof(OP) / 2; ++i) parts.v[i] = q[i].bits;
    return __builtin_bit_cast(OP, parts);
}

__device__ __forceinline__ void hold_operand(uint4 &v) {
    asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w));
}
__device__ __forceinline__ void hold_operand(uint2 &v) { asm volatile("" : "+v"(v.x), "+v"(v.y)); }

}  // namespace pikv
