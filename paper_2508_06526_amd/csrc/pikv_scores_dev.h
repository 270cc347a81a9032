// Capped scores: cap tanh(s / cap).
#pragma once

#include "pikv_common.h"

#include <math.h>

namespace pikv {

// tanh x.  Small, for |x| < 1/2: x + x^3 P(x^2), P of degree 4 through tanh's values at the nodes of Chebyshev's polynomial over that range (off by
// 1.04 * 2^-24 of the value, roundings included).  Large: from exp(2 |x|), off by some 2^-23 whatever the value.
__device__ __forceinline__ float tanh_small(float x) {
    const float y = x * x;
    float t = -0.0069470033f;
    t = fmaf(t, y, 0.0214727204f);
    t = fmaf(t, y, -0.0539337881f);
    t = fmaf(t, y, 0.133332267f);
    t = fmaf(t, y, -0.333333313f);
    return fmaf(t * y, x, x);
}
__device__ __forceinline__ float tanh_large(float x) {
    const float e = __expf(2.0f * fabsf(x));         // (infinite: 1)
    return copysignf(fmaf(-2.0f, __builtin_amdgcn_rcpf(e + 1.0f), 1.0f), x);
}
// N products to parts of a cap, tanh(dot * by), by = scale / cap.  Where a wave holds one that is large, all of them are taken for such: off by
// 2^-23 of the cap, which is 2^-22 of that score.
template <int N>
__device__ __forceinline__ void cap_parts(float (&s)[N], float by) {
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] *= by;
        most = fmaxf(most, fabsf(s[i]));
    }
    if (__any(most >= 0.5f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = tanh_large(s[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = tanh_small(s[i]);
    }
}
template <int N>
__device__ __forceinline__ void cap_scores(float (&s)[N], float scale, float cap, float cap_rcp) {
    cap_parts(s, scale * cap_rcp);
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] *= cap;
}

}  // namespace pikv
