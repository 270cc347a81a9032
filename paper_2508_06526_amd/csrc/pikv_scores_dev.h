// Capped scores: cap tanh(s / cap).
#pragma once

#include "pikv_common.h"

#include <math.h>

namespace pikv {

// tanh x.  Small: the odd Taylor polynomial to x^15, for |x| < 1/2 (the next term is 0.15 * 2^-24 of the value).  Large: from exp(2 |x|), off by
// some 2^-23 whatever the value.
__device__ __forceinline__ float tanh_small(float x) {
    const float y = x * x;
    float t = -0.00145583438f;           // -929569 / 638512875
    t = fmaf(t, y, 0.00359212803f);      // 21844 / 6081075
    t = fmaf(t, y, -0.00886323552f);     // -1382 / 155925
    t = fmaf(t, y, 0.0218694885f);       // 62 / 2835
    t = fmaf(t, y, -0.0539682540f);      // -17 / 315
    t = fmaf(t, y, 0.133333333f);        // 2 / 15
    t = fmaf(t, y, -0.333333333f);
    return fmaf(t * y, x, x);
}
__device__ __forceinline__ float tanh_large(float x) {
    const float e = __expf(2.0f * fabsf(x));         // (infinite: 1)
    return copysignf(fmaf(-2.0f, __builtin_amdgcn_rcpf(e + 1.0f), 1.0f), x);
}
// Products of N scores to capped ones, s = cap tanh(dot * scale / cap).  Where a wave holds a score that is large, all of them are taken
// for such: off by 2^-23 of the cap, which is 2^-22 of that score.
template <int N>
__device__ __forceinline__ void cap_scores(float (&s)[N], float scale, float cap, float cap_rcp) {
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] = s[i] * scale * cap_rcp;
        most = fmaxf(most, fabsf(s[i]));
    }
    if (__any(most >= 0.5f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = cap * tanh_large(s[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = cap * tanh_small(s[i]);
    }
}

}  // namespace pikv
