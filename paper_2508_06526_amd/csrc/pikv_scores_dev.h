// Capped scores: cap tanh(s / cap).  What a call may give for cap and scale.
#pragma once

#include "pikv_common.h"

#include <math.h>

namespace pikv {

// Host: a scale of a call as the kernels take it, and whether their factors are finite: an infinite one makes a NaN of a product that is zero.
inline float score_scale(float scale, int D) { return scale > 0.0f ? scale : 1.0f / sqrtf((float)D); }
inline bool score_factors_finite(float scale, int D, float cap) {
    if (cap == 0.0f) return true;
    const float rcp = 1.0f / cap, by = score_scale(scale, D) * rcp;
    return rcp - rcp == 0.0f && by - by == 0.0f;
}

// tanh x.  Small, for |x| < 1/2: x + x^3 P(x^2), P of degree 4 through tanh's values at the nodes of Chebyshev's polynomial over that range (off by
// 1.04 * 2^-24 of the value, roundings included).  Large, for the others: from exp(2 |x|), off by at most 3.6 * 2^-24 - of the exponential 1.4, of the
// sum and its reciprocal 1.6, of the result 0.5 -, which is less than 2^-21 of these values.
constexpr float kTanhSmall = 0.5f;
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
    const float e = __builtin_amdgcn_exp2f(fabsf(x) * 2.88539008177792681472f);      // (2 log2 e; infinite: 1)
    return copysignf(fmaf(-2.0f, __builtin_amdgcn_rcpf(e + 1.0f), 1.0f), x);
}
// N products to parts of a cap, tanh(dot * by), by = scale / cap.  Each score takes its own form: neither what is not seen nor another row of the wave
// has a part in its bits.  The larger form is only entered where a wave holds a score that needs it.
template <int N>
__device__ __forceinline__ void cap_parts(float (&s)[N], float by) {
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] *= by;
        most = fmaxf(most, fabsf(s[i]));
    }
    if (__any(most >= kTanhSmall)) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = fabsf(s[i]) < kTanhSmall ? tanh_small(s[i]) : tanh_large(s[i]);
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
