// jb_scores.cuh -- what attention does to a score, for the kernels of jb_attend.cu and jb_tree.cu.
#pragma once
#include <cuda_runtime.h>

namespace jb {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.0e38f;

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// scale q.k under the cap, in units of ln 2. p.cap_in is scale / cap, p.cap_out cap / ln 2.
template <typename P>
__device__ __forceinline__ float capped(const P& p, float dot) {
    const float x = dot * (p.a.scale * kLog2e);
    // tanh(y) = 1 - 2 / (1 + e^2y), to a few 2^-24; near 0 that is not enough of a small y, and
    // tanh(y) / y = 1 - y^2/3 + 2 y^4/15 - 17 y^6/315 is good to 6e-8 below 1/5
    const float y = dot * p.cap_in, y2 = y * y;
    const float e = exp2_approx(y * (2.0f * kLog2e));
    const float large = fmaf(-2.0f * p.cap_out, __fdividef(1.0f, 1.0f + e), p.cap_out);
    const float small = x * fmaf(y2, fmaf(y2, fmaf(y2, -17.0f / 315.0f, 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
    return fabsf(y) < 0.2f ? small : large;
}

// The same of two scores where |scale q.k / cap| is below kSmallCap: tanh(y) / y up to y^12, good to 5e-8 there (the next term
// of the series is 0.0015 y^14).
constexpr float kSmallCap = 0.45f;
template <typename P>
__device__ __forceinline__ float2 capped_small(const P& p, float2 dot) {
    const auto both = [](float x) { return make_float2(x, x); };
    const float2 x = __fmul2_rn(dot, both(p.a.scale * kLog2e)), y = __fmul2_rn(dot, both(p.cap_in)), y2 = __fmul2_rn(y, y);
    float2 t = both(21844.0f / 6081075.0f);
    t = __ffma2_rn(t, y2, both(-1382.0f / 155925.0f));
    t = __ffma2_rn(t, y2, both(62.0f / 2835.0f));
    t = __ffma2_rn(t, y2, both(-17.0f / 315.0f));
    t = __ffma2_rn(t, y2, both(2.0f / 15.0f));
    t = __ffma2_rn(t, y2, both(-1.0f / 3.0f));
    t = __ffma2_rn(t, y2, both(1.0f));
    return __fmul2_rn(x, t);
}

// The score as the softmax takes it, in units of ln 2, as is the slope.
template <bool kExtra, typename P>
__device__ __forceinline__ float score(const P& p, float dot, float slope, int back) {
    if constexpr (!kExtra) {
        return dot * (p.a.scale * kLog2e);
    } else {
        const float x = p.a.softcap > 0.0f ? capped(p, dot) : dot * (p.a.scale * kLog2e);
        return fmaf(slope, static_cast<float>(back), x);
    }
}

}  // namespace jb
