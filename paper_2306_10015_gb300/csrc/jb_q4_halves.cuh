// jb_q4_halves.cuh -- how inputs of products with 4-bit weights become fp16: scaled by a power of two for each row (or a part of
// it), fp32 as an upper and a lower part.
#pragma once
#include <cstdint>

#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "jb_draft.h"

namespace jb {

__device__ __forceinline__ uint32_t halves(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// With `most` the largest finite size in [2^e, 2^(e+1)), it becomes [2^14, 2^15): the exponent of a power of two that fp32 has with
// its inverse.
__device__ __forceinline__ int exponent_of(float most) { return most > 0.0f ? min(max((__float_as_int(most) >> 23) - 127 - 14, -126), 126) : 0; }
// What inputs are multiplied by, and what sums of products with levels are.
__device__ __forceinline__ float scaled_down(int e) { return __uint_as_float(static_cast<uint32_t>(127 - e) << 23); }
template <bool kF32>
__device__ __forceinline__ float scaled_up(int e) { return __uint_as_float(static_cast<uint32_t>(127 + e) << 23) * (1.0f / kLevelScale<kF32>); }

// Two scaled inputs. fp32: what is not finite is all lower part, which the lower parts of levels, which may be 0, do not meet.
template <bool kF32>
__device__ __forceinline__ void split(float a, float b, uint32_t& upper, uint32_t& lower) {
    if constexpr (!kF32) {
        upper = halves(a, b);
    } else {
        upper = halves(isfinite(a) ? a : 0.0f, isfinite(b) ? b : 0.0f);
        const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&upper));
        lower = halves(a - h.x, b - h.y);
    }
}

}  // namespace jb
