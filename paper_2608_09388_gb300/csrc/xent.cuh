// Shared by the kernels of the cross entropy: the exponential, and the pairs
// (largest, sum of exponentials below it) that sums of exponentials are kept in.
#pragma once

#include "tokens.cuh"

namespace hc {

#if defined(__CUDACC__)

constexpr float kLog2e = 1.4426950408889634f;

// 2^v, 2 units in the last place; results below the normal numbers are zero.
__device__ __forceinline__ float ex2(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// (top, sum) and another pair as one; tops of -infinity hold nothing, a NaN stays.
__device__ __forceinline__ float2 join_pairs(float2 a, float2 b) {
    const float least = -__int_as_float(0x7f800000);
    const float top = fmaxf(a.x, b.x), from = top == least ? 0.f : top;
    return make_float2(top, a.y * ex2((a.x - from) * kLog2e) + b.y * ex2((b.x - from) * kLog2e));
}
// The pairs of `kLanes` neighbouring lanes as one, in each of them.
template <int kLanes>
__device__ __forceinline__ float2 join_lanes(float2 p) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1)
        p = join_pairs(p, make_float2(__shfl_xor_sync(0xffffffffu, p.x, o),
                                      __shfl_xor_sync(0xffffffffu, p.y, o)));
    return p;
}

#endif  // __CUDACC__

}  // namespace hc
