// The 8-bit form's arithmetic, shared by the kernels that write it: the scale
// of a block from its largest magnitude, and e4m3(x / scale).
#pragma once

#include <cuda_fp8.h>

#include "tokens.cuh"

namespace hc {

#if defined(__CUDACC__)

constexpr float kE4m3Max = 448.f;
constexpr float kMinScale = 1.17549435e-38f;  // 2^-126

__device__ __forceinline__ float scale_of(float amax) {
    const float s = amax / kE4m3Max;
    return s < kMinScale ? kMinScale : s;  // a NaN passes
}
// (a, b) * (s, s), one instruction for both.
__device__ __forceinline__ float2 mul_pair(float a, float b, float s) {
    unsigned long long v, ss;
    float2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    asm("mov.b64 %0, {%1, %1};" : "=l"(ss) : "f"(s));
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(ss));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}

// The first n of a word's four bytes.
__device__ __forceinline__ uint32_t first_bytes(int n) {
    return n >= 4 ? 0xffffffffu : n > 0 ? (1u << 8 * n) - 1u : 0u;
}

// The e4m3 bytes of N values x / scale. With inv the rounded reciprocal,
// x * (inv * (1 - 2^-21)) and x * (inv * (1 + 2^-21)) enclose the fp32
// quotient (four roundings of at most 2^-24 each separate it from x * inv),
// and rounding to e4m3 is monotonic: where both products round alike, so does
// the quotient. Only the others are divided.
template <int N>
__device__ __forceinline__ void to_e4m3(const float (&x)[N], float scale, float inv,
                                        uint32_t (&w)[N / 4]) {
    const float below = inv * (1.f - 0x1p-21f), above = inv * (1.f + 0x1p-21f);
    uint32_t differ = 0;
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float2 a = mul_pair(x[i], x[i + 1], below), b = mul_pair(x[i + 2], x[i + 3], below);
        const float2 c = mul_pair(x[i], x[i + 1], above), d = mul_pair(x[i + 2], x[i + 3], above);
        w[i / 4] = pack_e4m3(a.x, a.y, b.x, b.y);
        differ |= w[i / 4] ^ pack_e4m3(c.x, c.y, d.x, d.y);
    }
    if (differ) {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            w[i / 4] = pack_e4m3(x[i] / scale, x[i + 1] / scale, x[i + 2] / scale, x[i + 3] / scale);
    }
}

// Largest magnitude of a lane's 16 bytes of channels as fp32 bits: magnitudes
// compare as unsigned numbers, a NaN above all.
__device__ __forceinline__ uint32_t amax_bits(const Piece<float, 4>& p) {
    const uint32_t a = max(__float_as_uint(fabsf(p.v.x)), __float_as_uint(fabsf(p.v.y)));
    const uint32_t b = max(__float_as_uint(fabsf(p.v.z)), __float_as_uint(fabsf(p.v.w)));
    return max(a, b);
}
__device__ __forceinline__ uint32_t amax_bits(const Piece<__nv_bfloat16, 8>& p) {
    constexpr uint32_t kMag = 0x7fff7fffu;
    const uint32_t m = __vmaxu2(__vmaxu2(p.v.x & kMag, p.v.y & kMag),
                                __vmaxu2(p.v.z & kMag, p.v.w & kMag));
    return max(m << 16, m & 0xffff0000u);
}

#endif  // __CUDACC__

}  // namespace hc
