// The 8-bit form's arithmetic, shared by the kernels that write it: the scale
// of a block from its largest magnitude, and e4m3(x / scale).
#pragma once

#include <cuda_fp8.h>

#include "tokens.cuh"

namespace hc {

#if defined(__CUDACC__)

constexpr float kE4m3Max = 448.f;
constexpr float kMinScale = 1.17549435e-38f;  // 2^-126

// Where a number lies below this, its block is worked on 2^64 times as large:
// a residual (see to_e4m3) would leave the range of fp32.
constexpr float kTiny = 0x1p-90f, kUp = 0x1p64f, kDown = 0x1p-64f;

// max(amax / 448, 2^-126) by Markstein's correction; an infinity or a NaN passes.
__device__ __forceinline__ float scale_of(float amax) {
    constexpr float kInv = 1.f / kE4m3Max;
    const bool tiny = amax < kTiny;
    const float a = tiny ? amax * kUp : amax, q = a * kInv;
    const float c = fmaf(fmaf(q, -kE4m3Max, a), kInv, q), s = tiny ? c * kDown : c;
    return !(amax < __int_as_float(0x7f800000)) ? amax : s < kMinScale ? kMinScale : s;
}
// The largest magnitude of three, a NaN if one of them is.
__device__ __forceinline__ float max_mag(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
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

// The e4m3 bytes of N values x / scale, inv the rounded reciprocal of scale. The
// quotient is q - (q * scale - x) * inv with q = x * inv (Markstein's
// correction): the residual is exact, and with a correctly rounded inv the
// result is the correctly rounded quotient, as the division gives it, also
// for a zero of either sign. Under a scale that is infinite or a NaN the
// values are divided.
template <int N>
__device__ __forceinline__ void to_e4m3(const float (&x)[N], float scale, float inv,
                                        uint32_t (&w)[N / 4]) {
    if (scale < __int_as_float(0x7f800000)) {
        const bool tiny = scale < kTiny;
        const float sc = tiny ? scale * kUp : scale, in = tiny ? inv * kDown : inv;
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = x[i];
        if (tiny) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= kUp;
        }
        const F2 s = make_f2(sc, sc), i1 = make_f2(in, in), i2 = make_f2(-in, -in);
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            float2 f[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float a = v[i + 2 * h], b = v[i + 2 * h + 1];
                const F2 q = mul(make_f2(a, b), i1);
                f[h] = split(fma(fma(q, s, make_f2(-a, -b)), i2, q));
            }
            w[i / 4] = pack_e4m3(f[0].x, f[0].y, f[1].x, f[1].y);
        }
    } else {
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
