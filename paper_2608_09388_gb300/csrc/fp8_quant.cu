// Rows and weights held in 8 bits: e4m3 values with one fp32 scale per block
// of 128 channels (rows) or per 128 x 128 block (weights).
//   scale = max(amax / 448, 2^-126),  q = e4m3(x / scale)
// with amax the block's largest magnitude, both quotients rounded to nearest
// even once, so that the largest magnitude of a block is held as 448. A block
// with a NaN has the scale NaN and NaN values; one with an infinity has the
// scale infinity, its infinities held as NaN: products of such a row are NaN.
#include <cuda_fp8.h>

#include "tokens.cuh"

namespace hc {
namespace {

constexpr int kThreads = 256;
constexpr float kE4m3Max = 448.f;
constexpr float kMinScale = 1.17549435e-38f;  // 2^-126

// Largest magnitude of two, NaN if either is NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
    return (a != a || a > b) ? a : b;
}
__device__ __forceinline__ float scale_of(float amax) {
    const float s = amax / kE4m3Max;
    return s < kMinScale ? kMinScale : s;  // a NaN passes
}
__device__ __forceinline__ uint8_t e4m3(float x, float scale) {
    return (uint8_t)__nv_cvt_float_to_fp8(x / scale, __NV_SATFINITE, __NV_E4M3);
}

// The e4m3 bytes of N values x / scale. x * (1 / scale) is within 2^-22 of
// the fp32 quotient (one rounding each of the reciprocal, the product and the
// quotient), so both round to the same e4m3 value unless a boundary between
// two of them is that near: a magnitude from 2^-6 up whose mantissa, cut to
// three bits, leaves one half give or take 4 units of the last place, or any
// magnitude below 2^-6, where e4m3 has fewer bits. Only those are divided.
template <int N>
__device__ __forceinline__ void to_e4m3(const float (&x)[N], float scale, float inv,
                                        uint32_t (&w)[N / 4]) {
    float t[N];
    bool near = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        t[i] = x[i] * inv;
        const uint32_t m = __float_as_uint(t[i]) & 0x7fffffffu;
        near |= (m & 0xfffffu) - 0x7fffcu <= 8u || (m < 0x3c800000u && m != 0u);
    }
    if (near) {
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = x[i] / scale;
    }
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const uint32_t lo =
            __nv_cvt_float2_to_fp8x2(make_float2(t[i], t[i + 1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi =
            __nv_cvt_float2_to_fp8x2(make_float2(t[i + 2], t[i + 3]), __NV_SATFINITE, __NV_E4M3);
        w[i / 4] = lo | hi << 16;
    }
}

// Blocks of 128 channels are numbered row by row. 128 / V lanes hold a block,
// V channels (16 bytes) each; a warp works on 32 V / 128 blocks at a time and
// has kAhead such steps in flight. VEC = V where rows allow 16-byte loads,
// else 1.
constexpr int kAhead = 4;

template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads)
    quant_rows_kernel(const T* __restrict__ x, const int32_t* count, long long capacity, int C,
                      int pitch, int nb, uint8_t* __restrict__ q, float* __restrict__ scales,
                      unsigned* status) {
    constexpr int V = 16 / (int)sizeof(T), kLanes = 128 / V, kBlocks = 32 / kLanes;
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    const int lane = threadIdx.x & 31, sub = lane / kLanes, part = lane % kLanes;
    const long long blocks = rows * nb;
    const long long step = (long long)gridDim.x * (kThreads / 32) * kBlocks * kAhead;
    long long g0 = (long long)((blockIdx.x * kThreads + threadIdx.x) >> 5) * kBlocks * kAhead;
    for (; g0 < blocks; g0 += step) {
        int b;
        long long n = div32(g0 + sub, nb, b);
        Piece<T, VEC> p[kAhead][V / VEC];
        long long at_n[kAhead];
        int at_b[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            at_n[k] = n;
            at_b[k] = b;
            const int c = b * 128 + part * V;
            const long long row = n < rows ? n : 0;  // absent blocks read row 0
#pragma unroll
            for (int v = 0; v < V / VEC; ++v)
                p[k][v].load(x + row * C + (c + v < C ? c + v : 0));
            b += kBlocks;
            while (b >= nb) {
                b -= nb;
                ++n;
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int c = at_b[k] * 128 + part * V;
            float f[V], m = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                f[v] = c + v < C ? p[k][v / VEC].get(v % VEC) : 0.f;
                m = max_nan(fabsf(f[v]), m);
            }
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1)
                m = max_nan(__shfl_xor_sync(0xffffffffu, m, o), m);
            if (at_n[k] >= rows) continue;
            const float sc = scale_of(m);
            uint32_t w[V / 4];
            to_e4m3<V>(f, sc, 1.f / sc, w);
            if (c < pitch) {
                uint8_t* const out = q + at_n[k] * pitch + c;
                if constexpr (V == 8)
                    *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
                else
                    *reinterpret_cast<uint32_t*>(out) = w[0];
            }
            if (part == 0) scales[(long long)at_b[k] * capacity + at_n[k]] = sc;
        }
    }
}

// A block per 128 x 128 block of W [C_in, C_out], written transposed.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    quant_weight_kernel(const T* __restrict__ W, int C_in, int C_out, int pitch, int nbi,
                        uint8_t* __restrict__ wq, float* __restrict__ ws) {
    __shared__ float red[kThreads / 32];
    __shared__ uint8_t tile[128][132];  // [channel in][channel out]
    pdl_wait();
    pdl_trigger();
    const int i0 = blockIdx.x * 128, o0 = blockIdx.y * 128;
    const int to = threadIdx.x & 127, ti = threadIdx.x >> 7;
    float m = 0.f;
    for (int i = ti; i < 128; i += 2)
        if (i0 + i < C_in && o0 + to < C_out)
            m = max_nan(fabsf(to_f32(W[(long long)(i0 + i) * C_out + o0 + to])), m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = max_nan(__shfl_xor_sync(0xffffffffu, m, o), m);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
    m = red[0];
    for (int w = 1; w < kThreads / 32; ++w) m = max_nan(red[w], m);
    const float sc = scale_of(m);
    if (threadIdx.x == 0) ws[(long long)blockIdx.y * nbi + blockIdx.x] = sc;
    for (int i = ti; i < 128; i += 2) {
        const bool in = i0 + i < C_in && o0 + to < C_out;
        tile[i][to] = in ? e4m3(to_f32(W[(long long)(i0 + i) * C_out + o0 + to]), sc) : 0;
    }
    __syncthreads();
    for (int j = threadIdx.x; j < 128 * 32; j += kThreads) {
        const int o = j >> 5, i = (j & 31) * 4;
        if (o0 + o < C_out && i0 + i < pitch) {
            const uint32_t w = (uint32_t)tile[i][o] | (uint32_t)tile[i + 1][o] << 8 |
                               (uint32_t)tile[i + 2][o] << 16 | (uint32_t)tile[i + 3][o] << 24;
            *reinterpret_cast<uint32_t*>(wq + (long long)(o0 + o) * pitch + i0 + i) = w;
        }
    }
}

template <typename T, int VEC>
hc_status quant_rows_as(const DeviceCtx* ctx, const void* x, const int32_t* count, int capacity,
                        int C, int pitch, int nb, uint8_t* q, float* scales, cudaStream_t s) {
    constexpr int kPerBlock = kThreads / 32 * kAhead * 32 / (128 * (int)sizeof(T) / 16);
    const long long need = ((long long)capacity * nb + kPerBlock - 1) / kPerBlock;
    const long long cap = (long long)ctx->num_sms * 16;
    return launch_pdl(quant_rows_kernel<T, VEC>, dim3((unsigned)(need < cap ? need : cap)),
                      dim3(kThreads), 0, s, "quant_rows_kernel", (const T*)x, count,
                      (long long)capacity, C, pitch, nb, q, scales, ctx->status);
}

template <typename T>
hc_status quant_rows(const DeviceCtx* ctx, const void* x, const int32_t* count, int capacity,
                     int C, int pitch, int nb, uint8_t* q, float* scales, cudaStream_t s) {
    constexpr int V = 16 / (int)sizeof(T);
    if (C % V == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0)
        return quant_rows_as<T, V>(ctx, x, count, capacity, C, pitch, nb, q, scales, s);
    return quant_rows_as<T, 1>(ctx, x, count, capacity, C, pitch, nb, q, scales, s);
}

}  // namespace

hc_status launch_quantize_fp8_rows(const DeviceCtx* ctx, const void* x, hc_dtype dt,
                                   const int32_t* count, int capacity, int C, uint8_t* q,
                                   float* scales, cudaStream_t s) {
    const int pitch = HC_FP8_PITCH(C), nb = (C + 127) / 128;
    return dt == HC_BF16 ? quant_rows<__nv_bfloat16>(ctx, x, count, capacity, C, pitch, nb, q, scales, s)
                         : quant_rows<float>(ctx, x, count, capacity, C, pitch, nb, q, scales, s);
}

hc_status launch_quantize_fp8_weight(const DeviceCtx*, const void* W, hc_dtype dt, int C_in,
                                     int C_out, uint8_t* wq, float* ws, cudaStream_t s) {
    const int pitch = HC_FP8_PITCH(C_in), nbi = (C_in + 127) / 128, nbo = (C_out + 127) / 128;
    if (nbo > 65535) {
        set_error("hc_quantize_fp8_weight: C_out=%d is too wide", C_out);
        return HC_ERR_UNSUPPORTED;
    }
    const dim3 grid((unsigned)nbi, (unsigned)nbo);
    if (dt == HC_BF16)
        return launch_pdl(quant_weight_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, s,
                          "quant_weight_kernel", (const __nv_bfloat16*)W, C_in, C_out, pitch, nbi,
                          wq, ws);
    return launch_pdl(quant_weight_kernel<float>, grid, dim3(kThreads), 0, s,
                      "quant_weight_kernel", (const float*)W, C_in, C_out, pitch, nbi, wq, ws);
}

}  // namespace hc
