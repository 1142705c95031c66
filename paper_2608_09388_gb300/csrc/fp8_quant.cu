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

// A warp per (row, block of 128 channels).
template <typename T>
__global__ void __launch_bounds__(kThreads)
    quant_rows_kernel(const T* __restrict__ x, const int32_t* count, long long capacity, int C,
                      int pitch, int nb, uint8_t* __restrict__ q, float* __restrict__ scales,
                      unsigned* status) {
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    const int lane = threadIdx.x & 31;
    const long long items = rows * nb;
    for (long long it = (blockIdx.x * (long long)kThreads + threadIdx.x) >> 5; it < items;
         it += (long long)gridDim.x * (kThreads / 32)) {
        int b;
        const long long n = div32(it, nb, b);
        float v[4], m = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = b * 128 + lane * 4 + j;
            v[j] = c < C ? to_f32(x[n * C + c]) : 0.f;
            m = max_nan(fabsf(v[j]), m);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = max_nan(__shfl_xor_sync(0xffffffffu, m, o), m);
        const float sc = scale_of(m);
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w |= (b * 128 + lane * 4 + j < C ? (uint32_t)e4m3(v[j], sc) : 0u) << (8 * j);
        if (b * 128 + lane * 4 < pitch)
            *reinterpret_cast<uint32_t*>(q + n * pitch + b * 128 + lane * 4) = w;
        if (lane == 0) scales[(long long)b * capacity + n] = sc;
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

}  // namespace

hc_status launch_quantize_fp8_rows(const DeviceCtx* ctx, const void* x, hc_dtype dt,
                                   const int32_t* count, int capacity, int C, uint8_t* q,
                                   float* scales, cudaStream_t s) {
    const int pitch = HC_FP8_PITCH(C), nb = (C + 127) / 128;
    long long blocks = ((long long)capacity * nb + kThreads / 32 - 1) / (kThreads / 32);
    const long long cap = (long long)ctx->num_sms * 16;
    if (blocks > cap) blocks = cap;
    if (dt == HC_BF16)
        return launch_pdl(quant_rows_kernel<__nv_bfloat16>, dim3((unsigned)blocks), dim3(kThreads),
                          0, s, "quant_rows_kernel", (const __nv_bfloat16*)x, count,
                          (long long)capacity, C, pitch, nb, q, scales, ctx->status);
    return launch_pdl(quant_rows_kernel<float>, dim3((unsigned)blocks), dim3(kThreads), 0, s,
                      "quant_rows_kernel", (const float*)x, count, (long long)capacity, C, pitch,
                      nb, q, scales, ctx->status);
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
