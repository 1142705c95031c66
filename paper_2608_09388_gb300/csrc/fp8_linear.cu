// The 8-bit linear layer on compact rows:
//   y[n][o] = act( bias[o] + sum over blocks b of 128 channels of
//                  xs[b][n] * ws[o / 128][b] * sum_{c in b} xq[n][c] * wq[o][c] )
// Products of e4m3 values are exact in fp32 and are summed there; a block's
// sum is scaled in fp32 and added to the fp32 total.
#include <cuda_fp8.h>

#include "tokens.cuh"

namespace hc {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;
constexpr int kStep = 32;  // channels staged at a time

__device__ __forceinline__ float e4m3_value(uint8_t q) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(q, __NV_E4M3)));
}

// 64 rows x 64 output channels per block, 4 x 4 per thread.
template <typename T>
__global__ void __launch_bounds__(kThreads) fp8_linear_kernel(const Fp8LinearArgs a) {
    __shared__ float xt[kStep][kTile + 1], wt[kStep][kTile + 1];
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(a.count, a.capacity, a.status);
    const long long n0 = (long long)blockIdx.x * kTile;
    const int o0 = blockIdx.y * kTile;
    if (n0 >= rows) return;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int nbi = (a.C_in + 127) / 128;
    float tot[4][4] = {};
    for (int b = 0; b < nbi; ++b) {
        float acc[4][4] = {};
        for (int k0 = b * 128; k0 < b * 128 + 128 && k0 < a.pitch; k0 += kStep) {
            __syncthreads();
            for (int j = threadIdx.x; j < kTile * kStep; j += kThreads) {
                const int r = j / kStep, k = j % kStep;
                const bool in = k0 + k < a.pitch;
                xt[k][r] = in && n0 + r < rows ? e4m3_value(a.xq[(n0 + r) * a.pitch + k0 + k]) : 0.f;
                wt[k][r] = in && o0 + r < a.C_out
                               ? e4m3_value(a.wq[(long long)(o0 + r) * a.pitch + k0 + k])
                               : 0.f;
            }
            __syncthreads();
#pragma unroll 8
            for (int k = 0; k < kStep; ++k) {
                float xv[4], wv[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    xv[i] = xt[k][ty * 4 + i];
                    wv[i] = wt[k][tx * 4 + i];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xv[i], wv[j], acc[i][j]);
            }
        }
        const float w = a.ws[(long long)(o0 / 128) * nbi + b];  // a tile lies in one block of 128
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long n = n0 + ty * 4 + i;
            const float sc = n < rows ? a.xs[(long long)b * a.capacity + n] * w : 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) tot[i][j] = fmaf(acc[i][j], sc, tot[i][j]);
        }
    }
    T* y = static_cast<T*>(a.y);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long n = n0 + ty * 4 + i;
            const int o = o0 + tx * 4 + j;
            if (n < rows && o < a.C_out)
                y[n * a.C_out + o] =
                    from_f32<T>(act_apply(tot[i][j] + (a.bias ? a.bias[o] : 0.f), a.act));
        }
}

}  // namespace

hc_status launch_fp8_linear(const DeviceCtx*, const Fp8LinearArgs& a, cudaStream_t s) {
    const dim3 grid((unsigned)((a.capacity + kTile - 1) / kTile),
                    (unsigned)((a.C_out + kTile - 1) / kTile));
    if (grid.y > 65535u) {
        set_error("hc_fp8_linear_fwd: C_out=%d is too wide", a.C_out);
        return HC_ERR_UNSUPPORTED;
    }
    return a.y_dt == HC_BF16
               ? launch_pdl(fp8_linear_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, s,
                            "fp8_linear_kernel", a)
               : launch_pdl(fp8_linear_kernel<float>, grid, dim3(kThreads), 0, s,
                            "fp8_linear_kernel", a);
}

}  // namespace hc
