// Sums over blocks of rows, joined: out[c] = sum of part[p][c] in a fixed
// order. Used where a gradient of a per-channel parameter is summed by many
// blocks, each of which leaves its own sums of every channel.
#include "tokens.cuh"

namespace hc {
namespace {

// 32 channels per block; 32 warps add every 32nd part in order, then the
// warps' sums are added in order. 4 us for 152 parts of 2048 channels.
constexpr int kWarps = 32;

__global__ void __launch_bounds__(kWarps * 32)
    column_sum_kernel(const float* __restrict__ part, int parts, long long pitch, int C,
                      float* __restrict__ out, const int* rows) {
    __shared__ float sh[kWarps][33];
    pdl_wait();
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long c = blockIdx.x * 32ll + lane;
    if (rows) parts = min(parts, (int)((*rows + 31ll) / 32));
    float v = 0.f;
    if (c < C) {
#pragma unroll 8
        for (int p = warp; p < parts; p += kWarps) v += part[p * pitch + c];
    }
    sh[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && c < C) {
        v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += sh[w][lane];
        out[c] = v;
    }
}

}  // namespace

hc_status launch_column_sum(const float* part, int parts, long long pitch, int C, float* out,
                            cudaStream_t s, const int* rows) {
    const unsigned grid = (unsigned)(((long long)C + 31) / 32);
    return launch_pdl(column_sum_kernel, dim3(grid), dim3(kWarps * 32), 0, s, "column_sum_kernel",
                      part, parts, pitch, C, out, rows);
}

}  // namespace hc
