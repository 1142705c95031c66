// Shared device helpers of the token operators (layer norm, row embedding,
// 8-bit quantisation and linear layer): the row count, 16-byte pieces of a
// row as fp32, and the reductions over a row's threads.
#pragma once

#include <cuda_bf16.h>

#include "hc_internal.cuh"

namespace hc {

#if defined(__CUDACC__)

// Rows in use: *count clamped to [0, capacity] (reported when it was
// outside), or every row when count is NULL.
__device__ __forceinline__ long long token_rows(const int32_t* count, long long capacity,
                                                unsigned* status) {
    if (count == nullptr) return capacity;
    long long n = *count;
    if (n < 0) {
        report(status, kErrIndex);
        return 0;
    }
    if (n > capacity) {
        report(status, kErrCapacity);
        return capacity;
    }
    return n;
}

__device__ __forceinline__ float to_f32(float v) {
    return v;
}
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) {
    return __bfloat162float(v);
}
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) {
    return v;
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) {
    return __float2bfloat16_rn(v);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Sum over the block, the same value in every thread; sh holds one float per
// warp and is free again when the next call's first barrier has been passed.
__device__ __forceinline__ float block_sum(float v, float* sh) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    v = warp_sum(v);
    __syncthreads();
    if (lane == 0) sh[warp] = v;
    __syncthreads();
    return warp_sum(lane < warps ? sh[lane] : 0.f);
}

#endif  // __CUDACC__

}  // namespace hc
