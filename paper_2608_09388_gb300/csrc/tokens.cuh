// Shared device helpers of the token operators (layer norm, row embedding,
// 8-bit quantisation and linear layer): the row count, 16-byte pieces of a
// row as fp32, and the reductions over a row's threads.
#pragma once

#include <cuda_bf16.h>

#include "hc_internal.cuh"

namespace hc {

#if defined(__CUDACC__)

// launch_pdl with `cluster` neighbouring blocks of the grid to a cluster.
template <typename... KArgs, typename... Args>
hc_status launch_cluster(void (*kernel)(KArgs...), unsigned blocks, unsigned cluster, int threads,
                         size_t smem, cudaStream_t s, const char* what, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return check_cuda(cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...), what);
}

// Every thread of every block of the cluster; what was written before it, to
// shared or global memory, is seen after it by all of them.
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;\n" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The shared-memory address of block `rank` of the cluster that `addr` is here.
__device__ __forceinline__ uint32_t cluster_map(uint32_t addr, uint32_t rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(at) : "r"(addr), "r"(rank));
    return at;
}

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

// Arithmetic units of a piece: two fp32 values that one instruction adds,
// multiplies or accumulates, or one where a piece is a single element.
struct F1 {
    float v;
};
struct F2 {
    unsigned long long v;
};
__device__ __forceinline__ F2 make_f2(float a, float b) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 split(F2 a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ F1 add(F1 a, F1 b) {
    return {a.v + b.v};
}
__device__ __forceinline__ F1 mul(F1 a, F1 b) {
    return {a.v * b.v};
}
__device__ __forceinline__ F1 fma(F1 a, F1 b, F1 c) {
    return {fmaf(a.v, b.v, c.v)};
}
__device__ __forceinline__ float total(F1 a) {
    return a.v;
}
__device__ __forceinline__ F2 add(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 mul(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ float total(F2 a) {
    const float2 f = split(a);
    return f.x + f.y;
}
template <int VEC>
struct UnitOf {
    using type = F2;
    static constexpr int count = VEC / 2;
    static __device__ __forceinline__ F2 splat(float v) { return make_f2(v, v); }
    static __device__ __forceinline__ void store(float* p, F2 u) {
        const float2 f = split(u);
        p[0] = f.x;
        p[1] = f.y;
    }
};
template <>
struct UnitOf<1> {
    using type = F1;
    static constexpr int count = 1;
    static __device__ __forceinline__ F1 splat(float v) { return {v}; }
    static __device__ __forceinline__ void store(float* p, F1 u) { *p = u.v; }
};

// A piece of a row: VEC elements of T as loaded (16 bytes, or one element).
template <typename T, int VEC>
struct Piece;
template <typename T>
struct Piece<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T* p) { v = *p; }
    __device__ __forceinline__ void store(T* p) const { *p = v; }
    __device__ __forceinline__ float get(int) const { return to_f32(v); }
    __device__ __forceinline__ void set(int, float f) { v = from_f32<T>(f); }
    __device__ __forceinline__ void set_all(const float (&f)[1]) { v = from_f32<T>(f[0]); }
    __device__ __forceinline__ F1 unit(int) const { return {to_f32(v)}; }
    __device__ __forceinline__ void set_units(const F1 (&u)[1]) { v = from_f32<T>(u[0].v); }
};
template <>
struct Piece<float, 4> {
    float4 v;
    __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = v; }
    __device__ __forceinline__ float get(int i) const {
        return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
    }
    __device__ __forceinline__ void set(int i, float f) {
        (i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w) = f;
    }
    __device__ __forceinline__ void set_all(const float (&f)[4]) {
        v = make_float4(f[0], f[1], f[2], f[3]);
    }
    __device__ __forceinline__ F2 unit(int i) const {
        return i ? make_f2(v.z, v.w) : make_f2(v.x, v.y);
    }
    __device__ __forceinline__ void set_units(const F2 (&u)[2]) {
        const float2 a = split(u[0]), b = split(u[1]);
        v = make_float4(a.x, a.y, b.x, b.y);
    }
};
template <>
struct Piece<__nv_bfloat16, 2> {
    uint32_t v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        v = *reinterpret_cast<const uint32_t*>(p);
    }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const {
        *reinterpret_cast<uint32_t*>(p) = v;
    }
    __device__ __forceinline__ float get(int i) const {
        return __uint_as_float(i ? v & 0xffff0000u : v << 16);
    }
    __device__ __forceinline__ F2 unit(int) const { return make_f2(get(0), get(1)); }
    __device__ __forceinline__ void set_units(const F2 (&u)[1]) {
        const float2 a = split(u[0]);
        const __nv_bfloat162 b = __floats2bfloat162_rn(a.x, a.y);
        v = *reinterpret_cast<const uint32_t*>(&b);
    }
};
template <>
struct Piece<__nv_bfloat16, 4> {
    uint2 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        v = *reinterpret_cast<const uint2*>(p);
    }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const {
        *reinterpret_cast<uint2*>(p) = v;
    }
    __device__ __forceinline__ void set_all(const float (&f)[4]) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
        v = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    }
    __device__ __forceinline__ float get(int i) const {
        const uint32_t w = i >> 1 ? v.y : v.x;
        return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    }
};
template <>
struct Piece<__nv_bfloat16, 8> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        v = *reinterpret_cast<const uint4*>(p);
    }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const {
        *reinterpret_cast<uint4*>(p) = v;
    }
    __device__ __forceinline__ uint32_t word(int i) const {
        return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
    }
    // bf16 is the upper half of an fp32
    __device__ __forceinline__ float get(int i) const {
        const uint32_t w = word(i >> 1);
        return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    }
    __device__ __forceinline__ void set(int i, float f) {
        const uint32_t b = __bfloat16_as_ushort(__float2bfloat16_rn(f));
        uint32_t& w = (i >> 1) == 0 ? v.x : (i >> 1) == 1 ? v.y : (i >> 1) == 2 ? v.z : v.w;
        w = i & 1 ? (w & 0xffffu) | b << 16 : (w & 0xffff0000u) | b;
    }
    // two values to a word in one conversion
    __device__ __forceinline__ void set_all(const float (&f)[8]) {
        v = make_uint4(pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7]));
    }
    __device__ __forceinline__ F2 unit(int i) const {
        return make_f2(get(2 * i), get(2 * i + 1));
    }
    __device__ __forceinline__ void set_units(const F2 (&u)[4]) {
        const float2 a = split(u[0]), b = split(u[1]), c = split(u[2]), d = split(u[3]);
        v = make_uint4(pair(a.x, a.y), pair(b.x, b.y), pair(c.x, c.y), pair(d.x, d.y));
    }
    static __device__ __forceinline__ uint32_t pair(float lo, float hi) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&b);
    }
};

// p[c .. c + VEC), 16-byte aligned when VEC > 2, or `none` without a p.
template <int VEC>
__device__ __forceinline__ void load_units(const float* __restrict__ p, int c, float none,
                                           typename UnitOf<VEC>::type (&u)[UnitOf<VEC>::count]) {
    if constexpr (VEC == 1) {
        u[0].v = p ? __ldg(p + c) : none;
    } else if constexpr (VEC == 2) {
        u[0] = p ? make_f2(__ldg(p + c), __ldg(p + c + 1)) : make_f2(none, none);
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; i += 2) {
            const float4 f = p ? __ldg(reinterpret_cast<const float4*>(p + c + 2 * i))
                               : make_float4(none, none, none, none);
            u[i] = make_f2(f.x, f.y);
            u[i + 1] = make_f2(f.z, f.w);
        }
    }
}

// The same as plain numbers.
template <int VEC>
__device__ __forceinline__ void load_floats(const float* __restrict__ p, int c, float none,
                                            float (&f)[VEC]) {
    typename UnitOf<VEC>::type u[UnitOf<VEC>::count];
    load_units<VEC>(p, c, none, u);
    if constexpr (VEC == 1) {
        f[0] = u[0].v;
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const float2 v = split(u[i]);
            f[2 * i] = v.x;
            f[2 * i + 1] = v.y;
        }
    }
}

// a + b, rounded to their type. (bf16 pairs in one instruction: one rounding,
// as a sum in fp32 rounded again gives it too, since that one is exact wherever the
// smaller number reaches the last place of the result.)
template <typename P>
__device__ __forceinline__ P sum_of(const P& a, const P& b) {
    P r;
    r.v = a.v;
    if constexpr (sizeof(r.v) == 16) {
        r.v = make_float4(a.v.x + b.v.x, a.v.y + b.v.y, a.v.z + b.v.z, a.v.w + b.v.w);
    } else {
        const float f[1] = {a.get(0) + b.get(0)};
        r.set_all(f);
    }
    return r;
}
__device__ __forceinline__ uint32_t sum_words(uint32_t a, uint32_t b) {
    const __nv_bfloat162 s = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&a),
                                     *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&s);
}
__device__ __forceinline__ Piece<__nv_bfloat16, 2> sum_of(const Piece<__nv_bfloat16, 2>& a,
                                                          const Piece<__nv_bfloat16, 2>& b) {
    Piece<__nv_bfloat16, 2> r;
    r.v = sum_words(a.v, b.v);
    return r;
}
__device__ __forceinline__ Piece<__nv_bfloat16, 8> sum_of(const Piece<__nv_bfloat16, 8>& a,
                                                          const Piece<__nv_bfloat16, 8>& b) {
    Piece<__nv_bfloat16, 8> r;
    r.v = make_uint4(sum_words(a.v.x, b.v.x), sum_words(a.v.y, b.v.y), sum_words(a.v.z, b.v.z),
                     sum_words(a.v.w, b.v.w));
    return r;
}

// Sum over a group of TPR threads (a power of two; group g of the block owns
// threads g * TPR ..), the same value in each of them. A group of several
// warps passes the warps' sums through sh, [2][warps of the block] floats
// used in turn (`turn` 0, 1, 0, ..), so that one barrier a call is enough.
template <int TPR>
__device__ __forceinline__ float group_sum(float v, float* sh, int turn) {
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1)
        v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (TPR > 32) {
        constexpr int kWarps = TPR / 32;
        static_assert(kWarps % 4 == 0, "the warps' sums are read four at a time");
        const int g = threadIdx.x / TPR;
        float* const at = sh + (turn ? blockDim.x / 32 : 0) + g * kWarps;  // 16-byte aligned
        if ((threadIdx.x & 31) == 0) at[(threadIdx.x % TPR) >> 5] = v;
        asm volatile("bar.sync %0, %1;\n" ::"r"(g + 1), "r"(TPR) : "memory");
        v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; w += 4) {
            const float4 f = *reinterpret_cast<const float4*>(at + w);
            v += (f.x + f.y) + (f.z + f.w);
        }
    }
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
