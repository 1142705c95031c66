// The cross entropy behind a linear layer for a small head: up to 128 classes of
// up to 256 channels, 8192 weights at most (the semantic label of a vertex). The
// formulas are those of linear_xent.cu. W stays in shared memory as fp32, and a
// block takes 32 tokens at a time through all products on the CUDA cores, in
// fp32 throughout: no gather, no G in memory, one launch forward and two
// backward, where the tensor-core path waits for eleven.
//
// 256 threads as 16 x 16. Logits: thread (ty, tx) has the tokens 2 ty, 2 ty + 1 and
// the classes tx + 16 j, all channels. dx: the same tokens, the channels 4 (tx +
// 16 k) .. + 3, all classes. dW: the classes ty + 16 j and those channels, all
// tokens of the block, kept in registers over its tiles. Rows of shared
// memory are 4 floats longer than a multiple of 64, so that 16 rows' 16-byte
// pieces fall into different banks. Bound by launches and, behind them, by shared
// memory: 5 wavefronts for 12 products of four channels.
#include "xent.cuh"

namespace hc {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 32;
constexpr int kMaxPerThread = 8;  // VJ * CJ: 32 sums of dW a thread

// Blocks of a multiprocessor, by the registers of a thread's sums (64 where there are
// four). Loss and gradients of 16763 of 42 x 64 fp32: 30 us so, 33 with four blocks
// backward, 36 with three of both; of a million of 5 x 16 418 us, 504 with two backward.
template <int VJ, int CJ>
constexpr int kForward = VJ * CJ <= 4 ? 4 : 2;
template <int VJ, int CJ>
constexpr int kBackward = VJ * CJ <= 2 ? 4 : 2;

struct SmallArgs {
    const void* x;
    const void* W;
    const float* bias;
    const int32_t* targets;
    const int32_t* count;
    long long capacity;
    int C, V;
    float* loss;  // forward
    float* lse_out;
    const float* lse;  // backward
    const float* dloss;
    void* dx;
    float* part;  // [blocks][V * C + V], or NULL
    bool wide_x, wide_dx;  // rows allow four elements at a time
    unsigned* status;
};

template <typename T>
__device__ __forceinline__ void load4(const T* p, int left, bool wide, float (&f)[4]) {
    if (wide) {
        Piece<T, 4> q;
        q.load(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = q.get(e);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = e < left ? to_f32(p[e]) : 0.f;
    }
}

template <typename T, int VJ, int CJ>
struct Head {
    static constexpr int kRow = 64 * CJ + 4;   // floats of a row of x or W
    static constexpr int kGRow = 16 * VJ + 4;  // of a token's classes
    static constexpr size_t kSmem = 4 * (16 * VJ * kRow + kTokens * kRow + kTokens * kGRow);

    // W, zero where there is no class or channel.
    static __device__ __forceinline__ void load_weight(const SmallArgs& a, float* w) {
        const T* const from = static_cast<const T*>(a.W);
        for (int i = threadIdx.x; i < 16 * VJ * 64 * CJ; i += kThreads) {
            const int v = i / (64 * CJ), c = i % (64 * CJ);
            w[v * kRow + c] = v < a.V && c < a.C ? to_f32(from[(long long)v * a.C + c]) : 0.f;
        }
    }
    // The tile's rows, zero for tokens that take no part (whatever they hold).
    static __device__ __forceinline__ void load_rows(const SmallArgs& a, long long n0, long long rows,
                                                     float* x) {
        const T* const from = static_cast<const T*>(a.x);
#pragma unroll
        for (int i = threadIdx.x; i < kTokens * 16 * CJ; i += kThreads) {
            const int r = i / (16 * CJ), c = i % (16 * CJ) * 4;
            float f[4] = {0.f, 0.f, 0.f, 0.f};
            if (n0 + r < rows && c < a.C) {
                const int t = a.targets[n0 + r];
                load4(from + (n0 + r) * a.C + c, a.C - c, a.wide_x, f);
                if (t < 0 || t >= a.V) f[0] = f[1] = f[2] = f[3] = 0.f;
            }
            *reinterpret_cast<float4*>(x + r * kRow + c) = make_float4(f[0], f[1], f[2], f[3]);
        }
    }
    // Target of token n: -1 where it takes no part.
    static __device__ __forceinline__ int target(const SmallArgs& a, long long n, long long rows) {
        if (n >= rows) return -1;
        const int t = a.targets[n];
        if (t < -1 || t >= a.V) {
            if (threadIdx.x % 16 == 0) report(a.status, kErrIndex);
            return -1;
        }
        return t;
    }
    // l[k][j]: token 2 ty + k, class tx + 16 j; -infinity where there is no class.
    static __device__ __forceinline__ void logits(const SmallArgs& a, const float* x, const float* w,
                                                  float (&l)[2][VJ]) {
        const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < VJ; ++j) l[k][j] = 0.f;
        const int n4 = (a.C + 3) / 4;
#pragma unroll 4
        for (int c = 0; c < n4; ++c) {
            float4 f[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
                f[k] = *reinterpret_cast<const float4*>(x + (2 * ty + k) * kRow + 4 * c);
#pragma unroll
            for (int j = 0; j < VJ; ++j) {
                const float4 g = *reinterpret_cast<const float4*>(w + (tx + 16 * j) * kRow + 4 * c);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    l[k][j] = fmaf(f[k].x, g.x, l[k][j]);
                    l[k][j] = fmaf(f[k].y, g.y, l[k][j]);
                    l[k][j] = fmaf(f[k].z, g.z, l[k][j]);
                    l[k][j] = fmaf(f[k].w, g.w, l[k][j]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < VJ; ++j) {
            const int v = tx + 16 * j;
            const float b = a.bias && v < a.V ? __ldg(a.bias + v) : 0.f;
#pragma unroll
            for (int k = 0; k < 2; ++k) l[k][j] = v < a.V ? l[k][j] + b : -__int_as_float(0x7f800000);
        }
    }
};

template <typename T, int VJ, int CJ>
__global__ void __launch_bounds__(kThreads, kForward<VJ, CJ>) xent_small_fwd_kernel(const SmallArgs a) {
    using H = Head<T, VJ, CJ>;
    extern __shared__ __align__(16) float smem[];
    float *const w = smem, *const x = w + 16 * VJ * H::kRow;
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(a.count, a.capacity, a.status);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    if (blockIdx.x * (long long)kTokens >= rows) return;
    H::load_weight(a, w);
    for (long long n0 = blockIdx.x * (long long)kTokens; n0 < rows; n0 += gridDim.x * (long long)kTokens) {
        H::load_rows(a, n0, rows, x);
        __syncthreads();
        float l[2][VJ];
        H::logits(a, x, w, l);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const long long n = n0 + 2 * ty + k;
            const int t = H::target(a, n, rows);
            const float least = -__int_as_float(0x7f800000);
            float top = least, at = 0.f, sum = 0.f;
#pragma unroll
            for (int j = 0; j < VJ; ++j) {
                top = fmaxf(top, l[k][j]);
                at = tx + 16 * j == t ? l[k][j] : at;
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) {
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                at += __shfl_xor_sync(0xffffffffu, at, o);
            }
            const float from = top == least ? 0.f : top;
#pragma unroll
            for (int j = 0; j < VJ; ++j) sum += ex2((l[k][j] - from) * kLog2e);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (tx == 0 && n < rows) {
                const float lse = t < 0 ? 0.f : top + logf(sum);
                if (a.lse_out) a.lse_out[n] = lse;
                if (a.loss) a.loss[n] = t < 0 ? 0.f : lse - at;
            }
        }
        __syncthreads();
    }
}

template <typename T, int VJ, int CJ>
__global__ void __launch_bounds__(kThreads, kBackward<VJ, CJ>) xent_small_bwd_kernel(const SmallArgs a) {
    using H = Head<T, VJ, CJ>;
    extern __shared__ __align__(16) float smem[];
    float *const w = smem, *const x = w + 16 * VJ * H::kRow, *const g = x + kTokens * H::kRow;
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(a.count, a.capacity, a.status);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    if (blockIdx.x * (long long)kTokens >= rows) return;
    H::load_weight(a, w);
    float dw[VJ][CJ][4] = {}, db[VJ] = {};
    for (long long n0 = blockIdx.x * (long long)kTokens; n0 < rows; n0 += gridDim.x * (long long)kTokens) {
        H::load_rows(a, n0, rows, x);
        __syncthreads();
        float l[2][VJ];
        bool used[2];
        H::logits(a, x, w, l);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const long long n = n0 + 2 * ty + k;
            const int t = H::target(a, n, rows);
            used[k] = t >= 0;
            const float lse = t < 0 ? 0.f : a.lse[n], dloss = t < 0 ? 0.f : a.dloss[n];
#pragma unroll
            for (int j = 0; j < VJ; ++j) {
                const int v = tx + 16 * j;
                float p = ex2((l[k][j] - lse) * kLog2e);
                p -= v == t ? 1.f : 0.f;
                p = t >= 0 && v < a.V ? p * dloss : 0.f;
                g[(2 * ty + k) * H::kGRow + v] = p;
                db[j] += p;
            }
        }
        __syncthreads();
        if (a.dx) {
            float d[2][CJ][4] = {};
#pragma unroll 2
            for (int v = 0; v < a.V; v += 4) {
                float q[2][4];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float4 f = *reinterpret_cast<const float4*>(g + (2 * ty + k) * H::kGRow + v);
                    q[k][0] = f.x, q[k][1] = f.y, q[k][2] = f.z, q[k][3] = f.w;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < CJ; ++c) {
                        const float4 f = *reinterpret_cast<const float4*>(
                            w + (v + e) * H::kRow + 4 * (tx + 16 * c));
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            d[k][c][0] = fmaf(q[k][e], f.x, d[k][c][0]);
                            d[k][c][1] = fmaf(q[k][e], f.y, d[k][c][1]);
                            d[k][c][2] = fmaf(q[k][e], f.z, d[k][c][2]);
                            d[k][c][3] = fmaf(q[k][e], f.w, d[k][c][3]);
                        }
                    }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const long long n = n0 + 2 * ty + k;
                if (n >= rows) continue;
#pragma unroll
                for (int c = 0; c < CJ; ++c) {
                    if (!used[k])  // whatever W holds
                        d[k][c][0] = d[k][c][1] = d[k][c][2] = d[k][c][3] = 0.f;
                    const int at = 4 * (tx + 16 * c);
                    T* const to = static_cast<T*>(a.dx) + n * a.C + at;
                    if (at >= a.C) continue;
                    if (a.wide_dx) {
                        if constexpr (sizeof(T) == 4)
                            *reinterpret_cast<float4*>(to) =
                                make_float4(d[k][c][0], d[k][c][1], d[k][c][2], d[k][c][3]);
                        else
                            *reinterpret_cast<uint2*>(to) =
                                make_uint2(Piece<__nv_bfloat16, 8>::pair(d[k][c][0], d[k][c][1]),
                                           Piece<__nv_bfloat16, 8>::pair(d[k][c][2], d[k][c][3]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (at + e < a.C) to[e] = from_f32<T>(d[k][c][e]);
                    }
                }
            }
        }
        if (a.part) {
#pragma unroll 4
            for (int t = 0; t < kTokens; ++t) {
                float q[VJ];
#pragma unroll
                for (int j = 0; j < VJ; ++j) q[j] = g[t * H::kGRow + ty + 16 * j];
#pragma unroll
                for (int c = 0; c < CJ; ++c) {
                    const float4 f = *reinterpret_cast<const float4*>(x + t * H::kRow + 4 * (tx + 16 * c));
#pragma unroll
                    for (int j = 0; j < VJ; ++j) {
                        dw[j][c][0] = fmaf(q[j], f.x, dw[j][c][0]);
                        dw[j][c][1] = fmaf(q[j], f.y, dw[j][c][1]);
                        dw[j][c][2] = fmaf(q[j], f.z, dw[j][c][2]);
                        dw[j][c][3] = fmaf(q[j], f.w, dw[j][c][3]);
                    }
                }
            }
        }
        __syncthreads();
    }
    if (!a.part) return;
    float* const part = a.part + (long long)blockIdx.x * a.V * (a.C + 1);
#pragma unroll
    for (int j = 0; j < VJ; ++j) {
        const int v = ty + 16 * j;
#pragma unroll
        for (int c = 0; c < CJ; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = 4 * (tx + 16 * c) + e;
                if (v < a.V && at < a.C) part[v * a.C + at] = dw[j][c][e];
            }
        g[ty * H::kGRow + tx + 16 * j] = db[j];
    }
    __syncthreads();
    for (int v = threadIdx.x; v < a.V; v += kThreads) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) s += g[k * H::kGRow + v];
        part[a.V * a.C + v] = s;
    }
}

// dW and dbias from the blocks' parts (those of blocks that had tokens), 32
// values a block: every 32nd part a warp, then the warps in order.
template <typename T>
__global__ void __launch_bounds__(1024)
    xent_small_join_kernel(const float* __restrict__ part, int blocks, const int32_t* count,
                           long long capacity, int weights, int V, T* dW, float* dbias,
                           unsigned* status) {
    __shared__ float sh[32][33];
    pdl_wait();
    pdl_trigger();
    const long long tiles = (token_rows(count, capacity, status) + kTokens - 1) / kTokens;
    const int parts = tiles < blocks ? (int)tiles : blocks;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int i = blockIdx.x * 32 + lane, all = weights + V;
    float v = 0.f;
    if (i < all) {
#pragma unroll 8
        for (int p = warp; p < parts; p += 32) v += part[(long long)p * all + i];
    }
    sh[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && i < all) {
        v = 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) v += sh[k][lane];
        if (i < weights) {
            if (dW) dW[i] = from_f32<T>(v);
        } else if (dbias) {
            dbias[i - weights] = v;
        }
    }
}

SmallArgs args_of(const DeviceCtx* ctx, const LinearXentArgs& a, size_t size) {
    auto aligned = [&](const void* p) { return a.C % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & (4 * size - 1)) == 0; };
    SmallArgs s{};
    s.x = a.x;
    s.W = a.W;
    s.bias = a.bias;
    s.targets = a.targets;
    s.count = a.count;
    s.capacity = a.capacity;
    s.C = a.C;
    s.V = a.V;
    s.loss = a.loss_out;
    s.lse_out = a.lse_out;
    s.lse = a.lse;
    s.dloss = a.dloss;
    s.dx = a.dx;
    s.wide_x = aligned(a.x);
    s.wide_dx = aligned(a.dx);
    s.status = ctx->status;
    return s;
}

template <typename T, int VJ, int CJ>
hc_status run(const DeviceCtx* ctx, const LinearXentArgs& a, bool back, cudaStream_t s) {
    using H = Head<T, VJ, CJ>;
    static_assert(VJ * CJ <= kMaxPerThread, "sums of dW a thread");
    SmallArgs k = args_of(ctx, a, sizeof(T));
    const long long tiles = ((long long)a.capacity + kTokens - 1) / kTokens;
    const long long cap = (long long)(back ? kBackward<VJ, CJ> : kForward<VJ, CJ>)*ctx->num_sms;
    const unsigned grid = (unsigned)(tiles < 1 ? 1 : tiles < cap ? tiles : cap);
    auto kern = back ? xent_small_bwd_kernel<T, VJ, CJ> : xent_small_fwd_kernel<T, VJ, CJ>;
    static bool done[2][64];
    if (H::kSmem > 48 * 1024 && !done[back][ctx->device]) {
        const hc_status st = check_cuda(
            cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)H::kSmem),
            "xent_small_kernel");
        if (st != HC_OK) return st;
        done[back][ctx->device] = true;
    }
    const int weights = a.V * a.C;
    if (back && (a.dW || a.dbias)) {
        k.part = (float*)stream_workspace(s, (size_t)grid * (weights + a.V) * 4);
        if (!k.part) return HC_ERR_CUDA;
    }
    const hc_status st =
        launch_pdl(kern, dim3(grid), dim3(kThreads), H::kSmem, s, "xent_small_kernel", k);
    if (st != HC_OK || !k.part) return st;
    return launch_pdl(xent_small_join_kernel<T>, dim3((unsigned)((weights + a.V + 31) / 32)), dim3(1024), 0,
                      s, "xent_small_join_kernel", (const float*)k.part, (int)grid, a.count,
                      (long long)a.capacity, weights, a.V, (T*)a.dW, a.dbias, ctx->status);
}

template <typename T, int VJ>
hc_status by_channels(const DeviceCtx* ctx, const LinearXentArgs& a, bool back, cudaStream_t s) {
    if (a.C <= 64) return run<T, VJ, 1>(ctx, a, back, s);
    if constexpr (VJ <= 4) {
        if (a.C <= 128) return run<T, VJ, 2>(ctx, a, back, s);
    }
    if constexpr (VJ <= 2) return run<T, VJ, 4>(ctx, a, back, s);
    set_error("cross entropy: V=%d C=%d is no small head", a.V, a.C);
    return HC_ERR_UNSUPPORTED;
}

template <typename T>
hc_status by_classes(const DeviceCtx* ctx, const LinearXentArgs& a, bool back, cudaStream_t s) {
    if (a.V <= 16) return by_channels<T, 1>(ctx, a, back, s);
    if (a.V <= 32) return by_channels<T, 2>(ctx, a, back, s);
    if (a.V <= 48) return by_channels<T, 3>(ctx, a, back, s);
    if (a.V <= 64) return by_channels<T, 4>(ctx, a, back, s);
    if (a.V <= 96) return by_channels<T, 6>(ctx, a, back, s);
    return by_channels<T, 8>(ctx, a, back, s);
}

}  // namespace

// Forward and gradients against the tensor-core path: 42 x 64 bf16, 2048 tokens 34 and 52
// us (the host's time), 65536 78 and 187 (fp32 241), a million 1.06 and 2.79 ms; the
// largest heads, 128 x 64 bf16, 16384 tokens 55 and 84 us, a million 2.26 and 2.86 ms, and
// 32 x 256, 66 and 99 us, 3.12 and 3.52 ms.
bool xent_small_supported(const LinearXentArgs& a) {
    if (a.V <= 32) return a.C <= 256;
    if (a.V <= 64) return a.C <= 128;
    return a.V <= 128 && a.C <= 64;
}

hc_status launch_xent_small_fwd(const DeviceCtx* ctx, const LinearXentArgs& a, cudaStream_t s) {
    return a.dt == HC_BF16 ? by_classes<__nv_bfloat16>(ctx, a, false, s)
                           : by_classes<float>(ctx, a, false, s);
}

hc_status launch_xent_small_bwd(const DeviceCtx* ctx, const LinearXentArgs& a, cudaStream_t s) {
    return a.dt == HC_BF16 ? by_classes<__nv_bfloat16>(ctx, a, true, s)
                           : by_classes<float>(ctx, a, true, s);
}

}  // namespace hc
