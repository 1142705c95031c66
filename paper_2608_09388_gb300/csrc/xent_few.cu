// The cross entropy behind a linear layer for up to eight tokens (a scoring or
// decoding step, and the gradients of one). The formulas are those of
// linear_xent.cu. Bound by the one read of W, and backward the write of dW, so the sums
// are taken on the CUDA cores, in fp32 throughout, straight from the rows as
// they are.
//
// A warp takes kRows classes at a time, 16 bytes of each a lane, against the
// tokens' rows in shared memory (fp32; the 16-byte pieces of a lane's channels lie
// 512 bytes apart, so that neither side has bank conflicts). Backward, a block
// forms G of its warps' classes in the same order of additions, so that the G of a
// sure token's target, p - 1, has no rounding of a logit in it, then goes over the classes' rows again (from
// L2), a thread for the same channels of all of them: dW is written, dx added up in
// shared memory and, over the blocks, by a last kernel.
//
// One of 32000 x 4096 bf16: 49 us, 39 at the copy rate; its gradients 150 us, 77 at
// the copy rate (286 on the tensor cores, which take 256 tokens at a time). There a
// block's two phases alternate behind barriers, and half of W's second read comes
// from memory (405 MB are read for 262). Four of 32000 x 1024 fp32: 94 us (303).
#include "xent.cuh"

namespace hc {
namespace {

constexpr int kFew = 8;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kRows = 4;

template <int VEC>
__device__ __forceinline__ int place(int c) {
    if (VEC < 8) return c;
    return (c & ~255) + (c & 4) * 32 + ((c & 255) >> 3) * 4 + (c & 3);
}
__host__ __device__ __forceinline__ int pitch_of(int C) {
    return (C + 255) & ~255;
}
// N floats of a row in shared memory from channel c on.
template <int VEC, int N>
__device__ __forceinline__ void get(const float* row, int c, float (&f)[N]) {
    if constexpr (VEC == 1) {
        f[0] = row[c];
    } else {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const float4 q = *reinterpret_cast<const float4*>(row + place<VEC>(c + e));
            f[e] = q.x, f[e + 1] = q.y, f[e + 2] = q.z, f[e + 3] = q.w;
        }
    }
}
template <int VEC, int N>
__device__ __forceinline__ void set(float* row, int c, const float (&f)[N]) {
    if constexpr (VEC == 1) {
        row[c] = f[0];
    } else {
#pragma unroll
        for (int e = 0; e < N; e += 4)
            *reinterpret_cast<float4*>(row + place<VEC>(c + e)) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
    }
}

// Of the kRows * kT sums of a round (class r, token t) a lane keeps one, the
// lane's upper bits being r and t.
template <int kTokens>
struct Lanes {
    static constexpr int kT = kTokens == 3 ? 4 : kTokens == 6 ? 8 : kTokens, kValues = kRows * kT;
    static constexpr int kSame = 32 / kValues;  // lanes with the same value
    int r, t;
    bool first;
    __device__ __forceinline__ Lanes() {
        const int lane = threadIdx.x & 31;
        r = lane / (32 / kRows);
        t = lane / kSame % kT;
        first = lane % kSame == 0 && t < kTokens;
    }
};

// This lane's sum over the channels, for the classes v0 .. v0 + take - 1.
template <typename T, int VEC, int kTokens>
__device__ __forceinline__ float sums(const float* rows, int pitch, const T* __restrict__ W,
                                      long long v0, int take, int C, int V) {
    using L = Lanes<kTokens>;
    const int lane = threadIdx.x & 31;
    float s[kRows][kTokens] = {};
#pragma unroll kTokens <= 4 ? 2 : 1
    for (int c = lane * VEC; c < C; c += 32 * VEC) {
        Piece<T, VEC> p[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (r < take && v0 + r < V) p[r].load(W + (v0 + r) * C + c);
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
            float f[VEC];
            get<VEC>(rows + t * pitch, c, f);
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int e = 0; e < VEC; ++e) s[r][t] = fmaf(p[r].get(e), f[e], s[r][t]);
        }
    }
    // over the lanes, half of the values left to each at every step
    float v[L::kValues];
#pragma unroll
    for (int k = 0; k < L::kValues; ++k) v[k] = k % L::kT < kTokens ? s[k / L::kT][k % L::kT] : 0.f;
    int o = 16;
#pragma unroll
    for (int half = L::kValues / 2; half > 0; half /= 2, o /= 2) {
        const bool up = lane & o;
#pragma unroll
        for (int k = 0; k < half; ++k) {
            const float send = up ? v[k] : v[k + half], keep = up ? v[k + half] : v[k];
            v[k] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
    }
#pragma unroll
    for (int q = L::kSame / 2; q > 0; q /= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], q);
    return v[0];
}

// Blocks of a multiprocessor forward: the sums of more tokens, or of eight channels for
// three, take more registers than four blocks have (two of 32000 x 4096 bf16 70 us, 74
// with three, of 121848 x 152 25 and 29, though of 131072 x 4096 201 and 192; four of
// 32000 x 1024 fp32 43, 47 with two, of 121848 x 151 bf16 33, 45 with two; four of
// 32000 x 2048 bf16 49 with two, 70 with four).
template <int VEC, int kTokens>
constexpr int kForwardBlocks = kTokens <= 2 || (kTokens <= 4 && VEC < 8) ? 4 : 2;

template <typename T, int VEC, int kTokens>
__global__ void __launch_bounds__(kThreads, kForwardBlocks<VEC, kTokens>)
    xent_few_kernel(const T* __restrict__ x, const T* __restrict__ W, const float* __restrict__ bias,
                    const int32_t* targets, int tokens, int C, int V, float2* __restrict__ pairs,
                    float* __restrict__ at_target) {
    extern __shared__ __align__(16) float rows[];  // [kTokens][pitch]
    __shared__ float2 sh[kWarps][kTokens];
    const int warp = threadIdx.x >> 5, pitch = pitch_of(C);
    const float least = -__int_as_float(0x7f800000);
    pdl_wait();
    pdl_trigger();
    const Lanes<kTokens> me;
    int my_target = -1;
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
        const int target = t < tokens ? targets[t] : -1;
        my_target = me.t == t ? target : my_target;
        for (int c = threadIdx.x; c < C; c += kThreads)
            rows[t * pitch + place<VEC>(c)] = t < tokens ? to_f32(x[(long long)t * C + c]) : 0.f;
    }
    __syncthreads();
    float2 mine = make_float2(least, 0.f);
    // whole rounds of kRows classes a warp, then what is left in one round of as
    // few as it takes: every warp ends at the same time
    const int warps = gridDim.x * kWarps, w = (int)blockIdx.x * kWarps + warp;
    const int whole = V / (warps * kRows), left = V - whole * warps * kRows;
    const int last = (left + warps - 1) / warps;
    for (int i = 0; i <= whole; ++i) {
        const int take = i < whole ? kRows : last;
        const long long v0 = (long long)i * warps * kRows + (long long)w * take;
        if (v0 >= V || take == 0) break;
        const float sum = sums<T, VEC, kTokens>(rows, pitch, W, v0, take, C, V);
        const long long cls = v0 + me.r;
        if (me.r < take && cls < V && me.t < kTokens) {
            const float l = sum + (bias ? __ldg(bias + cls) : 0.f);
            if (me.first && cls == my_target) at_target[me.t] = l;
            mine = join_pairs(mine, make_float2(l, 1.f));
        }
    }
#pragma unroll
    for (int o = 16; o >= 32 / kRows; o /= 2)  // the classes of a token
        mine = join_pairs(mine, make_float2(__shfl_xor_sync(0xffffffffu, mine.x, o),
                                            __shfl_xor_sync(0xffffffffu, mine.y, o)));
    if (me.r == 0 && me.first) sh[warp][me.t] = mine;
    __syncthreads();
    if (threadIdx.x < kTokens) {
        float2 p = sh[0][threadIdx.x];
        for (int k = 1; k < kWarps; ++k) p = join_pairs(p, sh[k][threadIdx.x]);
        pairs[(long long)blockIdx.x * kFew + threadIdx.x] = p;
    }
}

// The blocks' pairs of a token -> loss and lse, a warp per token.
__global__ void __launch_bounds__(kFew * 32)
    xent_few_join_kernel(const int32_t* count, long long capacity, const int32_t* targets, int V,
                         const float2* __restrict__ pairs, int blocks, const float* at_target, float* loss,
                         float* lse, unsigned* status) {
    pdl_wait();
    pdl_trigger();
    const float least = -__int_as_float(0x7f800000);
    const int n = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (n >= token_rows(count, capacity, status)) return;
    const int t = targets[n];
    const bool in = t >= 0 && t < V;
    if (!in && t != -1 && lane == 0) report(status, kErrIndex);
    float2 p = make_float2(least, 0.f);
#pragma unroll 8
    for (int b = lane; b < blocks; b += 32) p = join_pairs(p, pairs[(long long)b * kFew + n]);
    p = join_lanes<32>(p);
    if (lane != 0) return;
    const float all = p.x + logf(p.y);
    if (lse) lse[n] = in ? all : 0.f;
    if (loss) loss[n] = in ? all - at_target[n] : 0.f;
}

struct GradArgs {
    const void* x;
    const void* W;
    const float* bias;
    const int32_t* targets;
    const int32_t* count;
    const float* lse;
    const float* dloss;
    int capacity, C, V;
    void* dW;      // or NULL
    float* dbias;  // or NULL
    float* part;   // [blocks][kTokens][C]: the blocks' sums of dx, or NULL
    unsigned* status;
};

constexpr int kBatch = kWarps * kRows;  // classes of a block at a time

// Blocks of a multiprocessor backward. Three have 80 registers a thread: one of
// 32000 x 4096 bf16 156 us against 150, two of 131072 x 4096 633 against 543.
constexpr int kBackBlocks = 2;

// Groups of threads, each of which holds all channels and takes its share of a
// batch's classes (three of 121848 x 152 bf16: 49 us, 74 with one group).
__host__ __device__ __forceinline__ int groups_of(int C, int vec) {
    const int units = (C + vec - 1) / vec, n = kThreads / units;
    return n < 1 ? 1 : n < 8 ? n : 8;
}

// Channels a thread takes at a time there: those of all tokens, and of dx, are in registers.
template <int VEC, int kTokens>
constexpr int kChannels = kTokens > 4 && VEC > 4 ? 4 : VEC;

template <typename T, int VEC, int kTokens>
__global__ void __launch_bounds__(kThreads, kBackBlocks)
    xent_few_bwd_kernel(const GradArgs a) {
    extern __shared__ __align__(16) float smem[];  // the rows of x, then each group's of dx
    __shared__ float g[kBatch][kTokens];
    const int warp = threadIdx.x >> 5, C = a.C, V = a.V, pitch = pitch_of(C);
    constexpr int kC = kChannels<VEC, kTokens>;
    const int groups = groups_of(C, kC), span = groups > 1 ? (C + kC - 1) / kC : kThreads;
    const int group = (int)threadIdx.x / span;
    float *const rows = smem, *const sum_dx = smem + kTokens * pitch;
    float* const dx = sum_dx + group * kTokens * pitch;  // of the threads with group < groups
    pdl_wait();
    pdl_trigger();
    const long long used = token_rows(a.count, a.capacity, a.status);
    const T *const x = static_cast<const T*>(a.x), *const W = static_cast<const T*>(a.W);
    const Lanes<kTokens> me;
    int my_target = -1;
    float my_lse = 0.f, my_dloss = 0.f;
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
        int target = t < used ? a.targets[t] : -1;
        if (target < -1 || target >= V) {
            if (blockIdx.x == 0 && threadIdx.x == 0) report(a.status, kErrIndex);
            target = -1;
        }
        if (me.t == t) {
            my_target = target;
            my_lse = target < 0 ? 0.f : a.lse[t];
            my_dloss = target < 0 ? 0.f : a.dloss[t];
        }
        // zero for a token that takes no part, whatever it holds
        for (int c = threadIdx.x; c < pitch; c += kThreads) {
            rows[t * pitch + place<VEC>(c)] = target >= 0 && c < C ? to_f32(x[(long long)t * C + c]) : 0.f;
        }
    }
    for (int i = threadIdx.x; i < groups * kTokens * pitch; i += kThreads) sum_dx[i] = 0.f;
    for (long long b0 = (long long)blockIdx.x * kBatch; b0 < V; b0 += (long long)gridDim.x * kBatch) {
        __syncthreads();  // the rows are there, or the last batch's G has been used
        {
            const long long v0 = b0 + warp * kRows, cls = v0 + me.r;
            const float sum = v0 < V ? sums<T, VEC, kTokens>(rows, pitch, W, v0, kRows, C, V) : 0.f;
            if (me.first) {
                float v = 0.f;
                if (my_target >= 0 && cls < V) {
                    v = ex2((sum + (a.bias ? __ldg(a.bias + cls) : 0.f) - my_lse) * kLog2e);
                    v = (v - (cls == my_target ? 1.f : 0.f)) * my_dloss;
                }
                g[warp * kRows + me.r][me.t] = v;
            }
        }
        __syncthreads();
        const int classes = V - b0 < kBatch ? (int)(V - b0) : kBatch;
        if (a.dbias && (int)threadIdx.x < classes) {
            float s = 0.f;
#pragma unroll
            for (int t = 0; t < kTokens; ++t) s += g[threadIdx.x][t];
            a.dbias[b0 + threadIdx.x] = s;
        }
        for (int c = (threadIdx.x - group * span) * kC; c < C && group < groups; c += span * kC) {
            float f[kTokens][kC], d[kTokens][kC];
#pragma unroll
            for (int t = 0; t < kTokens; ++t) {
                get<VEC>(rows + t * pitch, c, f[t]);
                get<VEC>(dx + t * pitch, c, d[t]);
            }
#pragma unroll 4
            for (int k = group; k < classes; k += groups) {
                const long long at = (b0 + k) * C + c;
                float gk[kTokens];
#pragma unroll
                for (int t = 0; t < kTokens; ++t) gk[t] = g[k][t];
                if (a.part) {
                    Piece<T, kC> p;
                    p.load(W + at);
#pragma unroll
                    for (int t = 0; t < kTokens; ++t)
#pragma unroll
                        for (int e = 0; e < kC; ++e) d[t][e] = fmaf(gk[t], p.get(e), d[t][e]);
                }
                if (a.dW) {
                    float o[kC];
#pragma unroll
                    for (int e = 0; e < kC; ++e) {
                        o[e] = gk[0] * f[0][e];
#pragma unroll
                        for (int t = 1; t < kTokens; ++t) o[e] = fmaf(gk[t], f[t][e], o[e]);
                    }
                    Piece<T, kC> p;
                    p.set_all(o);
                    p.store(static_cast<T*>(a.dW) + at);
                }
            }
#pragma unroll
            for (int t = 0; t < kTokens; ++t) set<VEC>(dx + t * pitch, c, d[t]);
        }
    }
    if (!a.part) return;
    __syncthreads();
    for (int t = 0; t < kTokens; ++t)
        for (int c = threadIdx.x; c < C; c += kThreads) {
            float v = 0.f;
            for (int k = 0; k < groups; ++k) v += sum_dx[(k * kTokens + t) * pitch + place<VEC>(c)];
            a.part[((long long)blockIdx.x * kTokens + t) * C + c] = v;
        }
}

// dx from the blocks' sums, 32 channels of a token a block: every 32nd part a
// warp, then the warps in order; zero for a token that takes no part.
template <typename T>
__global__ void __launch_bounds__(1024)
    xent_few_input_kernel(const float* __restrict__ part, int blocks, int slots, const int32_t* count, int capacity,
                          const int32_t* targets, int C, int V, T* dx, unsigned* status) {
    __shared__ float sh[32][33];
    pdl_wait();
    pdl_trigger();
    const int n = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = blockIdx.x * 32 + lane;
    if (n >= token_rows(count, capacity, status)) return;
    const int t = targets[n];
    const bool in = t >= 0 && t < V;
    float v = 0.f;
    if (in && c < C) {
#pragma unroll 8
        for (int p = warp; p < blocks; p += 32) v += part[((long long)p * slots + n) * C + c];
    }
    sh[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && c < C) {
        v = 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) v += sh[k][lane];
        dx[(long long)n * C + c] = from_f32<T>(v);
    }
}

// ---------------------------------------------------------------- host side
template <typename T, int VEC, int kTokens>
hc_status forward(const DeviceCtx* ctx, const LinearXentArgs& a, cudaStream_t s) {
    // as many blocks as run at a time, a class a warp at least
    const long long need = ((long long)a.V + kWarps - 1) / kWarps;
    const long long cap = (long long)kForwardBlocks<VEC, kTokens> * ctx->num_sms;
    const int blocks = (int)(need < cap ? need : cap);
    float2* const pairs = (float2*)stream_workspace(s, ((size_t)blocks * kFew + kFew) * sizeof(float2));
    if (!pairs) return HC_ERR_CUDA;
    float* const at_target = reinterpret_cast<float*>(pairs + (size_t)blocks * kFew);
    const hc_status st =
        launch_pdl(xent_few_kernel<T, VEC, kTokens>, dim3((unsigned)blocks), dim3(kThreads),
                   (size_t)kTokens * pitch_of(a.C) * 4, s, "xent_few_kernel", (const T*)a.x,
                   (const T*)a.W, a.bias, a.targets, a.capacity, a.C, a.V, pairs, at_target);
    if (st != HC_OK) return st;
    return launch_pdl(xent_few_join_kernel, dim3(1), dim3(kFew * 32), 0, s, "xent_few_join_kernel",
                      a.count, (long long)a.capacity, a.targets, a.V, (const float2*)pairs, blocks,
                      (const float*)at_target, a.loss_out, a.lse_out, ctx->status);
}

template <typename T, int VEC, int kTokens>
hc_status backward(const DeviceCtx* ctx, const LinearXentArgs& a, cudaStream_t s) {
    const long long need = ((long long)a.V + kBatch - 1) / kBatch;
    const long long cap = (long long)kBackBlocks * ctx->num_sms;
    const int blocks = (int)(need < cap ? need : cap);
    GradArgs g{a.x, a.W, a.bias, a.targets, a.count, a.lse, a.dloss, a.capacity, a.C, a.V, a.dW, a.dbias, nullptr,
               ctx->status};
    if (a.dx) {
        g.part = (float*)stream_workspace(s, (size_t)blocks * kTokens * a.C * 4);
        if (!g.part) return HC_ERR_CUDA;
    }
    // At most 92 KiB: with one group twice what xent_few_supported allows, with more, which
    // have C <= 1024 (512 with five tokens or more), 72 KiB
    const size_t smem = (1 + groups_of(a.C, kChannels<VEC, kTokens>)) * (size_t)kTokens * pitch_of(a.C) * 4;
    auto kern = xent_few_bwd_kernel<T, VEC, kTokens>;
    static bool done[64];
    if (smem > 47 * 1024 && !done[ctx->device]) {
        const hc_status st = check_cuda(
            cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 94 * 1024),
            "xent_few_bwd_kernel");
        if (st != HC_OK) return st;
        done[ctx->device] = true;
    }
    const hc_status st = launch_pdl(kern, dim3((unsigned)blocks), dim3(kThreads), smem, s,
                                    "xent_few_bwd_kernel", g);
    if (st != HC_OK || !a.dx) return st;
    return launch_pdl(xent_few_input_kernel<T>, dim3((unsigned)((a.C + 31) / 32), (unsigned)a.capacity),
                      dim3(1024), 0, s, "xent_few_input_kernel", (const float*)g.part, blocks, kTokens, a.count,
                      a.capacity, a.targets, a.C, a.V, (T*)a.dx, ctx->status);
}

template <typename T, int VEC>
hc_status by_tokens(const DeviceCtx* ctx, const LinearXentArgs& a, bool back, cudaStream_t s) {
    switch (a.capacity) {
        case 1: return back ? backward<T, VEC, 1>(ctx, a, s) : forward<T, VEC, 1>(ctx, a, s);
        case 2: return back ? backward<T, VEC, 2>(ctx, a, s) : forward<T, VEC, 2>(ctx, a, s);
        case 3: return back ? backward<T, VEC, 3>(ctx, a, s) : forward<T, VEC, 3>(ctx, a, s);
        case 4: return back ? backward<T, VEC, 4>(ctx, a, s) : forward<T, VEC, 4>(ctx, a, s);
        case 5:
        case 6: return back ? backward<T, VEC, 6>(ctx, a, s) : forward<T, VEC, 6>(ctx, a, s);
        default: return back ? backward<T, VEC, 8>(ctx, a, s) : forward<T, VEC, 8>(ctx, a, s);
    }
}

template <typename T>
hc_status run(const DeviceCtx* ctx, const LinearXentArgs& a, bool back, cudaStream_t s) {
    constexpr int kVec = 16 / (int)sizeof(T);
    auto aligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    if (a.C % kVec == 0 && aligned(a.W) && aligned(a.dW)) return by_tokens<T, kVec>(ctx, a, back, s);
    return by_tokens<T, 1>(ctx, a, back, s);
}

}  // namespace

// Their rows in fp32 have to fit the 48 KiB of shared memory that every launch may have.
// Forward and gradients against the tensor cores: eight of 33776 x 1168 fp32 226 and 544
// us, of 32000 x 1024 bf16 125 and 135, six 110 and 137. More than four of a bf16 W that is
// larger than the L2 lose, the products being cheap there and W read twice: six of
// 131072 x 1280 465 and 432, eight 524 and 434.
bool xent_few_supported(const LinearXentArgs& a) {
    if (a.capacity < 1 || a.capacity > kFew) return false;
    if (a.dt == HC_BF16 && a.capacity > 4 && (long long)a.V * a.C > 1ll << 26) return false;
    const long long slots = a.capacity <= 4 ? a.capacity : (a.capacity + 1) / 2 * 2;
    return slots * ((a.C + 255ll) / 256 * 256) * 4 <= 46 * 1024;
}

hc_status launch_xent_few_fwd(const DeviceCtx* ctx, const LinearXentArgs& a, cudaStream_t s) {
    return a.dt == HC_BF16 ? run<__nv_bfloat16>(ctx, a, false, s) : run<float>(ctx, a, false, s);
}

hc_status launch_xent_few_bwd(const DeviceCtx* ctx, const LinearXentArgs& a, cudaStream_t s) {
    return a.dt == HC_BF16 ? run<__nv_bfloat16>(ctx, a, true, s) : run<float>(ctx, a, true, s);
}

}  // namespace hc
