// Root-mean-square norm of compact rows behind the residual's addition, its
// 8-bit output, and its gradient. For every row n < N', over its C channels:
//   h = x + res, rounded to the rows' type (h = x without a residual)
//   rstd = 1 / sqrt(sum h^2 / C + eps)
//   v = h * rstd * gamma;  y = v rounded, or q, scales = the 8-bit form of v
// and backwards, with hh = h * rstd and g = dy * gamma:
//   dx     = dres + rstd * (g - hh * sum (g * hh) / C)
//   dgamma = sum over rows of dy * hh
// All sums in fp32. The statistics are those of the row as stored, and v is
// taken to 8 bits from fp32, so that the 8-bit form has one rounding only.
// dgamma is summed per thread over its rows, per block, then joined in a
// fixed order: every result is the same from run to run.
//
// Bound by memory: forward reads two rows and writes two (8 bits: one and a
// half), the gradient reads three and writes one. Rows of up to 8192 channels
// stay in registers between the sum of squares and the output, and the next
// rows are on their way before this one is reduced. At 65536 x 2048 bf16 (GB300)
// forward and gradient take 327 us (317 at the copy rate), 16384 x 8192 bf16 to 8
// bits 156 (139), 1 x 4096 to 8 bits 2.5.
#include "fp8.cuh"

namespace hc {
namespace {

constexpr int kThreads = 512;

// ms = sum h^2 / C + eps outside of what fp32 squares hold (or NaN): the row
// is summed again as h * f, and rstd = f / sqrt(sum (h f)^2 / C + eps f^2).
// Squares that overflow: the root mean square is above 2^47 (2^31 channels),
// so that 2^-100 takes the largest value to 2^28 and loses nothing that
// matters; small ones: below 2^-34, 2^84 takes them to 2^50.
constexpr float kSmallest = 0x1p-100f, kLessen = 0x1p-100f, kEnlarge = 0x1p84f;
__device__ __forceinline__ bool outside(float ms) {
    return !(ms >= kSmallest && ms < __int_as_float(0x7f800000));
}
__device__ __forceinline__ float factor(float ms) {
    return ms < kSmallest ? kEnlarge : kLessen;
}
__device__ __forceinline__ float rstd_scaled(float sum2, float inv, float eps, float f) {
    return rsqrtf(fmaf(sum2, inv, eps * f * f)) * f;
}

// Largest magnitude as bits: compares as an unsigned number, a NaN above all.
__device__ __forceinline__ uint32_t mag(float v) {
    return __float_as_uint(fabsf(v));
}

// Four channels of v to 8 bits with the scale of their block's largest
// magnitude `top`; the first `left` of them are channels of the row.
__device__ __forceinline__ uint32_t quantise4(const float (&v)[4], float scale, int left) {
    uint32_t w[1];
    to_e4m3<4>(v, scale, 1.f / scale, w);
    return w[0] & first_bytes(left);
}

// ---------------------------------------------------------------- rows in registers
// As in the layer norm: a group of TPR threads holds a row, NV pieces of VEC
// elements each, piece i of thread t at channel (i * TPR + t) * VEC. A block of
// 128 channels of the 8-bit form then lies in 128 / VEC neighbouring threads.
constexpr int kGroupThreads = 512;

// Rows in flight: 16 registers' worth of x and as much of res, four rows at most
// (65536 x 2048 bf16 forward and gradient 326 us; with 32 registers' worth 337).
template <int VEC, int NV>
constexpr int kRowRegs = NV * (VEC <= 2 ? 1 : 4);
template <int VEC, int NV>
constexpr int kFwdAhead = kRowRegs<VEC, NV> >= 16 ? 1 : kRowRegs<VEC, NV> >= 8 ? 2 : 4;

struct RmsArgs8 {
    uint8_t* q;
    float* scales;
    int pitch;
};

// Threads of a group meet: its named barrier, or its warp.
template <int TPR>
__device__ __forceinline__ void group_sync() {
    if constexpr (TPR > 32)
        asm volatile("bar.sync %0, %1;\n" ::"r"(threadIdx.x / TPR + 1), "r"(TPR) : "memory");
    else
        __syncwarp();
}

template <typename T, int VEC, int TPR, int NV, bool kQ>
__global__ void __launch_bounds__(kGroupThreads)
    rms_fwd_rows_kernel(const T* x, const T* res, const int32_t* count, long long capacity, int C,
                        float eps, const float* __restrict__ gamma, T* h, T* y, float* rstd_out,
                        RmsArgs8 o8, unsigned* status) {
    __shared__ __align__(16) float sh[2 * kGroupThreads / 32];
    extern __shared__ __align__(16) float vrow[];  // VEC <= 2 and kQ: a row of v a group
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    constexpr int kGroups = kGroupThreads / TPR;
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31;
    const long long step = (long long)gridDim.x * kGroups;
    // every thread of a warp takes part in the shuffles: groups of a warp run
    // the same number of rounds
    const long long n0 = (long long)blockIdx.x * kGroups + threadIdx.x / TPR;
    const long long w0 = TPR < 32 ? n0 - lane / TPR : n0;
    using Unit = UnitOf<VEC>;
    using U = typename Unit::type;
    constexpr int kU = Unit::count;
    const float inv = 1.f / (float)C;
    constexpr int kAhead = kFwdAhead<VEC, NV>;
    Piece<T, VEC> ring[kAhead][NV], ringr[kAhead][NV];
    U ga[NV][kU];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * VEC;
        if (c < C) load_units<VEC>(gamma, c, 1.f, ga[i]);
    }
    auto load = [&](long long n, Piece<T, VEC>(&p)[NV], Piece<T, VEC>(&r)[NV]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VEC;
            if (n < rows && c < C) {
                p[i].load(x + n * C + c);
                if (res) r[i].load(res + n * C + c);
            }
        }
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(n0 + u * step, ring[u], ringr[u]);
    int turn = 0;
    for (long long w = w0, n = n0; w < rows;) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u, w += step, n += step) {
            if (w >= rows) break;
            U s = Unit::splat(0.f), d[NV][kU];
            const bool in = n < rows;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * TPR + t) * VEC;
                if (res) ring[u][i] = sum_of(ring[u][i], ringr[u][i]);
#pragma unroll
                for (int e = 0; e < kU; ++e) d[i][e] = ring[u][i].unit(e);
                if (c < C) {
                    if (h && in) ring[u][i].store(h + n * C + c);
#pragma unroll
                    for (int e = 0; e < kU; ++e) s = fma(d[i][e], d[i][e], s);
                }
            }
            load(n + kAhead * step, ring[u], ringr[u]);
            const float ms = fmaf(group_sum<TPR>(total(s), sh, turn), inv, eps);
            turn ^= 1;
            float rstd = rsqrtf(ms);
            const bool out = in && outside(ms);
            if (TPR < 32 ? __any_sync(0xffffffffu, out) : out) {
                const float f = factor(ms);
                const U by = Unit::splat(f);
                s = Unit::splat(0.f);
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if ((i * TPR + t) * VEC < C)
#pragma unroll
                        for (int e = 0; e < kU; ++e) {
                            const U v = mul(d[i][e], by);
                            s = fma(v, v, s);
                        }
                const float again = rstd_scaled(group_sum<TPR>(total(s), sh, turn), inv, eps, f);
                turn ^= 1;
                if (out) rstd = again;
            }
            const U times = Unit::splat(rstd);
            if (rstd_out && in && t == 0) rstd_out[n] = rstd;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < kU; ++e) d[i][e] = mul(mul(d[i][e], times), ga[i][e]);
            if (!kQ || y) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = (i * TPR + t) * VEC;
                    if (c < C && in) {
                        Piece<T, VEC> p;
                        p.set_units(d[i]);
                        p.store(y + n * C + c);
                    }
                }
            }
            if constexpr (kQ && VEC > 2) {
                constexpr int kBlockLanes = 128 / VEC < TPR ? 128 / VEC : TPR;
                float v[NV][VEC];
                uint32_t top[NV];
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const bool there = (i * TPR + t) * VEC < C;
#pragma unroll
                    for (int e = 0; e < kU; ++e) {
                        const float2 f = split(d[i][e]);
                        v[i][2 * e] = there ? f.x : 0.f;
                        v[i][2 * e + 1] = there ? f.y : 0.f;
                    }
                    float most = 0.f;
#pragma unroll
                    for (int e = 0; e < VEC; e += 2) most = max_mag(most, v[i][e], v[i][e + 1]);
                    top[i] = __float_as_uint(most);
                }
                // the maxima of a lane's NV blocks: each exchange leaves it with
                // half of them, after which lane l goes on with block l % NV
                const int own = lane % NV;
                uint32_t m = top[0];
                if constexpr (NV == 2) {
                    m = max(own ? top[1] : top[0],
                            __shfl_xor_sync(0xffffffffu, own ? top[0] : top[1], 1));
                } else if constexpr (NV == 4) {
                    const bool b0 = lane & 1, b1 = lane & 2;
                    const uint32_t m01 = max(b0 ? top[1] : top[0],
                                             __shfl_xor_sync(0xffffffffu, b0 ? top[0] : top[1], 1));
                    const uint32_t m23 = max(b0 ? top[3] : top[2],
                                             __shfl_xor_sync(0xffffffffu, b0 ? top[2] : top[3], 1));
                    m = max(b1 ? m23 : m01, __shfl_xor_sync(0xffffffffu, b1 ? m01 : m23, 2));
                }
                static_assert(NV == 1 || NV == 2 || NV == 4, "blocks of a lane");
#pragma unroll
                for (int o = NV; o < kBlockLanes; o <<= 1)
                    m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                const float my_scale = scale_of(__uint_as_float(m)), my_inv = 1.f / my_scale;
                {
                    const int c = (own * TPR + t) * VEC;
                    if (in && lane % kBlockLanes < NV && (c & ~127) < C)
                        o8.scales[(long long)(c / 128) * capacity + n] = my_scale;
                }
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = (i * TPR + t) * VEC;
                    const int from = (lane & ~(kBlockLanes - 1)) + i;
                    const float scale = NV == 1 ? my_scale : __shfl_sync(0xffffffffu, my_scale, from);
                    const float inv = NV == 1 ? my_inv : __shfl_sync(0xffffffffu, my_inv, from);
                    uint32_t word[VEC / 4];
                    to_e4m3<VEC>(v[i], scale, inv, word);
                    if (c >= C) {
#pragma unroll
                        for (int k = 0; k < VEC / 4; ++k) word[k] = 0u;  // the pitch's end
                    }
                    if (in && c < o8.pitch) {
                        uint8_t* const at = o8.q + n * o8.pitch + c;
                        if constexpr (VEC == 8)
                            *reinterpret_cast<uint2*>(at) = make_uint2(word[0], word[1]);
                        else
                            *reinterpret_cast<uint32_t*>(at) = word[0];
                    }
                }
            }
            if constexpr (kQ && VEC <= 2) {
                // narrow pieces: the row through shared memory, four channels a lane
                const int cpad = (C + 127) / 128 * 128;
                float* const vr = vrow + (threadIdx.x / TPR) * cpad;
                group_sync<TPR>();  // the row before has been read
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if ((i * TPR + t) * VEC < C) Unit::store(vr + (i * TPR + t) * VEC, d[i][0]);
                group_sync<TPR>();
                constexpr int kLanes = TPR < 32 ? TPR : 32, kWords = 32 / kLanes;
                const int sub = t % kLanes;
                for (int b = t / kLanes; b * 128 < C; b += TPR / kLanes) {
                    float v[kWords][4];
                    uint32_t top = 0;
#pragma unroll
                    for (int k = 0; k < kWords; ++k) {
                        const int c = b * 128 + (k * kLanes + sub) * 4;
                        const float4 f = *reinterpret_cast<const float4*>(vr + c);
                        v[k][0] = c < C ? f.x : 0.f;
                        v[k][1] = c + 1 < C ? f.y : 0.f;
                        v[k][2] = c + 2 < C ? f.z : 0.f;
                        v[k][3] = c + 3 < C ? f.w : 0.f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) top = max(top, mag(v[k][e]));
                    }
#pragma unroll
                    for (int o = 1; o < kLanes; o <<= 1)
                        top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const float scale = scale_of(__uint_as_float(top));
#pragma unroll
                    for (int k = 0; k < kWords; ++k) {
                        const int c = b * 128 + (k * kLanes + sub) * 4;
                        const uint32_t word = quantise4(v[k], scale, C - c);
                        if (in && c < o8.pitch)
                            *reinterpret_cast<uint32_t*>(o8.q + n * o8.pitch + c) = word;
                    }
                    if (in && sub == 0) o8.scales[(long long)b * capacity + n] = scale;
                }
            }
        }
    }
}

// The gradient in the same layout. A thread owns its channels for all its
// rows, so dgamma is summed in registers; the groups of a block are added in
// order through shared memory, the blocks by column_sum_kernel.
template <typename T, int VEC, int TPR, int NV>
__global__ void __launch_bounds__(kGroupThreads)
    rms_bwd_rows_kernel(const T* h, const T* dy, const T* dres, const int32_t* count,
                        long long capacity, int C, const float* __restrict__ gamma,
                        const float* __restrict__ rstd, T* dx, float* __restrict__ part,
                        unsigned* status) {
    __shared__ __align__(16) float sh[2 * kGroupThreads / 32];
    extern __shared__ __align__(16) float psum[];  // [groups][C] when the block has several
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    constexpr int kGroups = kGroupThreads / TPR;
    const int t = threadIdx.x % TPR;
    const long long step = (long long)gridDim.x * kGroups;
    const long long n0 = (long long)blockIdx.x * kGroups + threadIdx.x / TPR;
    const long long w0 = TPR < 32 ? n0 - (threadIdx.x & 31) / TPR : n0;
    using Unit = UnitOf<VEC>;
    using U = typename Unit::type;
    constexpr int kU = Unit::count;
    const float inv = 1.f / (float)C;
    Piece<T, VEC> ch[NV], cd[NV], cr[NV], nh[NV], nd[NV], nr[NV];
    float r1 = 0.f;
    U ga[NV][kU], dg[NV][kU];
    auto load = [&](long long n) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VEC;
            if (n < rows && c < C) {
                nh[i].load(h + n * C + c);
                nd[i].load(dy + n * C + c);
                if (dres && dx) nr[i].load(dres + n * C + c);
            }
        }
        if (n < rows) r1 = rstd[n];
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * VEC;
#pragma unroll
        for (int e = 0; e < kU; ++e) ga[i][e] = Unit::splat(1.f), dg[i][e] = Unit::splat(0.f);
        if (c < C) load_units<VEC>(gamma, c, 1.f, ga[i]);
    }
    // the next row is on its way while this one is worked on; 16 single elements
    // of three inputs twice would spill (16384 x 5001 bf16 951 us so)
    constexpr bool kNext = !(VEC == 1 && NV == 16);
    if (kNext) load(n0);
    int turn = 0;
    for (long long w = w0, n = n0; w < rows; w += step, n += step) {
        const bool in = n < rows;
        if (!kNext) load(n);
        const U times = Unit::splat(r1);
        U s = Unit::splat(0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            ch[i] = nh[i];
            cd[i] = nd[i];
            cr[i] = nr[i];
        }
        if (kNext) load(n + step);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (in && (i * TPR + t) * VEC < C)
#pragma unroll
                for (int e = 0; e < kU; ++e) {
                    const U p = mul(cd[i].unit(e), mul(ch[i].unit(e), times));  // dy * hh
                    s = fma(p, ga[i][e], s);
                    dg[i][e] = add(dg[i][e], p);
                }
        if (dx == nullptr) continue;
        const float mean = group_sum<TPR>(total(s), sh, turn) * inv;
        turn ^= 1;
        if (!in) continue;
        const U less = Unit::splat(-mean);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VEC;
            if (c < C) {
                U f[kU];
#pragma unroll
                for (int e = 0; e < kU; ++e) {
                    const U hh = mul(ch[i].unit(e), times);
                    f[e] = fma(hh, less, mul(cd[i].unit(e), ga[i][e]));
                    f[e] = dres ? fma(f[e], times, cr[i].unit(e)) : mul(f[e], times);
                }
                ch[i].set_units(f);
                ch[i].store(dx + n * C + c);
            }
        }
    }
    if (part == nullptr) return;
    float* const out = part + (long long)blockIdx.x * C;
    float* const mine = kGroups > 1 ? psum + (threadIdx.x / TPR) * C : out;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < kU; ++e) {
            const int c = (i * TPR + t) * VEC + e * (VEC / kU);
            if (c < C) Unit::store(mine + c, dg[i][e]);
        }
    if constexpr (kGroups > 1) {
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += kGroupThreads) {
            float v = 0.f;
#pragma unroll 8
            for (int g = 0; g < kGroups; ++g) v += psum[g * C + c];
            out[c] = v;
        }
    }
}

// ---------------------------------------------------------------- wide rows
// A block per row, read a second time for the output (from the caches). A
// lane holds four neighbouring channels, so that a warp holds a block of the
// 8-bit form, and the same ones in every pass: what it wrote it may read.
template <typename T, bool kWide>
struct Four {
    float f[4];
    __device__ __forceinline__ void load(const T* p, int left) {
        if constexpr (kWide) {
            Piece<T, 4> q;
            q.load(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = q.get(e);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = e < left ? to_f32(p[e]) : 0.f;
        }
    }
    __device__ __forceinline__ void store(T* p, int left) const {
        if constexpr (kWide) {
            if constexpr (sizeof(T) == 4)
                *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
            else
                *reinterpret_cast<uint2*>(p) = make_uint2(Piece<__nv_bfloat16, 8>::pair(f[0], f[1]),
                                                          Piece<__nv_bfloat16, 8>::pair(f[2], f[3]));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) p[e] = from_f32<T>(f[e]);
        }
    }
};

template <typename T, bool kWide>
__global__ void __launch_bounds__(kThreads)
    rms_fwd_kernel(const T* x, const T* res, const int32_t* count, long long capacity, int C,
                   float eps, const float* __restrict__ gamma, T* h, T* y, float* rstd_out,
                   RmsArgs8 o8, unsigned* status) {
    __shared__ float sh[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    const float inv = 1.f / (float)C;
    constexpr int kStep = kThreads * 4;
    for (long long n = blockIdx.x; n < rows; n += gridDim.x) {
        // the row's channels c .. c + 3 as the norm takes them
        auto row = [&](int c, bool again) {
            Four<T, kWide> p;
            if (again && h) {
                p.load(h + n * C + c, C - c);
                return p;
            }
            p.load(x + n * C + c, C - c);
            if (res) {
                Four<T, kWide> r;
                r.load(res + n * C + c, C - c);
#pragma unroll
                for (int e = 0; e < 4; ++e) p.f[e] = to_f32(from_f32<T>(p.f[e] + r.f[e]));
            }
            return p;
        };
        float s = 0.f;
#pragma unroll 4
        for (int c = threadIdx.x * 4; c < C; c += kStep) {
            const Four<T, kWide> p = row(c, false);
            if (h) p.store(h + n * C + c, C - c);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = fmaf(p.f[e], p.f[e], s);
        }
        const float ms = fmaf(block_sum(s, sh), inv, eps);
        float rstd = rsqrtf(ms);
        if (outside(ms)) {
            const float f = factor(ms);
            s = 0.f;
            for (int c = threadIdx.x * 4; c < C; c += kStep) {
                const Four<T, kWide> p = row(c, true);
#pragma unroll
                for (int e = 0; e < 4; ++e) s = fmaf(p.f[e] * f, p.f[e] * f, s);
            }
            rstd = rstd_scaled(block_sum(s, sh), inv, eps, f);
        }
        if (rstd_out && threadIdx.x == 0) rstd_out[n] = rstd;
        // whole blocks of 128 channels a warp, so that its lanes stay together
        for (int c = threadIdx.x * 4; (c & ~127) < C; c += kStep) {
            Four<T, kWide> p{};
            if (c < C) {
                p = row(c, true);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float g = gamma && c + e < C ? __ldg(gamma + c + e) : 1.f;
                    p.f[e] = p.f[e] * rstd * g;
                }
            }
            if (o8.q) {
                uint32_t top = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) top = max(top, c + e < C ? mag(p.f[e]) : 0u);
#pragma unroll
                for (int o = 1; o < 32; o <<= 1)
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float scale = scale_of(__uint_as_float(top));
                const uint32_t word = quantise4(p.f, scale, C - c);
                if (c < o8.pitch) *reinterpret_cast<uint32_t*>(o8.q + n * o8.pitch + c) = word;
                if ((threadIdx.x & 31) == 0)
                    o8.scales[(long long)(c / 128) * capacity + n] = scale;
            }
            if (y && c < C) p.store(y + n * C + c, C - c);
        }
    }
}

// sums[n] = sum (g * hh) / C.
template <typename T, bool kWide>
__global__ void __launch_bounds__(kThreads)
    rms_bwd_sums_kernel(const T* h, const T* dy, const int32_t* count, long long capacity, int C,
                        const float* __restrict__ gamma, const float* __restrict__ rstd,
                        float* __restrict__ sums, unsigned* status) {
    __shared__ float sh[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    for (long long n = blockIdx.x; n < rows; n += gridDim.x) {
        const float r = rstd[n];
        float s = 0.f;
#pragma unroll 4
        for (int c = threadIdx.x * 4; c < C; c += kThreads * 4) {
            Four<T, kWide> p, d;
            p.load(h + n * C + c, C - c);
            d.load(dy + n * C + c, C - c);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float g = gamma && c + e < C ? __ldg(gamma + c + e) : 1.f;
                s = fmaf(d.f[e] * (p.f[e] * r), g, s);
            }
        }
        s = block_sum(s, sh);
        if (threadIdx.x == 0) sums[n] = s / (float)C;
    }
}

// Four channels a thread, rows blockIdx.y, + gridDim.y, ...: dx, and the
// thread's own sums of dy * hh into part[blockIdx.y][C]. Four rows are loaded
// before the first is worked on: dx may be one of the inputs, so no load
// would be moved up over a store.
constexpr int kColRows = 4;

template <typename T, bool kWide>
__global__ void __launch_bounds__(kThreads)
    rms_bwd_cols_kernel(const T* h, const T* dy, const T* dres, const int32_t* count,
                        long long capacity, int C, const float* __restrict__ gamma,
                        const float* __restrict__ rstd, const float* __restrict__ sums, T* dx,
                        float* __restrict__ part, unsigned* status) {
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    const int c = (int)(blockIdx.x * kThreads + threadIdx.x) * 4;
    if (c >= C) return;
    const int left = C - c;
    float ga[4], dg[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e) ga[e] = gamma && e < left ? __ldg(gamma + c + e) : 1.f;
    for (long long m = blockIdx.y; m < rows; m += (long long)kColRows * gridDim.y) {
        Four<T, kWide> p[kColRows], d[kColRows], r[kColRows];
        float rs[kColRows], s[kColRows];
#pragma unroll
        for (int u = 0; u < kColRows; ++u) {
            // a row past the end is loaded as the first and not used
            const long long at = m + (long long)u * gridDim.y, n = at < rows ? at : m;
            p[u].load(h + n * C + c, left);
            d[u].load(dy + n * C + c, left);
            r[u] = Four<T, kWide>{};
            if (dres && dx) r[u].load(dres + n * C + c, left);
            rs[u] = rstd[n];
            s[u] = dx ? sums[n] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kColRows; ++u) {
            const long long n = m + (long long)u * gridDim.y;
            if (n >= rows) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float hh = p[u].f[e] * rs[u];
                dg[e] = fmaf(d[u].f[e], hh, dg[e]);
                p[u].f[e] = fmaf(fmaf(hh, -s[u], d[u].f[e] * ga[e]), rs[u], r[u].f[e]);
            }
            if (dx) p[u].store(dx + n * C + c, left);
        }
    }
    if (part) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) part[(long long)blockIdx.y * C + c + e] = dg[e];
    }
}

// ---------------------------------------------------------------- host side
RmsArgs8 out8(const RmsNormArgs& a) {
    return {a.q, a.scales, HC_FP8_PITCH(a.C)};
}

template <typename T, int VEC, int TPR, int NV, bool kQ>
hc_status launch_fwd_rows(const DeviceCtx* ctx, const RmsNormArgs& a, cudaStream_t s) {
    constexpr int kGroups = kGroupThreads / TPR;
    const long long need = ((long long)a.capacity + kGroups - 1) / kGroups;
    const long long cap = (long long)ctx->num_sms;
    // a row of v a group, padded to whole blocks of 128: 4 bytes for each of the at
    // most 512 * VEC * NV channels held (64 KiB with 16 pairs a thread, 32 with
    // single elements) or, below 128 channels, for the 128 of 64 groups' rows (32
    // KiB). More than 48 KiB, the sums' 128 bytes among them, have to be allowed.
    const size_t smem = kQ && VEC <= 2 ? (size_t)kGroups * ((a.C + 127) / 128 * 128) * 4 : 0;
    auto kern = rms_fwd_rows_kernel<T, VEC, TPR, NV, kQ>;
    constexpr size_t kMost = (size_t)4 * kGroupThreads * VEC * NV;
    static bool done[64];
    if (kQ && VEC <= 2 && kMost > 47 * 1024 && smem > 47 * 1024 && !done[ctx->device]) {
        const hc_status st = check_cuda(
            cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMost),
            "rms_fwd_rows_kernel");
        if (st != HC_OK) return st;
        done[ctx->device] = true;
    }
    return launch_pdl(kern, dim3((unsigned)(need < cap ? need : cap)), dim3(kGroupThreads), smem, s,
                      "rms_fwd_rows_kernel", (const T*)a.x, (const T*)a.res, a.count,
                      (long long)a.capacity, a.C, a.eps, a.gamma, (T*)a.h, (T*)a.y, a.rstd_out,
                      out8(a), ctx->status);
}

template <typename T, int VEC, int TPR, int NV>
hc_status fwd_rows(const DeviceCtx* ctx, const RmsNormArgs& a, cudaStream_t s) {
    return a.q ? launch_fwd_rows<T, VEC, TPR, NV, true>(ctx, a, s)
               : launch_fwd_rows<T, VEC, TPR, NV, false>(ctx, a, s);
}

template <typename T, int VEC, int TPR, int NV>
hc_status bwd_rows(const DeviceCtx* ctx, const RmsNormArgs& a, cudaStream_t s) {
    constexpr int kGroups = kGroupThreads / TPR;
    const long long need = ((long long)a.capacity + kGroups - 1) / kGroups;
    const long long cap = (long long)ctx->num_sms;
    const int grid = (int)(need < 1 ? 1 : need < cap ? need : cap);
    float* part = nullptr;
    if (a.dgamma) {
        part = (float*)stream_workspace(s, (size_t)grid * a.C * 4);
        if (!part) return HC_ERR_CUDA;
    }
    // the groups' sums: at most 32 KiB, 4 bytes for each of the
    // kGroups * C <= 512 * 16 channels held
    const size_t smem = kGroups > 1 && part ? (size_t)kGroups * a.C * 4 : 0;
    const hc_status st = launch_pdl(
        rms_bwd_rows_kernel<T, VEC, TPR, NV>, dim3((unsigned)grid), dim3(kGroupThreads), smem, s,
        "rms_bwd_rows_kernel", (const T*)a.x, (const T*)a.dy, (const T*)a.res, a.count,
        (long long)a.capacity, a.C, a.gamma, a.rstd, (T*)a.dx, part, ctx->status);
    if (st != HC_OK || !part) return st;
    return launch_column_sum(part, grid, a.C, a.C, a.dgamma, s);
}

template <typename T, int VEC, int TPR, int NV>
hc_status rows_in_regs(const DeviceCtx* ctx, const RmsNormArgs& a, bool back, cudaStream_t s) {
    return back ? bwd_rows<T, VEC, TPR, NV>(ctx, a, s) : fwd_rows<T, VEC, TPR, NV>(ctx, a, s);
}

template <typename T, bool kWide>
hc_status fwd_wide(const DeviceCtx* ctx, const RmsNormArgs& a, cudaStream_t s) {
    const long long cap = (long long)ctx->num_sms * 4;
    const unsigned grid = (unsigned)(a.capacity < cap ? a.capacity : cap);
    return launch_pdl(rms_fwd_kernel<T, kWide>, dim3(grid), dim3(kThreads), 0, s, "rms_fwd_kernel",
                      (const T*)a.x, (const T*)a.res, a.count, (long long)a.capacity, a.C, a.eps,
                      a.gamma, (T*)a.h, (T*)a.y, a.rstd_out, out8(a), ctx->status);
}

template <typename T, bool kWide>
hc_status bwd_wide(const DeviceCtx* ctx, const RmsNormArgs& a, cudaStream_t s) {
    const unsigned ctiles = (unsigned)(((long long)a.C + kThreads * 4 - 1) / (kThreads * 4));
    long long parts = (ctx->num_sms * 4 + ctiles - 1) / ctiles;
    if (parts > a.capacity) parts = a.capacity;
    if (parts < 1) parts = 1;
    const size_t sums_n = ((size_t)a.capacity + 63) / 64 * 64;
    float* const ws = (float*)stream_workspace(
        s, 4 * (sums_n + (a.dgamma ? (size_t)parts * a.C : 0)));
    if (!ws) return HC_ERR_CUDA;
    float* const part = a.dgamma ? ws + sums_n : nullptr;
    hc_status st;
    if (a.capacity > 0 && a.dx) {
        const long long cap = (long long)ctx->num_sms * 4;
        st = launch_pdl(rms_bwd_sums_kernel<T, kWide>,
                        dim3((unsigned)(a.capacity < cap ? a.capacity : cap)), dim3(kThreads), 0, s,
                        "rms_bwd_sums_kernel", (const T*)a.x, (const T*)a.dy, a.count,
                        (long long)a.capacity, a.C, a.gamma, a.rstd, ws, ctx->status);
        if (st != HC_OK) return st;
    }
    st = launch_pdl(rms_bwd_cols_kernel<T, kWide>, dim3(ctiles, (unsigned)parts), dim3(kThreads), 0,
                    s, "rms_bwd_cols_kernel", (const T*)a.x, (const T*)a.dy, (const T*)a.res,
                    a.count, (long long)a.capacity, a.C, a.gamma, a.rstd, (const float*)ws,
                    (T*)a.dx, part, ctx->status);
    if (st != HC_OK || !part) return st;
    return launch_column_sum(part, (int)parts, a.C, a.C, a.dgamma, s);
}

// Rows of at most 8192 channels are held in registers by the smallest group that
// does so without spilling: forward up to 64 bytes a lane of a warp (300 to 1024 bf16
// channels by a warp each, which waits for no other: 600 channels 168 us for 268 MB
// in and out, by 128 threads with a barrier a row 229; to 8 bits 162 and 316), the
// gradient, which keeps three rows' pieces twice, gamma and its sums, half of
// that. Rows without 16-byte loads are read in 4-byte pieces where they allow it (602
// bf16 channels 188 us, 2050 258), else element by element (2047 bf16 265, fp32 165).
template <typename T>
hc_status run(const DeviceCtx* ctx, const RmsNormArgs& a, bool back, cudaStream_t s) {
    constexpr int kVec = 16 / (int)sizeof(T);
    const int C = a.C;
    auto aligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const bool wide = C % kVec == 0 && aligned(a.x) && aligned(a.res) && aligned(a.h) &&
                      aligned(a.y) && aligned(a.dy) && aligned(a.dx) && aligned(a.gamma);
    if (C > 8192) {
        if (wide) return back ? bwd_wide<T, true>(ctx, a, s) : fwd_wide<T, true>(ctx, a, s);
        return back ? bwd_wide<T, false>(ctx, a, s) : fwd_wide<T, false>(ctx, a, s);
    }
    if (wide) {
        if (C <= 8 * kVec) return rows_in_regs<T, kVec, 8, 1>(ctx, a, back, s);
        if (C <= 32 * kVec) return rows_in_regs<T, kVec, 32, 1>(ctx, a, back, s);
        if (C <= 64 * kVec) return rows_in_regs<T, kVec, 32, 2>(ctx, a, back, s);
        if (C <= 128 * kVec)
            return back ? bwd_rows<T, kVec, 128, 1>(ctx, a, s) : fwd_rows<T, kVec, 32, 4>(ctx, a, s);
        if (C <= 256 * kVec) return rows_in_regs<T, kVec, 128, 2>(ctx, a, back, s);
        if (C <= 512 * kVec) return rows_in_regs<T, kVec, 256, 2>(ctx, a, back, s);
        if (C <= 1024 * kVec) {
            // two groups a block, so that one works while the other waits for its
            // row's sum: 16384 x 8192 bf16 to 8 bits 155 us, one group 160
            if (a.q && !back) return launch_fwd_rows<T, kVec, 256, 4, true>(ctx, a, s);
            return rows_in_regs<T, kVec, 512, 2>(ctx, a, back, s);
        }
        if constexpr (kVec == 4) return rows_in_regs<T, kVec, 512, 4>(ctx, a, back, s);
    }
    if constexpr (kVec == 8) {
        // bf16 rows that allow 4-byte loads
        auto even = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; };
        if (C % 2 == 0 && even(a.x) && even(a.res) && even(a.h) && even(a.y) && even(a.dy) && even(a.dx)) {
            if (C <= 64) return rows_in_regs<T, 2, 8, 4>(ctx, a, back, s);
            if (C <= 128) return rows_in_regs<T, 2, 8, 8>(ctx, a, back, s);
            if (C <= 256) return rows_in_regs<T, 2, 32, 4>(ctx, a, back, s);
            if (C <= 512) return rows_in_regs<T, 2, 32, 8>(ctx, a, back, s);
            if (!back) {
                if (C <= 1024) return fwd_rows<T, 2, 32, 16>(ctx, a, s);
                if (C <= 4096) return fwd_rows<T, 2, 128, 16>(ctx, a, s);
                return fwd_rows<T, 2, 256, 16>(ctx, a, s);
            }
            if (C <= 1024) return bwd_rows<T, 2, 128, 4>(ctx, a, s);
            if (C <= 2048) return bwd_rows<T, 2, 128, 8>(ctx, a, s);
            if (C <= 4096) return bwd_rows<T, 2, 256, 8>(ctx, a, s);
            return bwd_rows<T, 2, 512, 8>(ctx, a, s);
        }
    }
    if (C <= 32) return rows_in_regs<T, 1, 8, 4>(ctx, a, back, s);
    if (C <= 64) return rows_in_regs<T, 1, 8, 8>(ctx, a, back, s);
    if (C <= 128) return rows_in_regs<T, 1, 32, 4>(ctx, a, back, s);
    if (C <= 256) return rows_in_regs<T, 1, 32, 8>(ctx, a, back, s);
    if (!back) {
        if (C <= 512) return fwd_rows<T, 1, 32, 16>(ctx, a, s);
        if (C <= 1024) return fwd_rows<T, 1, 128, 8>(ctx, a, s);
        if (C <= 2048) return fwd_rows<T, 1, 128, 16>(ctx, a, s);
        if (C <= 4096) return fwd_rows<T, 1, 256, 16>(ctx, a, s);
        return fwd_rows<T, 1, 512, 16>(ctx, a, s);
    }
    if (C <= 512) return bwd_rows<T, 1, 128, 4>(ctx, a, s);
    if (C <= 1024) return bwd_rows<T, 1, 128, 8>(ctx, a, s);
    if (C <= 2048) return bwd_rows<T, 1, 256, 8>(ctx, a, s);
    if (C <= 4096) return bwd_rows<T, 1, 512, 8>(ctx, a, s);
    return bwd_rows<T, 1, 512, 16>(ctx, a, s);
}

}  // namespace

hc_status launch_rms_norm_fwd(const DeviceCtx* ctx, const RmsNormArgs& a, cudaStream_t s) {
    return a.dt == HC_BF16 ? run<__nv_bfloat16>(ctx, a, false, s) : run<float>(ctx, a, false, s);
}

hc_status launch_rms_norm_bwd(const DeviceCtx* ctx, const RmsNormArgs& a, cudaStream_t s) {
    return a.dt == HC_BF16 ? run<__nv_bfloat16>(ctx, a, true, s) : run<float>(ctx, a, true, s);
}

}  // namespace hc
