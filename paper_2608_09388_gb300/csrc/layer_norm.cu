// Layer norm of compact rows and its gradient. For every row n < N', over its
// C channels:
//   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps)
//   y = (x - mean) * rstd * gamma + beta
// and backwards, with xh = (x - mean) * rstd and g = dy * gamma:
//   dx     = rstd * (g - sum g / C - xh * sum (g * xh) / C)
//   dgamma = sum over rows of dy * xh,  dbeta = sum over rows of dy
// All sums in fp32; the variance is taken around the mean, which is refined
// where it is far from zero against the row's spread. dgamma and dbeta
// are summed per block of rows and the blocks' sums joined in a fixed order,
// so every result is the same from run to run.
//
// Bound by memory: forward reads and writes a row once, the gradient reads two
// rows and writes one. Rows of up to 8192 channels therefore stay in registers
// between the passes over their channels, and the loads of the next rows are
// issued before this one is reduced. At 65536 x 2048 bf16 (GB300) the forward
// takes 91 us (79 at the copy rate) and the gradient 137 us (119), 4 us of it
// the joining of dgamma and dbeta; before the arithmetic went in pairs the
// issue slots bound it (103 us).
#include "tokens.cuh"

namespace hc {
namespace {

constexpr int kThreads = 512;

// ---------------------------------------------------------------- rows in registers
// A group of TPR threads holds a whole row: NV pieces of VEC elements each,
// piece i of thread t at channel (i * TPR + t) * VEC. The row is read once;
// the next rows of the group are loaded before this one is worked on, so that
// loads are in flight throughout. Groups stride over the rows.
constexpr int kGroupThreads = 512;  // threads per block: kGroupThreads / TPR groups
// Rows of a group in flight in the forward pass: 32 registers' worth, four at
// most. One block an SM then has 64 KB on the way, and gamma and beta stay in
// registers (read from L1 for every row they took 85% of its data path:
// 65536 x 2048 bf16 103 us).
template <typename T, int VEC, int NV>
constexpr int kRowRegs = NV * (VEC == 1 ? 1 : 4);
template <typename T, int VEC, int NV>
constexpr int kFwdAhead = 32 / kRowRegs<T, VEC, NV> < 4 ? 32 / kRowRegs<T, VEC, NV> : 4;

// p[c .. c + VEC), 16-byte aligned when VEC > 1, or `none` without a p.
template <int VEC>
__device__ __forceinline__ void load_units(const float* __restrict__ p, int c, float none,
                                           typename UnitOf<VEC>::type (&u)[UnitOf<VEC>::count]) {
    if constexpr (VEC == 1) {
        u[0].v = p ? __ldg(p + c) : none;
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

// Whether a row's mean is so far from zero, against the spread that its sum of
// squared differences shows, that the rounding of its sum may matter: 16 times.
// The mean of the differences is then taken off them as well. A row of one
// value is always so unless it is zero: its differences, all alike and a few
// units in the last place of the value, then vanish.
__device__ __forceinline__ bool is_far(float mean, float sum2, float inv) {
    return mean * mean >= sum2 * (256.f * inv) && mean != 0.f;
}
// sum / C with inv the rounded 1 / C: the product, corrected by its residual,
// is the quotient where that is an fp32 number.
__device__ __forceinline__ float mean_of(float sum, int C, float inv) {
    const float q = sum * inv;
    return fmaf(fmaf(-q, (float)C, sum), inv, q);
}

template <typename T, int VEC, int TPR, int NV>
__global__ void __launch_bounds__(kGroupThreads)
    ln_fwd_rows_kernel(const T* x, const int32_t* count, long long capacity, int C, float eps,
                       const float* __restrict__ gamma, const float* __restrict__ beta, T* y,
                       float* mean_out, float* rstd_out, unsigned* status) {
    __shared__ __align__(16) float sh[2 * kGroupThreads / 32];
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    constexpr int kGroups = kGroupThreads / TPR;
    const int t = threadIdx.x % TPR;
    const long long step = (long long)gridDim.x * kGroups;
    // every thread of a warp takes part in the shuffles: groups of a warp run
    // the same number of rounds
    const long long n0 = (long long)blockIdx.x * kGroups + threadIdx.x / TPR;
    const long long w0 = TPR < 32 ? n0 - (threadIdx.x & 31) / TPR : n0;
    using Unit = UnitOf<VEC>;
    using U = typename Unit::type;
    const float inv = 1.f / (float)C;
    constexpr int kAhead = kFwdAhead<T, VEC, NV>;
    // The second look at a row that is far from zero reads it again where single
    // elements fill the registers (keeping it spills: 32768 x 2047 bf16 230 us, 76 so).
    constexpr bool kReread = VEC == 1;
    Piece<T, VEC> ring[kAhead][NV];
    U ga[NV][Unit::count], be[NV][Unit::count];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * VEC;
        if (c < C) {
            load_units<VEC>(gamma, c, 1.f, ga[i]);
            load_units<VEC>(beta, c, 0.f, be[i]);
        }
    }
    auto load = [&](long long n, Piece<T, VEC>(&p)[NV]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VEC;
            if (n < rows && c < C) p[i].load(x + n * C + c);
        }
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(n0 + u * step, ring[u]);
    for (long long w = w0, n = n0; w < rows;) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u, w += step, n += step) {
            if (w >= rows) break;
            // the row as fp32, then its differences from the mean
            U s = Unit::splat(0.f), v = s, d[NV][Unit::count];
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < Unit::count; ++e) d[i][e] = ring[u][i].unit(e);
            load(n + kAhead * step, ring[u]);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if ((i * TPR + t) * VEC < C)
#pragma unroll
                    for (int e = 0; e < Unit::count; ++e) s = add(s, d[i][e]);
            // a product that is not fused into the differences: they are taken from
            // the number that is kept
            float mean = __fmul_rn(group_sum<TPR>(total(s), sh, 0), inv);
            const U less = Unit::splat(-mean);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if ((i * TPR + t) * VEC < C)
#pragma unroll
                    for (int e = 0; e < Unit::count; ++e) {
                        d[i][e] = add(d[i][e], less);
                        v = fma(d[i][e], d[i][e], v);
                    }
            float sum2 = group_sum<TPR>(total(v), sh, 1);
            const bool far = n < rows && is_far(mean, sum2, inv);
            if (TPR < 32 ? __any_sync(0xffffffffu, far) : far) {
                s = v = Unit::splat(0.f);
                if constexpr (kReread) {
#pragma unroll 1
                    for (int c = t; far && c < C; c += TPR) {
                        Piece<T, VEC> p;
                        p.load(x + n * C + c);
                        s = add(s, add(p.unit(0), less));
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < NV; ++i)
                        if ((i * TPR + t) * VEC < C)
#pragma unroll
                            for (int e = 0; e < Unit::count; ++e) s = add(s, d[i][e]);
                }
                const float off = mean_of(group_sum<TPR>(total(s), sh, 0), C, inv);
                if (far) {
                    mean += off;
                    const U less2 = Unit::splat(kReread ? -mean : -off);
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const int c = (i * TPR + t) * VEC;
                        if (c >= C) continue;
                        Piece<T, VEC> p;
                        if constexpr (kReread) p.load(x + n * C + c);
#pragma unroll
                        for (int e = 0; e < Unit::count; ++e) {
                            d[i][e] = add(kReread ? p.unit(e) : d[i][e], less2);
                            v = fma(d[i][e], d[i][e], v);
                        }
                    }
                }
                const float again = group_sum<TPR>(total(v), sh, 1);
                sum2 = far ? again : sum2;
            }
            const float rstd = rsqrtf(fmaf(sum2, inv, eps));
            if (n >= rows) continue;
            const U times = Unit::splat(rstd);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * TPR + t) * VEC;
                if (c < C) {
#pragma unroll
                    for (int e = 0; e < Unit::count; ++e)
                        d[i][e] = fma(mul(d[i][e], times), ga[i][e], be[i][e]);
                    Piece<T, VEC> out;
                    out.set_units(d[i]);
                    out.store(y + n * C + c);
                }
            }
            if (t == 0) {
                if (mean_out) mean_out[n] = mean;
                if (rstd_out) rstd_out[n] = rstd;
            }
        }
    }
}

// The gradient in the same layout. A thread owns its channels for all its
// rows, so dgamma and dbeta are summed in registers; the groups of a block
// are added in order through shared memory, the blocks by ln_param_grad_kernel.
template <typename T, int VEC, int TPR, int NV>
__global__ void __launch_bounds__(kGroupThreads)
    ln_bwd_rows_in_regs_kernel(const T* x, const T* dy, const int32_t* count, long long capacity,
                               int C, const float* __restrict__ gamma,
                               const float* __restrict__ mean, const float* __restrict__ rstd,
                               T* dx, float* __restrict__ part, unsigned* status) {
    __shared__ __align__(16) float sh[2 * kGroupThreads / 32];
    extern __shared__ float psum[];  // [groups][2][C] when the block has several groups
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
    Piece<T, VEC> cx[NV], cd[NV], nx[NV], nd[NV];
    float m1 = 0.f, r1 = 0.f;
    U ga[NV][kU], dg[NV][kU], db[NV][kU];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * VEC;
#pragma unroll
        for (int e = 0; e < kU; ++e) ga[i][e] = Unit::splat(1.f), dg[i][e] = db[i][e] = Unit::splat(0.f);
        if (c < C) load_units<VEC>(gamma, c, 1.f, ga[i]);
        if (n0 < rows && c < C) {
            nx[i].load(x + n0 * C + c);
            nd[i].load(dy + n0 * C + c);
        }
    }
    if (n0 < rows) {
        m1 = mean[n0];
        r1 = rstd[n0];
    }
    for (long long w = w0, n = n0; w < rows; w += step, n += step) {
        const bool in = n < rows, more = n + step < rows;
        const U less = Unit::splat(-m1), times = Unit::splat(r1);
        U s1 = Unit::splat(0.f), s2 = s1;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VEC;
            cx[i] = nx[i];
            cd[i] = nd[i];
            if (more && c < C) {
                nx[i].load(x + (n + step) * C + c);
                nd[i].load(dy + (n + step) * C + c);
            }
        }
        if (more) {
            m1 = mean[n + step];
            r1 = rstd[n + step];
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (in && (i * TPR + t) * VEC < C)
#pragma unroll
                for (int e = 0; e < kU; ++e) {
                    const U d = cd[i].unit(e), xh = mul(add(cx[i].unit(e), less), times);
                    const U g = mul(d, ga[i][e]);
                    s1 = add(s1, g);
                    s2 = fma(g, xh, s2);
                    dg[i][e] = fma(d, xh, dg[i][e]);
                    db[i][e] = add(db[i][e], d);
                }
        if (dx == nullptr) continue;
        const float c1 = group_sum<TPR>(total(s1), sh, 0) * inv;
        const float c2 = group_sum<TPR>(total(s2), sh, 1) * inv;
        if (!in) continue;
        const U less1 = Unit::splat(-c1), less2 = Unit::splat(-c2);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VEC;
            if (c < C) {
                U f[kU];
#pragma unroll
                for (int e = 0; e < kU; ++e) {
                    const U xh = mul(add(cx[i].unit(e), less), times);
                    f[e] = mul(fma(xh, less2, fma(cd[i].unit(e), ga[i][e], less1)), times);
                }
                cx[i].set_units(f);
                cx[i].store(dx + n * C + c);
            }
        }
    }
    if (part == nullptr) return;
    float* const out = part + 2ll * blockIdx.x * C;
    if constexpr (kGroups > 1) {
        float* const mine = psum + (threadIdx.x / TPR) * 2 * C;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < kU; ++e) {
                const int c = (i * TPR + t) * VEC + e * (VEC / kU);
                if (c < C) {
                    Unit::store(mine + c, dg[i][e]);
                    Unit::store(mine + C + c, db[i][e]);
                }
            }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * C; c += kGroupThreads) {
            float v = 0.f;
#pragma unroll 8
            for (int g = 0; g < kGroups; ++g) v += psum[g * 2 * C + c];
            out[c] = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < kU; ++e) {
                const int c = (i * TPR + t) * VEC + e * (VEC / kU);
                if (c < C) {
                    Unit::store(out + c, dg[i][e]);
                    Unit::store(out + C + c, db[i][e]);
                }
            }
    }
}

// ---------------------------------------------------------------- wide rows
// A block per row; the row is read once for the mean, once for the variance
// and once for the output (the second and third time from the caches).
// 16384 x 16384 bf16: forward 257 us, gradient 457 (158 and 237 at the copy
// rate; element by element 404 and 1115; forward with 256 threads 283).
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads)
    ln_fwd_kernel(const T* x, const int32_t* count, long long capacity, int C, float eps,
                  const float* __restrict__ gamma, const float* __restrict__ beta, T* y,
                  float* mean_out, float* rstd_out, unsigned* status) {
    __shared__ float sh[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    for (long long n = blockIdx.x; n < rows; n += gridDim.x) {
        const T* xr = x + n * C;
        T* yr = y + n * C;
        float s = 0.f;
#pragma unroll 4
        for (int c = threadIdx.x * VEC; c < C; c += kThreads * VEC) {
            Piece<T, VEC> p;
            p.load(xr + c);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s += p.get(e);
        }
        float mean = block_sum(s, sh) / (float)C;
        float v;
        for (bool again = false;; again = true) {
            v = 0.f;
#pragma unroll 4
            for (int c = threadIdx.x * VEC; c < C; c += kThreads * VEC) {
                Piece<T, VEC> p;
                p.load(xr + c);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float d = p.get(e) - mean;
                    v += d * d;
                }
            }
            v = block_sum(v, sh);
            if (again || !is_far(mean, v, 1.f / (float)C)) break;
            s = 0.f;
#pragma unroll 1
            for (int c = threadIdx.x * VEC; c < C; c += kThreads * VEC) {
                Piece<T, VEC> p;
                p.load(xr + c);
#pragma unroll
                for (int e = 0; e < VEC; ++e) s += p.get(e) - mean;
            }
            mean += block_sum(s, sh) / (float)C;
        }
        const float rstd = 1.f / sqrtf(v / (float)C + eps);
        for (int c = threadIdx.x * VEC; c < C; c += kThreads * VEC) {
            Piece<T, VEC> p;
            p.load(xr + c);
            float w[VEC], b[VEC], f[VEC];
            load_floats<VEC>(gamma, c, 1.f, w);
            load_floats<VEC>(beta, c, 0.f, b);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = (p.get(e) - mean) * rstd * w[e] + b[e];
            p.set_all(f);
            p.store(yr + c);
        }
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[n] = mean;
            if (rstd_out) rstd_out[n] = rstd;
        }
    }
}

// The two means of a row's gradient: sums[2n] = sum g / C, sums[2n + 1] =
// sum (g * xh) / C.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads)
    ln_bwd_rows_kernel(const T* x, const T* dy, const int32_t* count, long long capacity, int C,
                       const float* __restrict__ gamma, const float* __restrict__ mean,
                       const float* __restrict__ rstd, float* __restrict__ sums,
                       unsigned* status) {
    __shared__ float sh[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    for (long long n = blockIdx.x; n < rows; n += gridDim.x) {
        const float m = mean[n], r = rstd[n];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll 2
        for (int c = threadIdx.x * VEC; c < C; c += kThreads * VEC) {
            Piece<T, VEC> p, d;
            float w[VEC];
            p.load(x + n * C + c);
            d.load(dy + n * C + c);
            load_floats<VEC>(gamma, c, 1.f, w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float g = d.get(e) * w[e];
                s1 += g;
                s2 += g * ((p.get(e) - m) * r);
            }
        }
        s1 = block_sum(s1, sh);
        s2 = block_sum(s2, sh);
        if (threadIdx.x == 0) {
            sums[2 * n] = s1 / (float)C;
            sums[2 * n + 1] = s2 / (float)C;
        }
    }
}

// A thread per piece of VEC channels walks the rows blockIdx.y, + gridDim.y,
// ...: dx, and its own sums of dy * xh and dy into part[blockIdx.y][2][C].
// kColRows rows are loaded before the first is worked on: dx may be x or dy,
// so no load would be moved up over a store.
constexpr int kColRows = 4;

template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads)
    ln_bwd_cols_kernel(const T* x, const T* dy, const int32_t* count, long long capacity, int C,
                       const float* __restrict__ gamma, const float* __restrict__ mean,
                       const float* __restrict__ rstd, const float* __restrict__ sums, T* dx,
                       float* __restrict__ part, unsigned* status) {
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    const int c = (int)(blockIdx.x * kThreads + threadIdx.x) * VEC;
    if (c >= C) return;
    float w[VEC], dg[VEC], db[VEC];
    load_floats<VEC>(gamma, c, 1.f, w);
#pragma unroll
    for (int e = 0; e < VEC; ++e) dg[e] = db[e] = 0.f;
    for (long long n0 = blockIdx.y; n0 < rows; n0 += (long long)kColRows * gridDim.y) {
        Piece<T, VEC> p[kColRows], d[kColRows];
        float m[kColRows], r[kColRows], s1[kColRows], s2[kColRows];
#pragma unroll
        for (int u = 0; u < kColRows; ++u) {
            // a row past the end is loaded as the first and not used
            const long long at = n0 + (long long)u * gridDim.y, n = at < rows ? at : n0;
            p[u].load(x + n * C + c);
            d[u].load(dy + n * C + c);
            m[u] = mean[n];
            r[u] = rstd[n];
            s1[u] = dx ? sums[2 * n] : 0.f;
            s2[u] = dx ? sums[2 * n + 1] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kColRows; ++u) {
            const long long n = n0 + (long long)u * gridDim.y;
            if (n >= rows) break;
            float f[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float g = d[u].get(e), xh = (p[u].get(e) - m[u]) * r[u];
                f[e] = (g * w[e] - s1[u] - xh * s2[u]) * r[u];
                dg[e] += g * xh;
                db[e] += g;
            }
            if (dx) {
                p[u].set_all(f);
                p[u].store(dx + n * C + c);
            }
        }
    }
    if (part) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            part[(2ll * blockIdx.y) * C + c + e] = dg[e];
            part[(2ll * blockIdx.y + 1) * C + c + e] = db[e];
        }
    }
}

// dgamma and dbeta from the blocks' sums part[parts][2][C]: 32 values per
// block, 32 warps adding every 32nd part in order, then the warps in order.
constexpr int kGradWarps = 32;

__global__ void __launch_bounds__(kGradWarps * 32)
    ln_param_grad_kernel(const float* __restrict__ part, int parts, int C, float* dgamma,
                         float* dbeta) {
    __shared__ float sh[kGradWarps][33];
    pdl_wait();
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long c = blockIdx.x * 32ll + lane;  // of the 2 * C sums of a part
    float v = 0.f;
    if (c < 2ll * C) {
#pragma unroll 8
        for (int p = warp; p < parts; p += kGradWarps) v += part[2ll * p * C + c];
    }
    sh[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && c < 2ll * C) {
        v = 0.f;
#pragma unroll
        for (int w = 0; w < kGradWarps; ++w) v += sh[w][lane];
        float* const out = c < C ? dgamma : dbeta;
        if (out) out[c < C ? c : c - C] = v;
    }
}

hc_status param_grad(const LayerNormArgs& a, const float* part, int parts, cudaStream_t s) {
    const unsigned grid = (unsigned)((2ll * a.C + 31) / 32);
    return launch_pdl(ln_param_grad_kernel, dim3(grid), dim3(kGradWarps * 32), 0, s,
                      "ln_param_grad_kernel", part, parts, a.C, a.dgamma, a.dbeta);
}

template <typename T, int VEC, int TPR, int NV>
hc_status fwd_rows(const DeviceCtx* ctx, const LayerNormArgs& a, cudaStream_t s) {
    constexpr int kGroups = kGroupThreads / TPR;
    const long long need = ((long long)a.capacity + kGroups - 1) / kGroups;
    const long long cap = (long long)ctx->num_sms;
    return launch_pdl(ln_fwd_rows_kernel<T, VEC, TPR, NV>,
                      dim3((unsigned)(need < cap ? need : cap)), dim3(kGroupThreads), 0, s,
                      "ln_fwd_rows_kernel", (const T*)a.x, a.count, (long long)a.capacity, a.C,
                      a.eps, a.gamma, a.beta, (T*)a.y, a.mean_out, a.rstd_out, ctx->status);
}

template <typename T, int VEC, int TPR, int NV>
hc_status bwd_rows(const DeviceCtx* ctx, const LayerNormArgs& a, cudaStream_t s) {
    constexpr int kGroups = kGroupThreads / TPR;
    const long long need = ((long long)a.capacity + kGroups - 1) / kGroups;
    const long long cap = (long long)ctx->num_sms;
    const int grid = (int)(need < 1 ? 1 : need < cap ? need : cap);
    const bool params = a.dgamma || a.dbeta;
    float* part = nullptr;
    if (params) {
        part = (float*)stream_workspace(s, (size_t)grid * a.C * 8);
        if (!part) return HC_ERR_CUDA;
    }
    // the groups' sums: at most 64 KiB, two 4-byte sums for each of the
    // kGroups * C <= 512 * 16 channels held
    const size_t smem = kGroups > 1 && params ? (size_t)kGroups * a.C * 8 : 0;
    auto kern = ln_bwd_rows_in_regs_kernel<T, VEC, TPR, NV>;
    static bool done[64];
    if (smem > 48 * 1024 && !done[ctx->device]) {
        const hc_status st = check_cuda(
            cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kGroupThreads * NV * VEC * 8),
            "ln_bwd_rows_in_regs_kernel");
        if (st != HC_OK) return st;
        done[ctx->device] = true;
    }
    hc_status st = launch_pdl(kern, dim3((unsigned)grid), dim3(kGroupThreads), smem, s,
                              "ln_bwd_rows_in_regs_kernel", (const T*)a.x, (const T*)a.dy, a.count, (long long)a.capacity, a.C,
                              a.gamma, a.mean, a.rstd, (T*)a.dx, part, ctx->status);
    if (st != HC_OK || !params) return st;
    return param_grad(a, part, grid, s);
}

template <typename T, int VEC>
hc_status fwd_wide(const DeviceCtx* ctx, const LayerNormArgs& a, cudaStream_t s) {
    const long long cap = (long long)ctx->num_sms * 8;
    const unsigned grid = (unsigned)(a.capacity < cap ? a.capacity : cap);
    return launch_pdl(ln_fwd_kernel<T, VEC>, dim3(grid), dim3(kThreads), 0, s, "ln_fwd_kernel",
                      (const T*)a.x, a.count, (long long)a.capacity, a.C, a.eps, a.gamma, a.beta,
                      (T*)a.y, a.mean_out, a.rstd_out, ctx->status);
}

template <typename T, int VEC>
hc_status bwd_wide(const DeviceCtx* ctx, const LayerNormArgs& a, cudaStream_t s) {
    const bool params = a.dgamma || a.dbeta;
    const unsigned ctiles = (unsigned)((a.C + kThreads * VEC - 1) / (kThreads * VEC));
    long long parts = (ctx->num_sms * 8 + ctiles - 1) / ctiles;
    if (parts > a.capacity) parts = a.capacity;
    if (parts < 1) parts = 1;
    const size_t sums_b = (size_t)a.capacity * 8, part_b = params ? (size_t)parts * a.C * 8 : 0;
    float* ws = (float*)stream_workspace(s, sums_b + part_b);
    if (!ws) return HC_ERR_CUDA;
    float* part = params ? ws + 2 * (size_t)a.capacity : nullptr;
    const long long cap = (long long)ctx->num_sms * 8;
    hc_status st;
    if (a.capacity > 0 && a.dx) {
        st = launch_pdl(ln_bwd_rows_kernel<T, VEC>, dim3((unsigned)(a.capacity < cap ? a.capacity : cap)),
                        dim3(kThreads), 0, s, "ln_bwd_rows_kernel", (const T*)a.x, (const T*)a.dy,
                        a.count, (long long)a.capacity, a.C, a.gamma, a.mean, a.rstd, ws,
                        ctx->status);
        if (st != HC_OK) return st;
    }
    st = launch_pdl(ln_bwd_cols_kernel<T, VEC>, dim3(ctiles, (unsigned)parts), dim3(kThreads), 0, s,
                    "ln_bwd_cols_kernel", (const T*)a.x, (const T*)a.dy, a.count,
                    (long long)a.capacity, a.C, a.gamma, a.mean, a.rstd, (const float*)ws,
                    (T*)a.dx, part, ctx->status);
    if (st != HC_OK || !params) return st;
    return param_grad(a, part, (int)parts, s);
}

template <typename T, int VEC, int TPR, int NV>
hc_status rows_in_regs(const DeviceCtx* ctx, const LayerNormArgs& a, bool back, cudaStream_t s) {
    return back ? bwd_rows<T, VEC, TPR, NV>(ctx, a, s) : fwd_rows<T, VEC, TPR, NV>(ctx, a, s);
}

// Rows of at most 8192 channels are held in registers (16384 x 8192 bf16:
// forward 104 us, gradient 170; through the caches 145 and 244), by the
// smallest group that does so with two 16-byte pieces a thread (four for the
// widest fp32 rows): the gradient keeps two rows' pieces, gamma and both sums
// of every channel. Twice the threads for a row cost more than they hide
// (65536 x 2048 bf16: 135 and 183 us against 91 and 136; 65536 x 64: 14 and 18
// against 5 and 9), four pieces a thread slow the gradient (65536 x 256 bf16:
// 48 us against 22). Rows that allow no 16-byte loads are read element by
// element (32768 x 2047 bf16 75 and 143 us, half of 91 and 136 at 2048
// channels); there the forward holds 16 elements a thread from 257 channels on
// (8: 127 us), the gradient at most 8 (16: 252) up to 4096.
template <typename T>
hc_status run(const DeviceCtx* ctx, const LayerNormArgs& a, bool back, cudaStream_t s) {
    constexpr int kVec = 16 / (int)sizeof(T);
    const int C = a.C;
    auto aligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const bool wide = C % kVec == 0 && aligned(a.x) && aligned(a.y) && aligned(a.dy) &&
                      aligned(a.dx) && aligned(a.gamma) && aligned(a.beta);
    if (C > 8192) {
        if (wide) return back ? bwd_wide<T, kVec>(ctx, a, s) : fwd_wide<T, kVec>(ctx, a, s);
        return back ? bwd_wide<T, 1>(ctx, a, s) : fwd_wide<T, 1>(ctx, a, s);
    }
    if (wide) {
        if (C <= 8 * kVec) return rows_in_regs<T, kVec, 8, 1>(ctx, a, back, s);
        if (C <= 32 * kVec) return rows_in_regs<T, kVec, 32, 1>(ctx, a, back, s);
        if (C <= 64 * kVec) return rows_in_regs<T, kVec, 32, 2>(ctx, a, back, s);
        if (C <= 128 * kVec) return rows_in_regs<T, kVec, 128, 1>(ctx, a, back, s);
        if (C <= 256 * kVec) return rows_in_regs<T, kVec, 128, 2>(ctx, a, back, s);
        if (C <= 512 * kVec) return rows_in_regs<T, kVec, 256, 2>(ctx, a, back, s);
        if (C <= 1024 * kVec) return rows_in_regs<T, kVec, 512, 2>(ctx, a, back, s);
        if constexpr (kVec == 4) return rows_in_regs<T, kVec, 512, 4>(ctx, a, back, s);
    }
    if (C <= 32) return rows_in_regs<T, 1, 8, 4>(ctx, a, back, s);
    if (C <= 64) return rows_in_regs<T, 1, 8, 8>(ctx, a, back, s);
    if (C <= 128) return rows_in_regs<T, 1, 32, 4>(ctx, a, back, s);
    if (C <= 256) return rows_in_regs<T, 1, 32, 8>(ctx, a, back, s);
    if (C > 512 && C <= 1024) return rows_in_regs<T, 1, 128, 8>(ctx, a, back, s);
    if (back) {
        if (C <= 512) return bwd_rows<T, 1, 128, 4>(ctx, a, s);
        if (C <= 2048) return bwd_rows<T, 1, 256, 8>(ctx, a, s);
        if (C <= 4096) return bwd_rows<T, 1, 512, 8>(ctx, a, s);
    } else {
        if (C <= 512) return fwd_rows<T, 1, 32, 16>(ctx, a, s);
        if (C <= 2048) return fwd_rows<T, 1, 128, 16>(ctx, a, s);
        if (C <= 4096) return fwd_rows<T, 1, 256, 16>(ctx, a, s);
    }
    return rows_in_regs<T, 1, 512, 16>(ctx, a, back, s);
}

}  // namespace

hc_status launch_layer_norm_fwd(const DeviceCtx* ctx, const LayerNormArgs& a, cudaStream_t s) {
    return a.dt == HC_BF16 ? run<__nv_bfloat16>(ctx, a, false, s) : run<float>(ctx, a, false, s);
}

hc_status launch_layer_norm_bwd(const DeviceCtx* ctx, const LayerNormArgs& a, cudaStream_t s) {
    return a.dt == HC_BF16 ? run<__nv_bfloat16>(ctx, a, true, s) : run<float>(ctx, a, true, s);
}

}  // namespace hc
