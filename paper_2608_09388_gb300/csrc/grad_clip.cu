// The norm over all gradients of a network, and the gradients scaled so that
// it is at most max_norm:
//   norm = sqrt(sum over all tensors of g^2),  out = g * min(1, max_norm / norm)
// The tensors are cut into units of 4096 elements, numbered tensor after
// tensor; a block takes a range of units, whatever tensors they lie in.
//
// Squares are summed 32 at a time in fp32, those sums in a pair of fp32
// numbers that keeps what each addition rounds off, the threads' and blocks'
// sums in 64 bits: the norm of 10^9 values is off by a few units of fp32. The
// order is fixed by the sizes alone, so the result is the same from run to run.
//
// Bound by memory: the norm reads every value, the scaling reads it again (what
// the caches still hold of it: the units are walked in the other direction) and
// writes it.
#include <algorithm>
#include <exception>
#include <vector>

#include "tokens.cuh"

namespace hc {
namespace {

constexpr int kThreads = 512;
constexpr int kPer = 8;                      // elements of a unit per thread
constexpr int kUnit = kThreads * kPer;
constexpr int kAhead = 4;                    // units loaded before the first is worked on

// One tensor. Units count from the 16-byte boundary at or below `in`, `off`
// elements before its first; `first` numbers its first unit.
struct Entry {
    const void* in;
    void* out;
    long long numel;
    long long first;
    int off;
    int dt;
};

// A thread's elements of a unit: 16 bytes of bf16, or two times 16 bytes of fp32.
struct Elems {
    uint4 a[2];
};

template <typename T>
__device__ __forceinline__ uint4 load_piece(const T* p, long long at, long long numel) {
    constexpr int V = 16 / (int)sizeof(T);
    if (at >= 0 && at + V <= numel) return *reinterpret_cast<const uint4*>(p + at);
    alignas(16) T v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = at + i >= 0 && at + i < numel ? p[at + i] : from_f32<T>(0.f);
    return *reinterpret_cast<const uint4*>(v);
}
template <typename T>
__device__ __forceinline__ void store_piece(T* p, long long at, long long numel, uint4 v, bool wide) {
    constexpr int V = 16 / (int)sizeof(T);
    if (wide && at >= 0 && at + V <= numel) {
        *reinterpret_cast<uint4*>(p + at) = v;
        return;
    }
    alignas(16) T f[V];
    *reinterpret_cast<uint4*>(f) = v;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (at + i >= 0 && at + i < numel) p[at + i] = f[i];
}

// First element (of the tensor) of this thread's piece j of unit u.
__device__ __forceinline__ long long piece_at(const Entry& e, long long u, int j) {
    const long long base = (u - e.first) * kUnit - e.off;
    return e.dt == HC_BF16 ? base + threadIdx.x * 8 : base + j * (kUnit / 2) + threadIdx.x * 4;
}
__device__ __forceinline__ Elems load_unit(const Entry& e, long long u) {
    Elems r;
    if (e.dt == HC_BF16) {
        r.a[0] = load_piece(static_cast<const __nv_bfloat16*>(e.in), piece_at(e, u, 0), e.numel);
    } else {
        const float* p = static_cast<const float*>(e.in);
        r.a[0] = load_piece(p, piece_at(e, u, 0), e.numel);
        r.a[1] = load_piece(p, piece_at(e, u, 1), e.numel);
    }
    return r;
}
__device__ __forceinline__ void as_floats(const Elems& r, bool bf16, float (&f)[kPer]) {
    const uint32_t w[4] = {r.a[0].x, r.a[0].y, r.a[0].z, r.a[0].w};
    if (bf16) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    } else {
        const uint32_t z[4] = {r.a[1].x, r.a[1].y, r.a[1].z, r.a[1].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = __uint_as_float(w[i]);
            f[4 + i] = __uint_as_float(z[i]);
        }
    }
}

// The entry of unit u: the last one whose first unit is not above u.
__device__ __forceinline__ int find_entry(const Entry* table, int n, long long u) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (table[mid].first <= u)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_sum_f64(double v, double* sh) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) sh[warp] = v;
    __syncthreads();
    v = lane < warps ? sh[lane] : 0.0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Whether units u .. u + n - 1 lie wholly inside their tensor.
__device__ __forceinline__ bool inside(const Entry& e, long long u, int n) {
    const long long at = (u - e.first) * kUnit - e.off;
    return at >= 0 && at + (long long)n * kUnit <= e.numel;
}

// The block's units [first, last): part[blockIdx.x] = the sum of their squares.
__global__ void __launch_bounds__(kThreads, 2)
    sum_squares_kernel(const Entry* __restrict__ table, int n, long long units,
                       double* __restrict__ part) {
    __shared__ double sh[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    const long long u0 = units * blockIdx.x / gridDim.x, u1 = units * (blockIdx.x + 1) / gridDim.x;
    float hi = 0.f, lo = 0.f;
    double far = 0.0;  // squares that fp32 does not hold
    if (u0 >= u1) {
        if (threadIdx.x == 0) part[blockIdx.x] = 0.0;
        return;
    }
    int t = find_entry(table, n, u0);
    Entry e = table[t];
    long long end = table[t + 1].first;
    for (long long u = u0; u < u1; u += kAhead) {
        Elems r[kAhead];
        bool bf16[kAhead];
        while (end <= u) {
            e = table[++t];
            end = table[t + 1].first;
        }
        if (u + kAhead <= u1 && inside(e, u, kAhead)) {
            // the rule: no look at the ends, all loads at once
            if (e.dt == HC_BF16) {
                const uint4* const at = reinterpret_cast<const uint4*>(
                    static_cast<const __nv_bfloat16*>(e.in) + piece_at(e, u, 0));
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    bf16[k] = true;
                    r[k].a[0] = at[k * kThreads];
                }
            } else {
                const uint4* const at = reinterpret_cast<const uint4*>(
                    static_cast<const float*>(e.in) + piece_at(e, u, 0));
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    bf16[k] = false;
                    r[k].a[0] = at[2 * k * kThreads];
                    r[k].a[1] = at[(2 * k + 1) * kThreads];
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                bf16[k] = true;
                r[k].a[0] = make_uint4(0u, 0u, 0u, 0u);
                if (u + k < u1) {
                    while (end <= u + k) {
                        e = table[++t];
                        end = table[t + 1].first;
                    }
                    bf16[k] = e.dt == HC_BF16;
                    r[k] = load_unit(e, u + k);
                }
            }
        }
        F2 s = make_f2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float f[kPer];
            as_floats(r[k], bf16[k], f);
#pragma unroll
            for (int i = 0; i < kPer; i += 2) {
                const F2 v = make_f2(f[i], f[i + 1]);
                s = fma(v, v, s);
            }
        }
        const float p = total(s);
        if (p < __int_as_float(0x7f800000)) {
            // hi + p, and what the addition rounds off
            const float sum = hi + p, b = sum - hi;
            lo += (hi - (sum - b)) + (p - b);
            hi = sum;
        } else {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                float f[kPer];
                as_floats(r[k], bf16[k], f);
#pragma unroll 1
                for (int i = 0; i < kPer; ++i) far += (double)f[i] * (double)f[i];
            }
        }
    }
    const double v = block_sum_f64((double)hi + (double)lo + far, sh);
    if (threadIdx.x == 0) part[blockIdx.x] = v;
}

__global__ void __launch_bounds__(kThreads)
    norm_kernel(const double* __restrict__ part, int parts, float* norm) {
    __shared__ double sh[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    double v = 0.0;
    for (int p = threadIdx.x; p < parts; p += kThreads) v += part[p];
    v = block_sum_f64(v, sh);
    if (threadIdx.x == 0) *norm = (float)sqrt(v);
}

// kAhead units wholly inside a tensor, input and output aligned alike.
template <typename T>
__device__ __forceinline__ void scale_units(const Entry& e, long long u, float scale) {
    constexpr int V = 16 / (int)sizeof(T), kPieces = kPer / V;
    const long long at = piece_at(e, u, 0);
    const T* const in = static_cast<const T*>(e.in) + at;
    T* const out = static_cast<T*>(e.out) + at;
    Piece<T, V> p[kAhead * kPieces];
#pragma unroll
    for (int k = 0; k < kAhead * kPieces; ++k) p[k].load(in + k * kThreads * V);
#pragma unroll
    for (int k = 0; k < kAhead * kPieces; ++k) {
        float f[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = p[k].get(i) * scale;
        p[k].set_all(f);
        p[k].store(out + k * kThreads * V);
    }
}

// The same units as sum_squares_kernel's block, from the last one down.
__global__ void __launch_bounds__(kThreads, 2)
    scale_kernel(const Entry* __restrict__ table, int n, long long units, const float* norm,
                 float max_norm) {
    pdl_wait();
    pdl_trigger();
    const float size = *norm;
    const float scale = size <= max_norm ? 1.f : max_norm / size;  // a NaN passes
    const long long u0 = units * blockIdx.x / gridDim.x, u1 = units * (blockIdx.x + 1) / gridDim.x;
    if (u0 >= u1) return;
    int t = find_entry(table, n, u1 - 1);
    Entry e = table[t];
    auto wide = [](const Entry& e) {
        return ((reinterpret_cast<uintptr_t>(e.in) ^ reinterpret_cast<uintptr_t>(e.out)) & 15) == 0;
    };
    for (long long u = u1 - 1; u >= u0; u -= kAhead) {  // u and the ones below
        while (e.first > u) e = table[--t];
        const long long lo = u - (kAhead - 1);
        if (lo >= u0 && lo >= e.first && inside(e, lo, kAhead) && wide(e)) {
            if (scale == 1.f && e.in == e.out) continue;
            if (e.dt == HC_BF16)
                scale_units<__nv_bfloat16>(e, lo, scale);
            else
                scale_units<float>(e, lo, scale);
            continue;
        }
        Elems r[kAhead];
        int at[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            at[k] = -1;
            if (u - k >= u0) {
                while (e.first > u - k) e = table[--t];
                if (scale != 1.f || e.in != e.out) {
                    at[k] = t;
                    r[k] = load_unit(e, u - k);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (at[k] < 0) continue;
            const Entry o = table[at[k]];
            const bool bf16 = o.dt == HC_BF16;
            float f[kPer];
            as_floats(r[k], bf16, f);
#pragma unroll
            for (int i = 0; i < kPer; ++i) f[i] *= scale;
            if (bf16) {
                Piece<__nv_bfloat16, 8> p;
                p.set_all(f);
                store_piece(static_cast<__nv_bfloat16*>(o.out), piece_at(o, u - k, 0), o.numel, p.v,
                            wide(o));
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    store_piece(static_cast<float*>(o.out), piece_at(o, u - k, j), o.numel,
                                make_uint4(__float_as_uint(f[4 * j]), __float_as_uint(f[4 * j + 1]),
                                           __float_as_uint(f[4 * j + 2]),
                                           __float_as_uint(f[4 * j + 3])),
                                wide(o));
            }
        }
    }
}

unsigned grid_of(const DeviceCtx* ctx, long long units) {
    const long long cap = 2ll * ctx->num_sms;
    return (unsigned)(units < 1 ? 1 : units < cap ? units : cap);
}

}  // namespace

size_t tensor_list_bytes(int n) {
    return ((size_t)n + 1) * sizeof(Entry);
}

// Entries of n tensors and a last one that holds the number of units. false:
// outputs overlap each other or another tensor's input (`*bad` is one of them).
bool fill_tensor_list(const void* const* in, void* const* out, const long long* numel,
                      const int* dt, int n, void* table, long long* units, int* bad) {
    struct Range {
        uintptr_t from, to;
        int i;
    };
    std::vector<Range> outs;
    Entry* const e = static_cast<Entry*>(table);
    long long first = 0;
    for (int i = 0; i < n; ++i) {
        const int size = dt[i] == HC_BF16 ? 2 : 4;
        const int off = (int)((reinterpret_cast<uintptr_t>(in[i]) & 15) / size);
        void* const o = out ? out[i] : const_cast<void*>(in[i]);
        e[i] = Entry{in[i], o, numel[i], first, off, dt[i]};
        if (numel[i] == 0) continue;
        first += (numel[i] + off + kUnit - 1) / kUnit;
        const uintptr_t at = reinterpret_cast<uintptr_t>(o);
        outs.push_back({at, at + (uintptr_t)numel[i] * size, i});
    }
    e[n] = Entry{nullptr, nullptr, 0, first, 0, 0};
    *units = first;
    std::sort(outs.begin(), outs.end(),
              [](const Range& a, const Range& b) { return a.from < b.from; });
    for (size_t k = 1; k < outs.size(); ++k)
        if (outs[k].from < outs[k - 1].to) {
            *bad = outs[k].i;
            return false;
        }
    for (int i = 0; i < n; ++i) {
        if (numel[i] == 0) continue;
        const uintptr_t from = reinterpret_cast<uintptr_t>(in[i]);
        const uintptr_t to = from + (uintptr_t)numel[i] * (dt[i] == HC_BF16 ? 2 : 4);
        // outputs that end behind the input's start, up to those that start behind its end
        auto k = std::upper_bound(outs.begin(), outs.end(), from,
                                  [](uintptr_t v, const Range& r) { return v < r.to; });
        for (; k != outs.end() && k->from < to; ++k)
            if (k->i != i || k->from != from) {
                *bad = i;
                return false;
            }
    }
    return true;
}

hc_status launch_grad_norm(const DeviceCtx* ctx, const void* table, int n, long long units,
                           float* norm, cudaStream_t s) {
    const unsigned grid = grid_of(ctx, units);
    double* const part = (double*)stream_workspace(s, grid * sizeof(double));
    if (!part) return HC_ERR_CUDA;
    const hc_status st =
        launch_pdl(sum_squares_kernel, dim3(grid), dim3(kThreads), 0, s, "sum_squares_kernel",
                   static_cast<const Entry*>(table), n, units, part);
    if (st != HC_OK) return st;
    return launch_pdl(norm_kernel, dim3(1), dim3(kThreads), 0, s, "norm_kernel",
                      (const double*)part, (int)grid, norm);
}

hc_status launch_grad_clip(const DeviceCtx* ctx, const void* table, int n, long long units,
                           const float* norm, float max_norm, cudaStream_t s) {
    return launch_pdl(scale_kernel, dim3(grid_of(ctx, units)), dim3(kThreads), 0, s,
                      "scale_kernel", static_cast<const Entry*>(table), n, units, norm, max_norm);
}

}  // namespace hc
