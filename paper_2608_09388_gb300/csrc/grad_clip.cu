// The norm over all gradients of a network, and the gradients scaled so that
// it is at most max_norm:
//   norm = sqrt(sum over all tensors of g^2),  out = g * min(1, max_norm / norm)
// The tensors are cut into units of 16 KiB, numbered tensor after tensor; a
// block takes a range of units, whatever tensors they lie in.
//
// A thread's squares of a unit (8 fp32, 16 bf16) are summed in fp32, those sums in a
// pair of fp32 numbers that keeps what each addition rounds off, the threads'
// and blocks' sums in 64 bits: the norm of 10^9 values is off by a few units of
// fp32. The order is fixed by the sizes alone, so the result is the same from
// run to run.
//
// Bound by memory: the norm reads every value, the scaling reads it again (what
// the caches still hold of it: the units are walked in the other direction) and
// writes it. One compact loop for both types: what a short call waits for is
// the table, the first loads and the code itself, which come from memory too
// (71 MB in 60 tensors: unrolled paths for whole and for ragged units took 20
// us more).
#include <algorithm>
#include <exception>
#include <vector>

#include "tokens.cuh"

namespace hc {
namespace {

constexpr int kThreads = 512;
constexpr int kResident = 3;                 // blocks an SM
constexpr int kPieces = 2;                   // 16-byte pieces of a unit per thread
constexpr int kUnit = kThreads * kPieces * 16;
// Blocks of the grid: as many as run at a time, or several times that (up to
// kBlocks an SM) where each still gets kShare units: ranges that are taken as SMs
// get free even out what they wait.
constexpr int kBlocks = 32, kShare = 8;

// One tensor. Units count from the 16-byte boundary at or below `in`; `first`
// numbers its first unit.
struct Entry {
    const char* in;
    char* out;
    long long bytes;
    long long first;
    int bf16;
    int pad;
};

// The last entry whose first unit is not above u, the same in every thread: all
// entries looked at together, or by halves where they are many.
__device__ __forceinline__ int find_entry(const Entry* table, int n, long long u) {
    if (n <= kThreads)
        return __syncthreads_count((int)threadIdx.x < n && table[threadIdx.x].first <= u) - 1;
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (int)(((long long)lo + hi + 1) >> 1);
        if (table[mid].first <= u)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// A thread's 16 bytes at `at`, zero where they lie outside [from, to).
__device__ __forceinline__ uint4 load_piece(const char* at, const char* from, const char* to) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (at >= from && at + 16 <= to) {
        v = *reinterpret_cast<const uint4*>(at);
    } else if (at < to && at + 16 > from) {
        // both types as halves of words: an element is inside or outside as a whole
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const char* const p = at + 2 * i;
            if (p >= from && p < to)
                w[i >> 1] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16 * (i & 1);
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}
__device__ __forceinline__ void store_piece(char* at, const char* from, const char* to, uint4 v,
                                            bool wide) {
    if (wide && at >= from && at + 16 <= to) {
        *reinterpret_cast<uint4*>(at) = v;
    } else if (at < to && at + 16 > from) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            char* const p = at + 2 * i;
            if (p >= from && p < to)
                *reinterpret_cast<uint16_t*>(p) = (uint16_t)(w[i >> 1] >> 16 * (i & 1));
        }
    }
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

// The two values of a word.
__device__ __forceinline__ float2 halves(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// part[b] = the sum of the squares in the units [units * b / blocks, ..).
__global__ void __launch_bounds__(kThreads, kResident)
    sum_squares_kernel(const Entry* __restrict__ table, int n, long long units,
                       double* __restrict__ part) {
    __shared__ double sh[kThreads / 32];
    pdl_trigger();
    const long long u1 = units * (blockIdx.x + 1) / gridDim.x;
    long long u = units * blockIdx.x / gridDim.x;
    float hi = 0.f, lo = 0.f;
    double far = 0.0;  // squares and sums that fp32 does not hold
    // the table has been there since before the first call: its look-up runs
    // while the kernel before ends
    int t = u < u1 ? find_entry(table, n, u) : 0;
    pdl_wait();
    if (u < u1) {
        while (u < u1) {
            const char *const from = table[t].in, *const to = from + table[t].bytes;
            const bool bf16 = table[t].bf16;
            const long long next = table[t + 1].first, end = next < u1 ? next : u1;
            const char* at = from - (reinterpret_cast<uintptr_t>(from) & 15) +
                             (u - table[t].first) * kUnit + threadIdx.x * 16;
#pragma unroll 1
            for (; u < end; ++u, at += kUnit) {
                uint4 v[kPieces];
#pragma unroll
                for (int j = 0; j < kPieces; ++j) v[j] = load_piece(at + j * (kThreads * 16), from, to);
                float s0 = 0.f, s1 = 0.f;
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 f = bf16 ? halves(w[i]) : make_float2(__uint_as_float(w[i]), 0.f);
                        s0 = fmaf(f.x, f.x, s0);
                        s1 = fmaf(f.y, f.y, s1);
                    }
                }
                const float s = s0 + s1, sum = hi + s;
                if (sum < __int_as_float(0x7f800000)) {
                    // hi + s, and what the addition rounds off
                    const float b = sum - hi;
                    lo += (hi - (sum - b)) + (s - b);
                    hi = sum;
                } else if (s < __int_as_float(0x7f800000)) {
                    // the sums so far go to 64 bits, and begin again here
                    far += (double)hi + lo;
                    hi = s;
                    lo = 0.f;
                } else {
#pragma unroll 1
                    for (int i = 0; i < 4 * kPieces; ++i) {
                        uint4 q = v[0];
#pragma unroll
                        for (int j = 1; j < kPieces; ++j) q = i >> 2 == j ? v[j] : q;
                        const uint32_t w = (i & 2) ? ((i & 1) ? q.w : q.z) : ((i & 1) ? q.y : q.x);
                        const float2 f = bf16 ? halves(w) : make_float2(__uint_as_float(w), 0.f);
                        far += (double)f.x * f.x + (double)f.y * f.y;
                    }
                }
            }
            ++t;
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

// The units of sum_squares_kernel's blocks, from the last one down: what the
// norm has read last is in the caches.
__global__ void __launch_bounds__(kThreads, kResident)
    scale_kernel(const Entry* __restrict__ table, int n, long long units, const float* norm,
                 float max_norm) {
    pdl_trigger();
    const long long b = gridDim.x - 1 - blockIdx.x;
    const long long u0 = units * b / gridDim.x;
    long long u = units * (b + 1) / gridDim.x;  // the units below it are left
    int t = u > u0 ? find_entry(table, n, u - 1) : 0;  // see sum_squares_kernel
    pdl_wait();
    if (u <= u0) return;
    const float size = *norm;
    const float scale = size <= max_norm ? 1.f : max_norm / size;  // a NaN passes
    for (; u > u0; --t) {
        const char *const from = table[t].in, *const to = from + table[t].bytes;
        const bool bf16 = table[t].bf16;
        const long long first = table[t].first, end = first > u0 ? first : u0;
        const ptrdiff_t off = table[t].out - from;
        const bool wide = (off & 15) == 0;
        if (scale == 1.f && off == 0) u = end < u ? end : u;
        const char* at = from - (reinterpret_cast<uintptr_t>(from) & 15) + (u - 1 - first) * kUnit +
                         threadIdx.x * 16;
#pragma unroll 1
        for (; u > end; --u, at -= kUnit) {
            uint4 v[kPieces];
#pragma unroll
            for (int j = 0; j < kPieces; ++j) v[j] = load_piece(at + j * (kThreads * 16), from, to);
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = halves(w[i]);
                    w[i] = bf16 ? Piece<__nv_bfloat16, 8>::pair(f.x * scale, f.y * scale)
                                : __float_as_uint(__uint_as_float(w[i]) * scale);
                }
                store_piece(const_cast<char*>(at) + j * (kThreads * 16) + off, from + off, to + off,
                            make_uint4(w[0], w[1], w[2], w[3]), wide);
            }
        }
    }
}

unsigned grid_of(const DeviceCtx* ctx, long long units) {
    const long long once = (long long)kResident * ctx->num_sms, cap = (long long)kBlocks * ctx->num_sms;
    long long grid = units / kShare;
    if (grid < 4 * once) grid = once;  // a short second round would cost as much as the first
    if (grid > cap) grid = cap;
    if (grid > units) grid = units;
    return (unsigned)(grid < 1 ? 1 : grid);
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
        const long long off = (long long)(reinterpret_cast<uintptr_t>(in[i]) & 15);
        const long long bytes = numel[i] * size;
        void* const o = out ? out[i] : const_cast<void*>(in[i]);
        e[i] = Entry{(const char*)in[i], (char*)o, bytes, first, dt[i] == HC_BF16, 0};
        if (bytes == 0) continue;
        first += (bytes + off + kUnit - 1) / kUnit;
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
