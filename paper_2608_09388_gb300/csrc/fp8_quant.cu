// Rows and weights held in 8 bits: e4m3 values with one fp32 scale per block
// of 128 channels (rows) or per 128 x 128 block (weights).
//   scale = max(amax / 448, 2^-126),  q = e4m3(x / scale)
// with amax the block's largest magnitude, both quotients rounded to nearest
// even once, so that the largest magnitude of a block is held as 448. A block
// with a NaN has the scale NaN and NaN values; one with an infinity has the
// scale infinity, its infinities held as NaN: products of such a row are NaN.
//
// Bound by memory once the quotients are not divided one by one: 16384 x 8192
// bf16 takes 65 to 67 us (60 at the copy rate; 231 us with a division per value, 153
// with four scales a warp found one after another, 81 with two products that
// enclose the quotient in place of its correction), 16384 x 4932, whose rows
// allow 4-byte loads only, 67 to 72 us (36).
#include "fp8.cuh"

namespace hc {
namespace {

constexpr int kThreads = 256;

// Blocks of 128 channels are numbered row by row. 128 / V lanes hold a block,
// V channels (16 bytes) each; a warp takes 32 V / 128 blocks a step and four
// steps at a time, so that four loads are in flight and the four steps' scales
// are found together: the reduction over a block's lanes halves the steps a
// lane carries at its first two exchanges, after which lane l holds step l % 4
// and divides for it alone.
constexpr int kSteps = 4;
enum RowLoads {
    kScalar,  // elements one by one
    kWords,   // bf16 rows allow 4-byte loads
    kWide,    // rows allow 16-byte loads
    kFlat     // and hold whole blocks: block g lies at x + 128 g, whatever its row
};

template <typename T, RowLoads kLoads>
__global__ void __launch_bounds__(kThreads)
    quant_rows_kernel(const T* __restrict__ x, const int32_t* count, long long capacity, int C,
                      int pitch, int nb, uint8_t* __restrict__ q, float* __restrict__ scales,
                      unsigned* status) {
    constexpr int V = 16 / (int)sizeof(T), kLanes = 128 / V, kBlocks = 32 / kLanes;
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    const int lane = threadIdx.x & 31, sub = lane / kLanes, part = lane % kLanes;
    const long long blocks = rows * nb;
    const long long step = (long long)gridDim.x * (kThreads / 32) * kBlocks * kSteps;
    long long g0 = (long long)((blockIdx.x * kThreads + threadIdx.x) >> 5) * kBlocks * kSteps;
    for (; g0 < blocks; g0 += step) {
        Piece<T, V> p[kSteps];
        long long at[kSteps];   // of the lane's piece in q, -1: no such block
        uint32_t used = 0;      // bit k: the piece holds channels, not the row's end
        int b = 0;
        long long n = 0;
        if constexpr (kLoads != kFlat) n = div32(g0 + sub, nb, b);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            if constexpr (kLoads == kFlat) {
                const long long g = g0 + sub + k * kBlocks;
                at[k] = g < blocks ? g * 128 + part * V : -1;
                used |= 1u << k;
                p[k].load(x + (g < blocks ? at[k] : 0));  // absent blocks read the first
            } else {
                const int c = b * 128 + part * V;
                at[k] = n < rows && c < pitch ? n * pitch + c : -1;
                used |= (c < C ? 1u : 0u) << k;
                const long long xr = (n < rows ? n : 0) * C;
                if constexpr (kLoads == kWide) {
                    p[k].load(x + xr + (c < C ? c : 0));
                } else if constexpr (kLoads == kWords) {
                    uint32_t w[4];
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int at_c = c + 2 * v;  // both elements of a word exist, or neither
                        w[v] = *reinterpret_cast<const uint32_t*>(x + xr + (at_c < C ? at_c : 0));
                        w[v] = at_c < C ? w[v] : 0u;
                    }
                    p[k].v = make_uint4(w[0], w[1], w[2], w[3]);
                } else {
                    float f[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        f[v] = to_f32(x[xr + (c + v < C ? c + v : 0)]);
                        f[v] = c + v < C ? f[v] : 0.f;
                    }
                    p[k].set_all(f);
                }
                b += kBlocks;
                while (b >= nb) {
                    b -= nb;
                    ++n;
                }
            }
        }
        uint32_t m[kSteps];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) m[k] = used >> k & 1u ? amax_bits(p[k]) : 0u;
        const bool b0 = lane & 1, b1 = lane & 2;
        const uint32_t m01 =
            max(b0 ? m[1] : m[0], __shfl_xor_sync(0xffffffffu, b0 ? m[0] : m[1], 1));
        const uint32_t m23 =
            max(b0 ? m[3] : m[2], __shfl_xor_sync(0xffffffffu, b0 ? m[2] : m[3], 1));
        uint32_t top = max(b1 ? m23 : m01, __shfl_xor_sync(0xffffffffu, b1 ? m01 : m23, 2));
#pragma unroll
        for (int o = 4; o < kLanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float my_scale = scale_of(__uint_as_float(top)), my_inv = 1.f / my_scale;
        if (part < kSteps) {
            const long long mine = g0 + sub + (long long)part * kBlocks;
            int mb;
            const long long mn = div32(mine, nb, mb);
            if (mn < rows) scales[(long long)mb * capacity + mn] = my_scale;
        }
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const float sc = __shfl_sync(0xffffffffu, my_scale, sub * kLanes + k);
            const float inv = __shfl_sync(0xffffffffu, my_inv, sub * kLanes + k);
            if (at[k] < 0) continue;
            float f[V];
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] = p[k].get(v);
            uint32_t w[V / 4];
            to_e4m3<V>(f, sc, inv, w);
            if (kLoads != kFlat && !(used >> k & 1u)) {
#pragma unroll
                for (int v = 0; v < V / 4; ++v) w[v] = 0u;  // beyond C
            }
            if constexpr (kLoads == kScalar || kLoads == kWords) {
                // a piece that holds the row's end: the zeros behind it have no
                // quotient where the scale is a NaN
                if (sc != sc) {
                    const int left = C - (int)(at[k] % pitch);
#pragma unroll
                    for (int v = 0; v < V / 4; ++v) w[v] &= first_bytes(left - 4 * v);
                }
            }
            if constexpr (V == 8)
                *reinterpret_cast<uint2*>(q + at[k]) = make_uint2(w[0], w[1]);
            else
                *reinterpret_cast<uint32_t*>(q + at[k]) = w[0];
        }
    }
}

// Largest magnitude of two, NaN if either is NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
    return (a != a || a > b) ? a : b;
}
// A block per 128 x 128 block of W [C_in, C_out], written transposed: a thread
// holds 64 channels in of one channel out, all loaded before the first is
// used, and writes them as 64 bytes of that row. W is read once (8192 x 8192
// bf16: 67 us, 30 at the copy rate; read twice and transposed through shared
// memory 126; a warp's 16-byte stores go to 32 rows).
template <typename T>
__global__ void __launch_bounds__(kThreads)
    quant_weight_kernel(const T* __restrict__ W, int C_in, int C_out, int pitch, int nbi,
                        uint8_t* __restrict__ wq, float* __restrict__ ws) {
    constexpr int kHeld = 128 * 128 / kThreads;
    __shared__ float red[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int i0 = blockIdx.x * 128 + threadIdx.x / 128 * kHeld;
    const int o = blockIdx.y * 128 + threadIdx.x % 128;
    const T* const from = W + (o < C_out ? o : 0);
    T x[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)  // absent channels read the first
        x[k] = from[(long long)(i0 + k < C_in ? i0 + k : 0) * C_out];
    float m = 0.f;
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        m = max_nan(o < C_out && i0 + k < C_in ? fabsf(to_f32(x[k])) : 0.f, m);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = max_nan(__shfl_xor_sync(0xffffffffu, m, d), m);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
    m = red[0];
    for (int w = 1; w < kThreads / 32; ++w) m = max_nan(red[w], m);
    const float sc = scale_of(m), inv = 1.f / sc;
    if (threadIdx.x == 0) ws[(long long)blockIdx.y * nbi + blockIdx.x] = sc;
    if (o >= C_out) return;
    uint8_t* const to = wq + (long long)o * pitch + i0;
#pragma unroll
    for (int k = 0; k < kHeld; k += 16) {
        if (i0 + k >= pitch) break;
        float v[16];
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = to_f32(x[k + e]);
        to_e4m3<16>(v, sc, inv, w);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            w[q] &= first_bytes(C_in - (i0 + k + 4 * q));  // zero from C_in on
        }
        *reinterpret_cast<uint4*>(to + k) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <typename T>
hc_status quant_rows(const DeviceCtx* ctx, const void* x, const int32_t* count, int capacity,
                     int C, int pitch, int nb, uint8_t* q, float* scales, cudaStream_t s) {
    constexpr int V = 16 / (int)sizeof(T), kPerBlock = kThreads / 32 * kSteps * 32 * V / 128;
    const long long need = ((long long)capacity * nb + kPerBlock - 1) / kPerBlock;
    const long long cap = (long long)ctx->num_sms * 16;
    const uintptr_t at = reinterpret_cast<uintptr_t>(x);
    // 16-byte loads (16384 x 8192 bf16: 81 us, 169 element by element), without a
    // division a block to find its row where rows hold whole blocks (98 with it);
    // 4-byte loads of even bf16 rows (16384 x 4932: 85 us, 107 by elements)
    const bool wide = C % V == 0 && at % 16 == 0;
    auto kern = wide && C % 128 == 0 ? quant_rows_kernel<T, kFlat>
                : wide               ? quant_rows_kernel<T, kWide>
                                     : quant_rows_kernel<T, kScalar>;
    if constexpr (sizeof(T) == 2)
        if (!wide && C % 2 == 0 && at % 4 == 0) kern = quant_rows_kernel<T, kWords>;
    return launch_pdl(kern,
                      dim3((unsigned)(need < cap ? need : cap)), dim3(kThreads), 0, s,
                      "quant_rows_kernel", (const T*)x, count, (long long)capacity, C, pitch, nb,
                      q, scales, ctx->status);
}

}  // namespace

hc_status launch_quantize_fp8_rows(const DeviceCtx* ctx, const void* x, hc_dtype dt,
                                   const int32_t* count, int capacity, int C, uint8_t* q,
                                   float* scales, cudaStream_t s) {
    const int pitch = HC_FP8_PITCH(C), nb = (C + 127) / 128;
    return dt == HC_BF16 ? quant_rows<__nv_bfloat16>(ctx, x, count, capacity, C, pitch, nb, q, scales, s)
                         : quant_rows<float>(ctx, x, count, capacity, C, pitch, nb, q, scales, s);
}

hc_status launch_quantize_fp8_weight(const DeviceCtx*, const void* W, hc_dtype dt, int C_in,
                                     int C_out, uint8_t* wq, float* ws, cudaStream_t s) {
    const int pitch = HC_FP8_PITCH(C_in), nbi = (C_in + 127) / 128, nbo = (C_out + 127) / 128;
    if (nbo > 65535) {
        set_error("hc_quantize_fp8_weight: C_out=%d is too wide", C_out);
        return HC_ERR_UNSUPPORTED;
    }
    const dim3 grid((unsigned)nbi, (unsigned)nbo);
    if (dt == HC_BF16)
        return launch_pdl(quant_weight_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, s,
                          "quant_weight_kernel", (const __nv_bfloat16*)W, C_in, C_out, pitch, nbi,
                          wq, ws);
    return launch_pdl(quant_weight_kernel<float>, grid, dim3(kThreads), 0, s,
                      "quant_weight_kernel", (const float*)W, C_in, C_out, pitch, nbi, wq, ws);
}

}  // namespace hc
