// Layer norm of compact rows and its gradient. For every row n < N', over its
// C channels:
//   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps)
//   y = (x - mean) * rstd * gamma + beta
// and backwards, with xh = (x - mean) * rstd and g = dy * gamma:
//   dx     = rstd * (g - sum g / C - xh * sum (g * xh) / C)
//   dgamma = sum over rows of dy * xh,  dbeta = sum over rows of dy
// All sums in fp32; the variance is taken around the mean. dgamma and dbeta
// are summed per block of rows and the blocks' sums joined in a fixed order,
// so every result is the same from run to run.
#include "tokens.cuh"

namespace hc {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- any width
// A block per row; the row is read once for the mean, once for the variance
// and once for the output (the second and third time from the caches).
template <typename T>
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
        for (int c = threadIdx.x; c < C; c += kThreads) s += to_f32(xr[c]);
        const float mean = block_sum(s, sh) / (float)C;
        float v = 0.f;
        for (int c = threadIdx.x; c < C; c += kThreads) {
            const float d = to_f32(xr[c]) - mean;
            v += d * d;
        }
        const float rstd = 1.f / sqrtf(block_sum(v, sh) / (float)C + eps);
        for (int c = threadIdx.x; c < C; c += kThreads) {
            const float xh = (to_f32(xr[c]) - mean) * rstd;
            yr[c] = from_f32<T>(xh * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f));
        }
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[n] = mean;
            if (rstd_out) rstd_out[n] = rstd;
        }
    }
}

// The two means of a row's gradient: sums[2n] = sum g / C, sums[2n + 1] =
// sum (g * xh) / C.
template <typename T>
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
        for (int c = threadIdx.x; c < C; c += kThreads) {
            const float g = to_f32(dy[n * C + c]) * (gamma ? gamma[c] : 1.f);
            s1 += g;
            s2 += g * ((to_f32(x[n * C + c]) - m) * r);
        }
        s1 = block_sum(s1, sh);
        s2 = block_sum(s2, sh);
        if (threadIdx.x == 0) {
            sums[2 * n] = s1 / (float)C;
            sums[2 * n + 1] = s2 / (float)C;
        }
    }
}

// A thread per channel walks the rows blockIdx.y, + gridDim.y, ...: dx, and
// its own sums of dy * xh and dy into part[blockIdx.y][2][C].
template <typename T>
__global__ void __launch_bounds__(kThreads)
    ln_bwd_cols_kernel(const T* x, const T* dy, const int32_t* count, long long capacity, int C,
                       const float* __restrict__ gamma, const float* __restrict__ mean,
                       const float* __restrict__ rstd, const float* __restrict__ sums, T* dx,
                       float* __restrict__ part, unsigned* status) {
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= C) return;
    const float w = gamma ? gamma[c] : 1.f;
    float dg = 0.f, db = 0.f;
    for (long long n = blockIdx.y; n < rows; n += gridDim.y) {
        const float d = to_f32(dy[n * C + c]);
        const float xh = (to_f32(x[n * C + c]) - mean[n]) * rstd[n];
        if (dx) dx[n * C + c] = from_f32<T>((d * w - sums[2 * n] - xh * sums[2 * n + 1]) * rstd[n]);
        dg += d * xh;
        db += d;
    }
    if (part) {
        part[(2ll * blockIdx.y) * C + c] = dg;
        part[(2ll * blockIdx.y + 1) * C + c] = db;
    }
}

// dgamma and dbeta: a thread per channel adds the blocks' sums in order.
__global__ void __launch_bounds__(kThreads)
    ln_param_grad_kernel(const float* __restrict__ part, int parts, int C, float* dgamma,
                         float* dbeta) {
    pdl_wait();
    pdl_trigger();
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= C) return;
    float dg = 0.f, db = 0.f;
    for (int p = 0; p < parts; ++p) {
        dg += part[(2ll * p) * C + c];
        db += part[(2ll * p + 1) * C + c];
    }
    if (dgamma) dgamma[c] = dg;
    if (dbeta) dbeta[c] = db;
}

template <typename T>
hc_status fwd(const DeviceCtx* ctx, const LayerNormArgs& a, cudaStream_t s) {
    const long long cap = (long long)ctx->num_sms * 8;
    const unsigned grid = (unsigned)(a.capacity < cap ? a.capacity : cap);
    return launch_pdl(ln_fwd_kernel<T>, dim3(grid), dim3(kThreads), 0, s, "ln_fwd_kernel",
                      (const T*)a.x, a.count, (long long)a.capacity, a.C, a.eps, a.gamma, a.beta,
                      (T*)a.y, a.mean_out, a.rstd_out, ctx->status);
}

template <typename T>
hc_status bwd(const DeviceCtx* ctx, const LayerNormArgs& a, cudaStream_t s) {
    const bool params = a.dgamma || a.dbeta;
    const unsigned ctiles = (unsigned)((a.C + kThreads - 1) / kThreads);
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
        st = launch_pdl(ln_bwd_rows_kernel<T>, dim3((unsigned)(a.capacity < cap ? a.capacity : cap)),
                        dim3(kThreads), 0, s, "ln_bwd_rows_kernel", (const T*)a.x, (const T*)a.dy,
                        a.count, (long long)a.capacity, a.C, a.gamma, a.mean, a.rstd, ws,
                        ctx->status);
        if (st != HC_OK) return st;
    }
    st = launch_pdl(ln_bwd_cols_kernel<T>, dim3(ctiles, (unsigned)parts), dim3(kThreads), 0, s,
                    "ln_bwd_cols_kernel", (const T*)a.x, (const T*)a.dy, a.count,
                    (long long)a.capacity, a.C, a.gamma, a.mean, a.rstd, (const float*)ws,
                    (T*)a.dx, part, ctx->status);
    if (st != HC_OK || !params) return st;
    return launch_pdl(ln_param_grad_kernel, dim3(ctiles), dim3(kThreads), 0, s,
                      "ln_param_grad_kernel", (const float*)part, (int)parts, a.C, a.dgamma,
                      a.dbeta);
}

}  // namespace

hc_status launch_layer_norm_fwd(const DeviceCtx* ctx, const LayerNormArgs& a, cudaStream_t s) {
    return a.dt == HC_BF16 ? fwd<__nv_bfloat16>(ctx, a, s) : fwd<float>(ctx, a, s);
}

hc_status launch_layer_norm_bwd(const DeviceCtx* ctx, const LayerNormArgs& a, cudaStream_t s) {
    return a.dt == HC_BF16 ? bwd<__nv_bfloat16>(ctx, a, s) : bwd<float>(ctx, a, s);
}

}  // namespace hc
