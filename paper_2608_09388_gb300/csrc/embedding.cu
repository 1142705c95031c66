// Row embedding and its gradient.
//   fwd   y[n] = scale * table[ids[n]]  (zero for id -1)
//   sort  the token positions in order of their id, stable: row_ptr, order
//   bwd   dtable[v] = scale * sum of dy[order[i]], row_ptr[v] <= i < row_ptr[v+1]
// The sort is a least-significant-digit radix sort of the ids with 11-bit
// digits; ids that name no row (padding, out of range, positions past N')
// carry the key V and end up behind row_ptr[V]. Every sum runs in the order
// of the sort: results are the same from run to run.
#include "tokens.cuh"

namespace hc {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- forward
template <typename T>
__global__ void __launch_bounds__(kThreads)
    embed_fwd_kernel(const T* __restrict__ table, int V, int C, const int32_t* __restrict__ ids,
                     long long ids_stride, const int32_t* count, long long capacity, float scale,
                     T* __restrict__ y, unsigned* status) {
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    for (long long n = blockIdx.x; n < rows; n += gridDim.x) {
        const int id = ids[n * ids_stride];
        const bool ok = id >= 0 && id < V;
        if (!ok && id != -1 && threadIdx.x == 0) report(status, kErrIndex);
        for (int c = threadIdx.x; c < C; c += kThreads)
            y[n * C + c] =
                from_f32<T>(ok ? to_f32(table[(long long)id * C + c]) * scale : 0.f);
    }
}

// ---------------------------------------------------------------- sort
constexpr int kDigitBits = 11;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kMaxTiles = 64;
constexpr int kSortWarps = 8;
constexpr int kSortThreads = kSortWarps * 32;

struct SortArgs {
    const int32_t* ids;       // first pass: the ids themselves
    const int32_t* keys_in;   // later passes: keys and positions of the pass before
    const int32_t* pos_in;
    int32_t* keys_out;
    int32_t* pos_out;
    int32_t* hist;            // [tiles][kDigits]
    const int32_t* count;
    long long ids_stride;
    long long capacity;
    long long tile;           // keys per tile, a multiple of kSortThreads
    int V, shift;
    unsigned* status;
};

// Key of entry i of this pass.
__device__ __forceinline__ int sort_key(const SortArgs& a, long long i, long long rows) {
    if (a.ids == nullptr) return a.keys_in[i];
    if (i >= rows) return a.V;
    const int id = a.ids[i * a.ids_stride];
    if (id >= 0 && id < a.V) return id;
    if (id != -1) report(a.status, kErrIndex);
    return a.V;
}

__global__ void __launch_bounds__(kSortThreads) sort_hist_kernel(const SortArgs a) {
    __shared__ int h[kDigits];
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) h[d] = 0;
    pdl_wait();
    pdl_trigger();
    __syncthreads();
    const long long rows = token_rows(a.count, a.capacity, a.status);
    const long long b = blockIdx.x * a.tile;
    const long long e = b + a.tile < a.capacity ? b + a.tile : a.capacity;
    for (long long i = b + threadIdx.x; i < e; i += kSortThreads)
        atomicAdd(&h[(sort_key(a, i, rows) >> a.shift) & (kDigits - 1)], 1);
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads)
        a.hist[(long long)blockIdx.x * kDigits + d] = h[d];
}

// Places a tile's keys: an entry goes to the number of keys with a smaller
// digit, plus those with its digit in earlier tiles, in earlier warps' shares
// of this tile and earlier in its own warp's share.
constexpr size_t kScatterSmem = sizeof(int) * kDigits * (kSortWarps + 1);

__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(const SortArgs a) {
    extern __shared__ int sm[];
    __shared__ int sh[kSortWarps];
    int* const base = sm;                        // [kDigits]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int* const cnt = sm + kDigits * (1 + warp);  // this warp's [kDigits]
    for (int d = threadIdx.x; d < kDigits * kSortWarps; d += kSortThreads) sm[kDigits + d] = 0;
    pdl_wait();
    pdl_trigger();
    // Starts of the digit runs: thread t owns the kPer digits from t * kPer.
    constexpr int kPer = kDigits / kSortThreads;
    int before[kPer], total[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) before[j] = total[j] = 0;
    for (int t = 0; t < (int)gridDim.x; ++t) {
        const int* h = a.hist + (long long)t * kDigits + threadIdx.x * kPer;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int v = h[j];
            total[j] += v;
            if (t < (int)blockIdx.x) before[j] += v;
        }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) sum += total[j];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) sh[warp] = incl;
    __syncthreads();
    int run = incl - sum;
    for (int w = 0; w < warp; ++w) run += sh[w];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        base[threadIdx.x * kPer + j] = run + before[j];
        run += total[j];
    }
    // Digits of each warp's share.
    const long long rows = token_rows(a.count, a.capacity, a.status);
    const long long share = a.tile / kSortWarps;  // a multiple of 32
    const long long b = blockIdx.x * a.tile + warp * share;
    const long long e = b + share < a.capacity ? b + share : a.capacity;
    for (long long i = b + lane; i < e; i += 32)
        atomicAdd(&cnt[(sort_key(a, i, rows) >> a.shift) & (kDigits - 1)], 1);
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) {
        int at = base[d];
        for (int w = 0; w < kSortWarps; ++w) {
            const int c = sm[kDigits * (1 + w) + d];
            sm[kDigits * (1 + w) + d] = at;
            at += c;
        }
    }
    __syncthreads();
    for (long long i0 = b; i0 < e; i0 += 32) {
        const long long i = i0 + lane;
        const bool in = i < e;
        const int key = in ? sort_key(a, i, rows) : 0;
        const int digit = in ? (key >> a.shift) & (kDigits - 1) : kDigits;  // kDigits: no entry
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        const int rank = __popc(same & ((1u << lane) - 1u));
        int at = 0;
        if (in) at = cnt[digit] + rank;
        __syncwarp();
        if (in && rank == 0) cnt[digit] += __popc(same);
        __syncwarp();
        if (in) {
            a.keys_out[at] = key;
            a.pos_out[at] = a.ids ? (int)i : a.pos_in[i];
        }
    }
}

// row_ptr[v] = entries whose key is below v.
__global__ void __launch_bounds__(kThreads)
    sort_ptr_kernel(const int32_t* __restrict__ keys, int capacity, int V,
                    int32_t* __restrict__ row_ptr) {
    pdl_wait();
    pdl_trigger();
    const long long v = blockIdx.x * (long long)kThreads + threadIdx.x;
    if (v > V) return;
    int lo = 0, hi = capacity;
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (keys[mid] < v)
            lo = mid + 1;
        else
            hi = mid;
    }
    row_ptr[v] = lo;
}

// ---------------------------------------------------------------- gradient
// A block per (table row, 256 channels) adds the row's positions in order.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    embed_bwd_kernel(const T* __restrict__ dy, const int32_t* __restrict__ row_ptr,
                     const int32_t* __restrict__ order, int capacity, int V, int C, float scale,
                     float* __restrict__ dtable, unsigned* status) {
    pdl_wait();
    pdl_trigger();
    const int c = blockIdx.y * kThreads + threadIdx.x;
    for (long long v = blockIdx.x; v < V; v += gridDim.x) {
        int i = row_ptr[v], e = row_ptr[v + 1];
        if (i < 0 || e < i || e > capacity) {
            if (threadIdx.x == 0) report(status, kErrIndex);
            i = e = 0;
        }
        float s = 0.f;
        for (; i < e; ++i) {
            const int n = order[i];
            if (n < 0 || n >= capacity) {
                report(status, kErrIndex);
                continue;
            }
            if (c < C) s += to_f32(dy[(long long)n * C + c]);
        }
        if (c < C) dtable[v * C + c] = s * scale;
    }
}

}  // namespace

hc_status launch_embedding_fwd(const DeviceCtx* ctx, const EmbeddingArgs& a, const void* table,
                               void* y, cudaStream_t s) {
    const long long cap = (long long)ctx->num_sms * 8;
    const unsigned grid = (unsigned)(a.capacity < cap ? a.capacity : cap);
    if (a.dt == HC_BF16)
        return launch_pdl(embed_fwd_kernel<__nv_bfloat16>, dim3(grid), dim3(kThreads), 0, s,
                          "embed_fwd_kernel", (const __nv_bfloat16*)table, a.V, a.C, a.ids,
                          a.ids_stride, a.count, (long long)a.capacity, a.scale,
                          (__nv_bfloat16*)y, ctx->status);
    return launch_pdl(embed_fwd_kernel<float>, dim3(grid), dim3(kThreads), 0, s,
                      "embed_fwd_kernel", (const float*)table, a.V, a.C, a.ids, a.ids_stride,
                      a.count, (long long)a.capacity, a.scale, (float*)y, ctx->status);
}

hc_status launch_embedding_sort(const DeviceCtx* ctx, const EmbeddingArgs& a, int32_t* row_ptr,
                                int32_t* order, cudaStream_t s) {
    const long long n = a.capacity;
    hc_status st;
    const int32_t* sorted = nullptr;
    if (n > 0) {
        static bool done[64];
        if (!done[ctx->device]) {
            st = check_cuda(cudaFuncSetAttribute(sort_scatter_kernel,
                                                 cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)kScatterSmem),
                            "sort_scatter_kernel");
            if (st != HC_OK) return st;
            done[ctx->device] = true;
        }
        long long tile = (n + kMaxTiles - 1) / kMaxTiles;
        if (tile < 2048) tile = 2048;
        tile = (tile + kSortThreads - 1) / kSortThreads * kSortThreads;
        const unsigned tiles = (unsigned)((n + tile - 1) / tile);
        int passes = 1;
        while (passes < 3 && (a.V >> (kDigitBits * passes)) != 0) ++passes;
        // workspace: histograms, two buffers of keys and two of positions
        int32_t* ws = (int32_t*)stream_workspace(
            s, sizeof(int32_t) * ((size_t)kMaxTiles * kDigits + 4 * (size_t)n));
        if (!ws) return HC_ERR_CUDA;
        int32_t* keys[2] = {ws + (size_t)kMaxTiles * kDigits, ws + (size_t)kMaxTiles * kDigits + n};
        int32_t* pos[2] = {keys[1] + n, keys[1] + 2 * n};
        for (int p = 0; p < passes; ++p) {
            SortArgs k{};
            k.ids = p == 0 ? a.ids : nullptr;
            k.keys_in = keys[(p + 1) & 1];
            k.pos_in = pos[(p + 1) & 1];
            k.keys_out = keys[p & 1];
            k.pos_out = p == passes - 1 ? order : pos[p & 1];
            k.hist = ws;
            k.count = a.count;
            k.ids_stride = a.ids_stride;
            k.capacity = n;
            k.tile = tile;
            k.V = a.V;
            k.shift = p * kDigitBits;
            k.status = ctx->status;
            st = launch_pdl(sort_hist_kernel, dim3(tiles), dim3(kSortThreads), 0, s,
                            "sort_hist_kernel", k);
            if (st != HC_OK) return st;
            st = launch_pdl(sort_scatter_kernel, dim3(tiles), dim3(kSortThreads), kScatterSmem, s,
                            "sort_scatter_kernel", k);
            if (st != HC_OK) return st;
            sorted = k.keys_out;
        }
    }
    const unsigned grid = (unsigned)(((long long)a.V + 1 + kThreads - 1) / kThreads);
    return launch_pdl(sort_ptr_kernel, dim3(grid), dim3(kThreads), 0, s, "sort_ptr_kernel", sorted,
                      (int)n, a.V, row_ptr);
}

hc_status launch_embedding_bwd(const DeviceCtx* ctx, const EmbeddingArgs& a, const void* dy,
                               const int32_t* row_ptr, const int32_t* order, float* dtable,
                               cudaStream_t s) {
    const unsigned ctiles = (unsigned)((a.C + kThreads - 1) / kThreads);
    long long gx = (long long)ctx->num_sms * 32;
    if (gx > a.V) gx = a.V;
    if (ctiles > 65535u) {
        set_error("hc_embedding_bwd: C=%d is too wide", a.C);
        return HC_ERR_UNSUPPORTED;
    }
    const dim3 grid((unsigned)gx, ctiles);
    if (a.dt == HC_BF16)
        return launch_pdl(embed_bwd_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, s,
                          "embed_bwd_kernel", (const __nv_bfloat16*)dy, row_ptr, order, a.capacity,
                          a.V, a.C, a.scale, dtable, ctx->status);
    return launch_pdl(embed_bwd_kernel<float>, grid, dim3(kThreads), 0, s, "embed_bwd_kernel",
                      (const float*)dy, row_ptr, order, a.capacity, a.V, a.C, a.scale, dtable,
                      ctx->status);
}

}  // namespace hc
