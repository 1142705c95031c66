// Row embedding and its gradient.
//   fwd   y[n] = scale * table[ids[n]]  (zero for id -1)
//   sort  the token positions in order of their id, stable: row_ptr, order
//   bwd   dtable[v] = scale * sum of dy[order[i]], row_ptr[v] <= i < row_ptr[v+1]
// The sort is a least-significant-digit radix sort of the ids with digits of
// up to 11 bits; ids that name no row (padding, out of range, positions past
// N') carry the key V and end up behind row_ptr[V]. Every sum runs in a fixed
// order: results are the same from run to run.
//
// Forward and gradient are bound by memory (rows gathered, a table of fp32
// written whole), the sort by the round trips of its launches (two a pass, one
// for row_ptr). 65536 Zipf-distributed ids into 131072 x 1024 bf16 (GB300):
// forward 32 us (26 at the copy rate), sort 24 us, gradient 125 us (99).
#include "tokens.cuh"

namespace hc {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- forward
// A group of TPR threads copies NV pieces of TPR * VEC channels of a token's
// row at a time; all of them are loaded before the first is stored.
template <typename T, int VEC, int TPR, int NV>
__global__ void __launch_bounds__(kThreads)
    embed_fwd_kernel(const T* __restrict__ table, int V, int C, const int32_t* __restrict__ ids,
                     long long ids_stride, const int32_t* count, long long capacity, int slices,
                     float scale, T* __restrict__ y, unsigned* status) {
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    const int t = threadIdx.x % TPR;
    const long long items = rows * slices;
    const long long step = (long long)gridDim.x * (kThreads / TPR);
    for (long long it = (long long)blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR; it < items;
         it += step) {
        int slice;
        const long long n = div32(it, slices, slice);
        const int id = ids[n * ids_stride];
        const bool ok = id >= 0 && id < V;
        if (!ok && id != -1 && t == 0 && slice == 0) report(status, kErrIndex);
        const int c0 = (slice * NV * TPR + t) * VEC;
        Piece<T, VEC> p[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = c0 + i * TPR * VEC;
            if (ok && c < C) p[i].load(table + (long long)id * C + c);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = c0 + i * TPR * VEC;
            if (c < C) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) p[i].set(e, ok ? p[i].get(e) * scale : 0.f);
                p[i].store(y + n * C + c);
            }
        }
    }
}

// ---------------------------------------------------------------- sort
constexpr int kMaxDigitBits = 11;
constexpr int kMaxDigits = 1 << kMaxDigitBits;
constexpr int kMaxTiles = 64;
constexpr int kSortWarps = 16;
constexpr int kSortThreads = kSortWarps * 32;
constexpr int kSmallSort = 4 * kSortThreads;  // entries of a sort by one block

struct SortArgs {
    const int32_t* ids;       // first pass: the ids themselves
    const int32_t* keys_in;   // later passes: keys and positions of the pass before
    const int32_t* pos_in;
    int32_t* keys_out;
    int32_t* pos_out;
    int32_t* hist;            // [tiles][digits]
    const int32_t* count;
    long long ids_stride;
    long long capacity;
    int V, shift, bits;       // this pass sorts by key bits [shift, shift + bits)
    unsigned* status;
};

// Keys per tile, a multiple of R a thread, for at most kMaxTiles tiles. R keys a
// lane are held in registers at a time and placed one after another: few keys a
// tile shorten that chain, many tiles lengthen the sum of their histograms. With
// row_ptr 16763 ids take 16.4 us with R = 2, 17.8 with 4, 23.6 with 8, 65536 of
// 131072 rows 25.7, 23.7 and 26.2, 262144 of 32000 35, 35 and 31: R is 2 while
// that is 32 tiles at most, else 4 (8 would suit a large capacity that is used
// whole, but N' is often a small part of it).
template <int R>
__device__ __forceinline__ long long sort_tile(long long rows) {
    constexpr int kMinTile = kSortThreads * R;
    const long long t = (rows + kMaxTiles - 1) / kMaxTiles;
    return t < kMinTile ? kMinTile : (t + kMinTile - 1) / kMinTile * kMinTile;
}

// Key of entry i < N' of this pass.
__device__ __forceinline__ int sort_key(const SortArgs& a, long long i) {
    if (a.ids == nullptr) return a.keys_in[i];
    const int id = a.ids[i * a.ids_stride];
    if (id >= 0 && id < a.V) return id;
    if (id != -1) report(a.status, kErrIndex);
    return a.V;
}

template <int R>
__global__ void __launch_bounds__(kSortThreads) sort_hist_kernel(const SortArgs a) {
    __shared__ int h[kMaxDigits];
    const int digits = 1 << a.bits;
    for (int d = threadIdx.x; d < digits; d += kSortThreads) h[d] = 0;
    pdl_wait();
    pdl_trigger();
    __syncthreads();
    const long long rows = token_rows(a.count, a.capacity, a.status);
    const long long tile = sort_tile<R>(rows);
    const long long b = blockIdx.x * tile;
    if (b >= rows) return;
    const long long e = b + tile < rows ? b + tile : rows;
    for (long long i = b + threadIdx.x; i < e; i += kSortThreads)
        atomicAdd(&h[(sort_key(a, i) >> a.shift) & (digits - 1)], 1);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads)
        a.hist[(long long)blockIdx.x * digits + d] = h[d];
}

// Places a tile's keys: an entry goes to the number of keys with a smaller
// digit, plus those with its digit in earlier tiles, in earlier warps' shares
// of this tile and earlier in its own warp's share.
constexpr size_t scatter_smem(int bits) {
    return (sizeof(int) << bits) * (kSortWarps + 2);
}

template <int R>
__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(const SortArgs a) {
    extern __shared__ int sm[];
    __shared__ int sh[kSortWarps];
    const int digits = 1 << a.bits;
    int* const base = sm;                       // [digits] starts in this tile
    int* const tot = sm + digits;               // [digits] over all tiles
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int* const cnt = sm + digits * (2 + warp);  // [digits] of this warp
    for (int d = threadIdx.x; d < digits * kSortWarps; d += kSortThreads) sm[digits * 2 + d] = 0;
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(a.count, a.capacity, a.status);
    const long long tile = sort_tile<R>(rows);
    const int tiles = (int)((rows + tile - 1) / tile);
    if ((int)blockIdx.x >= tiles) return;
    // Starts of the digit runs. Column sums of the tiles' histograms first
    // (coalesced over the digits), then a scan with kPer digits a thread.
    for (int d = threadIdx.x; d < digits; d += kSortThreads) {
        int before = 0, total = 0;
#pragma unroll 8
        for (int t = 0; t < tiles; ++t) {
            const int v = a.hist[(long long)t * digits + d];
            total += v;
            before += t < (int)blockIdx.x ? v : 0;
        }
        base[d] = before;
        tot[d] = total;
    }
    __syncthreads();
    constexpr int kPer = kMaxDigits / kSortThreads;
    int sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int d = threadIdx.x * kPer + j;
        sum += d < digits ? tot[d] : 0;
    }
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
        const int d = threadIdx.x * kPer + j;
        if (d < digits) {
            base[d] += run;
            run += tot[d];
        }
    }
    // Digits of each warp's share: a multiple of 32 * R entries, that
    // many at a time in registers (the first batch stays for the placing).
    const long long share = tile / kSortWarps;
    const long long b = blockIdx.x * tile + warp * share;
    const long long e = b + share < rows ? b + share : rows;
    int key[R], pos[R];
    auto load = [&](long long i0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long i = i0 + r * 32 + lane;
            key[r] = i < e ? sort_key(a, i) : -1;
            pos[r] = a.ids ? (int)i : i < e ? a.pos_in[i] : 0;
        }
    };
    for (long long i0 = b; i0 < e; i0 += 32 * R) {
        load(i0);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (key[r] >= 0) atomicAdd(&cnt[(key[r] >> a.shift) & (digits - 1)], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads) {
        int at = base[d];
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            const int c = sm[digits * (2 + w) + d];
            sm[digits * (2 + w) + d] = at;
            at += c;
        }
    }
    __syncthreads();
    for (long long i0 = b; i0 < e; i0 += 32 * R) {
        if (share > 32 * R) load(i0);  // else the share is still held
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool in = key[r] >= 0;
            const int digit = in ? (key[r] >> a.shift) & (digits - 1) : digits;  // no entry
            const unsigned same = __match_any_sync(0xffffffffu, digit);
            const int rank = __popc(same & ((1u << lane) - 1u));
            int at = 0;
            if (in) at = cnt[digit] + rank;
            __syncwarp();
            if (in && rank == 0) cnt[digit] += __popc(same);
            __syncwarp();
            if (in) {
                a.keys_out[at] = key[r];
                a.pos_out[at] = pos[r];
            }
        }
    }
}

// All passes of a sort of at most R * kSortThreads entries by one block, the keys and
// positions handed from pass to pass through shared memory.
template <int R>
constexpr size_t small_smem(int bits) {
    return (sizeof(int) << bits) * (kSortWarps + 1) + 2 * sizeof(int) * R * kSortThreads;
}

template <int R>
__global__ void __launch_bounds__(kSortThreads) sort_small_kernel(const SortArgs a, int passes) {
    extern __shared__ int sm[];
    __shared__ int sh[kSortWarps];
    const int digits = 1 << a.bits;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int* const base = sm;                         // [digits]
    int* const cnt = sm + digits * (1 + warp);    // [digits] of this warp
    int* const skey = sm + digits * (1 + kSortWarps);
    int* const spos = skey + R * kSortThreads;
    pdl_wait();
    pdl_trigger();
    const int rows = (int)token_rows(a.count, a.capacity, a.status);
    const int i0 = warp * 32 * R + lane;
    int key[R], pos[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        pos[r] = i0 + r * 32;
        key[r] = pos[r] < rows ? sort_key(a, pos[r]) : -1;
    }
    for (int p = 0; p < passes; ++p) {
        const int shift = p * a.bits;
        for (int d = threadIdx.x; d < digits * kSortWarps; d += kSortThreads) sm[digits + d] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (key[r] >= 0) atomicAdd(&cnt[(key[r] >> shift) & (digits - 1)], 1);
        __syncthreads();
        // starts of the warps within a digit, then of the digits
        for (int d = threadIdx.x; d < digits; d += kSortThreads) {
            int at = 0;
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                const int c = sm[digits * (1 + w) + d];
                sm[digits * (1 + w) + d] = at;
                at += c;
            }
            base[d] = at;
        }
        __syncthreads();
        constexpr int kPer = kMaxDigits / kSortThreads;
        int tot[kPer], sum = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int d = threadIdx.x * kPer + j;
            tot[j] = d < digits ? base[d] : 0;
            sum += tot[j];
        }
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
            const int d = threadIdx.x * kPer + j;
            if (d < digits) base[d] = run;
            run += tot[j];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool in = key[r] >= 0;
            const int digit = in ? (key[r] >> shift) & (digits - 1) : digits;  // no entry
            const unsigned same = __match_any_sync(0xffffffffu, digit);
            const int rank = __popc(same & ((1u << lane) - 1u));
            int at = 0;
            if (in) at = base[digit] + cnt[digit] + rank;
            __syncwarp();
            if (in && rank == 0) cnt[digit] += __popc(same);
            __syncwarp();
            if (in) {
                skey[at] = key[r];
                spos[at] = pos[r];
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = i0 + r * 32;
            key[r] = i < rows ? skey[i] : -1;
            pos[r] = i < rows ? spos[i] : 0;
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = i0 + r * 32;
        if (i < rows) {
            a.keys_out[i] = key[r];
            a.pos_out[i] = pos[r];
        }
    }
}

// row_ptr[v] = entries whose key is below v: a binary search that starts
// among 1024 samples of the keys in shared memory, so that at most 2^-10 of
// the keys are left for the dependent global loads. Positions from N' on
// follow the sorted ones in order.
constexpr int kSampleBits = 10;

__global__ void __launch_bounds__(kThreads)
    sort_ptr_kernel(const int32_t* __restrict__ keys, const int32_t* count, int capacity, int V,
                    int32_t* __restrict__ row_ptr, int32_t* __restrict__ order, unsigned* status) {
    __shared__ int sample[1 << kSampleBits];
    pdl_wait();
    pdl_trigger();
    const int rows = (int)token_rows(count, capacity, status);
    const int stride = (rows >> kSampleBits) + 1;  // sample i is keys[i * stride]
    const int samples = (int)(((long long)rows + stride - 1) / stride);
    for (int i = threadIdx.x; i < samples; i += kThreads) sample[i] = keys[(long long)i * stride];
    __syncthreads();
    const long long g = blockIdx.x * (long long)kThreads + threadIdx.x;
    const long long all = (long long)gridDim.x * kThreads;
    for (long long v = g; v <= V; v += all) {
        int lo = 0, hi = samples;  // samples below v
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (sample[mid] < v)
                lo = mid + 1;
            else
                hi = mid;
        }
        // the answer lies after sample lo - 1 and not after sample lo
        hi = lo == samples ? rows : lo * stride;
        lo = lo == 0 ? 0 : (lo - 1) * stride + 1;
        while (lo < hi) {
            const int mid = lo + (hi - lo) / 2;
            if (keys[mid] < v)
                lo = mid + 1;
            else
                hi = mid;
        }
        row_ptr[v] = lo;
    }
    for (long long i = rows + g; i < capacity; i += all) order[i] = (int)i;
}

// ---------------------------------------------------------------- gradient
// Sorted entries are cut into chunks, of at least kMinChunk entries and at
// most `max_chunks`. A table row of at most one chunk's tokens is summed by
// one group of threads, so that no group walks a frequent token alone. A
// longer row is summed chunk by chunk, a block each: it holds the chunk's
// first entry or its last, so a chunk has at most two such sums, slot 0 for
// the row of its first entry and slot 1 for another row at its end. Both
// kinds of work are blocks of one launch (embed_bwd_kernel). The chunks' sums
// of a row are then added in a fixed order by the blocks of the chunk where
// the row starts (embed_bwd_join_kernel; at most one long row starts in a
// chunk, noted in `starts`).
// Fewer chunks leave frequent tokens to few groups, more mean more sums to join:
// 65536 ids of a 32000 x 512 bf16 table, frequent rows side by side, took 60 us with 8
// chunks an SM (79 with 4, 59 with 16), 16763 of 10475 x 128 fp32, frequent rows
// scattered, 14.3 (13.7, 16.3).
constexpr int kMinChunk = 64;
constexpr int kChunksPerSM = 8;

struct GradArgs {
    const int32_t* row_ptr;
    const int32_t* order;
    int capacity, V, C;
    int max_chunks;
    float scale;
    float* part;    // [chunks][2][C]
    int* starts;    // [chunks] the long row that starts there, or -1
    float* dtable;
    unsigned* status;
};

// Sorted entries in use, and entries per chunk.
__device__ __forceinline__ int entries(const GradArgs& a) {
    return min(max(__ldg(a.row_ptr + a.V), 0), a.capacity);
}
__device__ __forceinline__ int chunk_of(const GradArgs& a, int total) {
    return max(kMinChunk, (int)(((long long)total + a.max_chunks - 1) / a.max_chunks));
}

// Tokens of table row v; empty (and reported) where row_ptr is not a range of
// the capacity.
__device__ __forceinline__ int2 tokens_of(const GradArgs& a, int v) {
    int2 r = make_int2(__ldg(a.row_ptr + v), __ldg(a.row_ptr + v + 1));
    if (r.x < 0 || r.y < r.x || r.y > a.capacity) {
        report(a.status, kErrIndex);
        r = make_int2(0, 0);
    }
    return r;
}

// Whether the short rows of a group of `per` > 1 table rows are left to the
// chunks too, each to the chunk that its tokens start in: the group holds more
// than a chunk's tokens. Frequent rows are often neighbours (ids by falling
// frequency), and their group would end last: 65536 tokens of 131072 x 1024
// bf16 178 us so, 121 with this, of 32000 x 512 59 and 40.
__device__ __forceinline__ bool is_heavy(const GradArgs& a, int per, long long group, int chunk) {
    if (per == 1 || a.max_chunks == 1) return false;
    const long long v0 = group * per, v1 = v0 + per < a.V ? v0 + per : a.V;
    return (long long)__ldg(a.row_ptr + v1) - __ldg(a.row_ptr + v0) > chunk;
}

// The table rows whose tokens include the sorted entries i.x <= i.y <
// row_ptr[V], found by a warp with 32 probes a step, both at once (a binary
// search would be up to 17 dependent loads each).
__device__ __forceinline__ int2 rows_at(const GradArgs& a, int2 i) {
    const int lane = threadIdx.x & 31;
    int lo[2] = {0, 0}, hi[2] = {a.V - 1, a.V - 1};  // the first row with row_ptr[v + 1] > i
    const int want[2] = {i.x, i.y};
    while (lo[0] < hi[0] || lo[1] < hi[1]) {
        long long at[2];
        bool above[2];
        int step[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            step[q] = (hi[q] - lo[q]) / 32 + 1;  // probes every `step`, the last past hi
            at[q] = (long long)lo[q] + (long long)(lane + 1) * step[q] - 1;
            above[q] = at[q] >= hi[q] || __ldg(a.row_ptr + at[q] + 1) > want[q];
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int k = __ffs(__ballot_sync(0xffffffffu, above[q])) - 1;
            const long long top = (long long)lo[q] + (long long)(k + 1) * step[q] - 1;
            lo[q] += k * step[q];
            if (top < hi[q]) hi[q] = (int)top;
        }
    }
    return make_int2(lo[0], lo[1]);
}

// Rows of dy a group keeps in flight: up to 32 registers' worth, 8 at most
// (single elements count double for their addresses).
template <typename T, int VEC, int NV>
constexpr int kAheadRegs = VEC == 1 ? 2 * NV : NV * VEC * (int)sizeof(T) / 4;
template <typename T, int VEC, int NV>
constexpr int kAheadRows = 32 / kAheadRegs<T, VEC, NV> < 8 ? 32 / kAheadRegs<T, VEC, NV> : 8;

// acc += dy[order[i]] for i = b, b + step, .. < e, by a group of TPR threads
// (`mask` of its warp) holding NV pieces of TPR * VEC channels from c0 on. A
// group reads TPR entries of order at once and keeps kAhead rows in flight:
// absent rows and channels load from row 0 and channel 0 and add zero, since
// a load under a condition is moved down to its use, behind the one before.
template <typename T, int VEC, int TPR, int NV>
__device__ __forceinline__ void add_tokens(const GradArgs& a, const T* __restrict__ dy, long long b,
                                           int e, int step, int c0, unsigned mask, float (&acc)[NV * VEC]) {
    constexpr int kAhead = kAheadRows<T, VEC, NV>;
    const int t = threadIdx.x % TPR;
    for (long long i0 = b; i0 < e; i0 += (long long)TPR * step) {
        const long long mine = i0 + (long long)t * step;
        int pos = -1;
        if (mine < e) {
            pos = __ldg(a.order + mine);
            if (pos < 0 || pos >= a.capacity) {
                report(a.status, kErrIndex);
                pos = -1;
            }
        }
        const long long left = (e - i0 + step - 1) / step;
        const int n = left < TPR ? (int)left : TPR;
        for (int j = 0; j < n; j += kAhead) {
            Piece<T, VEC> p[kAhead][NV];
            int at[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                at[u] = __shfl_sync(mask, pos, (j + u) % TPR, TPR);
                if (j + u >= n) at[u] = -1;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    const int c = c0 + k * TPR * VEC;
                    p[u][k].load(dy + (long long)max(at[u], 0) * a.C + (c < a.C ? c : 0));
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int k = 0; k < NV * VEC; ++k)
                    acc[k] += at[u] >= 0 ? p[u][k / VEC].get(k % VEC) : 0.f;
        }
    }
}

template <int VEC>
__device__ __forceinline__ void store_floats(float* p, const float* v) {
    if constexpr (VEC == 1) {
        *p = *v;
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 4)
            *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    }
}

constexpr int kMaxPer = 16;  // table rows per group at most (below TPR + 1 for 8 threads: 8)

// A group takes `per` consecutive table rows, one slice of channels of each.
// Their tokens are consecutive sorted entries: they are walked as one list,
// kAhead rows of dy in flight across the table rows' ends.
template <typename T, int VEC, int TPR, int NV>
__device__ __forceinline__ void rows_role(const GradArgs& a, const T* __restrict__ dy, int per,
                                          long long group, int slice) {
    constexpr int kAhead = kAheadRows<T, VEC, NV>;
    const int t = threadIdx.x % TPR;
    const unsigned mask =
        TPR == 32 ? 0xffffffffu : ((1u << (TPR & 31)) - 1u) << (threadIdx.x % 32 / TPR * TPR);
    const int c0 = (slice * NV * TPR + t) * VEC;
    const long long v0 = group * per;
    if (v0 >= a.V) return;
    const int mine = a.V - v0 < per ? (int)(a.V - v0) : per;
    const int chunk = chunk_of(a, entries(a));
    // thread j < mine: the tokens of row v0 + j
    int2 r = make_int2(0, 0);
    if (t < mine) r = tokens_of(a, (int)v0 + t);
    const bool is_long = r.y - r.x > chunk;  // left to the chunks
    const bool heavy = is_heavy(a, per, group, chunk);
    // one list if the ranges follow each other, else (a long row, or a
    // row_ptr that is none) a list per row
    const int next = __shfl_down_sync(mask, r.x, 1, TPR);
    const unsigned odd = __ballot_sync(mask, is_long || (t + 1 < mine && r.y != next)) & mask;
    float acc[NV * VEC];
#pragma unroll
    for (int k = 0; k < NV * VEC; ++k) acc[k] = 0.f;
    auto flush = [&](int j) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * TPR * VEC;
            if (c < a.C) {
                float v[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    v[e] = acc[k * VEC + e] * a.scale;
                    acc[k * VEC + e] = 0.f;
                }
                store_floats<VEC>(a.dtable + (v0 + j) * a.C + c, v);
            }
        }
    };
    if (heavy) {
        for (unsigned none = __ballot_sync(mask, t < mine && r.x == r.y) & mask; none != 0;
             none &= none - 1)
            flush((__ffs(none) - 1) % TPR);
        return;
    }
    if (odd) {
        for (int j = 0; j < mine; ++j) {
            const int b = __shfl_sync(mask, r.x, j, TPR), e = __shfl_sync(mask, r.y, j, TPR);
            if (e - b > chunk) continue;
            add_tokens<T, VEC, TPR, NV>(a, dy, b, e, 1, c0, mask, acc);
            flush(j);
        }
        return;
    }
    const int b = __shfl_sync(mask, r.x, 0, TPR), e = __shfl_sync(mask, r.y, mine - 1, TPR);
    int j = 0, end = __shfl_sync(mask, r.y, 0, TPR);
    // unsigned: the step behind the last entry may pass the largest int
    unsigned i0 = (unsigned)b;
    for (int left = e - b; left > 0; left -= TPR, i0 += TPR) {
        int pos = -1;
        if (t < left) {
            pos = __ldg(a.order + i0 + t);
            if (pos < 0 || pos >= a.capacity) {
                report(a.status, kErrIndex);
                pos = -1;
            }
        }
        const int n = min(left, TPR);
        for (int q = 0; q < n; q += kAhead) {
            Piece<T, VEC> p[kAhead][NV];
            int at[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                at[u] = __shfl_sync(mask, pos, (q + u) % TPR, TPR);
                if (q + u >= n) at[u] = -1;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    const int c = c0 + k * TPR * VEC;
                    p[u][k].load(dy + (long long)max(at[u], 0) * a.C + (c < a.C ? c : 0));
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (q + u >= n) break;
                while (i0 + q + u >= (unsigned)end) {  // this token is of a later row
                    flush(j);
                    end = __shfl_sync(mask, r.y, ++j, TPR);
                }
#pragma unroll
                for (int k = 0; k < NV * VEC; ++k)
                    acc[k] += at[u] >= 0 ? p[u][k / VEC].get(k % VEC) : 0.f;
            }
        }
    }
    for (; j < mine; ++j) flush(j);
}

// The sums of a chunk's long rows, then its short rows of heavy groups. For a
// long row the 8 warps are `sl` slices of 32 * VEC channels times 8 / sl shares
// of the tokens; shares are joined in order. A short row's slices go to the
// warps in turn. Rows of more than 8 slices are `part`s of them, a block each
// (3517 tokens of 895 x 3038 fp32 22 us, 69 by one block; 16384 of 32000 x 4096
// bf16 117 and 139). Where the last part is narrow it loses: its warps share the
// slices of the whole row, not of what is left (34421 tokens of 336 x 543 bf16,
// three parts of 256 channels, 41 us, 35 by one block).
template <typename T, int VEC>
__device__ __forceinline__ void chunk_role(const GradArgs& a, const T* __restrict__ dy, int index,
                                           int part, int per, float (*sh)[32 * VEC]) {
    constexpr int kWarps = kThreads / 32, kWidth = 32 * VEC;
    const int total = entries(a), chunk = chunk_of(a, total);
    const long long b = (long long)index * chunk;
    if (b >= total) {
        if (threadIdx.x == 0 && part == 0) a.starts[index] = -1;
        return;
    }
    const int p0 = (int)b, p1 = (int)(b + chunk < total ? b + chunk : total);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int2 row = rows_at(a, make_int2(p0, p1 - 1));
    if (threadIdx.x == 0 && part == 0) {
        const int2 r = tokens_of(a, row.y);
        a.starts[index] = r.y - r.x > chunk && r.x >= p0 ? row.y : -1;
    }
    int sl = 1;
    while (sl < kWarps && sl * kWidth < a.C) sl *= 2;
    const int shares = kWarps / sl, share = warp / sl;
    for (int slot = 0; slot < (row.y == row.x ? 1 : 2); ++slot) {
        const int2 r = tokens_of(a, slot ? row.y : row.x);
        if (r.y - r.x <= chunk) continue;
        float* const out = a.part + (2ll * index + slot) * a.C;
        const int c = (part * sl + warp % sl) * kWidth + lane * VEC;
        float acc[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[k] = 0.f;
        add_tokens<T, VEC, 32, 1>(a, dy, (long long)max(r.x, p0) + share, min(r.y, p1), shares, c,
                                  0xffffffffu, acc);
        if (shares > 1) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < VEC; ++v) sh[warp][lane * VEC + v] = acc[v];
            __syncthreads();
            if (share == 0)
                for (int q = 1; q < shares; ++q)
#pragma unroll
                    for (int v = 0; v < VEC; ++v) acc[v] += sh[warp + q * sl][lane * VEC + v];
        }
        if (share == 0 && c < a.C) store_floats<VEC>(out + c, acc);
    }
    // a heavy group holds more entries than a chunk: none lies between the
    // groups of the chunk's first and last entry
    const int from = part * kWarps, pieces = min((a.C + kWidth - 1) / kWidth, from + kWarps);
    int turn = 0;
    for (int q = 0; q < 2; ++q) {
        const int group = (q ? row.y : row.x) / per;
        if (q && group == row.x / per) break;
        if (!is_heavy(a, per, group, chunk)) continue;
        const long long v0 = (long long)group * per;
        int2 r = make_int2(0, 0);
        if (lane < per && v0 + lane < a.V) r = tokens_of(a, (int)v0 + lane);
        unsigned which = __ballot_sync(
            0xffffffffu, r.x < r.y && r.y - r.x <= chunk && r.x >= p0 && r.x < p1);
        for (; which != 0; which &= which - 1) {
            const int j = __ffs(which) - 1;
            const int b0 = __shfl_sync(0xffffffffu, r.x, j), e0 = __shfl_sync(0xffffffffu, r.y, j);
            for (int p = from; p < pieces; ++p, ++turn) {
                if (turn % kWarps != warp) continue;
                const int c = p * kWidth + lane * VEC;
                float acc[VEC];
#pragma unroll
                for (int k = 0; k < VEC; ++k) acc[k] = 0.f;
                add_tokens<T, VEC, 32, 1>(a, dy, b0, e0, 1, c, 0xffffffffu, acc);
#pragma unroll
                for (int k = 0; k < VEC; ++k) acc[k] *= a.scale;
                if (c < a.C) store_floats<VEC>(a.dtable + (v0 + j) * a.C + c, acc);
            }
        }
    }
}

// Blocks [0, chunks * parts): chunks; the others: groups of table rows.
// Three blocks an SM: with fewer registers a thread and 256 channels a group
// the 131072 x 1024 bf16 table of 65536 tokens took 135 us, with 512 channels
// and two blocks 147 us (loads in flight per warp against warps).
template <typename T, int VEC, int TPR, int NV>
__global__ void __launch_bounds__(kThreads, 3)
    embed_bwd_kernel(const GradArgs a, const T* __restrict__ dy, int chunks, int parts,
                     int slices, int per) {
    __shared__ float sh[kThreads / 32][32 * VEC];
    pdl_wait();
    pdl_trigger();
    if ((int)blockIdx.x < chunks * parts) {
        int part;
        const int index = div32((int)blockIdx.x, parts, part);
        chunk_role<T, VEC>(a, dy, index, part, per, sh);
    } else {
        int slice;
        const long long block = div32((int)blockIdx.x - chunks * parts, slices, slice);
        rows_role<T, VEC, TPR, NV>(a, dy, per, block * (kThreads / TPR) + threadIdx.x / TPR, slice);
    }
}

// Block (slice, chunk): if a long row starts in the chunk, 32 * V channels of
// the sum of the row's chunks' sums. Warp w adds every 8th from the w-th on,
// then the warps' sums are added in order. (One block a row, each thread walking
// all sums of its channels: 131 us instead of 125 for the gradient of 131072 x
// 1024, 21 instead of 17 for 65536 tokens of 10475 x 128 fp32.)
template <int V>
__global__ void __launch_bounds__(kThreads) embed_bwd_join_kernel(const GradArgs a) {
    constexpr int kWarps = kThreads / 32;
    __shared__ float sh[kWarps][32 * V];
    pdl_wait();
    pdl_trigger();
    const int row = __ldg(a.starts + blockIdx.y);
    if (row < 0) return;
    const int total = entries(a), chunk = chunk_of(a, total);
    const int2 r = tokens_of(a, row);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = ((int)blockIdx.x * 32 + lane) * V;
    // the row starts in this chunk: at its first entry (slot 0) or later
    // (slot 1); it holds the first entry of every later chunk (slot 0). Where
    // row_ptr decreases, its end may lie behind the last chunk.
    const int k0 = (int)blockIdx.y, k1 = (min(r.y, total) - 1) / chunk;
    const int slot0 = r.x == (long long)k0 * chunk ? 0 : 1;
    Piece<float, V> s;
#pragma unroll
    for (int v = 0; v < V; ++v) s.set(v, 0.f);
    if (c < a.C) {
#pragma unroll 4
        for (int k = k0 + warp; k <= k1; k += kWarps) {
            Piece<float, V> f;
            f.load(a.part + (2ll * k + (k == k0 ? slot0 : 0)) * a.C + c);
#pragma unroll
            for (int v = 0; v < V; ++v) s.set(v, s.get(v) + f.get(v));
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) sh[warp][lane * V + v] = s.get(v);
    __syncthreads();
    if (warp != 0 || c >= a.C) return;
#pragma unroll
    for (int w = 1; w < kWarps; ++w)
#pragma unroll
        for (int v = 0; v < V; ++v) s.set(v, s.get(v) + sh[w][lane * V + v]);
#pragma unroll
    for (int v = 0; v < V; ++v) s.set(v, s.get(v) * a.scale);
    s.store(a.dtable + (long long)row * a.C + c);
}

bool aligned16(const void* p) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0;
}

hc_status sort_smem(const DeviceCtx* ctx, const void* kern, size_t bytes, bool (&done)[64],
                    const char* name) {
    if (done[ctx->device]) return HC_OK;
    const hc_status st = check_cuda(
        cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes), name);
    done[ctx->device] = st == HC_OK;
    return st;
}

template <int R>
hc_status sort_small(const DeviceCtx* ctx, SortArgs k, int passes, int32_t* order,
                     const int32_t** sorted, cudaStream_t s) {
    static bool done[64];
    auto kern = sort_small_kernel<R>;
    hc_status st = sort_smem(ctx, (const void*)kern, small_smem<R>(kMaxDigitBits), done,
                             "sort_small_kernel");
    if (st != HC_OK) return st;
    k.keys_out = (int32_t*)stream_workspace(s, sizeof(int32_t) * (size_t)k.capacity);
    if (!k.keys_out) return HC_ERR_CUDA;
    k.pos_out = order;
    *sorted = k.keys_out;
    return launch_pdl(kern, dim3(1), dim3(kSortThreads), small_smem<R>(k.bits), s,
                      "sort_small_kernel", k, passes);
}

template <int R>
hc_status sort_tiles(const DeviceCtx* ctx, SortArgs k, int passes, int32_t* order,
                     const int32_t** sorted, cudaStream_t s) {
    static bool done[64];
    auto scatter = sort_scatter_kernel<R>;
    hc_status st = sort_smem(ctx, (const void*)scatter, scatter_smem(kMaxDigitBits), done,
                             "sort_scatter_kernel");
    if (st != HC_OK) return st;
    const long long n = k.capacity, need = (n + R * kSortThreads - 1) / (R * kSortThreads);
    const unsigned tiles = (unsigned)(need < kMaxTiles ? need : kMaxTiles);
    // workspace: histograms, two buffers of keys and two of positions
    const size_t hist = (size_t)kMaxTiles * kMaxDigits;
    int32_t* ws = (int32_t*)stream_workspace(s, sizeof(int32_t) * (hist + 4 * (size_t)n));
    if (!ws) return HC_ERR_CUDA;
    int32_t* keys[2] = {ws + hist, ws + hist + n};
    int32_t* pos[2] = {keys[1] + n, keys[1] + 2 * n};
    k.hist = ws;
    for (int p = 0; p < passes; ++p) {
        if (p > 0) k.ids = nullptr;
        k.keys_in = keys[(p + 1) & 1];
        k.pos_in = pos[(p + 1) & 1];
        k.keys_out = keys[p & 1];
        k.pos_out = p == passes - 1 ? order : pos[p & 1];
        k.shift = p * k.bits;
        st = launch_pdl(sort_hist_kernel<R>, dim3(tiles), dim3(kSortThreads), 0, s,
                        "sort_hist_kernel", k);
        if (st != HC_OK) return st;
        st = launch_pdl(scatter, dim3(tiles), dim3(kSortThreads), scatter_smem(k.bits), s,
                        "sort_scatter_kernel", k);
        if (st != HC_OK) return st;
        *sorted = k.keys_out;
    }
    return HC_OK;
}

template <typename T, int VEC, int TPR, int NV>
hc_status fwd(const DeviceCtx* ctx, const EmbeddingArgs& a, const void* table, void* y,
              cudaStream_t s) {
    const int slices = (a.C + NV * TPR * VEC - 1) / (NV * TPR * VEC);
    const long long need = ((long long)a.capacity * slices + kThreads / TPR - 1) / (kThreads / TPR);
    const long long cap = (long long)ctx->num_sms * 8;
    return launch_pdl(embed_fwd_kernel<T, VEC, TPR, NV>,
                      dim3((unsigned)(need < cap ? need : cap)), dim3(kThreads), 0, s,
                      "embed_fwd_kernel", (const T*)table, a.V, a.C, a.ids, a.ids_stride, a.count,
                      (long long)a.capacity, slices, a.scale, (T*)y, ctx->status);
}

// 16-byte pieces where the rows allow them (65536 of 131072 x 1024 bf16: 36 us,
// 57 element by element); 8 threads a row where that is enough (65536 of 10475 x
// 32 fp32: 3.7 us, 7.8 with a warp), else a warp with up to 4 pieces each (one:
// 39 us).
template <typename T>
hc_status run_fwd(const DeviceCtx* ctx, const EmbeddingArgs& a, const void* table, void* y,
                  cudaStream_t s) {
    constexpr int kVec = 16 / (int)sizeof(T);
    if (a.C % kVec == 0 && aligned16(table) && aligned16(y)) {
        if (a.C <= 8 * kVec) return fwd<T, kVec, 8, 1>(ctx, a, table, y, s);
        if (a.C <= 32 * kVec) return fwd<T, kVec, 32, 1>(ctx, a, table, y, s);
        return fwd<T, kVec, 32, 4>(ctx, a, table, y, s);
    }
    if (a.C <= 32) return fwd<T, 1, 8, 4>(ctx, a, table, y, s);
    return fwd<T, 1, 32, 8>(ctx, a, table, y, s);
}

template <typename T, int VEC, int TPR, int NV>
hc_status bwd(const DeviceCtx* ctx, const GradArgs& a, const void* dy, cudaStream_t s) {
    const int slices = (a.C + NV * TPR * VEC - 1) / (NV * TPR * VEC);
    const int chunks = a.max_chunks > 1 ? a.max_chunks : 0;  // one chunk: no row is longer
    // table rows per group: one while the groups fill the SMs (always one: 302
    // us instead of 225 for 65536 tokens of 131072 x 1024 bf16)
    const long long groups = (long long)ctx->num_sms * 16 * (kThreads / TPR);
    long long per = ((long long)a.V * slices + groups - 1) / groups;
    const int most = TPR < kMaxPer ? TPR : kMaxPer;
    per = per < 1 ? 1 : per > most ? most : per;
    const long long blocks = (a.V + per * (kThreads / TPR) - 1) / (per * (kThreads / TPR));
    constexpr int kPart = kThreads * VEC;  // channels of a chunk's block
    const int parts = (int)(((long long)a.C + kPart - 1) / kPart);
    const long long grid = blocks * slices + (long long)chunks * parts;
    if (grid > 0x7fffffffll) {
        set_error("hc_embedding_bwd: V=%d C=%d is too large", a.V, a.C);
        return HC_ERR_UNSUPPORTED;
    }
    hc_status st = launch_pdl(embed_bwd_kernel<T, VEC, TPR, NV>, dim3((unsigned)grid),
                              dim3(kThreads), 0, s, "embed_bwd_kernel", a, (const T*)dy, chunks,
                              parts, slices, (int)per);
    if (st != HC_OK || chunks == 0) return st;
    return launch_pdl(embed_bwd_join_kernel<VEC>,
                      dim3((unsigned)((a.C + 32 * VEC - 1) / (32 * VEC)), (unsigned)chunks),
                      dim3(kThreads), 0, s, "embed_bwd_join_kernel", a);
}

// Pieces of four channels: the fp32 sums of a warp's pieces then leave as
// whole 16-byte stores side by side (pieces of eight bf16 channels would
// store every other 16 bytes at a time); element by element the 225 us of 65536
// tokens of 131072 x 1024 bf16 were 295. 8 threads a row of up to 32 channels:
// 16763 tokens of 10475 x 32 fp32 take 8 us, with a warp 11.
template <typename T>
hc_status run_bwd(const DeviceCtx* ctx, const GradArgs& a, const void* dy, cudaStream_t s) {
    if (a.C % 4 == 0 && aligned16(dy) && aligned16(a.dtable)) {
        if (a.C <= 32) return bwd<T, 4, 8, 1>(ctx, a, dy, s);
        if (a.C <= 128) return bwd<T, 4, 32, 1>(ctx, a, dy, s);
        return bwd<T, 4, 32, 2>(ctx, a, dy, s);
    }
    if (a.C <= 32) return bwd<T, 1, 8, 4>(ctx, a, dy, s);
    return bwd<T, 1, 32, 4>(ctx, a, dy, s);
}

}  // namespace

hc_status launch_embedding_fwd(const DeviceCtx* ctx, const EmbeddingArgs& a, const void* table,
                               void* y, cudaStream_t s) {
    return a.dt == HC_BF16 ? run_fwd<__nv_bfloat16>(ctx, a, table, y, s)
                           : run_fwd<float>(ctx, a, table, y, s);
}

hc_status launch_embedding_sort(const DeviceCtx* ctx, const EmbeddingArgs& a, int32_t* row_ptr,
                                int32_t* order, cudaStream_t s) {
    const long long n = a.capacity;
    const int32_t* sorted = nullptr;
    if (n > 0) {
        // the keys 0 .. V in as few passes as 11-bit digits allow, of equal width
        int key_bits = 1;
        while (key_bits < 31 && (a.V >> key_bits) != 0) ++key_bits;
        const int passes = (key_bits + kMaxDigitBits - 1) / kMaxDigitBits;
        SortArgs k{};
        k.ids = a.ids;
        k.count = a.count;
        k.ids_stride = a.ids_stride;
        k.capacity = n;
        k.V = a.V;
        k.bits = (key_bits + passes - 1) / passes;
        k.status = ctx->status;
        // One launch instead of two a pass while a block holds the keys: 2000 ids
        // 10.5 us with row_ptr, 13.2 with tiles. 4000 by one block would take
        // 15.5, with tiles 14.1.
        const hc_status st = n <= 2 * kSortThreads    ? sort_small<2>(ctx, k, passes, order, &sorted, s)
                             : n <= kSmallSort        ? sort_small<4>(ctx, k, passes, order, &sorted, s)
                             : n <= 64 * kSortThreads ? sort_tiles<2>(ctx, k, passes, order, &sorted, s)
                                                      : sort_tiles<4>(ctx, k, passes, order, &sorted, s);
        if (st != HC_OK) return st;
    }
    const long long need = ((a.V + 1ll > n ? a.V + 1ll : n) + kThreads - 1) / kThreads;
    const long long cap = (long long)ctx->num_sms * 8;
    return launch_pdl(sort_ptr_kernel, dim3((unsigned)(need < cap ? need : cap)), dim3(kThreads), 0,
                      s, "sort_ptr_kernel", sorted, a.count, (int)n, a.V, row_ptr, order,
                      ctx->status);
}

hc_status launch_embedding_bwd(const DeviceCtx* ctx, const EmbeddingArgs& a, const void* dy,
                               const int32_t* row_ptr, const int32_t* order, float* dtable,
                               cudaStream_t s) {
    const long long need = ((long long)a.capacity + kMinChunk - 1) / kMinChunk;
    const int chunks = (int)(need < ctx->num_sms * kChunksPerSM ? need : ctx->num_sms * kChunksPerSM);
    GradArgs b{row_ptr, order, a.capacity, a.V, a.C, chunks < 1 ? 1 : chunks, a.scale, nullptr,
               nullptr, dtable, ctx->status};
    if (chunks > 1) {
        b.part = (float*)stream_workspace(s, (size_t)chunks * (2 * (size_t)a.C + 1) * sizeof(float));
        if (!b.part) return HC_ERR_CUDA;
        b.starts = (int*)(b.part + (size_t)chunks * 2 * a.C);
    }
    return a.dt == HC_BF16 ? run_bwd<__nv_bfloat16>(ctx, b, dy, s)
                           : run_bwd<float>(ctx, b, dy, s);
}

}  // namespace hc
