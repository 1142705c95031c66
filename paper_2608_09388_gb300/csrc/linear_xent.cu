// Softmax cross entropy behind a linear layer, and its gradients, without the
// logits ever being kept. For every token n < N' with a class t[n] >= 0:
//   l[v] = x[n] . W[v] + bias[v],  lse = log sum_v exp(l[v]),  loss = lse - l[t]
//   G[n][v] = dloss[n] * (exp(l[v] - lse) - (v == t))
//   dx = G W,  dW = G^T x,  dbias[v] = sum_n G[n][v]
// The tokens that take part are gathered first, in their order, into M rows
// of the workspace. Forward, a tile of logits leaves a (largest, sum of
// exponentials) pair per row and 64 classes, joined by a last kernel. Backward,
// the vocabulary is taken in pieces: the logits of a piece are formed again,
// G of the piece is written to the workspace in 16 bits, and both products
// with it follow; dx is summed over the pieces in fp32.
//
// All four products are tcgen05 products of bf16 with fp32 accumulators. fp32
// operands (and then G) are held as three bf16 numbers whose sum is the value
// to 2^-24 of it, and six of the nine partial products are summed, the small
// ones first: what is left out is below 2^-24 of a product. For bf16 operands
// G is rounded to bf16 once, as its factors are; its sums over tokens and classes
// stay in fp32. In dx one value of a row may outweigh all others, its target's: what
// the rounding takes off that one is kept in fp32 and added with the row of W
// at the end (8192 of 131072 x 2048: dx off by 0.0027 of its size without, 0.0017
// is the rounding of dx itself).
//
// The products run on pairs of CTAs (cta_group::2): a tile of 256 x 256, 128
// rows of both operands in each CTA's shared memory, and 2 x 256 columns of
// TMEM, so that a tile's epilogue runs under the next one's products.
//
// Measured on a GB300: forward and gradients of 8192 of 131072 x 2048 bf16 10.4 to
// 10.8 ms (17.6 TFLOP at 1.63 to 1.70 PFLOP/s; a plain product sustains 1.72 at the
// power limit), of 2048 of 32000 x 1024 371 to 377 us (284 at the burst rate). There
// the tensor pipe is busy 74 to 83% of the products' time: 13.2 rounds of tiles in
// 14, and a tile of 16 blocks is not much longer than its epilogue. Up to eight tokens go
// to xent_few.cu, small heads to xent_small.cu.
#include "pipeline.cuh"
#include "xent.cuh"

namespace hc {
namespace {

// ---------------------------------------------------------------- layout of a call
struct Rows {
    int* m;            // tokens that take part
    int* row_of;       // [capacity] their row, -1 for the others
    int* token_of;     // [capacity]
    int* target;       // [mpad]
    float* lse;        // [mpad] backward
    float* dloss;      // [mpad] backward
    float* at_target;  // [mpad] forward: the target's logit
    float* rest;       // [mpad] backward, bf16: what rounding took off the target's G
    __nv_bfloat16* x;  // [planes][mpad][pitch]
};

// ---------------------------------------------------------------- gather
__device__ __forceinline__ void planes_of(float v, __nv_bfloat16 (&p)[3]) {
    // an infinity or a NaN is all in the first; what would round to an
    // infinity is cut
    const bool plain = fabsf(v) < __int_as_float(0x7f800000);
    p[0] = fabsf(v) > 0x1.fep127f && plain ? __float2bfloat16_rz(v) : __float2bfloat16_rn(v);
    const float r = plain ? v - __bfloat162float(p[0]) : 0.f;
    p[1] = __float2bfloat16_rn(r);
    p[2] = __float2bfloat16_rn(r - __bfloat162float(p[1]));
}

constexpr int kGatherThreads = 256;

// Sum over the block of small counts.
__device__ __forceinline__ int block_count(int v, int* sh) {
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < kGatherThreads / 32; ++w) v += sh[w];
    return v;
}

struct GatherArgs {
    const void* x;
    const int32_t* targets;
    const int32_t* count;
    long long capacity, mpad;
    int C, V;
    long long pitch;        // of a gathered row
    const float* lse;       // backward
    const float* dloss;
    float* loss_out;        // forward: zero for tokens that take no part
    float* lse_out;
    unsigned* status;
};

// Block b takes the tokens [N' b / blocks, N' (b + 1) / blocks): it counts the
// ones that take part before them, then gives its own their rows in order. The
// last block zeroes the rows up to the next multiple of 64 (a block of the
// products over tokens).
template <typename T>
__global__ void __launch_bounds__(kGatherThreads)
    xent_gather_kernel(const GatherArgs a, const Rows r) {
    constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
    __shared__ int sh[kGatherThreads / 32];
    __shared__ int token[kGatherThreads];
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(a.count, a.capacity, a.status);
    const long long n0 = rows * blockIdx.x / gridDim.x, n1 = rows * (blockIdx.x + 1) / gridDim.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto valid = [&](long long n) {
        const int t = a.targets[n];
        return t >= 0 && t < a.V;
    };
    // the block's first targets are on their way while the ones before are counted
    int ahead = n0 + threadIdx.x < n1 ? a.targets[n0 + threadIdx.x] : -1;
    int before = 0;
#pragma unroll 8
    for (long long n = threadIdx.x; n < n0; n += kGatherThreads) before += valid(n);
    long long at = block_count(before, sh);
    const T* const x = static_cast<const T*>(a.x);
    const bool wide = a.C % 8 == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0;
    for (long long first = n0; first < n1; first += kGatherThreads) {
        const long long n = first + threadIdx.x;
        int t = -1;
        if (n < n1) {
            t = first == n0 ? ahead : a.targets[n];
            if (t < -1 || t >= a.V) {
                report(a.status, kErrIndex);
                t = -1;
            }
            if (t < 0) {
                r.row_of[n] = -1;
                if (a.loss_out) a.loss_out[n] = 0.f;
                if (a.lse_out) a.lse_out[n] = 0.f;
            }
        }
        const unsigned mask = __ballot_sync(0xffffffffu, t >= 0);
        __syncthreads();
        if (lane == 0) sh[warp] = __popc(mask);
        __syncthreads();
        int mine = __popc(mask & ((1u << lane) - 1u)), all = 0;
#pragma unroll
        for (int w = 0; w < kGatherThreads / 32; ++w) {
            if (w < warp) mine += sh[w];
            all += sh[w];
        }
        if (t >= 0) {
            const long long row = at + mine;
            token[mine] = (int)n;
            r.row_of[n] = (int)row;
            r.token_of[row] = (int)n;
            r.target[row] = t;
            if (a.dloss) {
                r.lse[row] = a.lse[n];
                r.dloss[row] = a.dloss[n];
            }
        }
        __syncthreads();
        for (int j = warp; j < all; j += kGatherThreads / 32) {
            const T* const from = x + (long long)token[j] * a.C;
            __nv_bfloat16* const to = r.x + (at + j) * a.pitch;
            if (wide && kPlanes == 1) {
#pragma unroll 4
                for (int c = lane * 8; c < a.C; c += 256)
                    *reinterpret_cast<uint4*>(to + c) = *reinterpret_cast<const uint4*>(from + c);
            } else if (wide) {
#pragma unroll 4
                for (int c = lane * 4; c < a.C; c += 128) {
                    const float4 f = *reinterpret_cast<const float4*>(from + c);
                    __nv_bfloat16 p[4][3];
                    planes_of(f.x, p[0]);
                    planes_of(f.y, p[1]);
                    planes_of(f.z, p[2]);
                    planes_of(f.w, p[3]);
#pragma unroll
                    for (int k = 0; k < kPlanes; ++k) {
                        alignas(8) __nv_bfloat16 q[4] = {p[0][k], p[1][k], p[2][k], p[3][k]};
                        *reinterpret_cast<uint2*>(to + k * a.mpad * a.pitch + c) =
                            *reinterpret_cast<const uint2*>(q);
                    }
                }
            } else {
#pragma unroll 4
                for (int c = lane; c < a.C; c += 32) {
                    __nv_bfloat16 p[3];
                    if constexpr (kPlanes == 1)
                        p[0] = from[c];
                    else
                        planes_of(from[c], p);
#pragma unroll
                    for (int k = 0; k < kPlanes; ++k) to[k * a.mpad * a.pitch + c] = p[k];
                }
            }
        }
        at += all;
    }
    if (blockIdx.x == gridDim.x - 1) {
        if (threadIdx.x == 0) *r.m = (int)at;
        const long long end = (at + 63) / 64 * 64;
        for (int k = 0; k < kPlanes; ++k) {
            // (rows are a multiple of 16 bytes apart)
            uint4* const p = reinterpret_cast<uint4*>(r.x + k * a.mpad * a.pitch);
            for (long long i = at * a.pitch / 8 + threadIdx.x; i < end * a.pitch / 8; i += kGatherThreads)
                p[i] = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

// W in the form the products read where it is not: three planes of bf16, or
// rows with a pitch that is a multiple of 16 bytes. kN channels a lane, where
// rows of fp32 allow it.
template <typename T, int kN>
__global__ void __launch_bounds__(256)
    xent_weight_kernel(const T* __restrict__ W, int V, int C, long long pitch,
                       __nv_bfloat16* __restrict__ out) {
    constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
    pdl_wait();
    pdl_trigger();
    const int warp = (int)((blockIdx.x * 256 + threadIdx.x) >> 5), lane = threadIdx.x & 31;
    for (long long v = warp; v < V; v += (long long)gridDim.x * 8)
#pragma unroll 4
        for (int c = lane * kN; c < C; c += 32 * kN) {
            __nv_bfloat16 p[kN][3];
            if constexpr (kPlanes == 1) {
                p[0][0] = W[v * C + c];
            } else {
                alignas(16) float f[kN];
                if constexpr (kN == 4)
                    *reinterpret_cast<float4*>(f) = *reinterpret_cast<const float4*>(W + v * C + c);
                else if constexpr (kN == 2)
                    *reinterpret_cast<float2*>(f) = *reinterpret_cast<const float2*>(W + v * C + c);
                else
                    f[0] = W[v * C + c];
#pragma unroll
                for (int i = 0; i < kN; ++i) planes_of(f[i], p[i]);
            }
#pragma unroll
            for (int k = 0; k < kPlanes; ++k) {
                __nv_bfloat16* const to = out + (k * (long long)V + v) * pitch + c;
                alignas(8) __nv_bfloat16 q[kN];
#pragma unroll
                for (int i = 0; i < kN; ++i) q[i] = p[i][k];
                if constexpr (kN == 4)
                    *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(q);
                else if constexpr (kN == 2)
                    *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(q);
                else
                    *to = q[0];
            }
        }
}

// ---------------------------------------------------------------- products
enum Product {
    kStats,  // x W^T -> the pairs of the forward pass
    kGrad,   // x W^T -> G of a piece
    kBack,   // G W -> fp32 slabs of dx, and G^T x -> rows of dW or fp32 slabs of them
};

constexpr int kTile = 256;                       // rows of a tile, 128 in each CTA
constexpr int kHalf = 128;
constexpr int kKB = 64;                          // elements per block of the sum: 128 bytes
constexpr int kOperandBytes = kHalf * kKB * 2;   // 16 KiB
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kStages = 5;
// Sixteen warps take a tile from TMEM, 32 rows and kCols columns each: with eight
// the loads, exponentials and stores of a tile of G, one behind the other,
// took longer than its products up to a depth of 1600.
constexpr int kStoreWarps = 16;
constexpr int kCols = 64;
constexpr int kLoadWarp = kStoreWarps;
constexpr int kMmaWarp = kStoreWarps + 1;
constexpr int kThreads = (kStoreWarps + 2) * 32;
constexpr int kOutBytes = 32 * 128;              // staging of a storing warp
constexpr int kGroupM = 16;                      // row tiles walked per column of tiles
// Blocks of the sum behind which the accumulator is added to fp32 registers,
// with fp32 operands and for logits. The tensor cores truncate at every step of 16,
// always towards zero: 784 steps at full size left 1.7e-5 of a weight's
// gradient, 128 steps 1.6e-6 of a loss (1.25e-8 a step). The logits of G are taken
// in the loss's chains, so that what is left in them is in lse too: in chains
// twice as long (2048 of 32000 x 1024 84 us, 88 so) dbias was off by 4e-6, not 5e-7.
// Results that are rounded to bf16 keep one accumulator.
template <Product kP, typename T>
constexpr bool kPromoted = sizeof(T) == 4 || kP != kBack;
template <typename T>
constexpr int kChain = sizeof(T) == 4 ? 4 : 8;
constexpr int kBars = 2 * kStages + 5;
constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + kStoreWarps * kOutBytes + kBars * 8 + 64;
static_assert(kSmem <= 232448, "shared memory of a block");

struct ProductArgs {
    const int* m;        // rows of x and G
    int cols;            // classes of the piece
    int C;
    int bn;              // columns of a tile: 256, 128 or (logits) 64
    int planes;          // 1, or 3: six products a block
    int v0;              // first class of the piece
    const float* bias;
    const int* target;
    const float* lse;
    const float* dloss;
    float* rest;         // kGrad, bf16
    float2* pairs;       // kStats: [classes / kCols][mpad]
    float* at_target;
    float* dbias_part;   // kGrad: [mpad / 32][piece], or NULL
    long long mpad, piece;
    int split;           // kBack: parts of the sums of dx, a slab each; 0: no dx
    int wsplit;          // of dW; 1: its rows directly; 0: no dW
    bool add;            // dx: onto what earlier pieces left
    void* dw;            // rows from v0 on
    bool wide;           // they are 16-byte aligned: stored by TMA
    unsigned* status;
};
struct Maps {
    CUtensorMap a, b, bx, out, out_w;
};

__device__ __forceinline__ uint64_t desc_sw128(uint32_t saddr, uint32_t lbo) {
    // 128-byte swizzle, groups of 8 rows 1024 bytes apart; MN-major: the next
    // 64 columns lbo bytes further on
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(lbo >> 4) << 16) |
           ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc,
                                         uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(da), "l"(db), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Arrive on `bar` of both CTAs once the products issued so far are done.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64"
        " [%0], %1;\n" ::"r"(bar),
        "h"((unsigned short)3)
        : "memory");
}
// Gives the accumulator back. All that has to come before it are the warp's loads
// from TMEM, and those are not ordered by the barrier's memory semantics: they are
// done at tcgen05.wait::ld (by the whole warp), tcgen05.fence::before_thread_sync
// puts them before the arrival, and tcgen05.fence::after_thread_sync behind the
// wait puts the products after it; with that pair of fences the arrival may be
// relaxed. With release semantics it also waited for the global stores of the
// tile before, which nobody waits for here: 1000 clocks a tile.
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(bar)
                 : "memory");
}
// A box of this CTA's, whose bytes are counted by the pair's first CTA.
__device__ __forceinline__ void load_pair(uint32_t dst, const void* tmap, int c0, int c1, int c2,
                                          uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void store_box(const void* tmap, uint32_t src, int c0, int c1, int c2,
                                          bool add) {
    if (add)
        asm volatile(
            "cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group"
            " [%0, {%2, %3, %4}], [%1];\n" ::"l"(reinterpret_cast<uint64_t>(tmap)),
            "r"(src), "r"(c0), "r"(c1), "r"(c2)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group"
            " [%0, {%2, %3, %4}], [%1];\n" ::"l"(reinterpret_cast<uint64_t>(tmap)),
            "r"(src), "r"(c0), "r"(c1), "r"(c2)
            : "memory");
    asm volatile("cp.async.bulk.commit_group;\n" ::: "memory");
}

// The tiles, walked in groups of kGroupM row tiles, the tiles of a group column by
// column, so that the pairs at work share both operands in L2. `at` is the tile's
// place in its group; going on needs no division but in the last group.
struct Walk {
    uint32_t tm, tn, first, in, at;
    __device__ __forceinline__ Walk(uint32_t tm_, uint32_t tn_, uint32_t t) : tm(tm_), tn(tn_) {
        const uint32_t g = t / ((uint32_t)kGroupM * tn);
        first = g * kGroupM;
        at = t - first * tn;
        size();
    }
    __device__ __forceinline__ void size() {
        in = tm - first < (uint32_t)kGroupM ? tm - first : (uint32_t)kGroupM;
    }
    // false behind the last tile
    __device__ __forceinline__ bool go(uint32_t by) {
        at += by;
        while (first < tm && at >= in * tn) {
            at -= in * tn;
            first += kGroupM;
            if (first < tm) size();
        }
        return first < tm;
    }
    __device__ __forceinline__ void tile(int& m, int& n) const {
        n = (int)(in == (uint32_t)kGroupM ? at / (uint32_t)kGroupM : at / in);
        m = (int)(first + at - (uint32_t)n * in);
    }
};

// The planes of operand A and B in product p of six, small ones first.
__device__ __forceinline__ int plane_a(int planes, int p) {
    return planes == 1 ? 0 : (0x021010 >> (4 * (5 - p))) & 3;
}
__device__ __forceinline__ int plane_b(int planes, int p) {
    return planes == 1 ? 0 : (0x201100 >> (4 * (5 - p))) & 3;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// f[j] += bias[j] for the `left` of 32 classes that there are; the same ones
// in every lane, 16 bytes at a time where their address allows it.
__device__ __forceinline__ void add_bias(float (&f)[32], const float* bias, int left) {
    if (left >= 32 && (reinterpret_cast<uintptr_t>(bias) & 15) == 0) {
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
            const float4 b = __ldg(reinterpret_cast<const float4*>(bias + j));
            f[j] += b.x, f[j + 1] += b.y, f[j + 2] += b.z, f[j + 3] += b.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < left) f[j] += __ldg(bias + j);
    }
}

// Sums of v[i] over the warp's lanes, column i in lane i.
__device__ __forceinline__ float column_sums(float (&v)[32]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < o; ++i) {
            const float send = up ? v[i] : v[i + o], keep = up ? v[i + o] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
    }
    return v[0];
}

// G of bf16 operands is held divided by a number in [1, 2) that takes the
// mantissa off the first row's dloss. Where all tokens have the same dloss (a mean
// over tokens), a target far from sure then is a power of two to the last
// place, and rounding it costs nothing; with the mantissa, all of them were
// rounded by the same part (dW off by 0.0019 to 0.0027 of its size by what
// the number of tokens happened to be). Products with G are multiplied by it.
__device__ __forceinline__ float scale_of_g(const float* dloss, int M) {
    if (M <= 0) return 1.f;
    const uint32_t b = __float_as_uint(__ldg(dloss)), e = b & 0x7f800000u;
    return e == 0u || e == 0x7f800000u ? 1.f : __uint_as_float((b & 0x007fffffu) | 0x3f800000u);
}

// What the pair does: a tile of one of the results, and the blocks [k0, k1)
// of its sum.
struct Work {
    bool weight;  // kBack: of dW
    int m, n, part, k0, k1;
};

// The i-th work of pair p of P. kBack has two lists, `first` units that cost
// about `times` as much as the `second` ones: the long ones go round the pairs,
// the pairs that got one less make up for it with short ones, and the rest
// of those goes round again. Returns the unit, counted through both lists.
__device__ __forceinline__ uint32_t scheduled(uint32_t i, uint32_t p, uint32_t P, uint32_t first,
                                              uint32_t second, uint32_t times) {
    const uint32_t r = first % P, mine = first / P + (p < r ? 1u : 0u);
    if (i < mine) return p + i * P;
    i -= mine;
    const uint32_t more = r && p >= r ? times : 0u;
    uint32_t u;
    if (i < more)
        u = p - r + i * (P - r);
    else
        u = (r ? times * (P - r) : 0u) + (p + P - r) % P + (i - more) * P;
    return u < second ? first + u : first + second;
}

template <Product kP, typename T>
__global__ void __launch_bounds__(kThreads, 1)
    xent_product_kernel(const ProductArgs a, const __grid_constant__ Maps maps) {
    constexpr bool kPromote = kPromoted<kP, T>, kPlanes3 = sizeof(T) == 4;
    constexpr bool kBMn = kP == kBack;  // B's rows are along the sum
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    const uint32_t out_at = base + kStages * kStageBytes;
    const uint32_t bars = out_at + kStoreWarps * kOutBytes;
    auto full_bar = [&](uint32_t s) { return bars + 8u * s; };
    auto empty_bar = [&](uint32_t s) { return bars + 8u * (kStages + s); };
    auto tfull_bar = [&](uint32_t b) { return bars + 8u * (2 * kStages + b); };
    auto tempty_bar = [&](uint32_t b) { return bars + 8u * (2 * kStages + 2 + b); };
    const uint32_t fin_bar = bars + 8u * (2 * kStages + 4);
    uint8_t* const misc = smem_raw + (bars - raw) + 8 * kBars;
    volatile uint32_t* const tmem_holder = reinterpret_cast<volatile uint32_t*>(misc);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(misc + 4);
    const uint32_t issued_at = bars + 8u * kBars + 8u;  // copies issued, read by the first CTA
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(tfull_bar(b), 1);
            mbar_init(tempty_bar(b), 2 * kStoreWarps);
        }
        mbar_init(fin_bar, 1);
        *abort_flag = 0;
        sts_s32(issued_at, 0);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        prefetch_tensormap(&maps.a);
        prefetch_tensormap(&maps.b);
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(
                         smem_u32((const void*)tmem_holder)),
                     "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_barrier();  // both CTAs' barriers are there
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;
    pdl_wait();
    pdl_trigger();

    const unsigned long long limit =
        reinterpret_cast<const volatile DeviceWord*>(a.status)->wait_limit_ns;
    const int M = *a.m;
    auto tiles_of = [](long long n, int by) { return (uint32_t)((n + by - 1) / by); };
    const int products = a.planes == 1 ? 1 : 6;
    const uint32_t pair = blockIdx.x >> 1, P = gridDim.x >> 1;
    // tiles and blocks of the logits or of dx, and of dW; unit counts are
    // below 2^31 (checked by the host)
    const uint32_t tm = tiles_of(M, kTile), tn = tiles_of(kP == kBack ? a.C : a.cols, a.bn);
    const uint32_t tmw = tiles_of(a.cols, kTile);
    const int blocks = (int)tiles_of(kP == kBack ? a.cols : a.C, kKB), wblocks = (int)tiles_of(M, kKB);
    const uint32_t units = tm * tn * (kP == kBack ? (uint32_t)a.split : 1u);
    const uint32_t wunits = kP == kBack ? tmw * tn * (uint32_t)a.wsplit : 0u;
    // the list with the longer units goes first
    const int each = a.split > 0 ? blocks / a.split : 0, weach = a.wsplit > 0 ? wblocks / a.wsplit : 0;
    const bool weight_first = kP == kBack && weach > each;
    const uint32_t times =
        (uint32_t)(weight_first ? weach / (each < 1 ? 1 : each) : each / (weach < 1 ? 1 : weach));

    // the logits' tiles go round the pairs
    Walk walk(tm, tn < 1 ? 1 : tn, pair);
    auto work_at = [&](uint32_t i, Work& w) -> bool {
        w.weight = false;
        w.part = 0;
        if constexpr (kP == kBack) {
            uint32_t u = weight_first ? scheduled(i, pair, P, wunits, units, times)
                             : scheduled(i, pair, P, units, wunits, times);
            if (u >= units + wunits) return false;
            w.weight = weight_first ? u < wunits : u >= units;
            if (w.weight != weight_first) u -= weight_first ? wunits : units;
            const uint32_t tiles = (w.weight ? tmw : tm) * tn;
            const int split = w.weight ? a.wsplit : a.split, all = w.weight ? wblocks : blocks;
            w.part = (int)(u / tiles);
            u -= (uint32_t)w.part * tiles;
            w.k0 = (int)((long long)all * w.part / split);
            w.k1 = (int)((long long)all * (w.part + 1) / split);
            const Walk at(w.weight ? tmw : tm, tn, u);
            at.tile(w.m, w.n);
        } else {
            if (i == 0 ? pair >= units : !walk.go(P)) return false;
            w.k0 = 0;
            w.k1 = blocks;
            walk.tile(w.m, w.n);
        }
        return true;
    };

    // In all roles every lane of the warp walks the loop, so that its state is
    // uniform; the copies and products are issued by one lane.
    if (warp == kLoadWarp) {
        const bool leader = elect_one();
        const uint32_t full0 = cluster_map(full_bar(0), 0);  // the first CTA's
        // a box of B holds its rows (the channels are innermost: bn / 2 rows),
        // or 64 columns of 64 rows each
        const uint32_t b_bytes = (uint32_t)a.bn / 2 * kKB * 2;
        const uint32_t both = 2 * (kOperandBytes + b_bytes);
        uint32_t issued = 0;
        bool ok = true;
        Work w;
        for (uint32_t i = 0; ok && work_at(i, w); ++i) {
            const int row = w.m * kTile + (int)rank * kHalf, col = w.n * a.bn + (int)rank * a.bn / 2;
            const int chain = kPromote ? kChain<T> : w.k1 - w.k0;
            for (int kc = w.k0; kc < w.k1 && ok; kc += chain)
                for (int p = 0; p < products && ok; ++p) {
                    const int pa = plane_a(a.planes, p), pb = plane_b(a.planes, p);
                    const int end = w.k1 - kc < chain ? w.k1 : kc + chain;
                    for (int k = kc; k < end; ++k, ++issued) {
                        const uint32_t s = issued % kStages;
                        ok = wait_bar(empty_bar(s), ((issued / kStages) & 1) ^ 1u, abort_flag,
                                      a.status, limit);
                        if (!ok) break;
                        if (leader) {
                            const uint32_t sa = base + s * kStageBytes, sb = sa + kOperandBytes;
                            const uint32_t bar = full0 + 8u * s;
                            const int at = k * kKB;
                            if (rank == 0) mbar_arrive_expect_tx(full_bar(s), both);
                            if constexpr (kP == kBack) {
                                // boxes of 64 rows both ways: G's rows or columns
                                if (w.weight) {
                                    load_pair(sa, &maps.a, row, at, pa, bar);
                                    load_pair(sa + kOperandBytes / 2, &maps.a, row + 64, at, pa, bar);
                                } else {
                                    load_pair(sa, &maps.a, at, row, pa, bar);
                                    load_pair(sa + kOperandBytes / 2, &maps.a, at, row + 64, pa, bar);
                                }
                                const CUtensorMap* const mb = w.weight ? &maps.bx : &maps.b;
                                const int from = w.weight ? at : a.v0 + at;
                                load_pair(sb, mb, col, from, pb, bar);
                                if (a.bn == 256)
                                    load_pair(sb + kOperandBytes / 2, mb, col + 64, from, pb, bar);
                            } else {
                                load_pair(sa, &maps.a, at, row, pa, bar);
                                load_pair(sb, &maps.b, at, a.v0 + col, pb, bar);
                            }
                        }
                        __syncwarp();
                    }
                }
        }
        if (lane == 0) sts_s32(issued_at, (int)issued);
    } else if (warp == kMmaWarp) {
        if (rank == 0) {
            const bool leader = elect_one();
            const uint32_t idesc0 = (1u << 4) | (1u << 7) | (1u << 10) | (kBMn ? 1u << 16 : 0u) |
                                    ((uint32_t)(a.bn >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
            uint32_t it = 0, tile = 0;
            bool ok = true;
            Work w;
            for (uint32_t i = 0; ok && work_at(i, w); ++i) {
                // A of dW is G read along its columns
                const uint32_t idesc = idesc0 | (w.weight ? 1u << 15 : 0u);
                const uint32_t lbo = w.weight ? kOperandBytes / 2 : 16, step = w.weight ? 128 : 2;
                const int chain = kPromote ? kChain<T> : w.k1 - w.k0;
                int kc = w.k0;
                do {  // an empty sum of bf16 operands still passes its accumulator on
                    if (kPromote && kc >= w.k1) break;
                    const uint32_t b = tile & 1;
                    ok = wait_bar(tempty_bar(b), ((tile >> 1) & 1) ^ 1u, abort_flag, a.status, limit);
                    if (!ok) break;
                    tc_fence_after();
                    const int total = (w.k1 - kc < chain ? w.k1 - kc : chain) * products;
                    for (int k = 0; k < total; ++k, ++it) {
                        const uint32_t s = it % kStages;
                        ok = wait_bar(full_bar(s), (it / kStages) & 1, abort_flag, a.status, limit);
                        if (!ok) break;
                        tc_fence_after();
                        if (leader) {
                            const uint32_t sa = base + s * kStageBytes;
                            const uint64_t da = desc_sw128(sa, lbo);
                            const uint64_t db =
                                desc_sw128(sa + kOperandBytes, kBMn ? kOperandBytes / 2 : 16);
#pragma unroll
                            for (int j = 0; j < kKB / 16; ++j)  // 16 elements of the sum further on
                                mma_pair(tmem_base + b * 256u, da + step * j, db + (kBMn ? 128 : 2) * j,
                                         idesc, (k | j) != 0 ? 1u : 0u);
                            commit_pair(empty_bar(s));
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (leader) commit_pair(tfull_bar(b));
                    __syncwarp();
                    ++tile;
                    kc += chain;
                } while (kc < w.k1);
            }
            // every product issued here, and every arrival before this one, has
            // completed once fin_bar fires, in both CTAs
            if (leader) commit_pair(fin_bar);
            __syncwarp();
        }
    } else {
        const int quarter = warp & 3, group = warp >> 2;
        // rows that are used: of G those that the products over tokens take too,
        // whole blocks of them
        const int used = kP == kGrad ? (int)(((long long)M + kKB - 1) / kKB * kKB) : M;
        const uint32_t stage = out_at + (uint32_t)warp * kOutBytes;
        const uint32_t tempty0 = cluster_map(tempty_bar(0), 0);
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const float g_scale = kP != kStats && !kPlanes3 ? scale_of_g(a.dloss, M) : 1.f;
        uint32_t tile = 0;
        bool ok = true;
        Work w;
        for (uint32_t i = 0; work_at(i, w); ++i) {
            const int row0 = w.m * kTile + (int)rank * kHalf + quarter * 32, row = row0 + lane;
            // a narrow tile, or one with few rows, leaves some warps idle
            const bool mine = group * kCols < a.bn && row0 < (w.weight ? a.cols : used);
            // the next accumulator: where it is, and the barrier that gives it back
            uint32_t acc = 0, tempty = 0;
            auto next = [&] {
                const uint32_t b = tile & 1;
                ok = wait_bar(tfull_bar(b), (tile >> 1) & 1, abort_flag, a.status, limit);
                tc_fence_after();
                acc = tmem_base + lanes + b * 256u + (uint32_t)(group * kCols);
                tempty = tempty0 + 8u * b;
                ++tile;
            };
            auto give_back = [&] {
                tc_fence_before();
                if (lane == 0) arrive_cluster(tempty);
            };
            // 32 columns of this lane's row from the accumulator, which is given
            // back with the last ones
            auto direct = [&](int c, float (&f)[32]) {
                uint32_t r[32];
                tmem_ld_32x32b_x32(acc + (uint32_t)c, r);
                tmem_ld_wait();
                if (c + 32 == kCols) give_back();
#pragma unroll
                for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(r[j]);
                if (kP == kBack && w.k1 == w.k0) {  // an empty sum
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[j] = 0.f;
                }
            };
            const int col0 = w.n * a.bn + group * kCols;
            // 128 bytes of each of the warp's rows, swizzled, then one box
            auto staging_free = [&] {
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory");
                __syncwarp();
            };
            auto put = [&](int q, uint4 v) { sts_v4(stage + lane * 128 + ((q ^ (lane & 7)) << 4), v); };
            auto send = [&](const CUtensorMap* map, int c0, int c1, int c2, bool add) {
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) store_box(map, stage, c0, c1, c2, add);
            };
            auto pack = [](float lo, float hi) { return Piece<__nv_bfloat16, 8>::pair(lo, hi); };

            auto finish = [&](auto load, auto load_all) {
            if constexpr (kP == kStats) {
                const int target = row < M ? a.target[row] : -1;
                const float least = -__int_as_float(0x7f800000);
                float f[kCols];
                load_all(f);
                if (a.bias) {
                    add_bias(reinterpret_cast<float (&)[32]>(f[0]), a.bias + col0, a.cols - col0);
                    add_bias(reinterpret_cast<float (&)[32]>(f[32]), a.bias + col0 + 32, a.cols - col0 - 32);
                }
                if (col0 + kCols > a.cols) {
#pragma unroll
                    for (int j = 0; j < kCols; ++j)
                        if (col0 + j >= a.cols) f[j] = least;
                }
                float m4[4] = {least, least, least, least};
#pragma unroll
                for (int j = 0; j < kCols; j += 2) m4[j / 2 & 3] = max3(m4[j / 2 & 3], f[j], f[j + 1]);
                const float top = max3(fmaxf(m4[0], m4[1]), m4[2], m4[3]);
                if (target >= col0 && target < col0 + kCols) {
                    float v = 0.f;
#pragma unroll
                    for (int j = 0; j < kCols; ++j) v = col0 + j == target ? f[j] : v;
                    a.at_target[row] = v;
                }
                // classes masked with -infinity leave it at that; a NaN goes
                // past the maximum and into the sum
                const float from = top == least ? 0.f : top;
                const F2 less = make_f2(-from, -from), scale = make_f2(kLog2e, kLog2e);
                F2 s4[4];
#pragma unroll
                for (int j = 0; j < kCols; j += 2) {
                    const float2 e = split(mul(add(make_f2(f[j], f[j + 1]), less), scale));
                    const F2 p = make_f2(ex2(e.x), ex2(e.y));
                    s4[j / 2 & 3] = j < 8 ? p : add(s4[j / 2 & 3], p);
                }
                const float sum = total(add(add(s4[0], s4[1]), add(s4[2], s4[3])));
                if (row < M && col0 < a.cols)
                    a.pairs[(long long)(col0 / kCols) * a.mpad + row] = make_float2(top, sum);
            } else if constexpr (kP == kGrad) {
                const bool in = row < M;
                const float lse = in ? a.lse[row] : 0.f;
                const float dloss = in ? a.dloss[row] / g_scale : 0.f;
                const int target = in ? a.target[row] - a.v0 : -1;
                // the whole of it inside: no looks at rows and columns
                const bool whole = row0 + 32 <= M && col0 + kCols <= a.cols;
                [[maybe_unused]] float keep[kPlanes3 ? kCols : 1];
                if (!kPlanes3) staging_free();
#pragma unroll
                for (int c = 0; c < kCols; c += 32) {
                    float f[32];
                    load(c, f);
                    const int col = col0 + c;
                    if (a.bias) add_bias(f, a.bias + a.v0 + col, a.cols - col);
                    const F2 less = make_f2(-lse, -lse), scale = make_f2(kLog2e, kLog2e);
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        const float2 e = split(mul(add(make_f2(f[j], f[j + 1]), less), scale));
                        f[j] = ex2(e.x);
                        f[j + 1] = ex2(e.y);
                    }
                    if (target >= col && target < col + 32) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) f[j] -= col + j == target ? 1.f : 0.f;
                    }
                    if (whole) {
                        const F2 times = make_f2(dloss, dloss);
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const float2 e = split(mul(make_f2(f[j], f[j + 1]), times));
                            f[j] = e.x;
                            f[j + 1] = e.y;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            f[j] = in && col + j < a.cols ? f[j] * dloss : 0.f;
                    }
                    if constexpr (kPlanes3) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) keep[c + j] = f[j];
                    } else {
                        if (target >= col && target < col + 32) {
                            float v = 0.f;
#pragma unroll
                            for (int j = 0; j < 32; ++j) v = col + j == target ? f[j] : v;
                            a.rest[row] = (v - __bfloat162float(__float2bfloat16_rn(v))) * g_scale;
                        }
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            put(c / 8 + q,
                                make_uint4(pack(f[8 * q], f[8 * q + 1]), pack(f[8 * q + 2], f[8 * q + 3]),
                                           pack(f[8 * q + 4], f[8 * q + 5]), pack(f[8 * q + 6], f[8 * q + 7])));
                    }
                    if (a.dbias_part) {
                        const float s = column_sums(f);
                        if (col + lane < a.cols)
                            a.dbias_part[(long long)(row0 / 32) * a.piece + col + lane] = s * g_scale;
                    }
                }
                if constexpr (kPlanes3) {
                    // three planes, each what the ones before leave
#pragma unroll
                    for (int k = 0; k < 3; ++k) {
                        staging_free();
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            float v[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                v[j] = __bfloat162float(__float2bfloat16_rn(keep[8 * q + j]));
                                keep[8 * q + j] -= v[j];
                            }
                            put(q, make_uint4(pack(v[0], v[1]), pack(v[2], v[3]), pack(v[4], v[5]),
                                              pack(v[6], v[7])));
                        }
                        send(&maps.out, col0, row0, k, false);
                    }
                } else {
                    send(&maps.out, col0, row0, 0, false);
                }
            } else if (!w.weight || kPromote || a.wsplit > 1) {
                // fp32 results, 32 columns at a time
                const bool slab = !w.weight || a.wsplit > 1;
                const CUtensorMap* const map = w.weight ? &maps.out_w : &maps.out;
                const int rows = w.weight ? a.cols : M;
#pragma unroll
                for (int c = 0; c < kCols; c += 32) {
                    float f[32];
                    load(c, f);
                    staging_free();
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        put(q, make_uint4(__float_as_uint(f[4 * q]), __float_as_uint(f[4 * q + 1]),
                                          __float_as_uint(f[4 * q + 2]), __float_as_uint(f[4 * q + 3])));
                    const int col = col0 + c;
                    if (slab) {
                        if (col < a.C) send(map, col, row0, w.part, !w.weight && a.add);
                    } else if (a.wide) {
                        if (col < a.C && row0 < rows) send(map, col, a.v0 + row0, 0, false);
                    } else {
                        __syncwarp();
                        for (int r = 0; r < 32; ++r) {
                            const uint32_t at = stage + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4;
                            if (row0 + r < rows && col + lane < a.C)
                                static_cast<float*>(a.dw)[(long long)(a.v0 + row0 + r) * a.C + col + lane] =
                                    __int_as_float(lds_s32(at));
                        }
                        __syncwarp();
                    }
                }
            } else {
                // bf16 rows of dW, 64 columns
                staging_free();
#pragma unroll
                for (int c = 0; c < kCols; c += 32) {
                    float f[32];
                    load(c, f);
#pragma unroll
                    for (int j = 0; j < 32; ++j) f[j] *= g_scale;
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        put(c / 8 + q,
                            make_uint4(pack(f[8 * q], f[8 * q + 1]), pack(f[8 * q + 2], f[8 * q + 3]),
                                       pack(f[8 * q + 4], f[8 * q + 5]), pack(f[8 * q + 6], f[8 * q + 7])));
                }
                if (a.wide) {
                    if (col0 < a.C && row0 < a.cols) send(&maps.out_w, col0, a.v0 + row0, 0, false);
                } else {
                    __syncwarp();
                    // two values a lane where the row's place in memory allows it; with
                    // the row one off, its first and last go by themselves
                    auto value = [&](int r, int j) {
                        const uint32_t at = stage + r * 128 + (((j >> 3) ^ (r & 7)) << 4) + (j & 7) * 2;
                        uint16_t v;
                        asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(v) : "r"(at) : "memory");
                        return v;
                    };
                    for (int r = 0; r < 32; ++r) {
                        if (row0 + r >= a.cols) break;
                        uint16_t* const to = static_cast<uint16_t*>(a.dw) +
                                             (long long)(a.v0 + row0 + r) * a.C + col0;
                        const int left = a.C - col0, off = (int)(reinterpret_cast<uintptr_t>(to) >> 1 & 1);
                        const int j = 2 * lane + off;
                        const uint16_t lo = value(r, j), hi = value(r, j + 1 < kCols ? j + 1 : 0);
                        if (j + 1 < kCols && j + 1 < left)
                            *reinterpret_cast<uint32_t*>(to + j) = (uint32_t)hi << 16 | lo;
                        else if (j < left)
                            to[j] = lo;
                        if (j + 1 == kCols && left > 0) to[0] = hi;
                    }
                    __syncwarp();
                }
            }
            };
            // one accumulator holds the whole sum, or its chains are added up here
            if (!kPromote || (w.k1 > w.k0 && w.k1 - w.k0 <= kChain<T>)) {
                next();
                if (!ok) break;
                if (mine)
                    finish(direct, [&](float (&f)[kCols]) {
                        uint32_t r0[32], r1[32];
                        tmem_ld_32x32b_x32(acc, r0);
                        tmem_ld_32x32b_x32(acc + 32u, r1);
                        tmem_ld_wait();
                        give_back();
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            f[j] = __uint_as_float(r0[j]);
                            f[32 + j] = __uint_as_float(r1[j]);
                        }
                    });
                else
                    give_back();
            } else {
                float sums[kCols];
#pragma unroll
                for (int j = 0; j < kCols; ++j) sums[j] = 0.f;
                for (int kc = w.k0; kc < w.k1 && ok; kc += kChain<T>) {
                    next();
                    if (!ok) break;
                    if (!mine) {
                        give_back();
                        continue;
                    }
#pragma unroll
                    for (int c = 0; c < kCols; c += 16) {
                        uint32_t r[16];
                        tmem_ld(acc + (uint32_t)c, r);
                        tmem_ld_wait();
                        if (c + 16 == kCols) give_back();
#pragma unroll
                        for (int j = 0; j < 16; ++j) sums[c + j] += __uint_as_float(r[j]);
                    }
                }
                if (!ok) break;
                if (mine)
                    finish(
                        [&](int c, float (&f)[32]) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) f[j] = sums[c + j];
                        },
                        [&](float (&f)[kCols]) {
#pragma unroll
                            for (int j = 0; j < kCols; ++j) f[j] = sums[j];
                        });
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory");
        __syncwarp();
    }

    // The copies already issued land before either CTA ends, also where a role
    // gave up: the first CTA's barriers count the bytes of both. A copy that one
    // CTA issued and the other did not is counted for both by hand.
    __syncthreads();
    cluster_barrier();
    if (warp == kMmaWarp && lane == 0) mbar_wait_drain(fin_bar, 0, a.status);
    if (rank == 0 && warp == kLoadWarp && lane == 0) {
        const uint32_t mine = (uint32_t)lds_s32(issued_at);
        uint32_t other;
        asm volatile("ld.shared::cluster.u32 %0, [%1];\n"
                     : "=r"(other)
                     : "r"(cluster_map(issued_at, 1))
                     : "memory");
        const uint32_t most = mine > other ? mine : other;
        const uint32_t one = kOperandBytes + (uint32_t)a.bn / 2 * kKB * 2;
        for (uint32_t j = most > kStages ? most - kStages : 0; j < most; ++j) {
            const uint32_t bar = full_bar(j % kStages);
            if (j >= mine)
                mbar_arrive_expect_tx(bar, one);
            else if (j >= other)
                asm volatile("mbarrier.complete_tx.relaxed.cluster.shared::cta.b64 [%0], %1;\n" ::"r"(
                                 bar),
                             "r"(one)
                             : "memory");
            mbar_wait_drain(bar, (j / kStages) & 1, a.status);
        }
    }
    __syncwarp();
    cluster_barrier();
    if (warp == kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem_base),
                     "r"(512)
                     : "memory");
    }
}

// ---------------------------------------------------------------- joins
// The pairs of a row -> loss and lse: 8 rows a block (64 neighbouring bytes of a
// part), every 128th part a thread; then a warp per row. Rows may be few
// and parts many: 1152 rows of 1261 parts took 25 us with 32 rows a block.
constexpr int kLossRows = 8, kLossThreads = 1024, kLossParts = kLossThreads / kLossRows;

__global__ void __launch_bounds__(kLossThreads)
    xent_loss_kernel(const Rows r, const float2* __restrict__ pairs, int parts, long long mpad,
                     float* loss, float* lse) {
    __shared__ float2 sh[kLossRows][kLossParts + 1];
    pdl_wait();
    pdl_trigger();
    const int M = *r.m, sub = threadIdx.x % kLossRows, first = threadIdx.x / kLossRows;
    const float least = -__int_as_float(0x7f800000);
    for (long long row0 = blockIdx.x * (long long)kLossRows; row0 < M;
         row0 += gridDim.x * (long long)kLossRows) {
        float2 p = make_float2(least, 0.f);
        if (row0 + sub < M) {
            constexpr int kLoads = 4;
            for (int h = first; h < parts; h += kLossParts * kLoads) {
                float2 q[kLoads];
#pragma unroll
                for (int k = 0; k < kLoads; ++k)
                    q[k] = h + kLossParts * k < parts
                               ? pairs[(h + (long long)kLossParts * k) * mpad + row0 + sub]
                               : make_float2(least, 0.f);
                p = join_pairs(p, join_pairs(join_pairs(q[0], q[1]), join_pairs(q[2], q[3])));
            }
        }
        __syncthreads();
        sh[sub][first] = p;
        __syncthreads();
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const long long row = row0 + warp;
        if (warp < kLossRows && row < M) {
            p = sh[warp][lane];
#pragma unroll
            for (int k = 32; k < kLossParts; k += 32) p = join_pairs(p, sh[warp][lane + k]);
            p = join_lanes<32>(p);
            if (lane == 0) {
                const float all = p.x + logf(p.y);
                const int n = r.token_of[row];
                if (lse) lse[n] = all;
                if (loss) loss[n] = all - r.at_target[row];
            }
        }
    }
}

// Rows of a result from its slabs. dx: the rows n < N', zero for tokens that
// take no part, with the `rest` of the target's G times its row of W where there
// is one; a piece of dW: all its rows. Four channels a lane.
template <typename T>
__global__ void __launch_bounds__(256)
    xent_slabs_kernel(const int32_t* count, long long capacity, const int* row_of,
                      const float* __restrict__ slabs, int split, long long slab_rows, long long pitch,
                      int C, bool wide, const float* __restrict__ rest, const int* __restrict__ target,
                      const T* __restrict__ W, const float* __restrict__ dloss, const int* m, T* out,
                      unsigned* status) {
    pdl_wait();
    pdl_trigger();
    const long long rows = token_rows(count, capacity, status);
    // a row's pieces of 128 channels, one after another
    const int lane = threadIdx.x & 31, per = (C + 127) / 128;
    const float g_scale = sizeof(T) == 4 ? 1.f : scale_of_g(dloss, *m);
    const long long step = (long long)gridDim.x * 8;
    for (long long i = (blockIdx.x * 256 + threadIdx.x) >> 5; i < rows * per; i += step) {
        int k;
        const long long n = div32(i, per, k);
        const int c = k * 128 + lane * 4;
        const long long row = row_of ? row_of[n] : n;
        if (c >= C) continue;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row >= 0) {
#pragma unroll 8
            for (int s = 0; s < split; ++s) {
                const float4 f = *reinterpret_cast<const float4*>(slabs + (s * slab_rows + row) * pitch + c);
                v.x += f.x, v.y += f.y, v.z += f.z, v.w += f.w;
            }
            v.x *= g_scale, v.y *= g_scale, v.z *= g_scale, v.w *= g_scale;
            if (rest) {
                const float by = rest[row];
                const T* const w = W + (long long)target[row] * C + c;
                float f[4];
                if (wide) {
                    Piece<T, 4> q;
                    q.load(w);
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] = q.get(e);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] = c + e < C ? to_f32(w[e]) : 0.f;
                }
                v.x = fmaf(by, f[0], v.x), v.y = fmaf(by, f[1], v.y);
                v.z = fmaf(by, f[2], v.z), v.w = fmaf(by, f[3], v.w);
            }
        }
        T* const to = out + n * C + c;
        if (wide) {
            if constexpr (sizeof(T) == 4)
                *reinterpret_cast<float4*>(to) = v;
            else
                *reinterpret_cast<uint2*>(to) = make_uint2(Piece<__nv_bfloat16, 8>::pair(v.x, v.y),
                                                           Piece<__nv_bfloat16, 8>::pair(v.z, v.w));
        } else {
            const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < C) to[e] = from_f32<T>(f[e]);
        }
    }
}

// ---------------------------------------------------------------- host side
// A 3-D map over [planes][rows][cols] elements, boxes of box_rows x 128 bytes
// with 128-byte swizzle; what lies outside reads as zero and is not written.
hc_status encode(CUtensorMap* m, CUtensorMapDataType type, const void* base, long long cols,
                 long long rows, int planes, long long pitch, int box_rows) {
    auto enc = tensor_map_encoder();
    if (!enc) {
        set_error("cuTensorMapEncodeTiled is unavailable");
        return HC_ERR_CUDA;
    }
    const int e = type == CU_TENSOR_MAP_DATA_TYPE_FLOAT32 ? 4 : 2;
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    cuuint64_t strides[2] = {(cuuint64_t)(pitch * e), (cuuint64_t)(pitch * e * rows)};
    cuuint32_t box[3] = {(cuuint32_t)(128 / e), (cuuint32_t)box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = enc(m, type, 3, const_cast<void*>(base), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_error("cuTensorMapEncodeTiled failed (%d)", (int)r);
        return HC_ERR_CUDA;
    }
    return HC_OK;
}
constexpr CUtensorMapDataType kBf16 = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
constexpr CUtensorMapDataType kF32 = CU_TENSOR_MAP_DATA_TYPE_FLOAT32;

template <Product kP, typename T>
hc_status product(const DeviceCtx* ctx, const ProductArgs& a, long long units, const Maps& maps, cudaStream_t s) {
    if (units > 0x7fffffffll) {
        set_error("cross entropy: %lld tiles are too many", units);
        return HC_ERR_UNSUPPORTED;
    }
    const long long pairs = ctx->num_sms / 2;
    const unsigned grid = (unsigned)(2 * (units < 1 ? 1 : units < pairs ? units : pairs));
    auto kern = xent_product_kernel<kP, T>;
    static bool done[64];
    if (!done[ctx->device]) {
        const hc_status st = check_cuda(
            cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem),
            "xent_product_kernel");
        if (st != HC_OK) return st;
        done[ctx->device] = true;
    }
    return launch_cluster(kern, grid, 2, kThreads, kSmem, s, "xent_product_kernel", a, maps);
}

long long up(long long v, long long to) {
    return (v + to - 1) / to * to;
}

// The workspace of a call, laid out part by part: once to count, once to place.
struct Layout {
    uint8_t* base;
    size_t used = 0;
    template <typename P>
    P* take(size_t n) {
        P* const p = reinterpret_cast<P*>(base + used);
        used = (used + n * sizeof(P) + 255) / 256 * 256;
        return p;
    }
};

template <typename T>
struct Call {
    static constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
    const DeviceCtx* ctx;
    const LinearXentArgs& a;
    cudaStream_t s;
    long long mpad, pitch;
    bool direct;         // the products read W where it is
    Rows r{};
    __nv_bfloat16* w = nullptr;

    Call(const DeviceCtx* ctx_, const LinearXentArgs& a_, cudaStream_t s_) : ctx(ctx_), a(a_), s(s_) {
        mpad = up(a.capacity < 1 ? 1 : a.capacity, kTile);
        pitch = up(a.C, 8);
        direct = kPlanes == 1 && a.C % 8 == 0 && (reinterpret_cast<uintptr_t>(a.W) & 15) == 0;
    }
    void rows(Layout& l, bool back) {
        r.m = l.take<int>(1);
        r.row_of = l.take<int>(mpad);
        r.token_of = l.take<int>(mpad);
        r.target = l.take<int>(mpad);
        if (back) {
            r.lse = l.take<float>(mpad);
            r.dloss = l.take<float>(mpad);
            r.rest = l.take<float>(mpad);
        } else {
            r.at_target = l.take<float>(mpad);
        }
        r.x = l.take<__nv_bfloat16>((size_t)kPlanes * mpad * pitch);
        if (!direct) w = l.take<__nv_bfloat16>((size_t)kPlanes * a.V * pitch);
    }
    hc_status gather(bool back) {
        GatherArgs g{a.x, a.targets, a.count, a.capacity, mpad, a.C, a.V, pitch,
                     back ? a.lse : nullptr, back ? a.dloss : nullptr, back ? nullptr : a.loss_out,
                     back ? nullptr : a.lse_out, ctx->status};
        const long long need = ((long long)a.capacity + 7) / 8, cap = 8ll * ctx->num_sms;
        hc_status st = launch_pdl(xent_gather_kernel<T>,
                                  dim3((unsigned)(need < 1 ? 1 : need < cap ? need : cap)),
                                  dim3(kGatherThreads), 0, s, "xent_gather_kernel", g, r);
        if (st != HC_OK || direct) return st;
        const long long wneed = ((long long)a.V + 7) / 8, wcap = 8ll * ctx->num_sms;
        const uintptr_t at = reinterpret_cast<uintptr_t>(a.W);
        auto kern = xent_weight_kernel<T, 1>;
        if constexpr (kPlanes == 3) {
            if (a.C % 4 == 0 && a.C >= 128 && at % 16 == 0)
                kern = xent_weight_kernel<T, 4>;
            else if (a.C % 2 == 0 && a.C >= 64 && at % 8 == 0)
                kern = xent_weight_kernel<T, 2>;
        }
        return launch_pdl(kern, dim3((unsigned)(wneed < wcap ? wneed : wcap)), dim3(256), 0, s,
                          "xent_weight_kernel", (const T*)a.W, a.V, a.C, pitch, w);
    }
    hc_status map_x(CUtensorMap* m, int box) {
        return encode(m, kBf16, r.x, a.C, mpad, kPlanes, pitch, box);
    }
    hc_status map_w(CUtensorMap* m, int box) {
        return encode(m, kBf16, direct ? a.W : (const void*)w, a.C, a.V, kPlanes,
                      direct ? a.C : pitch, box);
    }

    // Columns of a tile of logits: the ones whose rounds over the pairs of SMs take
    // least. A block of the sum takes 512 clocks with 256 columns, about 380 and
    // 320 with 128 and 64, which the loads bound (79 tokens of 113 x 2036 fp32: 63 us in
    // one tile of 256, 50 in two of 64).
    int columns(long long classes) const {
        const long long pairs = ctx->num_sms / 2;
        auto cost = [&](int bn) {
            const long long units = mpad / kTile * ((classes + bn - 1) / bn);
            return (units + pairs - 1) / pairs * (bn == 256 ? 8 : bn == 128 ? 6 : 5);
        };
        int bn = 256;
        if (cost(128) < cost(bn)) bn = 128;
        if (cost(64) < cost(bn)) bn = 64;
        return bn;
    }

    // The rows of `out` from `split` slabs (row_of: dx, else a piece of dW).
    hc_status join(const int32_t* count, long long rows_, const int* row_of, const float* slabs, int split,
                   long long slab_rows, long long xpitch, T* out) {
        const float* const rest = row_of && kPlanes == 1 ? r.rest : nullptr;
        auto aligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & (4 * sizeof(T) - 1)) == 0; };
        const bool wide = a.C % 4 == 0 && aligned(out) && (!rest || aligned(a.W));
        const long long need = (rows_ * ((a.C + 127) / 128) + 7) / 8, cap = 8ll * ctx->num_sms;
        return launch_pdl(xent_slabs_kernel<T>, dim3((unsigned)(need < cap ? need : cap)), dim3(256), 0, s,
                          "xent_slabs_kernel", count, rows_, row_of, slabs, split, slab_rows, xpitch, a.C,
                          wide, rest, (const int*)r.target, (const T*)a.W, (const float*)r.dloss, (const int*)r.m, out,
                          ctx->status);
    }

    hc_status forward() {
        const int bn = columns(a.V);
        const int parts = (int)(((long long)a.V + kCols - 1) / kCols);
        float2* pairs = nullptr;
        auto place = [&](Layout l) {
            rows(l, false);
            pairs = l.take<float2>((size_t)parts * mpad);
            return l.used;
        };
        uint8_t* const ws = (uint8_t*)stream_workspace(s, place({nullptr}));
        if (!ws) return HC_ERR_CUDA;
        place({ws});
        hc_status st = gather(false);
        if (st != HC_OK) return st;
        Maps maps{};
        if ((st = map_x(&maps.a, kHalf)) != HC_OK || (st = map_w(&maps.b, bn / 2)) != HC_OK) return st;
        ProductArgs p{};
        p.m = r.m;
        p.cols = a.V;
        p.C = a.C;
        p.bn = bn;
        p.planes = kPlanes;
        p.bias = a.bias;
        p.target = r.target;
        p.pairs = pairs;
        p.at_target = r.at_target;
        p.mpad = mpad;
        p.status = ctx->status;
        st = product<kStats, T>(ctx, p, mpad / kTile * ((a.V + (long long)bn - 1) / bn), maps, s);
        if (st != HC_OK) return st;
        const long long need = ((long long)a.capacity + kLossRows - 1) / kLossRows, cap = 2ll * ctx->num_sms;
        return launch_pdl(xent_loss_kernel, dim3((unsigned)(need < cap ? need : cap)), dim3(kLossThreads), 0, s,
                          "xent_loss_kernel", r, (const float2*)pairs, parts, mpad, a.loss_out, a.lse_out);
    }

    hc_status backward() {
        // pieces of the vocabulary: G of one takes at most 512 MiB, or 2048 classes
        const long long classes_all = up(a.V, kTile);
        long long most = (512ll << 20) / (mpad * 2 * kPlanes) / kTile * kTile;
        if (most < 2048) most = 2048;
        const long long pieces = (classes_all + most - 1) / most;
        const long long piece = up((classes_all + pieces - 1) / pieces, kTile);
        const long long xpitch = up(a.C, 4);
        const int bn_v = columns(piece < a.V ? piece : a.V), bn_c = a.C <= 128 ? 128 : 256;
        const long long tiles = mpad / kTile * ((a.C + bn_c - 1) / bn_c);
        // dx may have few tiles with long sums. They go first and the tiles of dW
        // fill up behind them, so that a part of a sum may be as long as two thirds of
        // a pair's whole work (2048 of 32000 x 1024: two parts; eight of them
        // cost 15 us for the slabs alone); 1024 classes at least. The same parts
        // without dW, so that dx does not depend on what else is asked for.
        const int pairs = ctx->num_sms / 2;
        const long long sum = piece / kKB;
        const long long all = tiles * sum + piece / kTile * ((a.C + bn_c - 1) / bn_c) * (mpad / kKB);
        long long split = (3 * sum * pairs + 2 * all - 1) / (2 * all);
        if (split > piece / 1024) split = piece / 1024;
        if (split < 1 || !a.dx) split = 1;
        // so has dW with few classes; 256 tokens at least
        const long long wtiles = piece / kTile * ((a.C + bn_c - 1) / bn_c);
        long long wsplit = pairs / wtiles;
        if (wsplit > a.capacity / 256) wsplit = a.capacity / 256;
        if (wsplit < 1 || !a.dW) wsplit = 1;
        __nv_bfloat16* G = nullptr;
        float *slabs = nullptr, *wslabs = nullptr, *part = nullptr;
        auto place = [&](Layout l) {
            rows(l, true);
            G = l.take<__nv_bfloat16>((size_t)kPlanes * mpad * piece);
            if (a.dx) slabs = l.take<float>((size_t)split * mpad * xpitch);
            if (wsplit > 1) wslabs = l.take<float>((size_t)wsplit * piece * xpitch);
            if (a.dbias) part = l.take<float>((size_t)(mpad / 32) * piece);
            return l.used;
        };
        uint8_t* const ws = (uint8_t*)stream_workspace(s, place({nullptr}));
        if (!ws) return HC_ERR_CUDA;
        place({ws});
        hc_status st = gather(true);
        if (st != HC_OK) return st;
        Maps grad{}, back{};
        const bool wide = (a.C * sizeof(T)) % 16 == 0 && (reinterpret_cast<uintptr_t>(a.dW) & 15) == 0;
        if ((st = map_x(&grad.a, kHalf)) != HC_OK || (st = map_w(&grad.b, bn_v / 2)) != HC_OK ||
            (st = encode(&grad.out, kBf16, G, piece, mpad, kPlanes, piece, 32)) != HC_OK ||
            (st = encode(&back.a, kBf16, G, piece, mpad, kPlanes, piece, kKB)) != HC_OK ||
            (st = map_w(&back.b, kKB)) != HC_OK || (st = map_x(&back.bx, kKB)) != HC_OK)
            return st;
        if (a.dx && (st = encode(&back.out, kF32, slabs, a.C, mpad, (int)split, xpitch, 32)) != HC_OK) return st;
        if (wsplit > 1)
            st = encode(&back.out_w, kF32, wslabs, a.C, piece, (int)wsplit, xpitch, 32);
        else if (a.dW && wide)
            st = encode(&back.out_w, sizeof(T) == 4 ? kF32 : kBf16, a.dW, a.C, a.V, 1, a.C, 32);
        if (st != HC_OK) return st;
        ProductArgs p{};
        p.m = r.m;
        p.C = a.C;
        p.planes = kPlanes;
        p.bias = a.bias;
        p.target = r.target;
        p.lse = r.lse;
        p.dloss = r.dloss;
        p.rest = r.rest;
        p.dbias_part = part;
        p.mpad = mpad;
        p.piece = piece;
        p.split = a.dx ? (int)split : 0;
        p.wsplit = a.dW ? (int)wsplit : 0;
        p.dw = a.dW;
        p.wide = wide;
        p.status = ctx->status;
        for (long long v0 = 0; v0 < a.V; v0 += piece) {
            const int classes = (int)(a.V - v0 < piece ? a.V - v0 : piece);
            p.v0 = (int)v0;
            p.cols = classes;
            p.bn = bn_v;
            p.add = v0 > 0;
            st = product<kGrad, T>(ctx, p, mpad / kTile * ((classes + bn_v - 1) / bn_v), grad, s);
            if (st != HC_OK) return st;
            if (a.dbias) {
                st = launch_column_sum(part, (int)(mpad / 32), piece, classes, a.dbias + v0, s, r.m);
                if (st != HC_OK) return st;
            }
            if (!a.dx && !a.dW) continue;
            p.bn = bn_c;
            const long long units = tiles * p.split + ((long long)classes + kTile - 1) / kTile *
                                                          ((a.C + bn_c - 1) / bn_c) * p.wsplit;
            st = product<kBack, T>(ctx, p, units, back, s);
            if (st != HC_OK) return st;
            if (p.wsplit > 1) {
                st = join(nullptr, classes, nullptr, wslabs, (int)wsplit, piece, xpitch,
                          (T*)a.dW + v0 * a.C);
                if (st != HC_OK) return st;
            }
        }
        if (!a.dx || a.capacity == 0) return HC_OK;
        return join(a.count, a.capacity, r.row_of, slabs, (int)split, mpad, xpitch, (T*)a.dx);
    }
};

}  // namespace

hc_status launch_linear_xent_fwd(const DeviceCtx* ctx, const LinearXentArgs& a, cudaStream_t s) {
    if (xent_small_supported(a)) return launch_xent_small_fwd(ctx, a, s);
    if (xent_few_supported(a)) return launch_xent_few_fwd(ctx, a, s);
    return a.dt == HC_BF16 ? Call<__nv_bfloat16>(ctx, a, s).forward() : Call<float>(ctx, a, s).forward();
}

hc_status launch_linear_xent_bwd(const DeviceCtx* ctx, const LinearXentArgs& a, cudaStream_t s) {
    if (xent_small_supported(a)) return launch_xent_small_bwd(ctx, a, s);
    if (xent_few_supported(a)) return launch_xent_few_bwd(ctx, a, s);
    return a.dt == HC_BF16 ? Call<__nv_bfloat16>(ctx, a, s).backward() : Call<float>(ctx, a, s).backward();
}

}  // namespace hc
