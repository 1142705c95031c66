// The 8-bit linear layer on compact rows:
//   y[n][o] = act( bias[o] + sum over blocks b of 128 channels of
//                  xs[b][n] * ws[o / 128][b] * sum_{c in b} xq[n][c] * wq[o][c] )
// on the tensor cores (tcgen05 kind::f8f6f4, e4m3 x e4m3). Products of e4m3
// values are exact in fp32; a block's 128 products are summed in the TMEM
// accumulator, then the block sum is scaled and added to the fp32 total in
// registers ("promotion"): the scales change from block to block, so an
// accumulator cannot run on over the blocks.
//
// A tile is 128 TMEM lanes x BN columns. Two orientations:
//   rows on lanes (BN = 128 or 256): lane = token, column = output channel.
//     The scale of a block is one number per thread.
//   channels on lanes (BN = 16, 32, 64; at most 64 tokens): lane = output
//     channel, column = token. A few tokens fill a narrow MMA instead of a
//     mostly empty 128-row tile, and the weight, which is all the traffic of
//     such a call, is read once, 128 output channels at a time.
// With fewer tiles than SMs the channel blocks of a tile are split over a
// cluster of 2, 4 or 8 CTAs, whose totals are added in rank order through
// distributed shared memory.
//
// Warps: 0-7 promote (warp w: TMEM lanes 32 (w % 4) .. + 31, columns half
// w / 4), 8 loads both operands of a block with TMA (128 bytes of channels =
// one swizzled row), 9 and 10 issue the even and the odd blocks' MMAs (four,
// K = 32 each; one warp's waits and issue took 800-900 clocks a block, more
// than the 512 of the MMAs). A block's accumulator is one of 512 / BN (at most
// 4) TMEM buffers, so the MMAs of the next blocks, and of the next tile, run
// while this one is promoted. Every mbarrier wait is bounded; on timeout the
// CTA records HC_ERR_TIMEOUT, waits for its own copies and MMAs and frees its
// TMEM.
//
// Measured on a GB300: 16384 x 8192 x 8192 in 825 to 870 us when it runs on at
// the 1.4 kW limit (1.6 GHz), 745 us in a burst (2.95 PFLOP/s, tensor pipe 64%
// of elapsed); the MMAs alone with their loads take 612 us. A tile of
// few blocks pays for its first scales and its epilogue, about 2 us (16384 x 640
// x 4096: 69 us, 41 without the stores and what leads to them). 1 x 8192 x 8192
// takes 14 us, 9.9 of them the weight at the copy rate.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <mutex>

#include "tokens.cuh"

namespace hc {
namespace {

constexpr int kLanes = 128;                   // TMEM lanes = rows of the first operand
constexpr int kKB = 128;                      // channels per block = bytes per smem row
constexpr int kPromoteWarps = 8;
constexpr int kLoadWarp = kPromoteWarps;
constexpr int kMmaWarp = kPromoteWarps + 1;  // and the next: even and odd blocks
constexpr int kMmaWarps = 2;
constexpr int kThreads = (kPromoteWarps + 4) * 32;  // three warpgroups; the last warp idles
// Registers of the third warpgroup and of the promoting ones: launched with
// 168 each (64512 in all), 128 * 88 + 256 * 208 = 64512 after the exchange.
constexpr int kRoleRegs = 88, kPromoteRegs = 208;
constexpr int kGroupM = 16;                   // token tiles walked per column of tiles
constexpr int kPrefetch = 8;                  // weight blocks of a CTA asked into L2 ahead

template <int BN>
struct Cfg {
    static constexpr int kStageBytes = (kLanes + BN) * kKB;
    // even: a stage's blocks then all belong to one MMA warp
    // Channels on the lanes: two CTAs an SM, so that the next call's are there,
    // and its first weights on their way into L2, while this one's finish.
    static constexpr bool kTwo = BN <= 64;
    static constexpr int kRing = kTwo ? 100 * 1024 : 192 * 1024;
    static constexpr int kStages = (kRing / kStageBytes < 10 ? kRing / kStageBytes : 10) & ~1;
    static constexpr int kBufs = 512 / BN < 4 ? 512 / BN : 4;
    static constexpr uint32_t kTmemCols = kBufs * BN;
    static constexpr int kCols = BN / 2;      // columns per promoting thread
    // kind::f8f6f4 instruction descriptor: D fp32 (bit 4), A and B e4m3 (0 at
    // bits 7 and 10), both K-major, N >> 3 at 17, M >> 4 at 24.
    static constexpr uint32_t kIdesc =
        (1u << 4) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(kLanes >> 4) << 24);
    // after the stages: bias of each promoting warp's columns, output staging
    // (32 rows x 64 bytes a warp), barriers
    static constexpr int kBiasBytes = kTwo ? 0 : kPromoteWarps * kCols * 4;
    static constexpr int kOutBytes = kTwo ? 0 : kPromoteWarps * 32 * 64;
    static constexpr size_t kSmem =
        1024 + (size_t)kStages * kStageBytes + kBiasBytes + kOutBytes + 256;
    // The totals of a split tile reuse the stages: [BN][128] fp32 with channels
    // on the lanes, [128][kTotalPitch] with tokens on the lanes (4 more than BN,
    // so that eight rows' 16-byte pieces fall into different banks).
    static constexpr int kTotalPitch = BN + 4;
    static_assert((size_t)kStages * kStageBytes >= (size_t)kTotalPitch * kLanes * 4, "split totals");
};

struct KernelArgs {
    Fp8LinearArgs a;
    int nkb;    // blocks of channels
    int split;  // CTAs of a cluster that share a tile's blocks
};

__device__ __forceinline__ uint64_t desc_sw128(uint32_t saddr) {
    // K-major, 128-byte swizzle: 8-row groups 1024 bytes apart, version bits
    // 46-48 = 0b001
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tc_mma_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc,
                                            uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
          "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7])
        : "r"(taddr)
        : "memory");
}
// A box of the tensor map into L2.
__device__ __forceinline__ void tma_prefetch_2d(const void* tmap, int c0, int c1) {
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];\n" ::"l"(
                     reinterpret_cast<uint64_t>(tmap)),
                 "r"(c0), "r"(c1)
                 : "memory");
}
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t e;
    asm volatile(
        "{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(e));
    return e != 0;
}
// (a0, a1) += (v0, v1) * (s, s), one instruction for both.
__device__ __forceinline__ void fma_pair(float& a0, float& a1, uint32_t v0, uint32_t v1, float s) {
    unsigned long long a, v, ss;
    asm("mov.b64 %0, {%1, %2};" : "=l"(a) : "f"(a0), "f"(a1));
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(v0), "r"(v1));
    asm("mov.b64 %0, {%1, %1};" : "=l"(ss) : "f"(s));
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(a) : "l"(v), "l"(ss));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a0), "=f"(a1) : "l"(a));
}
// A pipeline wait of this kernel, by a whole warp: a look at the phase, then
// tries that may suspend the warp, the abort flag and the clock after each.
// (mbar_wait reads its limit from global memory whenever its first try has
// failed, longer than most waits here last. Polling all the time instead drew
// power: 1.5% on the largest products, which run at the power limit. A limit
// lowered below a try's longest suspension is kept by polling.)
constexpr unsigned long long kLongestTryNs = 100000;
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n"
        " mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        " selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag,
                                          unsigned* status, unsigned long long limit) {
    const unsigned long long t0 = globaltimer_ns();
    bool ok;
    for (;;) {
        ok = limit > kLongestTryNs ? mbar_try_wait(bar, parity) : mbar_test(bar, parity);
        if (ok || *abort_flag) break;
        if (globaltimer_ns() - t0 > limit) {
            *abort_flag = 1;
            report(status, kErrTimeout);
            break;
        }
    }
    return __all_sync(0xffffffffu, ok);
}
__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity, volatile int* abort_flag,
                                         unsigned* status, unsigned long long limit) {
    if (__all_sync(0xffffffffu, mbar_test(bar, parity))) return true;
    return wait_slow(bar, parity, abort_flag, status, limit);
}
// Both phases, looked at together before either is waited for.
__device__ __forceinline__ bool wait_bars(uint32_t bar0, uint32_t parity0, uint32_t bar1,
                                          uint32_t parity1, volatile int* abort_flag,
                                          unsigned* status, unsigned long long limit) {
    const bool a = mbar_test(bar0, parity0), b = mbar_test(bar1, parity1);
    if (__all_sync(0xffffffffu, a && b)) return true;
    return wait_slow(bar0, parity0, abort_flag, status, limit) &&
           wait_slow(bar1, parity1, abort_flag, status, limit);
}
// A float at the same shared-memory offset of another CTA of the cluster.
__device__ __forceinline__ float lds_cluster_f32(uint32_t addr, uint32_t rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(v) : "r"(cluster_map(addr, rank)) : "memory");
    return v;
}

__device__ __forceinline__ float4 lds_cluster_f4(uint32_t addr, uint32_t rank) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];\n"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(cluster_map(addr, rank))
                 : "memory");
    return v;
}

// The tile t of the walk: token tiles in groups of kGroupM, the tiles of a
// group column by column, so that a wave of CTAs shares both operands in L2.
__device__ __forceinline__ void tile_at(uint32_t t, int tm, int tn, int& m, int& n) {
    const uint32_t per = (uint32_t)kGroupM * (uint32_t)tn;
    const uint32_t g = t / per;
    const int first = (int)g * kGroupM;
    const uint32_t in = (uint32_t)(tm - first < kGroupM ? tm - first : kGroupM);
    const uint32_t r = t - g * per;
    n = (int)(r / in);
    m = first + (int)(r - (uint32_t)n * in);
}

template <int kAct>
struct Act {
    static constexpr int value = kAct;
};

// Activation of an output. A NaN stays one: it marks a row whose 8-bit form
// holds a NaN or an infinity (fmaxf would make a zero of it). ELU's exp(z) - 1
// is taken from the fast exponential where z < -1/8: its two units in the last
// place are there at most 18 * 2^-24 of the difference. Nearer to zero, where
// nothing of a small z would be left, from the first five terms of its series (the sixth is
// below 2^-24 of the sum). 16384 x 640 x 4096 105 us so, with expm1f 195, 96
// with the exponential alone.
template <int kAct>
__device__ __forceinline__ float activate(float z) {
    if (kAct == HC_ACT_ELU) {
        float p = fmaf(z, 1.f / 120.f, 1.f / 24.f);
        p = fmaf(z, p, 1.f / 6.f);
        p = fmaf(z, p, 0.5f);
        p = fmaf(z * z, p, z);
        p = z < -0.125f ? __expf(z) - 1.f : p;
        return z > 0.f ? z : p;
    }
    if (kAct == HC_ACT_RELU) return z < 0.f ? 0.f : z;
    return z;
}
__device__ __forceinline__ float activate(float z, int act) {
    if (act == HC_ACT_ELU) return activate<HC_ACT_ELU>(z);
    if (act == HC_ACT_RELU) return activate<HC_ACT_RELU>(z);
    return z;
}

// Bias, activation and store of a warp's 32 rows (one per lane, from row r0
// on) x kCols channels from o0 on. 64 bytes of every row at a time go through
// the warp's staging buffer (16-byte pieces swizzled so that neither side has
// bank conflicts) and leave as whole 64-byte pieces of rows: straight from
// the registers a store would touch 32 rows with 16 bytes each.
template <typename T, int kCols, int kAct>
__device__ __forceinline__ void store_tile(const float (&acc)[kCols], const float* bias,
                                           uint32_t stage, T* y, long long r0, long long rows,
                                           int o0, int C_out) {
    constexpr int kV = 16 / (int)sizeof(T), kPass = 64 / (int)sizeof(T);
    const int lane = threadIdx.x & 31;
    const bool wide = C_out % kV == 0 && (reinterpret_cast<uintptr_t>(y) & 15) == 0;
#pragma unroll
    for (int p = 0; p < kCols; p += kPass) {
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float f[kV];
#pragma unroll
            for (int i = 0; i < kV; i += 4) {
                const int j = p + q * kV + i;
                const float4 b = *reinterpret_cast<const float4*>(bias + j);
                f[i] = activate<kAct>(acc[j] + b.x);
                f[i + 1] = activate<kAct>(acc[j + 1] + b.y);
                f[i + 2] = activate<kAct>(acc[j + 2] + b.z);
                f[i + 3] = activate<kAct>(acc[j + 3] + b.w);
            }
            Piece<T, kV> w;
            w.set_all(f);
            sts_v4(stage + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4),
                   *reinterpret_cast<const uint4*>(&w.v));
        }
        __syncwarp();
        if (wide) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = i * 8 + (lane >> 2), q = lane & 3;
                const int o = o0 + p + q * kV;
                const uint4 v = lds_u4(stage + r * 64 + ((q ^ ((r >> 1) & 3)) << 4));
                if (r0 + r < rows && o < C_out)
                    *reinterpret_cast<uint4*>(y + (r0 + r) * C_out + o) = v;
            }
        } else {
            // element by element, kPass lanes side by side in a row
            constexpr int kRows = 32 / kPass;  // rows at a time
            const int j = lane % kPass, q = j / kV, rl = lane / kPass;
            const bool in = o0 + p + j < C_out;
            T* at = y + (r0 + rl) * C_out + o0 + p + j;
            const uint32_t from = stage + rl * 64 + j % kV * (int)sizeof(T);
#pragma unroll
            for (int r = 0; r < 32; r += kRows) {
                const uint32_t a = from + r * 64 + ((q ^ (((r + rl) >> 1) & 3)) << 4);
                T v;
                if constexpr (sizeof(T) == 4) {
                    v = __int_as_float(lds_s32(a));
                } else {
                    uint16_t b;
                    asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(b) : "r"(a) : "memory");
                    v = __ushort_as_bfloat16(b);
                }
                if (in && r0 + r + rl < rows) *at = v;
                at += (long long)kRows * C_out;
            }
        }
    }
}

template <int BN, bool kSwap, typename T>
__global__ void __launch_bounds__(kThreads, Cfg<BN>::kTwo ? 2 : 1)
    fp8_linear_kernel(const KernelArgs k, const __grid_constant__ CUtensorMap map_x,
                      const __grid_constant__ CUtensorMap map_w) {
    using C = Cfg<BN>;
    const Fp8LinearArgs& a = k.a;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    const uint32_t bias_at = base + C::kStages * C::kStageBytes;
    const uint32_t out_at = bias_at + C::kBiasBytes;
    const uint32_t bars = out_at + C::kOutBytes;
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (C::kStages + s); };
    auto tfull_bar = [&](int b) { return bars + 8u * (2 * C::kStages + b); };
    auto tempty_bar = [&](int b) { return bars + 8u * (2 * C::kStages + C::kBufs + b); };
    const uint32_t fin_bar = bars + 8u * (2 * C::kStages + 2 * C::kBufs);
    uint8_t* const misc =
        smem_raw + (bars - raw) + 8 * (2 * C::kStages + 2 * C::kBufs + 1);
    volatile uint32_t* const tmem_holder = reinterpret_cast<volatile uint32_t*>(misc);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(misc + 4);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < C::kBufs; ++b) {
            mbar_init(tfull_bar(b), 1);
            mbar_init(tempty_bar(b), kPromoteWarps);
        }
        mbar_init(fin_bar, kMmaWarps);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        prefetch_tensormap(&map_x);
        prefetch_tensormap(&map_w);
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32((const void*)tmem_holder), C::kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;
    const uint32_t rank = k.split > 1 ? cluster_rank() : 0u;
    const int kb0 = (int)((long long)k.nkb * rank / k.split);
    const int kb1 = (int)((long long)k.nkb * (rank + 1) / k.split);
    const uint32_t first = blockIdx.x / (uint32_t)k.split, step = gridDim.x / (uint32_t)k.split;
    if constexpr (kSwap) {
        // The weight is all the traffic of these calls, and which tile a CTA
        // starts with does not depend on N': its first boxes are asked into L2
        // while the kernel before (the quantisation of the tokens, as a rule)
        // still runs. That kernel's writes land in L2 too: the loads below see
        // them whatever was asked for before.
        if (warp == kLoadWarp && first < (uint32_t)((a.C_out + kLanes - 1) / kLanes))
            for (int kb = kb0 + lane; kb < kb1 && kb < kb0 + kPrefetch; kb += 32)
                tma_prefetch_2d(&map_w, kb * kKB, (int)first * kLanes);
    }
    pdl_wait();
    pdl_trigger();

    const unsigned long long limit =
        reinterpret_cast<const volatile DeviceWord*>(a.status)->wait_limit_ns;
    const int rows = (int)token_rows(a.count, a.capacity, a.status);
    constexpr int kTileRows = kSwap ? BN : kLanes, kTileOut = kSwap ? kLanes : BN;
    const int tm = (int)(((long long)rows + kTileRows - 1) / kTileRows);
    const int tn = (int)(((long long)a.C_out + kTileOut - 1) / kTileOut);
    const uint32_t tiles = (uint32_t)tm * (uint32_t)tn;  // below 2^31 (checked by the host)

    // In all roles every lane of the warp walks the loop, so that its state is
    // uniform; the copies and MMAs are issued by one lane.
    if (warp >= kPromoteWarps) {
    if constexpr (!C::kTwo) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kRoleRegs));
    if (warp == kLoadWarp) {
        const bool leader = elect_one();
        uint32_t it = 0;
        bool ok = true;
        for (uint32_t t = first; t < tiles && ok; t += step) {
            int m, n;
            tile_at(t, tm, tn, m, n);
            const int ra = (kSwap ? n : m) * kLanes, rb = (kSwap ? m : n) * BN;
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const uint32_t s = it % C::kStages;
                ok = wait_bar(empty_bar(s), ((it / C::kStages) & 1) ^ 1u, abort_flag, a.status,
                              limit);
                if (!ok) break;
                if (leader) {
                    const uint32_t st = base + s * C::kStageBytes;
                    mbar_arrive_expect_tx(full_bar(s), C::kStageBytes);
                    tma_load_2d(st, kSwap ? &map_w : &map_x, kb * kKB, ra, full_bar(s));
                    tma_load_2d(st + kLanes * kKB, kSwap ? &map_x : &map_w, kb * kKB, rb,
                                full_bar(s));
                }
                __syncwarp();
            }
        }
        // the copies already issued end before the CTA does, also where another
        // role gave up and nobody waits for them
        if (leader)
            for (uint32_t j = it > C::kStages ? it - C::kStages : 0; j < it; ++j)
                mbar_wait_drain(full_bar(j % C::kStages), (j / C::kStages) & 1, a.status);
        __syncwarp();
    } else if (warp < kMmaWarp + kMmaWarps) {
        const bool leader = elect_one();
        const uint32_t mine = (uint32_t)(warp - kMmaWarp);
        // this CTA's blocks, all tiles one after another
        const uint32_t total =
            (tiles > first ? (tiles - first + step - 1) / step : 0u) * (uint32_t)(kb1 - kb0);
        bool ok = true;
        for (uint32_t it = mine; it < total; it += kMmaWarps) {
            const uint32_t s = it % C::kStages, b = it % C::kBufs;
            const uint64_t da = desc_sw128(base + s * C::kStageBytes);
            const uint64_t db = desc_sw128(base + s * C::kStageBytes + kLanes * kKB);
            ok = wait_bars(full_bar(s), (it / C::kStages) & 1, tempty_bar(b),
                           ((it / C::kBufs) & 1) ^ 1u, abort_flag, a.status, limit);
            if (!ok) break;
            tc_fence_after();
            if (leader) {
#pragma unroll
                for (int j = 0; j < kKB / 32; ++j)  // 32 bytes of channels further on
                    tc_mma_e4m3(tmem_base + b * BN, da + 2 * j, db + 2 * j, C::kIdesc, j != 0);
                tc_commit(tfull_bar(b));
                tc_commit(empty_bar(s));
            }
            __syncwarp();
        }
        // every MMA issued by these threads has completed once fin_bar fires
        if (leader) {
            tc_commit(fin_bar);
            mbar_wait_drain(fin_bar, 0, a.status);
        }
        __syncwarp();
    }
    } else {
        if constexpr (!C::kTwo)
            asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kPromoteRegs));
        const int quarter = warp & 3, half = warp >> 2;
        const uint32_t tm_lane = (uint32_t)(quarter * 32) << 16;
        // TMEM columns read at a time: more would not fit beside the totals
        constexpr int kChunk = C::kCols < 16 ? C::kCols : 16;
        T* const y = static_cast<T*>(a.y);
        float* const bias_s =
            reinterpret_cast<float*>(smem_raw + (bias_at - raw)) + warp * C::kCols;
        const int nbo = (a.C_out + kKB - 1) / kKB;
        uint32_t it = 0;
        bool ok = true;
        // The two factors of a block's scale are loaded two blocks ahead and
        // multiplied when they are used (formed at once, the product would
        // wait for its loads); unrolled by two, so that no copy from one
        // set to the other waits either. A row that is not in use takes
        // row 0's scales and is not stored. The last block's are loaded
        // again rather than any past it.
        float fx[2], fw[2];
        const float *xs, *xs_last, *ws;
        float bias_r[C::kCols / 32 + 1];
        auto load_scale = [&](int u) {
            fx[u] = __ldg(xs);
            fw[u] = __ldg(ws);
            if (xs < xs_last) {
                xs += a.capacity;
                ++ws;
            }
        };
        // the first scales and the bias of tile t, asked for before the tile
        // before it is stored
        auto begin = [&](uint32_t t) {
            int m, n;
            tile_at(t, tm, tn, m, n);
            if constexpr (!kSwap) {
#pragma unroll
                for (int j = 0; j < C::kCols; j += 32) {
                    const int o = n * BN + half * C::kCols + j + lane;
                    bias_r[j / 32] = a.bias && o < a.C_out ? __ldg(a.bias + o) : 0.f;
                }
            }
            // rows on lanes: this thread's token, and the block of its channels;
            // channels on lanes: lane l holds the scale of the half's token l
            const int row = kSwap ? m * BN + half * C::kCols + lane
                                  : m * kLanes + quarter * 32 + lane;
            const bool row_in = row < rows && (!kSwap || lane < C::kCols);
            const int ob = kSwap ? n : (n * BN + half * C::kCols) / kKB;
            xs = a.xs + (long long)kb0 * a.capacity + (row_in ? row : 0);
            xs_last = xs + (long long)(kb1 - kb0 - 1) * a.capacity;
            ws = a.ws + (long long)(ob < nbo ? ob : 0) * k.nkb + kb0;
            load_scale(0);
            load_scale(1);
        };
        if (first < tiles) begin(first);
        for (uint32_t t = first; t < tiles && ok; t += step) {
            float acc[C::kCols];
#pragma unroll
            for (int j = 0; j < C::kCols; ++j) acc[j] = 0.f;
            if constexpr (!kSwap) {
                __syncwarp();  // the last tile's bias has been read
#pragma unroll
                for (int j = 0; j < C::kCols; j += 32) bias_s[j + lane] = bias_r[j / 32];
                __syncwarp();
            }
            for (int left = kb1 - kb0; left > 0 && ok; left -= 2) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (u == 1 && (left < 2 || !ok)) break;
                    const uint32_t b = it % C::kBufs, ph = (it / C::kBufs) & 1;
                    const float s = fx[u] * fw[u];
                    load_scale(u);
                    ok = wait_bar(tfull_bar(b), ph, abort_flag, a.status, limit);
                    ++it;
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t at = tmem_base + tm_lane + b * BN + (uint32_t)(half * C::kCols);
#pragma unroll
                    for (int c = 0; c < C::kCols; c += kChunk) {
                        uint32_t r[kChunk];
                        tmem_ld(at + (uint32_t)c, r);
                        tmem_ld_wait();
                        if (c + kChunk == C::kCols) {
                            tc_fence_before();
                            if (lane == 0) mbar_arrive(tempty_bar(b));
                        }
                        if constexpr (kSwap) {
#pragma unroll
                            for (int j = 0; j < kChunk; ++j)
                                acc[c + j] = fmaf(__uint_as_float(r[j]),
                                                  __shfl_sync(0xffffffffu, s, c + j), acc[c + j]);
                        } else {
#pragma unroll
                            for (int j = 0; j < kChunk; j += 2)
                                fma_pair(acc[c + j], acc[c + j + 1], r[j], r[j + 1], s);
                        }
                    }
                }
            }
            if (!ok) break;
            if (k.split > 1) {
                // totals of this CTA's blocks into the (now idle) stages; a split
                // launch has one tile per cluster
                if constexpr (kSwap) {
#pragma unroll
                    for (int j = 0; j < C::kCols; ++j)
                        sts_s32(base + (uint32_t)(((half * C::kCols + j) * kLanes + quarter * 32 + lane) * 4),
                                __float_as_int(acc[j]));
                } else {
#pragma unroll
                    for (int j = 0; j < C::kCols; j += 4)
                        sts_v4(base + (uint32_t)((quarter * 32 + lane) * C::kTotalPitch + half * C::kCols + j) * 4u,
                               make_uint4(__float_as_uint(acc[j]), __float_as_uint(acc[j + 1]),
                                          __float_as_uint(acc[j + 2]), __float_as_uint(acc[j + 3])));
                }
                break;
            }
            int m, n;
            tile_at(t, tm, tn, m, n);
            if (t + step < tiles) begin(t + step);
            if constexpr (kSwap) {
                const int o = n * kLanes + quarter * 32 + lane;
                if (o < a.C_out) {
                    const float bias = a.bias ? a.bias[o] : 0.f;
#pragma unroll
                    for (int j = 0; j < C::kCols; ++j) {
                        const long long nn = (long long)m * BN + half * C::kCols + j;
                        if (nn < rows)
                            y[nn * a.C_out + o] = from_f32<T>(activate(acc[j] + bias, a.act));
                    }
                }
            } else {
                auto finish = [&](auto act) {
                    store_tile<T, C::kCols, decltype(act)::value>(
                        acc, bias_s, out_at + (uint32_t)warp * 2048u, y,
                        (long long)m * kLanes + quarter * 32, rows, n * BN + half * C::kCols,
                        a.C_out);
                };
                if (a.act == HC_ACT_ELU)
                    finish(Act<HC_ACT_ELU>{});
                else if (a.act == HC_ACT_RELU)
                    finish(Act<HC_ACT_RELU>{});
                else
                    finish(Act<HC_ACT_NONE>{});
            }
        }
    }
    if (k.split > 1) {
        // every CTA of the cluster passes both barriers, whatever happened above
        cluster_barrier();
        if (warp < kPromoteWarps && first < tiles && !*abort_flag) {
            int m, n;
            tile_at(first, tm, tn, m, n);
            T* const y = static_cast<T*>(a.y);
            if constexpr (kSwap) {
                // a share of the tokens each, a channel per lane
                const int quarter = warp & 3, half = warp >> 2;
                const int per = C::kCols / k.split, ln = quarter * 32 + lane;
                const int o = n * kLanes + ln;
                const float bias = a.bias && o < a.C_out ? __ldg(a.bias + o) : 0.f;
                for (int j = 0; j < per; ++j) {
                    const int col = half * C::kCols + (int)rank * per + j;
                    float v = 0.f;
                    for (int r = 0; r < k.split; ++r)
                        v += lds_cluster_f32(base + (uint32_t)((col * kLanes + ln) * 4), (uint32_t)r);
                    const long long nn = (long long)m * BN + col;
                    if (nn < rows && o < a.C_out)
                        y[nn * a.C_out + o] = from_f32<T>(activate(v + bias, a.act));
                }
            } else {
                // a share of the tokens each, a warp per token, 4 channels per lane
                const int per = kLanes / k.split;
                const bool wide = a.C_out % 4 == 0 && (reinterpret_cast<uintptr_t>(y) & 15) == 0;
                for (int c = lane * 4; c < BN; c += 128) {
                    const int o = n * BN + c;
                    float bias[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        bias[i] = a.bias && o + i < a.C_out ? __ldg(a.bias + o + i) : 0.f;
#pragma unroll 4
                    for (int q = warp; q < per; q += kPromoteWarps) {
                        const int ln = (int)rank * per + q;
                        const long long nn = (long long)m * kLanes + ln;
                        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                        for (int r = 0; r < k.split; ++r) {
                            const float4 f = lds_cluster_f4(
                                base + (uint32_t)(ln * C::kTotalPitch + c) * 4u, (uint32_t)r);
                            v.x += f.x, v.y += f.y, v.z += f.z, v.w += f.w;
                        }
                        if (nn >= rows) continue;
                        const float w[4] = {activate(v.x + bias[0], a.act), activate(v.y + bias[1], a.act),
                                            activate(v.z + bias[2], a.act), activate(v.w + bias[3], a.act)};
                        T* const yr = y + nn * a.C_out + o;
                        if (wide && o < a.C_out) {
                            if constexpr (sizeof(T) == 4)
                                *reinterpret_cast<float4*>(yr) = make_float4(w[0], w[1], w[2], w[3]);
                            else
                                *reinterpret_cast<uint2*>(yr) =
                                    make_uint2(Piece<T, 8>::pair(w[0], w[1]), Piece<T, 8>::pair(w[2], w[3]));
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (o + i < a.C_out) yr[i] = from_f32<T>(w[i]);
                        }
                    }
                }
            }
        }
        cluster_barrier();
    } else {
        __syncthreads();
    }
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem_base, C::kTmemCols);
    }
}

// ---------------------------------------------------------------- host side
PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                             &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    });
    return fn;
}

// A [rows, pitch] byte matrix in boxes of box_rows x 128 bytes, 128-byte
// swizzle; what lies outside reads as zero.
hc_status encode(CUtensorMap* m, const void* base, long long rows, int pitch, int box_rows) {
    auto enc = tensor_map_encoder();
    if (!enc) {
        set_error("cuTensorMapEncodeTiled is unavailable");
        return HC_ERR_CUDA;
    }
    cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)pitch};
    cuuint32_t box[2] = {kKB, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    const CUresult r =
        enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_error("cuTensorMapEncodeTiled failed (%d)", (int)r);
        return HC_ERR_CUDA;
    }
    return HC_OK;
}

template <int BN, bool kSwap, typename T>
hc_status launch(const DeviceCtx* ctx, const Fp8LinearArgs& a, cudaStream_t s) {
    using C = Cfg<BN>;
    KernelArgs k{a, (a.C_in + kKB - 1) / kKB, 1};
    CUtensorMap mx, mw;
    hc_status st = encode(&mx, a.xq, a.capacity, a.pitch, kSwap ? BN : kLanes);
    if (st != HC_OK) return st;
    st = encode(&mw, a.wq, a.C_out, a.pitch, kSwap ? kLanes : BN);
    if (st != HC_OK) return st;
    constexpr int kTileRows = kSwap ? BN : kLanes, kTileOut = kSwap ? kLanes : BN;
    const long long tiles = (((long long)a.capacity + kTileRows - 1) / kTileRows) *
                            (((long long)a.C_out + kTileOut - 1) / kTileOut);
    // Split while every CTA still gets an SM (or half) of its own and two blocks
    // or more: 1 x 8192 x 8192 takes 13.5 us, unsplit 22. Clusters of 8 find room
    // late unless they leave half of it free: 128 x 2048 x 2048 (16 tiles) 14.0
    // us, 7.1 with clusters of 4, 1 x 4096 x 4096 6.1 and 5.5; 128 x 8192 x 1024
    // (8 tiles) 8.9 against 9.8.
    const int slots = ctx->num_sms * (C::kTwo ? 2 : 1);
    while (k.split < 8 && tiles * k.split * (k.split == 4 ? 4 : 2) <= slots &&
           k.nkb >= 4 * k.split)
        k.split *= 2;
    if (tiles > 0x7fffffffll) {
        set_error("hc_fp8_linear_fwd: capacity=%d C_out=%d is too large", a.capacity, a.C_out);
        return HC_ERR_UNSUPPORTED;
    }
    const long long grid =
        k.split > 1 ? tiles * k.split : (tiles < slots ? tiles : slots);
    auto kern = fp8_linear_kernel<BN, kSwap, T>;
    static bool done[64];
    if (!done[ctx->device]) {
        st = check_cuda(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)C::kSmem),
                        "fp8_linear_kernel");
        if (st != HC_OK) return st;
        done[ctx->device] = true;
    }
    return launch_cluster(kern, (unsigned)grid, (unsigned)k.split, kThreads, C::kSmem, s,
                          "fp8_linear_kernel", k, mx, mw);
}

template <typename T>
hc_status dispatch(const DeviceCtx* ctx, const Fp8LinearArgs& a, cudaStream_t s) {
    // Few tokens on the columns, the narrowest that holds them: 16 x 4096 x 4096
    // 6.2 us, 10.8 with 64 columns, 10.1 with tokens on the lanes. At 33 to 64
    // it goes by the shape: 37 x 2000 x 1001 6.2 and 7.7 us, 64 x 8192 x 8192
    // 18.1 and 18.8, but 64 x 2048 x 8192 10.2 and 9.1, 64 x 4096 x 16384 19.8
    // and 15.6: wide outputs lose.
    if (a.capacity <= 16) return launch<16, true, T>(ctx, a, s);
    if (a.capacity <= 32) return launch<32, true, T>(ctx, a, s);
    if (a.capacity <= 64) return launch<64, true, T>(ctx, a, s);
    // A tile of 256 output channels takes 1.6 times as long as one of 128 (one
    // wave of each, 1024 x 4096 x 4096: 17.4 us against 22.1 for two waves of
    // 128): the width whose waves take less.
    const long long m = ((long long)a.capacity + kLanes - 1) / kLanes, sms = ctx->num_sms;
    const long long waves128 = (m * ((a.C_out + 127) / 128) + sms - 1) / sms;
    const long long waves256 = (m * ((a.C_out + 255) / 256) + sms - 1) / sms;
    if (a.C_out > 128 && 8 * waves256 <= 5 * waves128) return launch<256, false, T>(ctx, a, s);
    return launch<128, false, T>(ctx, a, s);
}

}  // namespace

hc_status launch_fp8_linear(const DeviceCtx* ctx, const Fp8LinearArgs& a, cudaStream_t s) {
    return a.y_dt == HC_BF16 ? dispatch<__nv_bfloat16>(ctx, a, s) : dispatch<float>(ctx, a, s);
}

}  // namespace hc
