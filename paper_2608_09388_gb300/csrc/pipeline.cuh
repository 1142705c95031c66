// Shared by the kernels that feed tcgen05 products by TMA from roles of their
// own: bounded waits of a warp on a barrier, and the tensor maps' encoder.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>

#include <mutex>

#include "tokens.cuh"

namespace hc {

#if defined(__CUDACC__)

// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t e;
    asm volatile(
        "{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(e));
    return e != 0;
}
// A pipeline wait, by a whole warp: a look at the phase, then
// tries that may suspend the warp, the abort flag and the clock after each.
// (mbar_wait reads its limit from global memory whenever its first try has
// failed, longer than most waits here last. Polling all the time instead drew
// power: 1.5% on the largest 8-bit products, which run at the power limit. A limit
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
    // one try before the clock is looked at
    if (limit > kLongestTryNs && __all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
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
// This lane's 16 or 8 columns from taddr on.
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

#endif  // __CUDACC__

// The driver's cuTensorMapEncodeTiled, nullptr where it has none.
inline PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
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

}  // namespace hc
