// PTX wrappers shared by the kernels on runs of rows (grouped products, adapters).
#pragma once

#include "mwu_gemm_dev.cuh"

namespace mwu {
namespace gemm {

// Limit of the bounded waits in cycles, and (testing aid, mwu_debug_rows_wait) a slot of the ring whose barrier waits for one arrival more
// than it gets; none: -1.  (Left to the barriers' set-up, since a test a stage in the producer's loop costs up to 5 % of a product.)
struct WaitLimits {
    long long cycles;
    int dead_slot;
};
WaitLimits wait_limits();               // mwu_grouped.cu

// The bounded waits with a limit of the caller's: polled for a while, then asleep in try_wait; false when aborted or out of time (then
// *abort is set).
__device__ __forceinline__ bool mbar_wait(unsigned bar, unsigned parity, volatile int *abort, long long limit) {
#pragma unroll 1
    for (int i = 0; i < 128; ++i)
        if (mbar_test(bar, parity)) return true;
    const long long t0 = clock64();
#pragma unroll 1
    while (true) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*abort) return false;
        if (clock64() - t0 > limit) { *abort = 1; return false; }
    }
}
// the same for a single latency-critical warp, polled for much longer first: every lane for itself
__device__ __forceinline__ bool mbar_wait_spin(unsigned bar, unsigned parity, volatile int *abort, long long limit) {
#pragma unroll 1
    for (int i = 0; i < 4096; ++i)
        if (mbar_test(bar, parity)) return true;
    return mbar_wait(bar, parity, abort, limit);
}
// ... and with the same answer in all lanes
__device__ __forceinline__ bool warp_wait_spin(unsigned bar, unsigned parity, volatile int *abort, long long limit) {
#pragma unroll 1
    for (int i = 0; i < 4096; ++i)
        if (__all_sync(0xffffffffu, mbar_test(bar, parity))) return true;
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort, limit));
}

// the two halves of a cluster barrier, for what can be done between them
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// 32 lanes x 16 columns of tensor memory
__device__ __forceinline__ void tmem_ld_16(unsigned taddr, unsigned (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}

}  // namespace gemm
}  // namespace mwu
