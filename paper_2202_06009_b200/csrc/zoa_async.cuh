// Barriers of the handle-free operators' kernels; every wait is bounded.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace zoa {
namespace {

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_init_done() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// kCluster: what arrives on the barrier are other blocks of the cluster, with data of theirs.
template <bool kCluster = false>
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    if constexpr (kCluster)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long timer_ns()
{
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
struct WaitLimit {
    int *error_word;            // set when a wait ran out: in host memory
    unsigned long long ns;
};
// False if the block has given up or the limit ran out (both flags are then set).
template <bool kCluster = false>
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up, const WaitLimit &limit)
{
    // The clock is first read after many tries: a read takes longer than most waits (it cost a product half its speed).
    unsigned long long start = 0;
    for (unsigned it = 1;; ++it) {
        if (mbar_try<kCluster>(bar, parity)) return true;
        if ((it & 255u) == 0) {
            if (*gave_up) return false;
            const unsigned long long now = timer_ns();
            if (start == 0) start = now;
            if (now - start > limit.ns) {
                *gave_up = 1;
                *reinterpret_cast<volatile int *>(limit.error_word) = 1;
                __threadfence_system();
                return false;
            }
        }
    }
}
// The same without a flag to look at: for copies that are known to be in flight.
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity, const WaitLimit &limit)
{
    const unsigned long long start = timer_ns();
    while (!mbar_try(bar, parity) && timer_ns() - start < limit.ns) {}
}
// Arrives on the barrier at the same place in block `rank` of this cluster.
__device__ __forceinline__ void mbar_arrive_at(uint32_t bar, uint32_t rank)
{
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(bar), "r"(rank));
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(remote) : "memory");
}
// Orders this thread's earlier accesses to its block's shared memory, and what it has seen of others', ahead of its later
// arrivals at cluster scope.  A release at that scope orders all memory and waits for what is on its way there: 1700 cycles in
// the pair product.
__device__ __forceinline__ void release_shared() { asm volatile("fence.release.sync_restrict::shared::cta.cluster;" ::: "memory"); }
// Arrives there without ordering earlier accesses: for tensor memory, whose own fences order it, or after release_shared.
__device__ __forceinline__ void mbar_tell(uint32_t bar, uint32_t rank)
{
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(bar), "r"(rank));
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(remote) : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

}  // namespace
}  // namespace zoa
