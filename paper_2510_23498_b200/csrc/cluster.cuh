// Exchange between the blocks of a cluster through distributed shared memory: asynchronous stores whose bytes count on the receiver's barrier, so
// that neither side needs a fence (one that made a block's stores visible first would wait for its results on the way to memory, about 1 us).
#pragma once
#include "common.cuh"

namespace mpode {

__device__ __forceinline__ unsigned smem_of(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ unsigned peer_of(unsigned local, unsigned rank) {
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ void send(unsigned at, float f, unsigned bar) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];" ::"r"(at), "f"(f), "r"(bar) : "memory");
}
__device__ __forceinline__ void send(unsigned at, float f, float g, unsigned bar) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(at), "f"(f), "f"(g), "r"(bar) : "memory");
}

// one lane of a converged warp, which the compiler knows to be one (behind lane == 0 a bulk copy's operands are moved in a loop over lanes)
__device__ __forceinline__ bool elected() {
    unsigned yes;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(yes));
    return yes != 0u;
}
__device__ __forceinline__ void bar_init(unsigned long long* bar, unsigned count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_of(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

// Barriers of sets of places that are used in turn, one thread of the block
__device__ __forceinline__ void sets_begin(unsigned long long* bar, int sets) {
    for (int i = 0; i < sets; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_of(&bar[i])) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
// one thread a block and round: the bytes that will come
__device__ __forceinline__ void set_expects(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool set_arrived(unsigned bar, unsigned parity) {
    unsigned ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0u;
}
// The blocks of a cluster run at the same time, so this wait ends; should it not within two seconds, the caller makes its results NaN and goes on
// without waiting again, so that the kernel ends.
static __device__ __noinline__ bool await_set(unsigned bar, unsigned parity) {
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t0));
    while (!set_arrived(bar, parity)) {
        asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
        if (t - t0 > 2000000000ull) return false;
    }
    return true;
}
__device__ __forceinline__ void wait_set(unsigned bar, unsigned parity, bool& broken) {
    if (!broken && !set_arrived(bar, parity)) broken = !await_set(bar, parity);
    __syncwarp();
}

}  // namespace mpode
