// Shared-memory barriers for asynchronous copies and tensor-core products, with bounded waits.
#pragma once
#include <cstdint>
#ifdef HPL_DEBUG_BOUNDS
#include <cstdio>
#include <cstdlib>
#endif

namespace hpl {

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_fence_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// Who waits: for room to load into, for operands and accumulators, for what results are made of.
enum Waiter { kLoads = 1, kProducts, kResults };
#ifdef HPL_DEBUG_BOUNDS
// Testing aid of the bounds-checking build: with HPL_DEBUG_EXPIRE=<waiter>,<block>,<n> in the environment, the waits of that Waiter in
// that block run out in the calls of this source file, all but the first n of them.
constexpr uint64_t kWaitNs = 200000000;
struct Expiry {
    int waiter, block, after, count;
};
static __device__ Expiry debug_expiry;
static __device__ inline bool expires(Waiter who) {
    return debug_expiry.waiter == who && debug_expiry.block == (int)blockIdx.x && atomicAdd(&debug_expiry.count, 1) >= debug_expiry.after;
}
static inline bool arm_expiry(cudaStream_t stream) {
    Expiry e = {};
    if (const char* v = getenv("HPL_DEBUG_EXPIRE")) sscanf(v, "%d,%d,%d", &e.waiter, &e.block, &e.after);
    return cudaMemcpyToSymbolAsync(debug_expiry, &e, sizeof e, 0, cudaMemcpyHostToDevice, stream) == cudaSuccess;
}
#else
constexpr uint64_t kWaitNs = 2000000000;
static __device__ __forceinline__ bool expires(Waiter) { return false; }
static inline bool arm_expiry(cudaStream_t) { return true; }
#endif
// Bounded: gives up after two seconds, or soon after another thread of the block has.  In a correct run none ever does; who
// gives up makes the results that depend on it NaN, and the block stays until what it has under way is over.
static __device__ inline bool mbar_wait_slow(uint32_t bar, uint32_t parity, volatile int* abort) {
    const uint64_t t0 = now_ns();
    for (int i = 1; i < (1 << 28); ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 63) == 0 && (*abort || now_ns() - t0 > kWaitNs)) break;
    }
    *abort = 1;
    return false;
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort, Waiter who) {
    if (expires(who)) {
        *abort = 1;
        return false;
    }
    if (mbar_try(bar, parity)) return true;
    return mbar_wait_slow(bar, parity, abort);
}
// Copies `bytes` (a multiple of 16; both addresses 16-byte aligned) to shared memory; `bar` counts them.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// After a wait was given up: time for copies and products on their way to end before their memory goes.
__device__ __forceinline__ void let_copies_land() {
    for (const uint64_t t0 = now_ns(); now_ns() - t0 < 1000000ull;) {
    }
}

}  // namespace hpl
