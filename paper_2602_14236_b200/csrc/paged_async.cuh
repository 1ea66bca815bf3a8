// Barriers in shared memory and bulk copies that arrive on them.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

constexpr int DRAIN_LIMIT = 1 << 16;         // tries for copies and matrix instructions under way to end

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {          // one arrival, and bytes to come
    asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
                 "r"(bar)
                 : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared.b64 p, [%1], %2; selp.b32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// True: the phase is complete.  False: the wait has been given up, after `limit` tries or because another role had given up;
// who gets that touches nothing that the phase stands for, arrives nowhere any more and leaves.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, int limit, volatile int* gave_up) {
#pragma unroll 1
    for (int i = 0; i < limit; ++i) {
        if (bar_try(bar, parity)) return true;
        if (*gave_up) return false;
    }
    *gave_up = 1;
    return false;
}
// The same for a whole warp, which stays together.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, int limit, volatile int* gave_up) {
    return __all_sync(0xffffffffu, bar_wait(bar, parity, limit, gave_up));
}
// ... with its loop in a function, for kernels with many waits and few values that live across them.  A vote at the first
// look keeps the warp's branch uniform (1149 us for frames over INT4; 1169 with a branch per lane).
static __device__ __noinline__ bool warp_wait_long(uint32_t bar, uint32_t parity, int limit, volatile int* gave_up) {
    return warp_wait(bar, parity, limit, gave_up);
}
__device__ __forceinline__ bool warp_wait_far(uint32_t bar, uint32_t parity, int limit, volatile int* gave_up) {
    if (__all_sync(0xffffffffu, limit > 0 && bar_try(bar, parity))) return true;
    return warp_wait_long(bar, parity, limit, gave_up);
}
// For what is under way when a block leaves early.
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity) {
#pragma unroll 1
    for (int i = 0; i < DRAIN_LIMIT && !bar_try(bar, parity); ++i) {}
}
// Every thread of the block, each role from its own place in the code.
__device__ __forceinline__ void join_roles() { asm volatile("barrier.cta.sync 0;" ::: "memory"); }

__device__ __forceinline__ void lds16(uint32_t* v, uint32_t addr) {
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
template <int W>
__device__ __forceinline__ void lds_words(uint32_t* v, uint32_t addr) {
    if (W == 4) lds16(v, addr);
    if (W == 2) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(addr) : "memory");
    if (W == 1) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v[0]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t lds_u16(uint32_t addr) {
    uint16_t x;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(addr) : "memory");
    return x;
}
// Work of the next kernel in the stream may begin; what it does before `grid_wait` must not touch this one's results.
__device__ __forceinline__ void grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// A launch that may begin while the kernel before it in the stream ends (each of these kernels waits for that one first).
template <typename... P, typename... A>
cudaError_t pt_launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
