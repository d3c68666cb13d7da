// kv_tma.cuh -- barriers in shared memory and copies of cache blocks by TMA, for kv_attend.cu and kv_prefix.cu.
#pragma once

#include <cuda.h>

#include "kv_internal.cuh"

namespace isjl {

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t phase) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(done) : "r"(bar), "r"(phase) : "memory");
    return done != 0;
}

// Waits end: after kLimit nanoseconds without the barrier's turn whoever waits gives up, waits for the copies (and
// products) that are under way, reports it and returns.
constexpr uint64_t kLimit = 2000000000ull;
__device__ __forceinline__ uint64_t now() {
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// false: it gave up, or `failed` (others' or its own giving up) was set
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t phase, volatile int32_t *failed = nullptr) {
    if (bar_try(bar, phase)) return true;
    const uint64_t begin = now();
    while (!bar_try(bar, phase)) {
        if (failed && *failed) return false;
        if (now() - begin > kLimit) {
            if (failed) *failed = 1;
            return false;
        }
    }
    return true;
}

__device__ __forceinline__ void tma_load(uint32_t to, const CUtensorMap *map, uint32_t bar, int slot, int half, int head, int block) {
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                 ::"r"(to), "l"(map), "r"(bar), "r"(0), "r"(slot), "r"(half), "r"(head), "r"(block) : "memory");
}
__device__ __forceinline__ void tma_prefetch(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// Kernels of one call start while the one before them ends; what waits sees all of its predecessor's writes.
__device__ __forceinline__ void start_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// A map of a cache side for copies of `rows` slots of one block and head and of `halves` times 64 values: in shared
// memory rows of 128 bytes, swizzled by 128, one 64 values' rows after the other's.  Coordinates: value in the 64
// (always 0), slot, which 64, head, block.  A block number beyond the cache reads as zeros.
bool encode_cache(void *encoder, CUtensorMap *map, void *p, const int64_t *stride, int rows, int halves, int n_blocks, int shift,
                  int n_kv_heads, int head_dim, int type);

// launch, started while the kernel before it in the stream ends (`early`) or after that
template <typename... Args>
cudaError_t launch_kernel(void (*kernel)(Args...), int grid, int threads, size_t smem, cudaStream_t st, bool early, const Args &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace isjl
