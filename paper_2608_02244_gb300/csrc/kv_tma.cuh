// kv_tma.cuh -- barriers in shared memory, copies of cache blocks and queries by TMA (kv_attend.cu, kv_prefix.cu, kv_prompt.cu),
// and launches (kv_attend4.cu too).
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

// true for one thread of a whole warp
__device__ __forceinline__ bool elect_one() {
    uint32_t mine;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(mine));
    return mine != 0;
}

// Copies are issued by one thread of a warp, between points where the whole warp is together: the lanes bring the block
// numbers by shuffles, the other operands are the same for all.  Issued by several threads, each with operands of its own,
// they ended with an illegal address in some builds of kv_prompt.cu; nothing in the source says which builds would.
__device__ __forceinline__ void tma_load(uint32_t to, const CUtensorMap *map, uint32_t bar, int slot, int half, int head, int block) {
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                 ::"r"(to), "l"(map), "r"(bar), "r"(0), "r"(slot), "r"(half), "r"(head), "r"(block) : "memory");
}
__device__ __forceinline__ void tma_load4(uint32_t to, const CUtensorMap *map, uint32_t bar, int half, int head, int token) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(to), "l"(map), "r"(bar), "r"(0), "r"(half), "r"(head), "r"(token) : "memory");
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
// A map of queries for copies of `tokens` tokens, each with `heads` heads, and 64 values of those: rows of 128 bytes,
// tokens outermost, swizzled by 128.  Coordinates: value in the 64 (always 0), which 64, head, token.  What is beyond
// the last head or token reads as zeros.
bool encode_queries(void *encoder, CUtensorMap *map, const void *p, const int64_t *stride, int tokens, int heads, int n_tokens, int n_heads,
                    int head_dim, int type);

// launch, started while the kernel before it in the stream ends (`early`) or after that
template <typename... Args>
cudaError_t launch_kernel(void (*kernel)(Args...), dim3 grid, int threads, size_t smem, cudaStream_t st, bool early, const Args &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
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
