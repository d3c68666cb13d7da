// kv_tensor.cuh -- tensor-core products with sums and weights in TMEM, for kv_prefix.cu and kv_prompt.cu.
#pragma once

#include "kv_tma.cuh"

namespace isjl {

// shared-memory operand with rows of 128 bytes, swizzled by 128 bytes
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t leading, uint32_t stride) {
    return (uint64_t)((at >> 4) & 0x3fff) | ((uint64_t)((leading >> 4) & 0x3fff) << 16) |
           ((uint64_t)((stride >> 4) & 0x3fff) << 32) | (1ull << 46) | (2ull << 61);
}

// operands by the low word and the (common) high word of their descriptors
__device__ __forceinline__ void mma_smem(uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t what, bool add) {
    asm volatile("{\n.reg .pred p;\n.reg .b64 x, y;\nmov.b64 x, {%1, %3};\nmov.b64 y, {%2, %3};\nsetp.ne.b32 p, %5, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, p;\n}"
                 ::"r"(d), "r"(a), "r"(b), "r"(high), "r"(what), "r"((int)add) : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t what, bool add) {
    asm volatile("{\n.reg .pred p;\n.reg .b64 y;\nmov.b64 y, {%2, %3};\nsetp.ne.b32 p, %5, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n}"
                 ::"r"(d), "r"(a), "r"(b), "r"(high), "r"(what), "r"((int)add) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

#define R8(v, i) "=r"((v)[(i)]), "=r"((v)[(i) + 1]), "=r"((v)[(i) + 2]), "=r"((v)[(i) + 3]), "=r"((v)[(i) + 4]), "=r"((v)[(i) + 5]), "=r"((v)[(i) + 6]), "=r"((v)[(i) + 7])
#define W8(v, i) "r"((v)[(i)]), "r"((v)[(i) + 1]), "r"((v)[(i) + 2]), "r"((v)[(i) + 3]), "r"((v)[(i) + 4]), "r"((v)[(i) + 5]), "r"((v)[(i) + 6]), "r"((v)[(i) + 7])

// two 32-bit operations in one instruction: for the exponents' arguments and sums, 378 -> 361 us with 512 queries of
// 64 + 8 heads over 32,768 tokens
__device__ __forceinline__ float2 fma2(float x, float y, float scale, float offset) {
    float2 z;
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %4};\nmov.b64 c, {%5, %5};\nfma.rn.f32x2 d, a, b, c;\n"
        "mov.b64 {%0, %1}, d;\n}" : "=f"(z.x), "=f"(z.y) : "f"(x), "f"(y), "f"(scale), "f"(offset));
    return z;
}
__device__ __forceinline__ void add2(float2 &sum, float x, float y) {
    asm("{\n.reg .b64 a, b;\nmov.b64 a, {%0, %1};\nmov.b64 b, {%2, %3};\nadd.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
        : "+f"(sum.x), "+f"(sum.y) : "f"(x), "f"(y));
}

// 32 columns of this thread's TMEM lane
__device__ __forceinline__ void tmem_load(uint32_t (&v)[32], uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : R8(v, 0), R8(v, 8), R8(v, 16), R8(v, 24) : "r"(at));
}
__device__ __forceinline__ void tmem_load(uint32_t (&v)[16], uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : R8(v, 0), R8(v, 8) : "r"(at));
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&v)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(at), W8(v, 0), W8(v, 8), W8(v, 16), W8(v, 24) : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

}  // namespace isjl
