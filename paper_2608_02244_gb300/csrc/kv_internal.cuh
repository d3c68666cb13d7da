// kv_internal.cuh -- what the decode-step entry points (kv.cu) and their kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "isjl_kv.h"

namespace isjl {

// the 16-bit types of a cache: packing with one rounding, and the tensor instruction
template <typename T>
struct Half;

template <>
struct Half<__nv_bfloat16> {
    static constexpr bool kIsBf16 = true;
    static constexpr int kTop = 0;             // its range is that of 32 bits
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<uint32_t *>(&v);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t w) {
        return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162 *>(&w));
    }
    // d += a (16 x 16, row) * b (16 x 8, column)
    static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};

template <>
struct Half<__half> {
    static constexpr bool kIsBf16 = false;
    // log2 of the largest softmax weight.  Weights below 2^-14 lose bits and below 2^-25 all of them, and tens of
    // thousands of those can count: with the largest at 2^15 that begins 2^29 and 2^40 below it.
    static constexpr int kTop = 15;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<uint32_t *>(&v);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t w) {
        return __half22float2(*reinterpret_cast<__half2 *>(&w));
    }
    static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};

// log2 of the growth of a maximum that is let pass, and of the largest weight of the tile that set it
template <typename T>
struct Grow {
    static constexpr float kPass = Half<T>::kIsBf16 ? 8.f : 4.f, kTop = Half<T>::kTop > 0 ? Half<T>::kTop - kPass : 0.f;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 1 over a sum of weights, 0 where there were none
__device__ __forceinline__ float inverse(float total) { return total > 0.f || total != total ? 1.f / total : 0.f; }
// the logarithm of a sum of exp2, in the natural base
__device__ __forceinline__ float log_of(float top, float total) {
    return total > 0.f || total != total ? (top + log2f(total)) * kLn2 : -INFINITY;
}

// x * y + z of both halves, rounded once
template <typename T>
__device__ __forceinline__ uint32_t fma2x16(uint32_t x, uint32_t y, uint32_t z) {
    uint32_t r;
    if (Half<T>::kIsBf16) asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(y), "r"(z));
    else asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(y), "r"(z));
    return r;
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

__device__ __forceinline__ void report(int32_t *status) { atomicOr(status, 1); }

// ---- assign (kv_assign.cu)
struct AssignArgs {
    isjl_kv_assign_args a;
    int32_t n_blocks, shift;      // block_size = 1 << shift
    int32_t *work;                // [8 + 4 n_rows], the sums for the kernel that fills
    int32_t aligned;              // the maps to 16 bytes
    int32_t *status;
};
cudaError_t launch_assign(const AssignArgs &a, int sms, cudaStream_t st);

// ---- append (kv_append.cu)
struct AppendArgs {
    isjl_kv_append_args a;
    isjl_kv_cache cache;
    isjl_kv_cache4 cache4;        // launch_append4: the cache
    int32_t n_q_heads, n_kv_heads, shift;
    int64_t n_slots;
    int32_t *status;
};
cudaError_t launch_append(const AppendArgs &a, int head_dim, int type, int sms, cudaStream_t st);
cudaError_t launch_append4(const AppendArgs &a, int head_dim, int type, int sms, cudaStream_t st);

// ---- read4 (kv_read4.cu)
struct Read4Args {
    isjl_kv_read4_args a;
    isjl_kv_cache4 cache;
    int32_t n_kv_heads, shift;
    int64_t n_slots;
    int32_t *status;
};
cudaError_t launch_read4(const Read4Args &a, int head_dim, int type, int sms, cudaStream_t st);

// ---- a shared prefix computed once for the batch (kv_prefix.cu)

// The line of (key head, pair of row tiles, token tile); a row tile holds the queries of whole tokens.
struct PrefixLine {
    int32_t tokens_of_tile, pairs, items, tiles;   // items: key heads x pairs, `tiles` token tiles each
    int32_t blocks, pieces;                        // 0 blocks: there is no such part
    __host__ __device__ int64_t work() const { return (int64_t)items * tiles; }
    // the first and last block that an item's run of the line belongs to
    __host__ __device__ int first_block(int item) const { return (int)((((int64_t)item * tiles + 1) * blocks - 1) / work()); }
    __host__ __device__ int last_block(int item) const { return (int)((((int64_t)item + 1) * tiles * blocks - 1) / work()); }
};

struct PrefixArgs {
    PrefixLine line;
    const void *q;
    int64_t q_stride[2];
    const int32_t *prefix;
    float *part_o;                // [pieces][n][n_q_heads][head_dim], sums of exp2(s - m) v; one more [n] for own tokens
    float2 *part_ml;              // [pieces][n][n_q_heads], m and the sum of exp2(s - m)
    int32_t *status;
    float scale;
    int32_t n, tokens, n_blocks, shift, n_kv_heads, group;
};
void *tensor_map_encoder();       // null if the driver has none
cudaError_t prepare_prefix(int head_dim, int type);   // once for a shape, before its first launch
PrefixLine prefix_line(int n, int group, int n_kv_heads, int tokens, int sms);
cudaError_t launch_prefix(const PrefixArgs &g, const isjl_kv_cache &cache, void *encoder, int head_dim, int type, cudaStream_t st);

// ---- attend (kv_attend.cu)
constexpr int kAttendWarps = 4;   // of a block
// an item (query t, key head or part of one h) in pieces: the warps in whose runs it begins and ends
struct alignas(16) CutItem {
    int32_t t, h;                 // t < 0: none
    int32_t first, last;
};

struct AttendArgs {
    isjl_kv_attend_args a;
    isjl_kv_cache cache;
    int32_t n_blocks, shift, n_kv_heads, group;
    PrefixLine line;              // blocks > 0: the prefix's tokens are done by kv_prefix.cu and merged here
    float *prefix_o;
    float2 *prefix_ml;
    float *part_o;                // [kAttendWarps * grid][2][16][head_dim] pieces of (query, key head) items
    float2 *part_ml;              // [kAttendWarps * grid][2][16]
    CutItem *cut;                 // for the kernel that joins: the cut items at the warps in whose runs they begin
                                  // [kAttendWarps * grid], or with a prefix all items [n * key heads (parts of them)]
    int32_t *status;
};
size_t attend_smem(int head_dim, int n);
// once for a shape, before its first launch: blocks that fit an SM, and the most queries of a call with which they do
// (with more, one block less fits: each holds 4 bytes a query)
cudaError_t prepare_attend(int head_dim, int type, int *blocks, int *queries);
cudaError_t launch_attend(const AttendArgs &g, void *encoder, int head_dim, int type, int grid, cudaStream_t st);

// ---- attend4 (kv_attend4.cu)
struct Attend4Args {
    isjl_kv_attend_args a;
    isjl_kv_cache4 cache;
    int32_t n_blocks, shift, n_kv_heads, group;
    float *part_o;                // [warps][2][16][head_dim] pieces of (query, key head) items: one that began earlier, one
    float2 *part_ml;              // [warps][2][16]           that goes on
    CutItem *cut;                 // [warps] items that begin in a warp's run and are cut by its end; first and last are teams
    int32_t *status;
};
// once for a shape, before its first launch: as prepare_attend; warps: most of a call
cudaError_t prepare_attend4(int head_dim, int type, int group, int sms, int *blocks, int *queries, int *warps);
cudaError_t launch_attend4(const Attend4Args &g, int head_dim, int type, int grid, cudaStream_t st);

// ---- prompt (kv_prompt.cu)
// an item that the end of its block's run cuts; the blocks up to `last` have a piece of it
struct alignas(16) PromptCut {
    int32_t row, head, item;      // row < 0: none
    int32_t last;
};

struct PromptArgs {
    isjl_kv_prompt_args a;
    isjl_kv_cache cache;
    int32_t n_blocks, shift, n_kv_heads, group;
    // by launch_prompt: rows of a tile for each token, tokens of a tile, and how many such parts a key head's queries make
    int32_t rows_of_token, tokens_of_tile, parts;
    int32_t out_wide;             // rows of out lie at multiples of 32 bytes
    float *part_o;                // [blocks][2][rows of an item][head_dim]: kPromptRows rows an SM
    float2 *part_ml;              // [blocks][2][rows of an item], as the prefix's
    PromptCut *cut;               // [blocks]
    int32_t *status;
};
constexpr int kPromptRows = 512;  // of the pieces of an SM's blocks
cudaError_t prepare_prompt(int head_dim, int type);   // once for a shape, before its first launch
cudaError_t launch_prompt(PromptArgs &g, void *encoder, int head_dim, int type, int sms, cudaStream_t st);

}  // namespace isjl
