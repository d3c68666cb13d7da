// kv_four.cuh -- what codes of 4 bits stand for: T(B + (1 + c / 16) S), with the group's scale S and offset B.
//
// 1 + c / 16 is a 16-bit number with the code in the top bits of its mantissa: a shift and one logical instruction make
// two of them, and one fused multiplication and addition, rounded once, their values.  That is why the format counts
// from 1 + c / 16: with c itself each pair would take another instruction to get rid of the constant.
#pragma once

#include "kv_internal.cuh"

namespace isjl {

template <typename T>
struct Four {
    static constexpr uint32_t kOne = Half<T>::kIsBf16 ? 0x3f803f80u : 0x3c003c00u;    // 1, 1
    static constexpr int kBit = Half<T>::kIsBf16 ? 3 : 6;                             // of the code's lowest bit
    static constexpr uint32_t kMask = 0x000f000fu << kBit;

    static __device__ __forceinline__ uint32_t fma(uint32_t x, uint32_t s, uint32_t b) { return fma2x16<T>(x, s, b); }
    // 1 + c / 16 of the codes at bits 4 kPlace of each half
    template <int kPlace>
    static __device__ __forceinline__ uint32_t ones(uint32_t word) {
        constexpr int kShift = kBit - 4 * kPlace;
        const uint32_t at = kShift >= 0 ? word << (kShift & 31) : word >> (-kShift & 31);
        uint32_t x;                  // (at & kMask) | kOne: said in C++ it became two instructions
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x) : "r"(at), "n"(kMask), "r"(kOne));
        return x;
    }
    // both halves of a scale and offset pair
    static __device__ __forceinline__ uint32_t scale2(uint32_t pair) { return __byte_perm(pair, 0, 0x1010); }
    static __device__ __forceinline__ uint32_t offset2(uint32_t pair) { return __byte_perm(pair, 0, 0x3232); }

    // the eight values of a word, in order
    static __device__ __forceinline__ void values(uint32_t (&v)[4], uint32_t word, uint32_t pair) {
        const uint32_t s = scale2(pair), b = offset2(pair);
        // places i and i + 4 of the word come together
        const uint32_t x[4] = {fma(ones<0>(word), s, b), fma(ones<1>(word), s, b), fma(ones<2>(word), s, b), fma(ones<3>(word), s, b)};
        v[0] = __byte_perm(x[0], x[1], 0x5410);
        v[1] = __byte_perm(x[2], x[3], 0x5410);
        v[2] = __byte_perm(x[0], x[1], 0x7632);
        v[3] = __byte_perm(x[2], x[3], 0x7632);
    }
};

}  // namespace isjl
