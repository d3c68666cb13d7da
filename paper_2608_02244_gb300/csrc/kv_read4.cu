// kv_read4.cu -- 16-bit values of slots of a cache in 4 bits (isjl_kv_read4).
//
// A thread takes 8 codes (4 bytes) to 8 values (16 bytes), the same place of eight tokens, whose loads are under way
// together.  Bound by memory, 5 bits a value in, 16 out: 98,309 tokens of 8 heads of 128 values, 529 MB, 95 us (5.6 TB/s; four
// tokens a thread 119, sixteen 120).
#include "kv_four.cuh"

#include <algorithm>

namespace isjl {
namespace {

constexpr int kThreads = 128, kTokens = 8;

template <int D, typename T>
__global__ void __launch_bounds__(kThreads) read4_kernel(const __grid_constant__ Read4Args g) {
    const isjl_kv_read4_args &a = g.a;
    constexpr int kLanes = D / 8;
    const int words = 2 * g.n_kv_heads * kLanes, groups = max(1, kThreads / words);        // of a token; tokens side by side
    const int group = threadIdx.x / words;                     // beyond groups - 1: nothing to do
    const int64_t first = ((int64_t)blockIdx.x * groups + group) * kTokens;
    if (words <= kThreads && group >= groups) return;
    for (int j = words <= kThreads ? threadIdx.x - group * words : threadIdx.x; j < words; j += kThreads) {
        const int side = j >= words / 2, c = j % kLanes, h = (side ? j - words / 2 : j) / kLanes;
        const int64_t *cs = side ? g.cache.v_stride : g.cache.k_stride, *ss = side ? g.cache.v_scale_stride : g.cache.k_scale_stride;
        const unsigned char *codes = static_cast<const unsigned char *>(side ? g.cache.v : g.cache.k) + h * cs[2] + 4 * c;
        const T *scales = static_cast<const T *>(side ? g.cache.v_scale : g.cache.k_scale) + h * ss[2] + c / 4 * 2;
        const int64_t *to_stride = side ? a.v_stride : a.k_stride;
        T *to = static_cast<T *>(side ? a.v_out : a.k_out) + first * to_stride[0] + h * to_stride[1] + 8 * c;
        int64_t slot[kTokens];
        uint32_t word[kTokens], pair[kTokens];
#pragma unroll
        for (int u = 0; u < kTokens; ++u) slot[u] = first + u < a.n_tokens ? a.slots[first + u] : -1;
#pragma unroll
        for (int u = 0; u < kTokens; ++u) {
            word[u] = pair[u] = 0;                             // stands for 0
            if (slot[u] >= g.n_slots) {
                if (j == 0) report(g.status);
            } else if (slot[u] >= 0) {
                const int64_t block = slot[u] >> g.shift, place = slot[u] & ((1 << g.shift) - 1);
                word[u] = __ldcs(reinterpret_cast<const uint32_t *>(codes + block * cs[0] + place * cs[1]));
                pair[u] = *reinterpret_cast<const uint32_t *>(scales + block * ss[0] + place * ss[1]);
            }
        }
#pragma unroll
        for (int u = 0; u < kTokens; ++u) {
            uint32_t v[4];
            Four<T>::values(v, word[u], pair[u]);
            if (first + u < a.n_tokens) __stcs(reinterpret_cast<uint4 *>(to + u * to_stride[0]), make_uint4(v[0], v[1], v[2], v[3]));
        }
    }
}

template <int D, typename T>
cudaError_t launch_of(const Read4Args &g, cudaStream_t st) {
    const int words = 2 * g.n_kv_heads * (D / 8), per = kTokens * std::max(1, kThreads / words);
    read4_kernel<D, T><<<(g.a.n_tokens - 1) / per + 1, kThreads, 0, st>>>(g);
    return cudaGetLastError();
}

template <int D>
cudaError_t launch_dim(const Read4Args &g, int type, cudaStream_t st) {
    return type == ISJL_KV_BF16 ? launch_of<D, __nv_bfloat16>(g, st) : launch_of<D, __half>(g, st);
}

}  // namespace

cudaError_t launch_read4(const Read4Args &g, int head_dim, int type, int, cudaStream_t st) {
    return head_dim == 64 ? launch_dim<64>(g, type, st) : head_dim == 128 ? launch_dim<128>(g, type, st) : launch_dim<256>(g, type, st);
}

}  // namespace isjl
