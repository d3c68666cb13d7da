// kv_read4.cu -- 16-bit values of slots of a cache in 4 bits (isjl_kv_read4).
//
// A thread takes 8 codes (4 bytes) to 8 values (16 bytes); a block has some tokens' keys and values.  Bound by memory:
// 5 bits a value in, 16 out.
#include "kv_four.cuh"

namespace isjl {
namespace {

constexpr int kThreads = 256;

template <int D, typename T>
__global__ void __launch_bounds__(kThreads) read4_kernel(const __grid_constant__ Read4Args g, int tokens_of_block) {
    const isjl_kv_read4_args &a = g.a;
    constexpr int kLanes = D / 8;
    const int words = 2 * g.n_kv_heads * kLanes;               // of a token
    const int first = blockIdx.x * tokens_of_block, tokens = min(tokens_of_block, a.n_tokens - first);
    for (int i = threadIdx.x; i < tokens * words; i += kThreads) {
        const int t = i / words, j = i - t * words, side = j >= words / 2, c = j % kLanes;
        const int h = (side ? j - words / 2 : j) / kLanes;
        const int64_t slot = a.slots[first + t];
        const int64_t *to_stride = side ? a.v_stride : a.k_stride;
        T *to = static_cast<T *>(side ? a.v_out : a.k_out) + (first + t) * to_stride[0] + h * to_stride[1] + 8 * c;
        uint32_t v[4] = {0, 0, 0, 0};
        if (slot >= 0 && slot < g.n_slots) {
            const int64_t block = slot >> g.shift, place = slot & ((1 << g.shift) - 1);
            const int64_t *cs = side ? g.cache.v_stride : g.cache.k_stride, *ss = side ? g.cache.v_scale_stride : g.cache.k_scale_stride;
            const uint32_t word = *reinterpret_cast<const uint32_t *>(
                static_cast<const unsigned char *>(side ? g.cache.v : g.cache.k) + block * cs[0] + place * cs[1] + h * cs[2] + 4 * c);
            const uint32_t pair = *reinterpret_cast<const uint32_t *>(
                static_cast<const T *>(side ? g.cache.v_scale : g.cache.k_scale) + block * ss[0] + place * ss[1] + h * ss[2] + c / 4 * 2);
            Four<T>::values(v, word, pair);
        } else if (slot >= g.n_slots && j == 0) {
            report(g.status);
        }
        *reinterpret_cast<uint4 *>(to) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

template <int D, typename T>
cudaError_t launch_of(const Read4Args &g, cudaStream_t st) {
    const int words = 2 * g.n_kv_heads * (D / 8), per = max(1, 4 * kThreads / words);
    read4_kernel<D, T><<<(g.a.n_tokens - 1) / per + 1, kThreads, 0, st>>>(g, per);
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
