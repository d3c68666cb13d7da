// kv_append.cu -- norms, position rotation and cache write of new tokens (isjl_kv_append).
//
// A head of D values is D / 8 threads of 8 values (16 bytes) each.  A thread keeps its place in the head and
// goes over the token's heads, so that the angles and weights of that place are loaded once per token; the
// sum of squares and the other half of a rotated pair come from the head's other threads by shuffles.  All
// arithmetic is in 32 bits with one rounding at the end.  Bound by memory: 4 bytes a value (49,152 tokens of
// 32 + 2 x 8 heads of 128 values 202 us, 6.1 TB/s).
#include "kv_internal.cuh"

namespace isjl {
namespace {

constexpr int kAhead = 3;      // values of a thread that are under way together, 16 bytes each

template <typename T>
__device__ __forceinline__ void unpack8(const uint4 &w, float (&x)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = Half<T>::unpack(u[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

template <int D, typename T, int kThreads>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendArgs g) {
    constexpr int kLanes = D / 8, kHeads = kThreads / kLanes;   // threads of a head, heads at a time
    const isjl_kv_append_args &a = g.a;
    const int t = blockIdx.x, c = threadIdx.x % kLanes, part = threadIdx.x / kLanes;
    const int hq = g.n_q_heads, hkv = g.n_kv_heads, heads = hq + 2 * hkv, half = a.rot / 2;
    const T *x_in = static_cast<const T *>(a.qkv) + t * a.qkv_stride + 8 * c;
    // values are asked for kAhead heads at a time, the first ones before anything that they do not need
    uint4 raw[kAhead];
    auto fetch = [&](int h0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int h = h0 + u * kHeads + part;
            raw[u] = h < heads ? *reinterpret_cast<const uint4 *>(x_in + (int64_t)h * D) : make_uint4(0, 0, 0, 0);
        }
    };
    fetch(0);
    const uint4 none = make_uint4(0, 0, 0, 0);
    const uint4 qw = a.q_weight ? *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.q_weight) + 8 * c) : none;
    const uint4 kw = a.k_weight ? *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.k_weight) + 8 * c) : none;
    int64_t slot = a.slots[t];
    int position = a.rot ? a.positions[t] : 0;
    if (slot >= 0 && (slot >= g.n_slots || position < 0 || (a.rot && position >= a.n_positions))) {
        if (threadIdx.x == 0) report(g.status);
        slot = -1;
    }
    T *q_out = static_cast<T *>(a.q_out) + t * a.q_out_stride;
    if (slot < 0) {
        for (int i = threadIdx.x; i < hq * kLanes; i += kThreads) reinterpret_cast<uint4 *>(q_out)[i] = none;
        return;
    }
    const int64_t block = slot >> g.shift, place = slot & ((1 << g.shift) - 1);
    T *k_out = static_cast<T *>(g.cache.k) + block * g.cache.k_stride[0] + place * g.cache.k_stride[1];
    T *v_out = static_cast<T *>(g.cache.v) + block * g.cache.v_stride[0] + place * g.cache.v_stride[1];

    // values 8 c .. 8 c + 7 of a head: their angles, and where their pairs are
    const bool turns = 8 * c < a.rot;
    const bool second = !a.interleaved && 8 * c >= half;
    float cosv[8], sinv[8];                  // sines with the sign that the pair's other value has
#pragma unroll
    for (int i = 0; i < 8; ++i) { cosv[i] = 1.f; sinv[i] = 0.f; }
    if (turns) {
        const float *angle = a.rope + (int64_t)position * a.rot;
        const int j = a.interleaved ? 4 * c : 8 * c - (second ? half : 0), count = a.interleaved ? 1 : 2;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (k >= count) break;
            const float4 x = *reinterpret_cast<const float4 *>(angle + j + 4 * k), y = *reinterpret_cast<const float4 *>(angle + half + j + 4 * k);
            const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (a.interleaved) {
                    cosv[2 * i] = cosv[2 * i + 1] = xs[i];
                    sinv[2 * i] = -ys[i];
                    sinv[2 * i + 1] = ys[i];
                } else {
                    cosv[4 * k + i] = xs[i];
                    sinv[4 * k + i] = second ? ys[i] : -ys[i];
                }
            }
        }
    }
    const int partner = turns && !a.interleaved ? (second ? c - half / 8 : c + half / 8) : c;
    const int lane = threadIdx.x & 31, from = lane - (lane % kLanes) + partner;

    // the same number of turns for every thread, so that whole warps take part in the shuffles
    for (int h0 = 0; h0 < heads; h0 += kAhead * kHeads) {
        if (h0) fetch(h0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (h0 + u * kHeads >= heads) break;
            __syncwarp();
            const int h = h0 + u * kHeads + part;
            const bool is_v = h >= hq + hkv, is_k = !is_v && h >= hq;
            float x[8];
            unpack8<T>(raw[u], x);
            uint4 w = raw[u];
            if (h0 + u * kHeads < hq + hkv) {        // some of the warps' heads are q or k heads
                const bool normed = is_k ? a.k_weight != nullptr : a.q_weight != nullptr;
                if (a.q_weight || a.k_weight) {
                    float sum = 0.f, scale[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
#pragma unroll
                    for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor_sync(~0u, sum, d);
                    unpack8<T>(is_k ? kw : qw, scale);
                    const float r = rsqrtf(sum * (1.f / D) + a.eps);
                    if (normed)
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] *= r * scale[i];
                }
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float other = __shfl_sync(~0u, x[i], from);
                    y[i] = turns ? x[i] * cosv[i] + (a.interleaved ? x[i ^ 1] : other) * sinv[i] : x[i];
                }
                if (!is_v) w = make_uint4(Half<T>::pack(y[0], y[1]), Half<T>::pack(y[2], y[3]), Half<T>::pack(y[4], y[5]), Half<T>::pack(y[6], y[7]));
            }
            if (h >= heads) continue;
            T *to = is_v ? v_out + (h - hq - hkv) * g.cache.v_stride[2]
                         : is_k ? k_out + (h - hq) * g.cache.k_stride[2] : q_out + (int64_t)h * D;
            *reinterpret_cast<uint4 *>(to + 8 * c) = w;
        }
    }
}

// Measured, 32 against 128 threads: 2,048 tokens of 32 + 2 x 8 heads of 128 values 15.5 and 12.6 us, 4,096 tokens 21.0 and
// 22.1, 49,152 tokens 201 and 226; with 28 + 2 x 4 heads of 64 values 5.9 and 6.4 at 2,048 tokens, 5.2 and 4.1 at 1,024.
// The rule goes by tokens alone and is that of the larger ones: with the smaller ones it loses 0.5 us at 2,048.
int many_tokens(int sms) { return 24 * sms; }

// A token is a block.  Few tokens: four warps each, which halve its latency.  Many: a warp each, for more of them under
// way on an SM without waiting for one another's longest.
template <int D, typename T>
cudaError_t launch_of(const AppendArgs &g, int sms, cudaStream_t st) {
    if (g.a.n_tokens >= many_tokens(sms)) append_kernel<D, T, 32><<<g.a.n_tokens, 32, 0, st>>>(g);
    else append_kernel<D, T, 128><<<g.a.n_tokens, 128, 0, st>>>(g);
    return cudaGetLastError();
}

template <int D>
cudaError_t launch_dim(const AppendArgs &g, int type, int sms, cudaStream_t st) {
    return type == ISJL_KV_BF16 ? launch_of<D, __nv_bfloat16>(g, sms, st) : launch_of<D, __half>(g, sms, st);
}

}  // namespace

cudaError_t launch_append(const AppendArgs &g, int head_dim, int type, int sms, cudaStream_t st) {
    return head_dim == 64 ? launch_dim<64>(g, type, sms, st)
         : head_dim == 128 ? launch_dim<128>(g, type, sms, st) : launch_dim<256>(g, type, sms, st);
}

}  // namespace isjl
