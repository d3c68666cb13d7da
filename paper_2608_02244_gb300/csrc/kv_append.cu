// kv_append.cu -- norms, position rotation and cache write of new tokens (isjl_kv_append, isjl_kv_append4).
//
// A head of D values is D / 8 threads of 8 values (16 bytes) each.  A thread keeps its place in the head and
// goes over the token's heads, so that the angles and weights of that place are loaded once per token; the
// sum of squares and the other half of a rotated pair come from the head's other threads by shuffles.  All
// arithmetic is in 32 bits with one rounding at the end.  Bound by memory: 4 bytes a value (49,152 tokens of
// 32 + 2 x 8 heads of 128 values 202 us, 6.1 TB/s).
//
// A cache in 4 bits: a group of 32 values is four neighbouring threads, whose least and largest value come by two
// shuffles; each thread makes a word of its eight codes, the first of the four writes scale and offset.  Bound by
// instructions: 20,011 tokens of 28 + 2 x 4 heads of 64 values 40 us, 31 into 16 bits, whose rows in memory are longer.
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

// The codes of this thread's 8 values of a group, and the group's scale and offset, in T.  16-bit values lie on borders
// between codes often, so the quotient d / S, with d = x - B, has to be rounded as the definition has it.  A border is
// t S with t = 1 + (c + 1/2) / 16, exact in 32 bits, and d is a number of 32 bits in the same or the next binade: where
// they differ, they do so by more than S 2^-24, and the rounded quotient is on the same side of t.  So an estimate with
// the reciprocal is put right by d's exact distance from the estimate's value: beyond half a step, or at it and odd.
template <typename T>
__device__ __forceinline__ uint32_t codes4(const float (&x)[8], uint32_t *scales) {
    float lo = x[0], hi = x[0];
    bool fine = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        fine = fine && fabsf(x[i]) < INFINITY;
    }
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(~0u, lo, d));
        hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, d));
        fine = __shfl_xor_sync(~0u, (int)fine, d) && fine;
    }
    const float s = Half<T>::unpack(Half<T>::pack((hi - lo) * (16.f / 15.f), 0.f)).x;
    const float b = Half<T>::unpack(Half<T>::pack(lo - s, 0.f)).x;
    fine = fine && s < INFINITY && b > -INFINITY;
    *scales = fine ? Half<T>::pack(s, b) : Half<T>::pack(NAN, NAN);
    uint32_t word = 0;
    if (fine && s > 0.f) {
        // A scale below the normal numbers: all of it by 2^64, which changes no quotient.  So do large ones by 2^-4, for
        // distances d of which 32 bits hold no number.
        const float up = s < 0x1p-100f ? 0x1p64f : s > 0x1p100f ? 0x1p-4f : 1.f, step = s * up * 0.0625f, inv = __fdividef(1.f, step);
        const float from = -b * up;
        constexpr float kWhole = 0x1.8p23f;         // a sum with it is rounded to a whole number, ties to even
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = fmaf(x[i], up, from), n = fmaf(d, inv, kWhole), off = fabsf(fmaf(kWhole - n, step, d));
            int c = __float_as_int(n) - __float_as_int(kWhole + 16.f);
            if (off > step * 0.5f || (off == step * 0.5f && (c & 1))) c += d > (n - kWhole) * step ? 1 : -1;
            word |= (uint32_t)min(max(c, 0), 15) << (4 * i);
        }
    }
    return word;
}

template <int D, typename T, int kThreads, bool kFour>
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
                // codes are made of y, which for a value head is what came; its 16 bits are kept as they are
                const bool normed = !(kFour && is_v) && (is_k ? a.k_weight != nullptr : a.q_weight != nullptr), turned = turns && !(kFour && is_v);
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
                if (a.interleaved) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = turned ? x[i] * cosv[i] + x[i ^ 1] * sinv[i] : x[i];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float other = __shfl_sync(~0u, x[i], from);
                        y[i] = turned ? x[i] * cosv[i] + other * sinv[i] : x[i];
                    }
                }
                if (!is_v) w = make_uint4(Half<T>::pack(y[0], y[1]), Half<T>::pack(y[2], y[3]), Half<T>::pack(y[4], y[5]), Half<T>::pack(y[6], y[7]));
                if (kFour)
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = y[i];
            }
            if (kFour && h0 + (u + 1) * kHeads > hq) {      // some of the warps' heads are k or v heads
                uint32_t pair;
                __syncwarp();
                const uint32_t word = codes4<T>(x, &pair);
                if (h >= hq && h < heads) {
                    const isjl_kv_cache4 &four = g.cache4;
                    const int64_t *cs = is_v ? four.v_stride : four.k_stride, *ss = is_v ? four.v_scale_stride : four.k_scale_stride;
                    const int head = is_v ? h - hq - hkv : h - hq;
                    *reinterpret_cast<uint32_t *>(static_cast<unsigned char *>(is_v ? four.v : four.k) + block * cs[0] + place * cs[1] + head * cs[2] + 4 * c) = word;
                    if (c % 4 == 0)
                        *reinterpret_cast<uint32_t *>(static_cast<T *>(is_v ? four.v_scale : four.k_scale) + block * ss[0] + place * ss[1] + head * ss[2] + c / 4 * 2) = pair;
                }
                if (h >= hq) continue;
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
// The rule goes by tokens alone and is that of the larger ones: with the smaller ones it loses 0.5 us at 2,048.  4-bit caches
// have the same rule, measured inside a graph (an empty one takes 8.8 us): with the larger heads 20.3 and 13.0 us at 1,024
// tokens, 23.0 and 20.7 at 2,048, 29.2 and 29.2 at 3,584, 128 and 137 at 20,011; with the smaller ones 10.5 and 9.2 at 1,024,
// 11.2 and 13.0 at 2,048, 13.5 and 18.6 at 3,584, 49 and 79 at 20,011: there it loses 2 to 5 us from 2,048 to 3,647.
int many_tokens(int sms) { return 24 * sms; }

// A token is a block.  Few tokens: four warps each, which halve its latency.  Many: a warp each, for more of them under
// way on an SM without waiting for one another's longest.
template <int D, typename T, bool kFour>
cudaError_t launch_of(const AppendArgs &g, int sms, cudaStream_t st) {
    if (g.a.n_tokens >= many_tokens(sms)) append_kernel<D, T, 32, kFour><<<g.a.n_tokens, 32, 0, st>>>(g);
    else append_kernel<D, T, 128, kFour><<<g.a.n_tokens, 128, 0, st>>>(g);
    return cudaGetLastError();
}

template <int D, bool kFour>
cudaError_t launch_dim(const AppendArgs &g, int type, int sms, cudaStream_t st) {
    return type == ISJL_KV_BF16 ? launch_of<D, __nv_bfloat16, kFour>(g, sms, st) : launch_of<D, __half, kFour>(g, sms, st);
}

template <bool kFour>
cudaError_t launch_any(const AppendArgs &g, int head_dim, int type, int sms, cudaStream_t st) {
    return head_dim == 64 ? launch_dim<64, kFour>(g, type, sms, st)
         : head_dim == 128 ? launch_dim<128, kFour>(g, type, sms, st) : launch_dim<256, kFour>(g, type, sms, st);
}

}  // namespace

cudaError_t launch_append(const AppendArgs &g, int head_dim, int type, int sms, cudaStream_t st) {
    return launch_any<false>(g, head_dim, type, sms, st);
}

cudaError_t launch_append4(const AppendArgs &g, int head_dim, int type, int sms, cudaStream_t st) {
    return launch_any<true>(g, head_dim, type, sms, st);
}

}  // namespace isjl
