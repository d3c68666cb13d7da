// kv_simple.cu -- attention of single queries over a cache in 4 bits (isjl_kv_attend4), a block for each
// query and query head: each warp takes every fourth visible token, a lane D / 32 of the values, with the running
// maximum and sum of a softmax; the warps' results are joined at the end.
#include "kv_four.cuh"

namespace isjl {
namespace {

constexpr int kWarps = 4;

template <int D, typename T>
__device__ __forceinline__ void load_values(float (&x)[D / 32], const T *p, int lane) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const float2 f = Half<T>::unpack(*reinterpret_cast<const uint32_t *>(p + 64 * i + 2 * lane));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

template <int D, typename T>
__device__ __forceinline__ void load_four(float (&x)[D / 32], const unsigned char *codes, const T *scales, int lane) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const int d = 64 * i + 2 * lane;
        const uint32_t byte = codes[d / 2], pair = *reinterpret_cast<const uint32_t *>(scales + d / 32 * 2);
        const uint32_t w = Four<T>::fma(Four<T>::template ones<0>((byte & 15) | (byte >> 4) << 16), Four<T>::scale2(pair), Four<T>::offset2(pair));
        const float2 f = Half<T>::unpack(w);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

// One query: tokens of `end` (prefix and own ones) from lo on and the first `sinks`; `load` gets a token's key or value.
template <int D, typename T, typename Load>
__device__ void attend_one(const T *q, T *out, float *lse, int32_t end, int32_t lo, int32_t sinks, float scale, const Load &load) {
    __shared__ float tops[kWarps], totals[kWarps], sums[kWarps][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float qx[D / 32], o[D / 32] = {}, top = -INFINITY, total = 0.f;
    load_values<D, T>(qx, q, lane);
    sinks = min(sinks, lo);
    for (int32_t i = warp; i < sinks + (end - lo); i += kWarps) {
        const int32_t y = i < sinks ? i : lo + (i - sinks);
        float x[D / 32], s = 0.f;
        load(x, y, false);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) s += qx[j] * x[j];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) s += __shfl_xor_sync(~0u, s, d);
        s *= scale;
        const float next = fmaxf(top, s), ref = next == -INFINITY ? 0.f : next, fix = expf(top - ref), p = expf(s - ref);
        top = next;
        total = total * fix + p;
        load(x, y, true);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) o[j] = o[j] * fix + p * x[j];
    }
    if (lane == 0) { tops[warp] = top; totals[warp] = total; }
    __syncthreads();
    float most = -INFINITY, sum = 0.f;
    for (int w = 0; w < kWarps; ++w) most = fmaxf(most, tops[w]);
    const float ref = most == -INFINITY ? 0.f : most;
    for (int w = 0; w < kWarps; ++w) sum += totals[w] * expf(tops[w] - ref);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) sums[warp][64 * (j / 2) + 2 * lane + j % 2] = o[j] * expf(top - ref);
    __syncthreads();
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    for (int d = 2 * threadIdx.x; d < D; d += 64 * kWarps) {
        float a = 0.f, b = 0.f;
        for (int w = 0; w < kWarps; ++w) { a += sums[w][d]; b += sums[w][d + 1]; }
        *reinterpret_cast<uint32_t *>(out + d) = Half<T>::pack(a * inv, b * inv);
    }
    if (lse && threadIdx.x == 0) *lse = sum > 0.f || sum != sum ? most + logf(sum) : -INFINITY;
}

template <int D, typename T>
__global__ void __launch_bounds__(32 * kWarps) attend4_kernel(const __grid_constant__ Attend4Args g) {
    const isjl_kv_attend_args &a = g.a;
    const int t = blockIdx.x, h = blockIdx.y, kv = h / g.group, lane = threadIdx.x & 31;
    const int32_t x = a.lens[t], row = a.rows ? a.rows[t] : t, prefix = a.n_prefix_blocks << g.shift;
    const bool bad = x > 0 && row >= 0 && (row >= a.n_table_rows || ((x - 1) >> g.shift) >= a.table_width);
    if (bad && threadIdx.x == 0) report(g.status);
    const int32_t end = x <= 0 || row < 0 || bad ? 0 : x + prefix, lo = a.window && end > a.window ? end - a.window : 0;
    attend_one<D, T>(static_cast<const T *>(a.q) + t * a.q_stride[0] + h * a.q_stride[1],
                     static_cast<T *>(a.out) + t * a.out_stride[0] + h * a.out_stride[1],
                     a.lse ? a.lse + (int64_t)t * gridDim.y + h : nullptr, end, lo, a.sinks, a.scale, [&](float (&v)[D / 32], int32_t y, bool value) {
        const int32_t j = y >> g.shift, place = y & ((1 << g.shift) - 1);
        const int32_t block = j < a.n_prefix_blocks ? a.prefix[j] : a.table[(int64_t)row * a.table_width + j - a.n_prefix_blocks];
        if ((uint32_t)block >= (uint32_t)g.n_blocks) {
            report(g.status);
            for (float &e : v) e = 0.f;
            return;
        }
        const int64_t *cs = value ? g.cache.v_stride : g.cache.k_stride, *ss = value ? g.cache.v_scale_stride : g.cache.k_scale_stride;
        load_four<D, T>(v, static_cast<const unsigned char *>(value ? g.cache.v : g.cache.k) + block * cs[0] + place * cs[1] + kv * cs[2],
                        static_cast<const T *>(value ? g.cache.v_scale : g.cache.k_scale) + block * ss[0] + place * ss[1] + kv * ss[2], lane);
    });
}

template <int D, typename T>
cudaError_t attend4_of(const Attend4Args &g, cudaStream_t st) {
    attend4_kernel<D, T><<<dim3(g.a.n, g.n_kv_heads * g.group), 32 * kWarps, 0, st>>>(g);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend4(const Attend4Args &g, int head_dim, int type, cudaStream_t st) {
    if (type == ISJL_KV_BF16)
        return head_dim == 64 ? attend4_of<64, __nv_bfloat16>(g, st) : head_dim == 128 ? attend4_of<128, __nv_bfloat16>(g, st) : attend4_of<256, __nv_bfloat16>(g, st);
    return head_dim == 64 ? attend4_of<64, __half>(g, st) : head_dim == 128 ? attend4_of<128, __half>(g, st) : attend4_of<256, __half>(g, st);
}

}  // namespace isjl
