// kv_prompt_wide.cu -- isjl_kv_prompt with heads of 256 values.
//
// The same line of items as kv_prompt.cu, with 64 rows an item and tiles of 64 tokens.  A row tile's scores, weights
// and 256 sums fit a warp's registers at 16 rows, so a block is four warps with one tile of keys and of values in shared
// memory between them: the next keys come in while the values are at work and the other way round, by asynchronous
// copies of 16 bytes, and two blocks share an SM.  The products are a warp's own (16 x 8 x 16): 128 rows' sums of 256
// values would fill the half of TMEM that two row tiles need for their scores.
#include "kv_prompt.cuh"

namespace isjl {
namespace {

constexpr int D = 256, kRows = 64, kKeys = 64, kThreads = 128, kBlocks = 2;      // blocks of an SM
constexpr int kRowBytes = 2 * D, kTileBytes = kKeys * kRowBytes, kSmem = 3 * kTileBytes;      // queries, keys, values

// where 16 bytes of a row lie: eight rows' same places on all banks
__device__ __forceinline__ uint32_t place16(int row, int c) { return row * kRowBytes + ((c ^ (row & 7)) << 4); }

__device__ __forceinline__ void copy16(uint32_t to, const void *from, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(real ? 16 : 0) : "memory");
}

template <typename T>
__global__ void __launch_bounds__(kThreads, kBlocks) prompt_wide_kernel(const __grid_constant__ PromptArgs g) {
    extern __shared__ __align__(128) unsigned char raw[];
    __shared__ RunWords words;
    __shared__ int32_t left_out;                       // a value of the item is not finite and not seen by all
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t q_at = smem_addr(raw), k_at = q_at + kTileBytes, v_at = k_at + kTileBytes;
    const PromptShape shape = {kKeys, g.tokens_of_tile, g.a.window, g.a.sinks};
    const float scale = g.a.scale * kLog2e;

    start_next();
    if (threadIdx.x == 0) g.cut[blockIdx.x].row = -1;
    Run run = find_run<kThreads>(g, shape, words);
    begin_run(g, shape, words, run);

    // a tile's keys or values: each thread's 16 bytes of every fourth row, zeros for what no query sees
    auto copy_tile = [&](const Item &x, int j, bool values) {
        const int32_t y0 = tile_at(shape, x, j);
        const T *side = static_cast<const T *>(values ? g.cache.v : g.cache.k);
        const int64_t *stride = values ? g.cache.v_stride : g.cache.k_stride;
        const uint32_t to = values ? v_at : k_at;
        const int c = lane;
        int32_t last = -1, block = -1;
#pragma unroll 4
        for (int i = 0; i < kKeys / 4; ++i) {
            // a warp has neighbouring rows, mostly of one cache block
            const int row = warp * (kKeys / 4) + i;
            const int32_t y = y0 + row;
            const bool seen = !(x.kind & kDead) && y < x.end && (y >= x.low || y < shape.sinks);
            if (seen && y >> g.shift != last) {
                last = y >> g.shift;
                block = block_at(g, x.row, y);
                if ((uint32_t)block >= (uint32_t)g.n_blocks) {
                    if (c == 0) report(g.status);
                    block = -1;
                }
            }
            const bool real = seen && block >= 0;
            const T *from = side + (real ? block * stride[0] + (y & ((1 << g.shift) - 1)) * stride[1] + x.kv * stride[2] + 8 * c : 0);
            copy16(to + place16(row, c), from, real);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

    const int r = lane >> 2, c2 = (lane & 3) * 2;       // this lane's rows r and r + 8 of the warp's 16, columns 8 i + c2 and + 1
    for (Item x = take_item(g, shape, run, threadIdx.x == 0); x.count > 0; x = take_item(g, shape, run, threadIdx.x == 0)) {
        __syncthreads();                               // all are done with the item before
        if (threadIdx.x == 0) left_out = 0;
        copy_tile(x, 0, false);
        for (int i = threadIdx.x; i < kRows * (D / 8); i += kThreads) {
            const int row = i / (D / 8), c = i % (D / 8), token = row / g.rows_of_token, member = row % g.rows_of_token;
            const bool live = token < g.tokens_of_tile && member < x.members && token < x.tokens;
            uint4 w = make_uint4(0, 0, 0, 0);
            if (live)
                w = *reinterpret_cast<const uint4 *>(static_cast<const T *>(g.a.q) + (int64_t)(x.start + token) * g.a.q_stride[0] +
                                                     (int64_t)(x.q_head + member) * g.a.q_stride[1] + 8 * c);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_at + place16(row, c)), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
        }
        copy_tile(x, 0, true);
        // this lane's two rows
        int token[2], q_head[2];
        bool live[2];
        int32_t seen_end[2], low[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = warp * 16 + r + 8 * h, member = row % g.rows_of_token;
            token[h] = row / g.rows_of_token;
            q_head[h] = x.q_head + member;
            live[h] = token[h] < g.tokens_of_tile && member < x.members && token[h] < x.tokens;
            seen_end[h] = x.kind & kDead ? 0 : x.place + token[h] + 1;
            low[h] = low_of(shape, x.place + token[h]);
        }
        float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
        for (int j = 0; j < x.count; ++j) {
            const int32_t y0 = tile_at(shape, x, j);
            asm volatile("cp.async.wait_group 1;" ::: "memory");       // the keys; the values are under way
            __syncthreads();
            float s[kKeys / 8][4] = {};
#pragma unroll 4
            for (int k = 0; k < D / 16; ++k) {
                uint32_t a[4];
                ldsm4(a, q_at + place16(warp * 16 + (lane & 15), 2 * k + (lane >> 4)));
#pragma unroll
                for (int t = 0; t < kKeys / 16; ++t) {
                    // lanes 0-7: tokens 0-7 low half of 16 values, 8-15: high half, 16-23: tokens 8-15 low, 24-31: high
                    uint32_t b[4];
                    ldsm4(b, k_at + place16(t * 16 + (lane & 7) + (lane >> 4) * 8, 2 * k + ((lane >> 3) & 1)));
                    Half<T>::mma(s[2 * t], a, b[0], b[1]);
                    Half<T>::mma(s[2 * t + 1], a, b[2], b[3]);
                }
            }
            __syncthreads();                           // all have read the keys
            if (j + 1 < x.count) copy_tile(x, j + 1, false);
            else asm volatile("cp.async.commit_group;" ::: "memory");
            // what a row does not see
            const bool part = edge(shape, x, y0);
            if (part) {
#pragma unroll
                for (int i = 0; i < kKeys / 8; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int32_t y = y0 + 8 * i + c2 + (e & 1);
                        if (y >= seen_end[e >> 1] || (y < low[e >> 1] && y >= shape.sinks)) s[i][e] = -INFINITY;
                    }
            }
            __syncwarp();
            float top[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float most = fmaxf(s[0][2 * h], s[0][2 * h + 1]);
#pragma unroll
                for (int i = 1; i < kKeys / 8; ++i) most = fmaxf(most, fmaxf(s[i][2 * h], s[i][2 * h + 1]));
                most *= scale;
                most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
                top[h] = fmaxf(most, __shfl_xor_sync(~0u, most, 2)) - Half<T>::kTop;
            }
            if (__any_sync(~0u, top[0] > m[0] || top[1] > m[1])) {
                float fix[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float next = fmaxf(m[h], top[h]);
                    fix[h] = m[h] == next ? 1.f : ex2(m[h] - next);
                    m[h] = next;
                    l[h] *= fix[h];
                }
#pragma unroll
                for (int i = 0; i < D / 8; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][e] *= fix[e >> 1];
            }
            const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
            float sum[2] = {0.f, 0.f};
            uint32_t w[kKeys / 16][4];
#pragma unroll
            for (int i = 0; i < kKeys / 8; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float u = ex2(fmaf(s[i][2 * h], scale, -ref[h])), v = ex2(fmaf(s[i][2 * h + 1], scale, -ref[h]));
                    sum[h] += u + v;
                    w[i / 2][(i & 1) * 2 + h] = Half<T>::pack(u, v);
                }
            l[0] += sum[0];
            l[1] += sum[1];
            asm volatile("cp.async.wait_group 1;" ::: "memory");       // the values; the next keys are under way
            __syncthreads();
            if (part) {                                // values that some query does not see, as in kv_prompt.cu
                for (int i = threadIdx.x; i < kKeys * (D / 8); i += kThreads) {
                    const int row = i / (D / 8), c = i % (D / 8);
                    if (!edge_token(shape, x, y0 + row)) continue;
                    const uint32_t at = v_at + place16(row, c);
                    uint32_t z[4], bad = 0;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(z[0]), "=r"(z[1]), "=r"(z[2]), "=r"(z[3]) : "r"(at) : "memory");
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t n = not_finite<T>(z[k]);        // bits 15 and 31
                        bad |= n;
                        z[k] &= ~((n >> 15) * 0xffffu);
                    }
                    if (!bad) continue;
                    left_out = 1;
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(z[0]), "r"(z[1]), "r"(z[2]), "r"(z[3]) : "memory");
                }
                __syncthreads();
            }
#pragma unroll
            for (int t = 0; t < kKeys / 16; ++t)
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    uint32_t b[4];
                    ldsm4t(b, v_at + place16(t * 16 + (lane & 15), 2 * k + (lane >> 4)));
                    Half<T>::mma(o[2 * k], w[t], b[0], b[1]);
                    Half<T>::mma(o[2 * k + 1], w[t], b[2], b[3]);
                }
            __syncthreads();                           // all have read the values
            if (j + 1 < x.count) copy_tile(x, j + 1, true);
            else asm volatile("cp.async.commit_group;" ::: "memory");
        }
        const bool spoils = left_out;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(~0u, l[h], 1);
            l[h] += __shfl_xor_sync(~0u, l[h], 2);
        }
        const bool whole = x.kind & kWhole;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (!live[h]) continue;
            if (spoils)
#pragma unroll
                for (int b = 0; b < D / 32; ++b) {
                    const Spoilt y = spoilt<D, T, 32>(g, shape, x, token[h], q_head[h], 32 * b, m[h], scale);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int at = 8 * (i / 2) + c2 + (i & 1);
                        float &z = o[4 * b + i / 2][2 * h + (i & 1)];
                        if (y.plus >> at & 1) z += INFINITY;
                        if (y.minus >> at & 1) z -= INFINITY;
                        if (y.none >> at & 1) z = NAN;
                    }
                }
            const int64_t query = x.start + token[h];
            if (whole) {
                const float inv = inverse(l[h]);
                T *out = static_cast<T *>(g.a.out) + query * g.a.out_stride[0] + q_head[h] * g.a.out_stride[1];
#pragma unroll
                for (int i = 0; i < D / 8; ++i)
                    *reinterpret_cast<uint32_t *>(out + 8 * i + c2) = Half<T>::pack(o[i][2 * h] * inv, o[i][2 * h + 1] * inv);
                if ((lane & 3) == 0 && g.a.lse) g.a.lse[query * (g.n_kv_heads * g.group) + q_head[h]] = log_of(m[h], l[h]);
            } else {
                const int64_t at = (int64_t)(2 * blockIdx.x + ((x.kind & kFirst) != 0)) * kRows + warp * 16 + r + 8 * h;
#pragma unroll
                for (int i = 0; i < D / 8; ++i)
                    *reinterpret_cast<float2 *>(g.part_o + at * D + 8 * i + c2) = make_float2(o[i][2 * h], o[i][2 * h + 1]);
                if ((lane & 3) == 0) g.part_ml[at] = make_float2(m[h], l[h]);
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename T>
cudaError_t launch_of(const PromptArgs &g, int blocks, int sms, cudaStream_t st) {
    const cudaError_t e = launch_kernel(prompt_wide_kernel<T>, dim3(blocks), kThreads, kSmem, st, false, g);
    if (e != cudaSuccess) return e;
    return launch_kernel(join_kernel<D, T, kRows, kRows, kKeys>, dim3(kJoinBlocks * sms), kJoinThreads, 0, st, true, g, blocks);
}

}  // namespace

cudaError_t prepare_prompt_wide(int type) {
    return type == ISJL_KV_BF16 ? cudaFuncSetAttribute(prompt_wide_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem)
                                : cudaFuncSetAttribute(prompt_wide_kernel<__half>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
}

cudaError_t launch_prompt_wide(PromptArgs &g, int type, int sms, cudaStream_t st) {
    share_rows(g, kRows);
    const int blocks = kBlocks * sms < kMostRuns ? kBlocks * sms : kMostRuns;
    static_assert(2 * kBlocks * kRows <= kPromptRows, "the pieces' memory");
    return type == ISJL_KV_BF16 ? launch_of<__nv_bfloat16>(g, blocks, sms, st) : launch_of<__half>(g, blocks, sms, st);
}

}  // namespace isjl
