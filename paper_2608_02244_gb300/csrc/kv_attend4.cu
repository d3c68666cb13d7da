// kv_attend4.cu -- attention of single queries over a paged cache in 4 bits (isjl_kv_attend4).
//
// The work is a line of slices of 32 or 64 tokens of each query.  The grid's warps are teams, a warp for each key head, and
// every team has an equal run of the line, wherever requests end, with what a query takes beside its slices counted in.  A
// team's warps go over the same tokens at about the same time, each by itself: where a token's heads lie side by side in
// memory, they share lines of it, of which a head's codes and scales are a part only (with a run of one head's slices for
// each warp, 128 queries over 4,096 tokens of 8 heads took 320 us in that order and 148 with a block's heads apart; now 151
// and 148).  A slice's codes and scales come by asynchronous copies of 16 bytes through a ring of the warp's own, keys and
// values in turn.  Items cut by the runs' ends leave pieces, which a second kernel joins in their order.
//
// 5 bits a value leave a token and head 160 bytes at 128 values, which the memory brings an SM in 7 cycles: what bounds
// the work is the instructions from codes to products.  So
// - both products take the codes as their left operand, tokens (S^T = K Q^T) and values' places (O^T = V^T P^T) as its
//   rows, and 8 query heads are the columns: nothing is spent on heads that are not there, and 16 heads use the same
//   operands twice;
// - which row is which token and which column of the sum which place of a head is free to choose: a thread takes whole
//   words of eight codes, a shift and one logical instruction makes a pair of them numbers (kv_four.cuh) and one fused
//   multiplication and addition their values, in the order in which the instruction wants them;
// - weights go from the first product's layout to the second's by a transposition in the warp (movmatrix).
//
// The weights are rounded to 16 bits for the second product, as its instruction takes them, each by at most half a step of
// itself; their sum is of the unrounded ones, and scores, maxima, sums and pieces have 32 bits.
//
// 512 queries of 64 + 8 heads of 128 values over 1.23 million tokens, 1.58 GB: 329 us, 4.8 TB/s; 690 instructions for 32
// tokens of a key head (290 make numbers of codes, 32 are products; the rest are the copies, each with a pointer from shared
// memory and its 64-bit sum, the softmax of eight columns whatever the number of heads, the weights' transposition and the
// ring's turns), issue slots 58% busy, the ALU 51%, the tensor pipe 21%.  128 queries over 4,096 tokens with 4 query heads on
// each of 8 key heads 148 us (4.5 TB/s), 16 on each of 4 106; 256 values, 4 on each of 4, 151 (4.5 TB/s).
//
// A prefix that the requests share is read and decoded by every query: 64 queries of 32 + 8 heads over 8,192 tokens of it and
// 256 of their own 147 us, 512 over 2,048 308.
#include "kv_four.cuh"
#include "kv_sight.cuh"
#include "kv_tma.cuh"

#include <algorithm>
#include <type_traits>

namespace isjl {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps, kJoinThreads = 256;
// A query's beginning and end, in slices, which the runs count with them: places of the line in front of its slices.  With 0,
// 1 and 2 of them 256 queries of 1 to 6,144 tokens (32 + 8 heads of 128 values) took 92.4, 88.7 and 90.7 us, 512 of up to 8,192
// (64 + 8 heads) 336, 329 and 331.
constexpr int kExtra = 1;

template <int D, int kTiles>
struct Shape {
    static constexpr int kCodes = D / 2, kScales = D / 8;          // bytes of a token's key (or value) in one head
    static constexpr int kChunks = kCodes / 16;                    // of 16 bytes, of its codes
    // tokens.  Longer slices have fewer instructions a token around their products: 64 against 32 with 128 values 337 and 381 us
    // (the case above), with 64 values 98 and 112; with 256 values, where fewer blocks' rings fit, 269 and 155.
    static constexpr int kSlice = D == 256 ? 32 : 64, kEights = kSlice / 8;
    static constexpr int kStageBytes = kSlice * (kCodes + kScales);
    static constexpr int kStages = D == 256 ? 5 : 3;                              // of a warp's ring: keys or values of a slice
    static_assert(kStages % 2 == 1, "a slice's keys and values are under way together");
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kBlocks = D == 256 || kTiles == 2 ? 2 : 3;      // per SM
};

template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t to, const void *from, bool real) {
    if (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(real ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to), "l"(from), "r"(real ? 8 : 0) : "memory");
}

// Of each eight tokens, the one in row r of a product's operand: with it and `chunk_at` a warp's loads meet no bank twice,
// by rows (keys) or by pairs of rows (values).
__device__ __forceinline__ int token_of(int r) { return r ^ ((r >> 1) & 1); }
// where 16 bytes of a token's codes lie in a stage
template <int D>
__device__ __forceinline__ uint32_t chunk_at(int token, int chunk) {
    if (D == 64) return (token ^ ((token >> 2) & 1)) * 32 + chunk * 16;
    if (D == 128) return token * 64 + ((chunk ^ ((token >> 1) & 3)) << 4);
    return token * 128 + ((chunk ^ (token & 7)) << 4);
}

// kWords neighbouring words of a stage
template <int kWords>
__device__ __forceinline__ void load_words(uint32_t (&w)[kWords], uint32_t at) {
    if constexpr (kWords == 1) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
    else if constexpr (kWords == 2) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
    else asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
}

__device__ __forceinline__ const unsigned char *load_pointer(uint32_t at) {
    uint64_t p;
    asm volatile("ld.shared.b64 %0, [%1];" : "=l"(p) : "r"(at) : "memory");
    return reinterpret_cast<const unsigned char *>(p);
}

__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

template <int kSlice>
__device__ __forceinline__ Sight sight(const Attend4Args &g, int t) {
    return sight_of<kSlice>(g.a, g.shift, g.a.n_prefix_blocks << g.shift, g.status, t);
}

// place on the line of slices: slice i of query t, with its first token
struct At {
    int t, i;
    int32_t x;
    Sight s;
};

template <int D, typename T, int kTiles>
__global__ void __launch_bounds__(kThreads, (Shape<D, kTiles>::kBlocks)) attend4_kernel(const __grid_constant__ Attend4Args g) {
    using S = Shape<D, kTiles>;
    constexpr int kSlice = S::kSlice, kEights = S::kEights;
    extern __shared__ __align__(128) unsigned char smem[];
    int32_t *before = reinterpret_cast<int32_t *>(smem + S::kRing);                  // [n + 1] places before a query
    __shared__ int32_t warp_sum[kWarps];
    __shared__ const unsigned char *eight_at[kWarps][4 * kEights];
    __shared__ int64_t eight_stride[kWarps][4][3];
    const isjl_kv_attend_args &a = g.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = a.n, parts = (g.group + 8 * kTiles - 1) / (8 * kTiles), H = g.n_kv_heads * parts, hq = g.n_kv_heads * g.group;
    const float scale = a.scale * kLog2e;

    start_next();
    // ---- places of the line before each query
    {
        const int per = (n + kThreads - 1) / kThreads;
        const int begin = min(n, (int)threadIdx.x * per), end = min(n, begin + per);
        int32_t sum = 0;
        for (int t = begin; t < end; ++t) {
            const int32_t k = sight<kSlice>(g, t).slices + kExtra;
            before[t] = k;
            sum += k;
        }
        __syncwarp();                // the threads come from loops of different lengths
        int32_t inc = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t p = __shfl_up_sync(~0u, inc, d);
            if (lane >= d) inc += p;
        }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        int32_t base = inc - sum;
        for (int w = 0; w < warp; ++w) base += warp_sum[w];
        for (int t = begin; t < end; ++t) {
            const int32_t k = before[t];
            before[t] = base;
            base += k;
        }
        if (threadIdx.x == kThreads - 1) before[n] = base;
        __syncthreads();
    }
    // A team is a warp for each (part of a) key head; the teams have equal runs of the queries' slices.
    const int64_t W = before[n];
    const int64_t C = min((int64_t)(gridDim.x * kWarps / H), W);         // teams with work
    const int64_t me = (int64_t)blockIdx.x * kWarps + warp, team = me / H;
    const int head = (int)(me - team * H), kv = head / parts;
    const int64_t f0 = team < C ? W * team / C : W, f1 = team < C ? W * (team + 1) / C : W;
    if (lane == 0) g.cut[me].t = -1;
    if (f0 == f1) return;

    auto advance = [&](At &p) {
        p.x = ++p.i == p.s.head ? p.s.lo / kSlice * kSlice : p.x + kSlice;
        if (p.i < p.s.slices) return;
        p.i = 0;
        if (++p.t < n) p.s = sight<kSlice>(g, p.t);
        p.x = slice_start<kSlice>(p.s, 0);
    };
    // the query that place f of the line is one of
    auto query_at = [&](int64_t f) {
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (before[mid] <= f) lo = mid; else hi = mid;
        }
        return lo;
    };
    // slices before place f
    auto slices_before = [&](int64_t f, int t) { return before[t] - (int64_t)kExtra * t + max((int64_t)0, f - before[t] - kExtra); };
    At here;
    here.t = query_at(f0);
    const int slices = (int)(slices_before(f1, f1 == W ? n - 1 : query_at(f1)) - slices_before(f0, here.t));
    if (slices == 0) return;
    here.s = sight<kSlice>(g, here.t);
    here.i = max(0, (int)(f0 - before[here.t]) - kExtra);
    here.x = slice_start<kSlice>(here.s, here.i);

    // ---- the ring: keys and values of a slice, one stage each.  A slice is four or eight times eight tokens, each eight in
    // one block; a lane for each eight and kind (keys' codes and scales, values' codes and scales) finds where it lies, and
    // looks up its block a slice ahead of that.
    const uint32_t ring = smem_addr(smem) + warp * S::kStages * S::kStageBytes;
    const int slot_mask = (1 << g.shift) - 1, kind = (lane / kEights) & 3, my_eight = lane % kEights;
    // whether something is seen of a lane's eight tokens
    auto seen_of = [&](const At &p) {
        const int32_t y = p.x + 8 * my_eight;
        return y < p.s.end && (y + 8 > p.s.lo || y < a.sinks);
    };
    auto block_of = [&](const At &p) {
        const int32_t y = p.x + 8 * my_eight;
        if (!seen_of(p)) return -1;
        const int32_t j = y >> g.shift;
        return j < a.n_prefix_blocks ? a.prefix[j] : a.table[(int64_t)p.s.row * a.table_width + (j - a.n_prefix_blocks)];
    };
    const unsigned char *const kind_base = static_cast<const unsigned char *>(kind == 0 ? g.cache.k : kind == 1 ? g.cache.k_scale : kind == 2 ? g.cache.v : g.cache.v_scale);
    if (lane < 4 * kEights && my_eight == 0)
        for (int i = 0; i < 3; ++i)                    // in bytes
            eight_stride[warp][kind][i] = (kind == 0 ? g.cache.k_stride : kind == 1 ? g.cache.k_scale_stride : kind == 2 ? g.cache.v_stride : g.cache.v_scale_stride)[i] << (kind & 1);
    __syncwarp();
    At ahead = here;
    int ahead_left = slices;                           // slices whose values are still to be asked for
    int32_t ahead_block = block_of(ahead);
    constexpr uint32_t kAll = (1u << kEights) - 1;
    uint32_t ahead_there = 0;                          // which of its eights are read: the others are zeros
    constexpr int kRows = 32 / S::kChunks;             // tokens that one copy of all lanes brings codes of
    const uint32_t copy_to = ring + chunk_at<D>(lane / S::kChunks, lane % S::kChunks);
    const int64_t code_off[2] = {lane / S::kChunks % 8 * g.cache.k_stride[1] + lane % S::kChunks * 16, lane / S::kChunks % 8 * g.cache.v_stride[1] + lane % S::kChunks * 16};
    const int64_t scale_off[2] = {2 * (lane & 7) * g.cache.k_scale_stride[1], 2 * (lane & 7) * g.cache.v_scale_stride[1]};
    const uint32_t eights = smem_addr(eight_at[warp]);
    auto copies = [&](uint32_t stage, auto values, auto all) {
        constexpr int v = decltype(values)::value;
        const int64_t half = 4 * (v ? g.cache.v_stride : g.cache.k_stride)[1];
#pragma unroll
        for (int i = 0; i < S::kChunks * kSlice / 32; ++i) {
            const uint32_t which = kRows == 16 ? 2 * i + (lane >> 4) : kRows * i / 8;
            copy_async<16>((copy_to + stage + i * kRows * S::kCodes) ^ (kRows == 4 && i % 2 ? 64 : 0), load_pointer(eights + (2 * kEights * v + which) * 8) + code_off[v] + (kRows == 4 && i % 2 ? half : 0),
                           decltype(all)::value || ahead_there >> which & 1);
        }
#pragma unroll
        for (int i = 0; i < kSlice / 32; ++i) {
            const uint32_t which = 4 * i + (lane >> 3);
            const unsigned char *from = load_pointer(eights + (2 * kEights * v + kEights + which) * 8) + scale_off[v];
            constexpr int kBytes = S::kScales < 16 ? S::kScales : 16;
#pragma unroll
            for (int b = 0; b < S::kScales; b += kBytes)
                copy_async<kBytes>(ring + stage + kSlice * S::kCodes + (32 * i + lane) * S::kScales + b, from + b, decltype(all)::value || ahead_there >> which & 1);
        }
    };
    auto feed_keys = [&](uint32_t stage) {
        if (ahead_left > 0) {
            const bool there = (uint32_t)ahead_block < (uint32_t)g.n_blocks;
            if (!there && seen_of(ahead)) report(g.status);          // beyond the cache: zeros
            if (lane < 4 * kEights) {
                const int slot = (ahead.x + 8 * my_eight) & slot_mask;
                const int64_t *stride = eight_stride[warp][kind];
                eight_at[warp][lane] = kind_base + (there ? ahead_block * stride[0] + slot * stride[1] + kv * stride[2] : 0);
            }
            ahead_there = __ballot_sync(~0u, there) & kAll;
            __syncwarp();
            if (ahead_there == kAll) copies(stage, std::false_type(), std::true_type());
            else copies(stage, std::false_type(), std::false_type());
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto feed_values = [&](uint32_t stage) {
        if (ahead_left > 0) {
            if (ahead_there == kAll) copies(stage, std::true_type(), std::true_type());
            else copies(stage, std::true_type(), std::false_type());
            if (--ahead_left > 0) {
                advance(ahead);
                ahead_block = block_of(ahead);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < S::kStages - 1; i += 2) {
        feed_keys(i * S::kStageBytes);
        feed_values((i + 1) * S::kStageBytes);
        __syncwarp();
    }
    uint32_t at_stage = 0;
    // the next stage of the ring, when it has come; the one before it, which all have read by now, is fed: when keys are
    // taken with keys, as an even number of stages is under way
    auto next_stage = [&](auto values) {
        asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 2) : "memory");
        __syncwarp();
        const uint32_t last = (at_stage == 0 ? S::kStages * S::kStageBytes : at_stage) - S::kStageBytes;
        if (decltype(values)::value) feed_values(last);
        else feed_keys(last);
        const uint32_t at = ring + at_stage;
        at_stage = at_stage == (S::kStages - 1) * S::kStageBytes ? 0 : at_stage + S::kStageBytes;
        return at;
    };

    const int r = lane >> 2, c = lane & 3;             // this lane's row of an operand, and its columns 2 c and 2 c + 1
    constexpr int kKeyWords = D / 32, kKeyLoad = kKeyWords < 4 ? kKeyWords : 4;        // of codes of a token's key: places c D / 4 ..
    constexpr int kValueWords = D / 64;                                                // of its value: places r D / 8 ..
    // where this lane's part of the first of each eight tokens' rows is: a key's, and a value's of two tokens
    const uint32_t key_at = chunk_at<D>(token_of(r), D == 64 ? c / 2 : D == 128 ? c : 2 * c) + (D == 64 ? c % 2 * 8 : 0);
    const uint32_t key_scale_at = kSlice * S::kCodes + token_of(r) * S::kScales + (D == 64 ? c / 2 * 4 : c * (D / 32));
    const int value_chunk = D == 64 ? r / 4 : D == 128 ? r / 2 : r, value_rest = D == 64 ? r % 4 * 4 : D == 128 ? r % 2 * 8 : 0;
    const uint32_t value_at[2] = {chunk_at<D>(token_of(2 * c), value_chunk) + value_rest, chunk_at<D>(token_of(2 * c + 1), value_chunk) + value_rest};
    const uint32_t value_scale_at[2] = {kSlice * S::kCodes + token_of(2 * c) * S::kScales + value_chunk * 4u, kSlice * S::kCodes + token_of(2 * c + 1) * S::kScales + value_chunk * 4u};
    uint32_t q[kTiles][D / 16][2];
    float o[kTiles][D / 16][4], m[kTiles][2], l[kTiles][2];     // of heads 2 c and 2 c + 1 of each eight
    int first = 0, live = 0;                           // query heads of the item
    auto begin_item = [&]() {
        first = kv * g.group + (head - kv * parts) * 8 * kTiles;
        live = min(8 * kTiles, (kv + 1) * g.group - first);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            m[t][0] = m[t][1] = -INFINITY;
            l[t][0] = l[t][1] = 0.f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[t][i][j] = 0.f;
            // values c D / 4 .. of head r, as the codes come: i and i + 4 of each eight together
            const bool is = 8 * t + r < live;
            const T *from = static_cast<const T *>(a.q) + here.t * a.q_stride[0] + (first + 8 * t + r) * a.q_stride[1] + c * (D / 4);
#pragma unroll
            for (int w = 0; w < kKeyWords; ++w) {
                const uint4 x = is ? *reinterpret_cast<const uint4 *>(from + 8 * w) : make_uint4(0, 0, 0, 0);
                q[t][2 * w][0] = __byte_perm(x.x, x.z, 0x5410);
                q[t][2 * w][1] = __byte_perm(x.x, x.z, 0x7632);
                q[t][2 * w + 1][0] = __byte_perm(x.y, x.w, 0x5410);
                q[t][2 * w + 1][1] = __byte_perm(x.y, x.w, 0x7632);
            }
        }
    };

    auto slice = [&]() {
        const int32_t x0 = here.x;
        const uint32_t keys = next_stage(std::false_type());
        constexpr int kSixteens = kSlice / 16;
        float s[kTiles][kSixteens][4] = {};
#pragma unroll
        for (int h = 0; h < kSixteens; ++h) {                  // sixteen tokens each
            uint32_t pair[2][kKeyWords / 4 + (kKeyWords < 4)];
#pragma unroll
            for (int e = 0; e < 2; ++e) load_words(pair[e], keys + key_scale_at + (16 * h + 8 * e) * S::kScales);
#pragma unroll
            for (int b = 0; b < kKeyWords / kKeyLoad; ++b) {
                uint32_t w[2][kKeyLoad];
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    load_words(w[e], keys + (b ? key_at ^ 16 : key_at) + (16 * h + 8 * e) * S::kCodes);
                const uint32_t s2[2] = {Four<T>::scale2(pair[0][b]), Four<T>::scale2(pair[1][b])}, b2[2] = {Four<T>::offset2(pair[0][b]), Four<T>::offset2(pair[1][b])};
#pragma unroll
                for (int i = 0; i < kKeyLoad; ++i) {
                    const int k = 2 * (b * kKeyLoad + i);
                    const uint32_t x[2][4] = {{Four<T>::fma(Four<T>::template ones<0>(w[0][i]), s2[0], b2[0]), Four<T>::fma(Four<T>::template ones<0>(w[1][i]), s2[1], b2[1]),
                                               Four<T>::fma(Four<T>::template ones<1>(w[0][i]), s2[0], b2[0]), Four<T>::fma(Four<T>::template ones<1>(w[1][i]), s2[1], b2[1])},
                                              {Four<T>::fma(Four<T>::template ones<2>(w[0][i]), s2[0], b2[0]), Four<T>::fma(Four<T>::template ones<2>(w[1][i]), s2[1], b2[1]),
                                               Four<T>::fma(Four<T>::template ones<3>(w[0][i]), s2[0], b2[0]), Four<T>::fma(Four<T>::template ones<3>(w[1][i]), s2[1], b2[1])}};
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) {
                        Half<T>::mma(s[t][h], x[0], q[t][k][0], q[t][k][1]);
                        Half<T>::mma(s[t][h], x[1], q[t][k + 1][0], q[t][k + 1][1]);
                    }
                }
            }
        }
        const bool edge = x0 + kSlice > here.s.end || x0 < here.s.lo;
        auto hidden = [&](int32_t y) { return y >= here.s.end || (y < here.s.lo && y >= a.sinks); };
        if (edge) {
#pragma unroll
            for (int h = 0; h < kSixteens; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (hidden(x0 + 16 * h + 8 * e + token_of(r)))
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) s[t][h][2 * e] = s[t][h][2 * e + 1] = -INFINITY;
        }
        __syncwarp();
        // weights are relative to a maximum that may lag behind by kPass: it is looked for only when one is beyond that
        uint32_t w[kTiles][kSixteens][2];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            float top[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                top[j] = fmaxf(s[t][0][j], s[t][0][2 + j]);
#pragma unroll
                for (int h = 1; h < kSixteens; ++h) top[j] = fmaxf(top[j], fmaxf(s[t][h][j], s[t][h][2 + j]));
                top[j] = top[j] * scale - Grow<T>::kTop;
            }
            if (__any_sync(~0u, top[0] > m[t][0] + Grow<T>::kPass || top[1] > m[t][1] + Grow<T>::kPass)) {
                float fix[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(~0u, top[j], d));
                    const float next = fmaxf(m[t][j], top[j]);
                    fix[j] = m[t][j] == next ? 1.f : ex2(m[t][j] - next);
                    m[t][j] = next;
                    l[t][j] *= fix[j];
                }
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[t][i][j] *= fix[j & 1];
            }
            const float ref[2] = {m[t][0] == -INFINITY ? 0.f : m[t][0], m[t][1] == -INFINITY ? 0.f : m[t][1]};
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int h = 0; h < kSixteens; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float u = ex2(fmaf(s[t][h][2 * e], scale, -ref[0])), v = ex2(fmaf(s[t][h][2 * e + 1], scale, -ref[1]));
                    sum[0] += u;
                    sum[1] += v;
                    w[t][h][e] = transposed(Half<T>::pack(u, v));
                }
            l[t][0] += sum[0];
            l[t][1] += sum[1];
        }
        const uint32_t values = next_stage(std::true_type());
        if (edge) {
            // a weight of 0 does not silence an infinite or undefined value: what is not seen stands for 0
            for (int i = lane; i < kSlice; i += 32)
                if (hidden(x0 + i))
                    for (int b = 0; b < S::kScales; b += 8)
                        asm volatile("st.shared.v2.b32 [%0], {%1, %1};" ::"r"(values + kSlice * S::kCodes + i * S::kScales + b), "r"(0) : "memory");
            __syncwarp();
        }
#pragma unroll
        for (int h = 0; h < kSixteens; ++h) {
            // this lane's four tokens: two of each eight
            uint32_t word[4][kValueWords], s2[2], b2[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                uint32_t pair[2][1];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    load_words(word[2 * e + k], values + value_at[k] + (16 * h + 8 * e) * S::kCodes);
                    load_words(pair[k], values + value_scale_at[k] + (16 * h + 8 * e) * S::kScales);
                }
                s2[e] = __byte_perm(pair[0][0], pair[1][0], 0x5410);
                b2[e] = __byte_perm(pair[0][0], pair[1][0], 0x7632);
            }
#pragma unroll
            for (int i = 0; i < kValueWords; ++i)
#pragma unroll
                for (int part = 0; part < 2; ++part) {             // places 0 .. 3 and 4 .. 7 of the word
                    uint32_t y[2], x[2][4];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        y[e] = __byte_perm(word[2 * e][i], word[2 * e + 1][i], part ? 0x7632 : 0x5410);
                        x[0][2 * e] = Four<T>::fma(Four<T>::template ones<0>(y[e]), s2[e], b2[e]);
                        x[0][2 * e + 1] = Four<T>::fma(Four<T>::template ones<1>(y[e]), s2[e], b2[e]);
                        x[1][2 * e] = Four<T>::fma(Four<T>::template ones<2>(y[e]), s2[e], b2[e]);
                        x[1][2 * e + 1] = Four<T>::fma(Four<T>::template ones<3>(y[e]), s2[e], b2[e]);
                    }
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) {
                        Half<T>::mma(o[t][4 * i + 2 * part], x[0], w[t][h][0], w[t][h][1]);
                        Half<T>::mma(o[t][4 * i + 2 * part + 1], x[1], w[t][h][0], w[t][h][1]);
                    }
                }
        }
    };

    // the end of an item in this warp's run, or of the run in it
    auto end_item = [&](bool begins, bool ends) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[t][j] += __shfl_xor_sync(~0u, l[t][j], d);
                const int row = 8 * t + 2 * c + j;
                if (row >= live) continue;
                if (begins && ends) {
                    const float inv = inverse(l[t][j]);
                    T *out = static_cast<T *>(a.out) + here.t * a.out_stride[0] + (first + row) * a.out_stride[1] + r * (D / 8);
#pragma unroll
                    for (int i = 0; i < D / 64; ++i) {
                        uint32_t u[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) u[k] = Half<T>::pack(o[t][4 * i + k][j] * inv, o[t][4 * i + k][2 + j] * inv);
                        *reinterpret_cast<uint4 *>(out + 8 * i) = make_uint4(u[0], u[1], u[2], u[3]);
                    }
                    if (r == 0 && a.lse) a.lse[(int64_t)here.t * hq + first + row] = log_of(m[t][j], l[t][j]);
                } else {
                    const int64_t at = (me * 2 + begins) * 16 + row;
#pragma unroll
                    for (int i = 0; i < D / 32; ++i)
                        *reinterpret_cast<float4 *>(g.part_o + at * D + r * (D / 8) + 4 * i) =
                            make_float4(o[t][2 * i][j], o[t][2 * i][2 + j], o[t][2 * i + 1][j], o[t][2 * i + 1][2 + j]);
                    if (r == 0) g.part_ml[at] = make_float2(m[t][j], l[t][j]);
                }
            }
        __syncwarp();
    };

    begin_item();
    int begun = here.i;                                // the slice that this warp's part of the item begins with
    for (int left = slices; left > 0; --left) {
        slice();
        const bool ends = here.i + 1 == here.s.slices;
        if (ends || left == 1) {
            end_item(begun == 0, ends);
            if (!ends && begun == 0 && lane == 0)       // its pieces are those of the teams from here on
                g.cut[me] = {here.t, head, (int)team, (int)(((int64_t)before[here.t + 1] * C - 1) / W)};
            begun = 0;
        }
        if (left > 1) {
            advance(here);
            if (here.i == 0) begin_item();
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// Joins the pieces of the items that runs' ends cut, a block for the warp in whose run one begins.
template <int D, typename T, int kTiles>
__global__ void __launch_bounds__(kJoinThreads) join4_kernel(const __grid_constant__ Attend4Args g) {
    const isjl_kv_attend_args &a = g.a;
    const int parts = (g.group + 8 * kTiles - 1) / (8 * kTiles), H = g.n_kv_heads * parts, hq = g.n_kv_heads * g.group;
    wait_for_previous();
    const CutItem item = g.cut[blockIdx.x];
    if (item.t < 0) return;
    const int kv = item.h / parts, from = kv * g.group + (item.h - kv * parts) * 8 * kTiles, rows = min(8 * kTiles, (kv + 1) * g.group - from);
    // where few rows have many pieces, several threads share them
    constexpr int kBatch = 8;                               // pieces whose loads are under way together
    __shared__ float4 part_sum[kJoinThreads];
    __shared__ float2 part_ml[kJoinThreads];
    const int units = rows * (D / 4), pieces = item.last - item.first + 1;
    const int shares = max(1, min(kJoinThreads / units, (pieces + kBatch - 1) / kBatch)), per = (pieces + shares - 1) / shares;
    for (int x0 = 0; x0 < units; x0 += kJoinThreads) {
        const int x = x0 + (units < kJoinThreads ? threadIdx.x % units : threadIdx.x), share = units < kJoinThreads ? threadIdx.x / units : 0;
        const int row = x / (D / 4), d = (x % (D / 4)) * 4;
        float top = -INFINITY, total = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](float2 ml, float4 v) {               // relative to top
            const float p = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
            total += ml.y * p;
            sum.x += v.x * p;
            sum.y += v.y * p;
            sum.z += v.z * p;
            sum.w += v.w * p;
        };
        auto raise = [&](float next) {
            const float fix = next == top ? 1.f : ex2(top - next);
            top = next;
            total *= fix;
            sum.x *= fix;
            sum.y *= fix;
            sum.z *= fix;
            sum.w *= fix;
        };
        const int last = min(item.last, item.first + (share + 1) * per - 1);
        if (x < units && share < shares)
            for (int w0 = item.first + share * per; w0 <= last; w0 += kBatch) {
                float2 ml[kBatch];
                float4 v[kBatch];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const int w = min(w0 + k, last);
                    const int64_t at = (((int64_t)w * H + item.h) * 2 + (w == item.first)) * 16 + row;
                    ml[k] = g.part_ml[at];
                    v[k] = *reinterpret_cast<const float4 *>(g.part_o + at * D + d);
                }
                float next = top;
#pragma unroll
                for (int k = 0; k < kBatch; ++k) next = fmaxf(next, ml[k].x);
                raise(next);
#pragma unroll
                for (int k = 0; k < kBatch; ++k)
                    if (w0 + k <= last) add(ml[k], v[k]);
            }
        if (shares > 1) {                                   // the same for the whole block, and then all units lie in it
            part_sum[threadIdx.x] = sum;
            part_ml[threadIdx.x] = make_float2(top, total);
            __syncthreads();
            if (share > 0) return;
            float next = top;
            for (int k = 1; k < shares; ++k) next = fmaxf(next, part_ml[k * units + threadIdx.x].x);
            raise(next);
            for (int k = 1; k < shares; ++k) add(part_ml[k * units + threadIdx.x], part_sum[k * units + threadIdx.x]);
        }
        if (x >= units || share > 0) continue;
        const float inv = inverse(total);
        *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + item.t * a.out_stride[0] + (from + row) * a.out_stride[1] + d) =
            make_uint2(Half<T>::pack(sum.x * inv, sum.y * inv), Half<T>::pack(sum.z * inv, sum.w * inv));
        if (d == 0 && a.lse) a.lse[(int64_t)item.t * hq + from + row] = log_of(top, total);
    }
}

template <int D, int kTiles>
size_t smem_of(int n) { return Shape<D, kTiles>::kRing + (size_t)(n + 1) * sizeof(int32_t); }

// Blocks: what fits the SMs at a time, and a warp for each head (or part of one) at least.  Runs are equal, so blocks that
// begin when others have ended cost a second time: 4,096 queries of 400 tokens (32 + 8 heads of 128 values), of whose places
// two blocks hold all that an SM has, 584 us, and 693 with a grid of three; 256 values, one block, 727 and 735 with two.
template <int D, typename T, int kTiles>
cudaError_t launch_of(const Attend4Args &g, int grid, cudaStream_t st) {
    const int heads = g.n_kv_heads * ((g.group + 8 * kTiles - 1) / (8 * kTiles));
    grid = std::max(grid, (heads + kWarps - 1) / kWarps);
    const cudaError_t e = launch_kernel(attend4_kernel<D, T, kTiles>, grid, kThreads, smem_of<D, kTiles>(g.a.n), st, false, g);
    if (e != cudaSuccess) return e;
    return launch_kernel(join4_kernel<D, T, kTiles>, grid * kWarps, kJoinThreads, 0, st, true, g);
}

template <int D, typename T, int kTiles>
cudaError_t prepare_of(int sms, int *blocks, int *queries, int *warps) {
    const auto kernel = attend4_kernel<D, T, kTiles>;
    // the limit belongs to the function, not to a handle: always the largest
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_of<D, kTiles>(ISJL_KV_MAX_ROWS));
    int lo = 1, hi = ISJL_KV_MAX_ROWS + 1, per = 0;
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(blocks, kernel, kThreads, smem_of<D, kTiles>(1));
    *blocks = std::min(*blocks, Shape<D, kTiles>::kBlocks);
    while (e == cudaSuccess && hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, kThreads, smem_of<D, kTiles>(mid));
        if (per >= *blocks) lo = mid; else hi = mid;
    }
    *queries = lo;
    *warps = std::max(*blocks * sms * kWarps, 1024);
    return e;
}

// 8 query heads at a time, or 16 where a key head has more, which then is read once for 16: 4 key heads with 16 query heads
// each, 128 queries over 4,096 tokens, 106 us against 150 in two times 8.  Not with 256 values, where 16 heads' sums do not
// fit the registers: 306 us against 286.
template <int D>
bool sixteen(int group) { return D < 256 && group > 8; }

template <int D, typename T>
cudaError_t prepare_tiles(int group, int sms, int *blocks, int *queries, int *warps) {
    return sixteen<D>(group) ? prepare_of<D, T, D < 256 ? 2 : 1>(sms, blocks, queries, warps) : prepare_of<D, T, 1>(sms, blocks, queries, warps);
}
template <int D, typename T>
cudaError_t launch_tiles(const Attend4Args &g, int grid, cudaStream_t st) {
    return sixteen<D>(g.group) ? launch_of<D, T, D < 256 ? 2 : 1>(g, grid, st) : launch_of<D, T, 1>(g, grid, st);
}

}  // namespace

cudaError_t prepare_attend4(int head_dim, int type, int group, int sms, int *blocks, int *queries, int *warps) {
    if (type == ISJL_KV_BF16)
        return head_dim == 64 ? prepare_tiles<64, __nv_bfloat16>(group, sms, blocks, queries, warps)
             : head_dim == 128 ? prepare_tiles<128, __nv_bfloat16>(group, sms, blocks, queries, warps) : prepare_tiles<256, __nv_bfloat16>(group, sms, blocks, queries, warps);
    return head_dim == 64 ? prepare_tiles<64, __half>(group, sms, blocks, queries, warps)
         : head_dim == 128 ? prepare_tiles<128, __half>(group, sms, blocks, queries, warps) : prepare_tiles<256, __half>(group, sms, blocks, queries, warps);
}

cudaError_t launch_attend4(const Attend4Args &g, int head_dim, int type, int grid, cudaStream_t st) {
    if (type == ISJL_KV_BF16)
        return head_dim == 64 ? launch_tiles<64, __nv_bfloat16>(g, grid, st)
             : head_dim == 128 ? launch_tiles<128, __nv_bfloat16>(g, grid, st) : launch_tiles<256, __nv_bfloat16>(g, grid, st);
    return head_dim == 64 ? launch_tiles<64, __half>(g, grid, st)
         : head_dim == 128 ? launch_tiles<128, __half>(g, grid, st) : launch_tiles<256, __half>(g, grid, st);
}

}  // namespace isjl
