// kv_attend.cu -- attention of single queries over paged tokens (isjl_kv_attend).
//
// A step reads every visible key and value once and does 4 D operations a query head with each: bound by
// memory.  The work is a line of tiles of 64 tokens: for each query, each key head (and each 16 of its query
// heads), its visible tiles in order, the first tokens' before the window's.  Every block of the grid gets an
// equal run of that line wherever requests end, so ragged batches keep all SMs loading to the end.  A warp
// takes 16 tokens of each tile through a ring of its own of asynchronous copies (no block barrier while an
// item lasts), with the running maximum and sum of a softmax over its tokens; the query heads of a key head
// are the 16 rows of a tensor instruction.  At an item's end the four warps join through shared memory, and
// an item cut by the run's ends is joined by the last of its blocks to arrive, in their order, so that the
// result does not depend on the order of arrival.
#include "kv_tma.cuh"

namespace isjl {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps, kSlice = 16, kTile = kWarps * kSlice;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int32_t kNone = INT32_MIN;

template <int D>
struct Shape {
    static constexpr int kStages = D == 64 ? 6 : 3;
    static constexpr int kBlocks = D == 256 ? 1 : 2;               // per SM
    static constexpr int kHalves = D / 64;                         // rows of 128 bytes hold 64 values
    static constexpr int kHalfBytes = kSlice * 128;
    static constexpr int kSideBytes = kHalves * kHalfBytes;        // keys (or values) of a slice
    static constexpr int kRing = kWarps * kStages * 2 * kSideBytes;
    static constexpr int kJoinRow = D + 8;                         // padded: 8 rows of a warp's store on all banks
    static constexpr int kJoin = 2 * 8 * kJoinRow * 4;
};

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

// what a query sees: tokens end - window .. end - 1 and 0 .. sinks - 1, counted from the first token that
// this kernel reads (the prefix's, or the own ones' where the prefix is done elsewhere)
struct Sight {
    int32_t end, lo, head;     // head: tiles with first tokens that lie before the window's first tile
    int32_t tiles;             // at least 1: an item without tokens still has a result
    int32_t row;
};

__device__ __forceinline__ Sight sight(const AttendArgs &g, int t) {
    const isjl_kv_attend_args &a = g.a;
    Sight s;
    const int32_t x = a.lens[t];
    s.row = a.rows ? a.rows[t] : t;
    const int32_t prefix = a.n_prefix_blocks << g.shift;
    const bool bad = x > 0 && s.row >= 0 && (s.row >= a.n_table_rows || ((x - 1) >> g.shift) >= a.table_width);
    if (bad) report(g.status);
    s.end = x <= 0 || s.row < 0 || bad ? 0 : x + (g.line.blocks ? 0 : prefix);
    s.lo = a.window && s.end > a.window ? s.end - a.window : 0;
    s.head = min((min(a.sinks, s.lo) + kTile - 1) / kTile, s.lo / kTile);
    s.tiles = max(1, s.head + (s.end + kTile - 1) / kTile - s.lo / kTile);
    return s;
}

__device__ __forceinline__ int32_t tile_start(const Sight &s, int tile) {
    return (tile < s.head ? tile : s.lo / kTile + tile - s.head) * kTile;
}

// place on the line of tiles
struct Place {
    int t, h, tile;
    Sight s;
};

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, Shape<D>::kBlocks)
attend_kernel(const __grid_constant__ AttendArgs g, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
    using S = Shape<D>;
    extern __shared__ __align__(1024) unsigned char smem[];
    float *join = reinterpret_cast<float *>(smem + S::kRing);                        // [2][8][kJoinRow]
    float2 *stats = reinterpret_cast<float2 *>(smem + S::kRing + S::kJoin);          // [kWarps][16]
    float2 *row_stat = stats + kWarps * 16;                                          // [16]
    int32_t *before = reinterpret_cast<int32_t *>(row_stat + 16);                    // [n + 1] tiles before a query
    __shared__ int32_t warp_sum[kWarps];
    __shared__ int32_t last_one;
    __shared__ __align__(8) uint64_t bars[kWarps * S::kStages];

    const isjl_kv_attend_args &a = g.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = a.n, parts = (g.group + 15) / 16, H = g.n_kv_heads * parts, hq = g.n_kv_heads * g.group;
    const float scale = a.scale * kLog2e;

    const uint32_t bar0 = smem_addr(bars) + warp * S::kStages * 8;
    if (lane == 0) {
        for (int i = 0; i < S::kStages; ++i) bar_init(bar0 + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // ---- tiles before each query
    {
        const int per = (n + kThreads - 1) / kThreads;
        const int begin = min(n, (int)threadIdx.x * per), end = min(n, begin + per);
        int32_t sum = 0;
        for (int t = begin; t < end; ++t) {
            const int32_t k = sight(g, t).tiles;
            before[t] = k;
            sum += k;
        }
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
    const int64_t W = (int64_t)before[n] * H;
    const int64_t C = min((int64_t)gridDim.x, W);
    const int64_t me = blockIdx.x;
    if (me >= C) return;
    const int64_t f0 = W * me / C, f1 = W * (me + 1) / C;

    auto place_at = [&](int64_t f) {
        Place p;
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((int64_t)before[mid] * H <= f) lo = mid; else hi = mid;
        }
        p.t = lo;
        p.s = sight(g, lo);
        const int32_t rest = (int32_t)(f - (int64_t)before[lo] * H);
        p.h = rest / p.s.tiles;
        p.tile = rest - p.h * p.s.tiles;
        return p;
    };
    auto advance = [&](Place &p) {
        if (++p.tile < p.s.tiles) return;
        p.tile = 0;
        if (++p.h < H) return;
        p.h = 0;
        if (++p.t < n) p.s = sight(g, p.t);
    };

    // ---- the ring
    const uint32_t ring = smem_addr(smem) + warp * S::kStages * 2 * S::kSideBytes;
    const int32_t prefix_blocks = g.line.blocks ? 0 : a.n_prefix_blocks;
    // block numbers of the slice's first and second 8 tokens, kNone where nothing of them is visible.  They
    // are asked for one tile ahead of the copies that use them, and looked at only there.
    auto blocks_of = [&](const Place &p, int32_t &b0, int32_t &b1) {
        const int32_t x = tile_start(p.s, p.tile) + warp * kSlice;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int32_t y = x + 8 * k;
            int32_t b = kNone;
            if (y < p.s.end && (y + 8 > p.s.lo || y < a.sinks)) {
                const int32_t j = y >> g.shift;
                b = j < prefix_blocks ? a.prefix[j] : a.table[(int64_t)p.s.row * a.table_width + (j - prefix_blocks)];
            }
            (k ? b1 : b0) = b;
        }
    };
    // one copy for the slice's rows of a block (16, or 8 of each of two blocks) and 64 of their values
    auto load = [&](const Place &p, int stage, int32_t b0, int32_t b1) {
        const uint32_t bar = bar0 + 8 * stage;
        if (b0 == kNone && b1 == kNone) {              // nothing to come: the stage's turn passes all the same
            bar_arrive(bar);
            return;
        }
        const int32_t slot = (tile_start(p.s, p.tile) + warp * kSlice) & ((1 << g.shift) - 1);
        const int kv = p.h / parts;
        const uint32_t to = ring + stage * 2 * S::kSideBytes;
        bar_expect(bar, 2 * S::kSideBytes);
        if (g.shift > 3 && b0 == kNone) b0 = b1;       // both halves are of one block
        if ((uint32_t)b0 >= (uint32_t)g.n_blocks) { if (b0 != kNone) report(g.status); b0 = g.n_blocks; }   // beyond the cache: zeros
        if (g.shift == 3 && (uint32_t)b1 >= (uint32_t)g.n_blocks) { if (b1 != kNone) report(g.status); b1 = g.n_blocks; }
#pragma unroll
        for (int half = 0; half < S::kHalves; ++half) {
            const uint32_t at = to + half * S::kHalfBytes;
            tma_load(at, &kmap, bar, half * 64, slot, kv, b0);
            tma_load(at + S::kSideBytes, &vmap, bar, half * 64, slot, kv, b0);
            if (g.shift == 3) {
                tma_load(at + 1024, &kmap, bar, half * 64, 0, kv, b1);
                tma_load(at + S::kSideBytes + 1024, &vmap, bar, half * 64, 0, kv, b1);
            }
        }
    };

    Place ahead = place_at(f0), here = ahead;
    int64_t fa = f0;
    int32_t b0, b1;
    blocks_of(ahead, b0, b1);
    auto feed = [&](int stage) {
        if (fa >= f1) return;
        if (lane == 0) load(ahead, stage, b0, b1);
        if (++fa < f1) {
            advance(ahead);
            blocks_of(ahead, b0, b1);
            if (ahead.tile == 0) {                     // the next item's queries
                const int kv = ahead.h / parts, first = kv * g.group + (ahead.h - kv * parts) * 16;
                const int live = min(16, (kv + 1) * g.group - first);
                const T *qt = static_cast<const T *>(a.q) + ahead.t * a.q_stride[0] + first * a.q_stride[1];
                if (warp == 0)
                    for (int i = lane; i < live * (D / 64); i += 32)
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(qt + i / (D / 64) * a.q_stride[1] + i % (D / 64) * 64));
            }
        }
    };
#pragma unroll
    for (int i = 0; i < S::kStages - 1; ++i) feed(i);

    uint32_t q[D / 16][4];
    float o[D / 8][4], m[2], l[2];
    auto begin_item = [&]() {
        const int kv = here.h / parts, first = kv * g.group + (here.h - kv * parts) * 16;
        const int live = min(16, (kv + 1) * g.group - first);
        const T *qt = static_cast<const T *>(a.q) + here.t * a.q_stride[0] + first * a.q_stride[1];
        const int r = lane >> 2, c = (lane & 3) * 2;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = r + (j & 1) * 8, col = k * 16 + c + (j >> 1) * 8;
                q[k][j] = row < live ? *reinterpret_cast<const uint32_t *>(qt + row * a.q_stride[1] + col) : 0u;
            }
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
        if (!g.line.blocks || here.tile != 0 || here.s.end == 0) return;
        // the prefix's pieces are where the item starts from, one warp each
        const int item = kv * g.line.pairs + here.t / g.line.tokens_of_tile / 2;
        const int pieces = g.line.last_block(item) - g.line.first_block(item) + 1;
        for (int k = warp; k < pieces; k += kWarps) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (r + 8 * j >= live) continue;
                const int64_t at = ((int64_t)k * n + here.t) * hq + first + r + 8 * j;
                const float2 ml = g.prefix_ml[at];
                const float next = fmaxf(m[j], ml.x), ref = next == -INFINITY ? 0.f : next;
                const float fix = ex2(m[j] - ref), w = ex2(ml.x - ref);
                m[j] = next;
                l[j] = l[j] * fix + ((lane & 3) == 0 ? ml.y * w : 0.f);
#pragma unroll
                for (int i = 0; i < D / 8; ++i) {
                    const float2 v = *reinterpret_cast<const float2 *>(g.prefix_o + at * D + i * 8 + c);
                    o[i][2 * j] = o[i][2 * j] * fix + v.x * w;
                    o[i][2 * j + 1] = o[i][2 * j + 1] * fix + v.y * w;
                }
            }
        }
    };

    auto compute = [&](int stage) {
        const int32_t x = tile_start(here.s, here.tile) + warp * kSlice;
        if (x >= here.s.end || (x + kSlice <= here.s.lo && x >= a.sinks)) return;   // nothing visible
        const uint32_t base = ring + stage * 2 * S::kSideBytes;
        float s[2][4] = {};
        {
            // lanes 0-7: tokens 0-7 low half of 16 values, 8-15: high half, 16-23: tokens 8-15 low, 24-31: high
            const int r = (lane & 7) + (lane >> 4) * 8, up = (lane >> 3) & 1;
            const uint32_t at = base + r * 128, turn = (up ^ (r & 7)) << 4;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                uint32_t b[4];
                ldsm4(b, at + (k / 4) * S::kHalfBytes + (turn ^ ((k % 4) << 5)));
                Half<T>::mma(s[0], q[k], b[0], b[1]);
                Half<T>::mma(s[1], q[k], b[2], b[3]);
            }
        }
        const int c = (lane & 3) * 2;
        if (x + kSlice > here.s.end || x < here.s.lo) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int32_t y = x + i * 8 + c + j;
                    if (y >= here.s.end || (y < here.s.lo && y >= a.sinks)) s[i][j] = s[i][2 + j] = -INFINITY;
                }
            // a weight of 0 does not silence an infinite or undefined value: what is not seen becomes 0
            for (int i = lane; i < kSlice * S::kHalves * 8; i += 32) {
                const int r = (i / 8) % kSlice;
                if (x + r >= here.s.end || (x + r < here.s.lo && x + r >= a.sinks))
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(base + S::kSideBytes + (i / 8) * 128 + (i % 8) * 16), "r"(0) : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // before the next copy to this stage
            __syncwarp();
        }
        float top[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            top[j] = fmaxf(fmaxf(s[0][2 * j], s[0][2 * j + 1]), fmaxf(s[1][2 * j], s[1][2 * j + 1])) * scale;
            top[j] = fmaxf(top[j], __shfl_xor_sync(~0u, top[j], 1));
            top[j] = fmaxf(top[j], __shfl_xor_sync(~0u, top[j], 2));
        }
        if (__any_sync(~0u, top[0] > m[0] || top[1] > m[1])) {
            float fix[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float next = fmaxf(m[j], top[j]);
                fix[j] = m[j] == next ? 1.f : ex2(m[j] - next);
                m[j] = next;
                l[j] *= fix[j];
            }
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                o[i][0] *= fix[0];
                o[i][1] *= fix[0];
                o[i][2] *= fix[1];
                o[i][3] *= fix[1];
            }
        }
        const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
        float p[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[i][j] = ex2(fmaf(s[i][j], scale, -ref[j >> 1]));
                l[j >> 1] += p[i][j];
            }
        // weights are rounded to the cache's type for the product, as the tensor instruction takes them;
        // the sum l is of the unrounded ones
        const uint32_t w[4] = {Half<T>::pack(p[0][0], p[0][1]), Half<T>::pack(p[0][2], p[0][3]),
                               Half<T>::pack(p[1][0], p[1][1]), Half<T>::pack(p[1][2], p[1][3])};
        {
            const int r = (lane & 7) + ((lane >> 3) & 1) * 8, up = lane >> 4;
            const uint32_t at = base + S::kSideBytes + r * 128, turn = (up ^ (r & 7)) << 4;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                uint32_t b[4];
                ldsm4t(b, at + (k / 4) * S::kHalfBytes + (turn ^ ((k % 4) << 5)));
                Half<T>::mma(o[2 * k], w, b[0], b[1]);
                Half<T>::mma(o[2 * k + 1], w, b[2], b[3]);
            }
        }
    };

    // ---- the end of an item, or of this block's piece of it
    auto end_item = [&]() {
        const int t = here.t, kv = here.h / parts, first = kv * g.group + (here.h - kv * parts) * 16;
        const int live = min(16, (kv + 1) * g.group - first);
        const int64_t i0 = (int64_t)before[t] * H + (int64_t)here.h * here.s.tiles, i1 = i0 + here.s.tiles;
        const int64_t c0 = ((i0 + 1) * C - 1) / W, c1 = (i1 * C - 1) / W;         // its first and last block
        const bool whole = c0 == c1;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            l[j] += __shfl_xor_sync(~0u, l[j], 1);
            l[j] += __shfl_xor_sync(~0u, l[j], 2);
            if ((lane & 3) == 0) stats[warp * 16 + (lane >> 2) + 8 * j] = make_float2(m[j], l[j]);
        }
        __syncthreads();
        float mine[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = (lane >> 2) + 8 * j;
            if (8 * j >= live) break;
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, stats[w * 16 + r].x);
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) sum += stats[w * 16 + r].y * ex2(stats[w * 16 + r].x - ref);
            mine[j] = ex2(m[j] - ref);
            if (warp == 0 && (lane & 3) == 0) row_stat[r] = make_float2(top, sum);
        }
        const int64_t mypart = (me * 2 + (me == c0 ? 1 : 0)) * 16;
        T *out = static_cast<T *>(a.out) + t * a.out_stride[0] + first * a.out_stride[1];
        const int rr = lane >> 2, cc = (lane & 3) * 2;
#pragma unroll
        for (int j = 0; j < 2; ++j) {                 // rows 8 j .. 8 j + 7
            if (8 * j >= live) break;
            float *to = join + (warp & 1) * 8 * S::kJoinRow + rr * S::kJoinRow + cc;
            if (j) __syncthreads();                   // the first rows have been read
            if (warp >= 2) {
#pragma unroll
                for (int i = 0; i < D / 8; ++i)
                    *reinterpret_cast<float2 *>(to + i * 8) = make_float2(o[i][2 * j] * mine[j], o[i][2 * j + 1] * mine[j]);
            }
            __syncthreads();
            if (warp < 2) {
#pragma unroll
                for (int i = 0; i < D / 8; ++i) {
                    float2 *at = reinterpret_cast<float2 *>(to + i * 8);
                    const float2 u = *at;
                    *at = make_float2(fmaf(o[i][2 * j], mine[j], u.x), fmaf(o[i][2 * j + 1], mine[j], u.y));
                }
            }
            __syncthreads();
            for (int i = threadIdx.x; i < min(8, live - 8 * j) * (D / 4); i += kThreads) {
                const int r = i / (D / 4), d = (i % (D / 4)) * 4;
                const float4 u = *reinterpret_cast<const float4 *>(join + r * S::kJoinRow + d);
                const float4 v = *reinterpret_cast<const float4 *>(join + (8 + r) * S::kJoinRow + d);
                const float4 sum = make_float4(u.x + v.x, u.y + v.y, u.z + v.z, u.w + v.w);
                if (whole) {
                    const float total = row_stat[8 * j + r].y, inv = total > 0.f || total != total ? 1.f / total : 0.f;
                    *reinterpret_cast<uint2 *>(out + (8 * j + r) * a.out_stride[1] + d) =
                        make_uint2(Half<T>::pack(sum.x * inv, sum.y * inv), Half<T>::pack(sum.z * inv, sum.w * inv));
                } else {
                    *reinterpret_cast<float4 *>(g.part_o + (mypart + 8 * j + r) * D + d) = sum;
                }
            }
        }
        if (threadIdx.x < live) {
            const float2 s = row_stat[threadIdx.x];
            if (whole) {
                if (a.lse) a.lse[(int64_t)t * hq + first + threadIdx.x] = s.y > 0.f || s.y != s.y ? (s.x + log2f(s.y)) * 0.6931471805599453f : -INFINITY;
            } else {
                g.part_ml[mypart + threadIdx.x] = s;
            }
        }
        if (whole) { __syncthreads(); return; }
        // the last of the item's blocks to arrive joins the pieces, in the order of the blocks
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            // c0's count is that of the one item that begins in c0 and ends beyond it
            const uint32_t all = (uint32_t)(c1 - c0);
            const uint32_t seen = atomicAdd(g.arrived + c0, 1u);
            last_one = seen == all;
            if (seen == all) g.arrived[c0] = 0u;
        }
        __syncthreads();
        if (!last_one) return;
        __threadfence();
        const int pieces = (int)(c1 - c0) + 1;
        auto piece = [&](int k) { return ((c0 + k) * 2 + (k == 0 ? 1 : 0)) * 16; };
        for (int i = threadIdx.x; i < live * (D / 4); i += kThreads) {
            const int r = i / (D / 4), d = (i % (D / 4)) * 4;
            float top = -INFINITY;
            for (int k = 0; k < pieces; ++k) top = fmaxf(top, __ldcg(&g.part_ml[piece(k) + r]).x);
            const float ref = top == -INFINITY ? 0.f : top;
            float total = 0.f;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            auto add = [&](float2 ml, float4 v) {
                const float w = ex2(ml.x - ref);
                total += ml.y * w;
                sum.x += v.x * w;
                sum.y += v.y * w;
                sum.z += v.z * w;
                sum.w += v.w * w;
            };
#pragma unroll 4
            for (int k = 0; k < pieces; ++k)
                add(__ldcg(&g.part_ml[piece(k) + r]), __ldcg(reinterpret_cast<const float4 *>(g.part_o + (piece(k) + r) * D + d)));
            const float inv = total > 0.f || total != total ? 1.f / total : 0.f;
            *reinterpret_cast<uint2 *>(out + r * a.out_stride[1] + d) =
                make_uint2(Half<T>::pack(sum.x * inv, sum.y * inv), Half<T>::pack(sum.z * inv, sum.w * inv));
            if (d == 0 && a.lse)
                a.lse[(int64_t)t * hq + first + r] = total > 0.f || total != total ? (top + log2f(total)) * 0.6931471805599453f : -INFINITY;
        }
    };

    int stage = 0;
    uint32_t phase = 0;
    bool stuck = false;
    begin_item();
    for (int64_t f = f0; f < f1; ++f) {
        __syncwarp();                                   // all have read the stage that is fed now
        feed(stage == 0 ? S::kStages - 1 : stage - 1);
        if (!stuck && !bar_wait(bar0 + 8 * stage, phase)) stuck = true;
        compute(stage);
        if (++stage == S::kStages) { stage = 0; phase ^= 1; }
        if (here.tile + 1 == here.s.tiles || f + 1 == f1) end_item();
        if (f + 1 < f1) {
            advance(here);
            if (here.tile == 0) begin_item();
        }
    }
    if (stuck) atomicOr(g.status, 2);
}

template <int D, typename T>
cudaError_t launch_of(const AttendArgs &g, const CUtensorMap &k, const CUtensorMap &v, int grid, cudaStream_t st) {
    attend_kernel<D, T><<<grid, kThreads, attend_smem(D, g.a.n), st>>>(g, k, v);
    return cudaGetLastError();
}

template <int D, typename T>
cudaError_t grid_of(int max_rows, int sms, int *grid) {
    const int bytes = (int)attend_smem(D, max_rows);
    // the limit belongs to the function, not to a handle: always the largest
    cudaError_t e = cudaFuncSetAttribute(attend_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)attend_smem(D, ISJL_KV_MAX_ROWS));
    if (e != cudaSuccess) return e;
    int per = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, attend_kernel<D, T>, kThreads, bytes);
    *grid = per * sms;
    return e;
}

}  // namespace

size_t attend_smem(int head_dim, int n) {
    const size_t fixed = head_dim == 64 ? Shape<64>::kRing + Shape<64>::kJoin
                       : head_dim == 128 ? Shape<128>::kRing + Shape<128>::kJoin : Shape<256>::kRing + Shape<256>::kJoin;
    return fixed + (kWarps + 1) * 16 * sizeof(float2) + (size_t)(n + 1) * sizeof(int32_t);
}

cudaError_t attend_grid(int head_dim, int type, int max_rows, int sms, int *grid) {
    if (type == ISJL_KV_BF16)
        return head_dim == 64 ? grid_of<64, __nv_bfloat16>(max_rows, sms, grid)
             : head_dim == 128 ? grid_of<128, __nv_bfloat16>(max_rows, sms, grid) : grid_of<256, __nv_bfloat16>(max_rows, sms, grid);
    return head_dim == 64 ? grid_of<64, __half>(max_rows, sms, grid)
         : head_dim == 128 ? grid_of<128, __half>(max_rows, sms, grid) : grid_of<256, __half>(max_rows, sms, grid);
}

cudaError_t launch_attend(const AttendArgs &g, void *encoder, int head_dim, int type, int grid, cudaStream_t st) {
    CUtensorMap k, v;
    const int rows = g.shift == 3 ? 8 : kSlice;
    if (!encode_cache(encoder, &k, g.cache.k, g.cache.k_stride, rows, g.n_blocks, g.shift, g.n_kv_heads, head_dim, type) ||
        !encode_cache(encoder, &v, g.cache.v, g.cache.v_stride, rows, g.n_blocks, g.shift, g.n_kv_heads, head_dim, type))
        return cudaErrorInvalidValue;
    if (type == ISJL_KV_BF16)
        return head_dim == 64 ? launch_of<64, __nv_bfloat16>(g, k, v, grid, st)
             : head_dim == 128 ? launch_of<128, __nv_bfloat16>(g, k, v, grid, st) : launch_of<256, __nv_bfloat16>(g, k, v, grid, st);
    return head_dim == 64 ? launch_of<64, __half>(g, k, v, grid, st)
         : head_dim == 128 ? launch_of<128, __half>(g, k, v, grid, st) : launch_of<256, __half>(g, k, v, grid, st);
}

}  // namespace isjl
