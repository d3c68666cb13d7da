// kv_attend.cu -- attention of single queries over paged tokens (isjl_kv_attend).
//
// A step reads every visible key and value once and does 4 D operations a query head with each: bound by
// memory.  The work is a line of slices of 32 tokens: for each query, each key head (and each 16 of its query
// heads), its visible slices in order, the first tokens' before the window's.  Every warp of the grid gets an
// equal run of that line wherever requests end, so ragged batches keep all SMs loading to the end.  A warp's
// slices come by TMA through a ring of its own and no warp waits for another: the running maximum and sum of
// the softmax, the sums and an item's result are the warp's own, and while one is between items the others
// keep the memory busy.  The query heads of a key head are the 16 rows of a tensor instruction.  An item cut
// by the runs' ends leaves pieces (those of neighbouring warps joined in shared memory first), which a second
// kernel joins in their order.  Joining them here, by the last of an item's warps to arrive, took a fence and an
// atomic under full memory load: 10 to 20 us of stall against 3 us of a small kernel that starts as this one ends.
//
// 512 queries of 64 + 8 heads of 128 values, 4 GB of keys and values: 627 us, 6.5 TB/s; 256 queries, 670 MB: 121 us,
// 5.5 TB/s (6 us until the rings are full, and SMs that end up to 15% apart).  The tensor pipe is 18% busy.  64 queries
// of 8 + 8 heads of 256 values, 2.1 GB: 354 us, 6.1 TB/s.  More than 16 query heads on a key head read it again for
// each 16: 256 queries of 16 + 1 heads over 8,192 tokens 214 us, of 64 + 1 heads 706.
#include "kv_ring.cuh"
#include "kv_tma.cuh"

namespace isjl {
namespace {

constexpr int kWarps = kAttendWarps, kThreads = 32 * kWarps, kSlice = 32;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int D>
struct Shape {
    static constexpr int kStages = D == 64 ? 6 : 3;                // of a warp's ring: keys or values of a slice
    static constexpr int kBlocks = D == 256 ? 1 : 2;               // per SM
    static constexpr int kHalves = D / 64;                         // rows of 128 bytes hold 64 values
    static constexpr int kHalfBytes = kSlice * 128;
    static constexpr int kStageBytes = kHalves * kHalfBytes;
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kJoinRow = D + 8;                         // padded: 8 rows of a warp's store on all banks
    static_assert(kWarps * 16 * kJoinRow * 4 <= kRing, "the joined pieces take the ring's place");
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
    int32_t end, lo, head;     // head: slices with first tokens that lie before the window's first slice
    int32_t slices;            // at least 1: an item without tokens still has a result
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
    s.head = min((min(a.sinks, s.lo) + kSlice - 1) / kSlice, s.lo / kSlice);
    s.slices = max(1, s.head + (s.end + kSlice - 1) / kSlice - s.lo / kSlice);
    return s;
}

// first token of a query's slice
__device__ __forceinline__ int32_t slice_start(const Sight &s, int i) {
    return (i < s.head ? i : s.lo / kSlice + i - s.head) * kSlice;
}

__device__ __forceinline__ float inverse(float total) { return total > 0.f || total != total ? 1.f / total : 0.f; }
// the logarithm of a sum of exp2, in the natural base
__device__ __forceinline__ float log_of(float top, float total) {
    return total > 0.f || total != total ? (top + log2f(total)) * kLn2 : -INFINITY;
}

// place on the line of slices
struct Place {
    int t, h, i;
    Sight s;
};

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, Shape<D>::kBlocks)
attend_kernel(const __grid_constant__ AttendArgs g, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
    using S = Shape<D>;
    extern __shared__ __align__(1024) unsigned char smem[];
    float2 *stats = reinterpret_cast<float2 *>(smem + S::kRing);                     // [kWarps][16]
    int32_t *before = reinterpret_cast<int32_t *>(stats + kWarps * 16);              // [n + 1] slices before a query
    __shared__ int32_t warp_sum[kWarps];
    __shared__ int64_t cut[kWarps];           // where on the line the item begins that a warp's run leaves cut, or -1
    __shared__ __align__(8) uint64_t bars[kWarps * S::kStages];

    const isjl_kv_attend_args &a = g.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = a.n, parts = (g.group + 15) / 16, H = g.n_kv_heads * parts, hq = g.n_kv_heads * g.group;
    const float scale = a.scale * kLog2e;

    const uint32_t bar0 = smem_addr(bars) + warp * S::kStages * 8;
    start_next();
    if (lane == 0) {
        tma_prefetch(&kmap);
        tma_prefetch(&vmap);
        for (int i = 0; i < S::kStages; ++i) bar_init(bar0 + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // ---- slices before each query
    {
        const int per = (n + kThreads - 1) / kThreads;
        const int begin = min(n, (int)threadIdx.x * per), end = min(n, begin + per);
        int32_t sum = 0;
        for (int t = begin; t < end; ++t) {
            const int32_t k = sight(g, t).slices;
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
    const int64_t W = (int64_t)before[n] * H;
    const int64_t C = min((int64_t)gridDim.x * kWarps, W);               // warps with work
    const int64_t me = (int64_t)blockIdx.x * kWarps + warp;
    const int64_t f0 = me < C ? W * me / C : W, f1 = me < C ? W * (me + 1) / C : W;

    auto advance = [&](Place &p) {
        if (++p.i < p.s.slices) return;
        p.i = 0;
        if (++p.h < H) return;
        p.h = 0;
        if (++p.t < n) p.s = sight(g, p.t);
    };

    // ---- the ring: keys and values of a slice, one stage each.  A lane has one copy of a stage: the rows of one
    // of the slice's blocks, or all of them where the block is larger.
    const uint32_t ring = smem_addr(smem) + warp * S::kStages * S::kStageBytes;
    const int32_t prefix_blocks = g.line.blocks ? 0 : a.n_prefix_blocks;
    const int rows_shift = min(g.shift, 5), piece = lane;
    const bool copies = piece < (kSlice >> rows_shift);
    const uint32_t half_bytes = 128u << rows_shift;                    // a copy's rows of 64 values
    const uint32_t copy_at = ring + piece * S::kHalves * half_bytes;
    // where a row lies in a stage
    auto row_at = [&](int row) { return (row >> rows_shift) * S::kHalves * half_bytes + (row & ((1 << rows_shift) - 1)) * 128; };
    // the number of this lane's block, asked for one slice ahead of the copies that use it and looked at only there
    constexpr int32_t kNone = INT32_MIN;
    auto block_of = [&](const Place &p) {
        const int32_t y = slice_start(p.s, p.i) + (piece << rows_shift);
        if (!copies || y >= p.s.end || (y + (1 << rows_shift) <= p.s.lo && y >= a.sinks)) return kNone;   // nothing is seen of it
        const int32_t j = y >> g.shift;
        return j < prefix_blocks ? a.prefix[j] : a.table[(int64_t)p.s.row * a.table_width + (j - prefix_blocks)];
    };

    Place here;
    here.t = here.h = here.i = 0;
    if (f0 < f1) {
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((int64_t)before[mid] * H <= f0) lo = mid; else hi = mid;
        }
        here.t = lo;
        here.s = sight(g, lo);
        const int64_t rest = f0 - (int64_t)before[lo] * H;
        here.h = (int)(rest / here.s.slices);
        here.i = (int)(rest - (int64_t)here.h * here.s.slices);
    }
    Place ahead = here;
    int64_t ahead_left = f1 - f0;                      // slices whose values are still to be asked for
    bool ahead_values = false;                         // what is next: keys or values
    int32_t ahead_block = f0 < f1 ? block_of(ahead) : kNone;
    auto feed = [&](int stage) {
        if (ahead_left == 0) return;
        const uint32_t bar = bar0 + 8 * stage;
        int32_t block = ahead_block;
        if ((uint32_t)block >= (uint32_t)g.n_blocks) {                 // beyond the cache: zeros
            if (block != kNone) report(g.status);
            block = g.n_blocks;
        }
        if (lane == 0) bar_expect(bar, S::kStageBytes);
        if (copies)
            tma_load(copy_at + stage * S::kStageBytes, ahead_values ? &vmap : &kmap, bar,
                     slice_start(ahead.s, ahead.i) & ((1 << g.shift) - 1) & ~((1 << rows_shift) - 1), 0, ahead.h / parts, block);
        ahead_values = !ahead_values;
        if (ahead_values) return;
        if (--ahead_left == 0) return;
        advance(ahead);
        ahead_block = block_of(ahead);
        if (ahead.i == 0) {                            // the next item's queries
            const int kv = ahead.h / parts, from = kv * g.group + (ahead.h - kv * parts) * 16;
            const int rows = min(16, (kv + 1) * g.group - from);
            const T *qt = static_cast<const T *>(a.q) + ahead.t * a.q_stride[0] + from * a.q_stride[1];
            for (int i = lane; i < rows * (D / 64); i += 32)
                asm volatile("prefetch.global.L2 [%0];" ::"l"(qt + i / (D / 64) * a.q_stride[1] + i % (D / 64) * 64));
        }
    };
#pragma unroll
    for (int i = 0; i < S::kStages - 1; ++i) feed(i);

    uint32_t q[D / 16][4];
    float o[D / 8][4], m[2], l[2];
    int first = 0, live = 0;                           // query heads of the item
    const int r = lane >> 2, c = (lane & 3) * 2;       // this lane's rows r and r + 8, its columns 8 i + c and + 1
    auto begin_item = [&]() {
        const int kv = here.h / parts;
        first = kv * g.group + (here.h - kv * parts) * 16;
        live = min(16, (kv + 1) * g.group - first);
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
        const T *qt = static_cast<const T *>(a.q) + here.t * a.q_stride[0] + first * a.q_stride[1];
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = r + (j & 1) * 8, col = k * 16 + c + (j >> 1) * 8;
                q[k][j] = row < live ? *reinterpret_cast<const uint32_t *>(qt + row * a.q_stride[1] + col) : 0u;
            }
    };

    RingPlace<S::kStages> place;
    int64_t f = f0;                                    // the slice at hand, on the line
    bool stuck = false;
    // The next stage of the ring (a slice's keys, 0, or values, 1), when it has come; the one before it, which all have
    // read by now, is fed.  Lanes leave the prefetches and the wait at different times, and the products that follow
    // are the whole warp's.  So is giving up: nothing is asked for after it, and what is under way is waited for, since
    // the ring's memory is used again and then becomes another block's.
    auto next_stage = [&](int values) {
        __syncwarp();
        feed(place.before());
        const uint32_t at = ring + place.stage * S::kStageBytes;
        if (!stuck) {
            stuck = !__all_sync(~0u, bar_wait(bar0 + 8 * place.stage, place.phase));
            if (stuck) {
                ahead_left = 0;
                for (int k = place.under_way(2 * (f1 - f) - values); k > 0; --k, place.take()) bar_wait(bar0 + 8 * place.stage, place.phase);
            }
            place.take();
        }
        __syncwarp();
        return at;
    };

    uint32_t key_row[2], value_row[2];                 // of this lane's rows in tensor operands
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        key_row[h] = row_at((lane & 7) + (lane >> 4) * 8 + 16 * h);
        value_row[h] = row_at((lane & 7) + ((lane >> 3) & 1) * 8 + 16 * h);
    }
    auto slice = [&]() {
        const int32_t x = slice_start(here.s, here.i);
        const uint32_t keys = next_stage(0);
        float s[4][4] = {};
        {
            // lanes 0-7: tokens 0-7 low half of 16 values, 8-15: high half, 16-23: tokens 8-15 low, 24-31: high
            const uint32_t turn = (((lane >> 3) & 1) ^ (lane & 7)) << 4;
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t b[4];
                    ldsm4(b, keys + key_row[h] + (k / 4) * half_bytes + (turn ^ ((k % 4) << 5)));
                    Half<T>::mma(s[2 * h], q[k], b[0], b[1]);
                    Half<T>::mma(s[2 * h + 1], q[k], b[2], b[3]);
                }
        }
        const bool edge = x + kSlice > here.s.end || x < here.s.lo;
        auto hidden = [&](int32_t y) { return y >= here.s.end || (y < here.s.lo && y >= a.sinks); };
        if (edge) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (hidden(x + i * 8 + c + j)) s[i][j] = s[i][2 + j] = -INFINITY;
        }
        float top[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float most = fmaxf(s[0][2 * j], s[0][2 * j + 1]);
#pragma unroll
            for (int i = 1; i < 4; ++i) most = fmaxf(most, fmaxf(s[i][2 * j], s[i][2 * j + 1]));
            most *= scale;
            most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
            top[j] = fmaxf(most, __shfl_xor_sync(~0u, most, 2)) - Half<T>::kTop;     // what weights are relative to
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
        // Weights are rounded to the cache's type for the product, as the tensor instruction takes them; the sum l is
        // of the unrounded ones, a slice's among themselves first: beside a large l small ones would be lost one by one.
        float part[2] = {0.f, 0.f};
        uint32_t w[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float u = ex2(fmaf(s[i][2 * j], scale, -ref[j])), v = ex2(fmaf(s[i][2 * j + 1], scale, -ref[j]));
                part[j] += u + v;
                w[i / 2][(i & 1) * 2 + j] = Half<T>::pack(u, v);
            }
        l[0] += part[0];
        l[1] += part[1];
        const uint32_t values = next_stage(1);
        if (edge) {
            // a weight of 0 does not silence an infinite or undefined value: what is not seen becomes 0
            for (int i = lane; i < kSlice * S::kHalves * 8; i += 32) {
                const int row = (i / 8) % kSlice;
                if (hidden(x + row))
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};"
                                 ::"r"(values + row_at(row) + i / (8 * kSlice) * half_bytes + i % 8 * 16), "r"(0) : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // before the next copy to this stage
            __syncwarp();
        }
        {
            const uint32_t turn = ((lane >> 4) ^ (lane & 7)) << 4;
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t b[4];
                    ldsm4t(b, values + value_row[h] + (k / 4) * half_bytes + (turn ^ ((k % 4) << 5)));
                    Half<T>::mma(o[2 * k], w[h], b[0], b[1]);
                    Half<T>::mma(o[2 * k + 1], w[h], b[2], b[3]);
                }
        }
    };

    // ---- results, and pieces of items
    auto sum_rows = [&]() {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            l[j] += __shfl_xor_sync(~0u, l[j], 1);
            l[j] += __shfl_xor_sync(~0u, l[j], 2);
        }
    };
    // the end of an item in this warp's run
    auto end_item = [&]() {
        const bool whole = (int64_t)before[here.t] * H + (int64_t)here.h * here.s.slices >= f0;
        sum_rows();
        if (whole && !g.line.blocks) {
            T *out = static_cast<T *>(a.out) + here.t * a.out_stride[0] + first * a.out_stride[1];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = r + 8 * j;
                if (row >= live) break;
                const float inv = inverse(l[j]);
#pragma unroll
                for (int i = 0; i < D / 8; ++i)
                    *reinterpret_cast<uint32_t *>(out + row * a.out_stride[1] + 8 * i + c) = Half<T>::pack(o[i][2 * j] * inv, o[i][2 * j + 1] * inv);
                if ((lane & 3) == 0 && a.lse) a.lse[(int64_t)here.t * hq + first + row] = log_of(m[j], l[j]);
            }
            return;
        }
        // a piece: beside the prefix's, or the last one of an item that earlier warps began
        if (whole && lane == 0) g.cut[here.t * H + here.h] = {here.t, here.h, (int)me, (int)me};
        const int64_t at = whole ? ((int64_t)g.line.pieces * n + here.t) * hq + first : me * 2 * 16;
        float *po = whole ? g.prefix_o : g.part_o;
        float2 *pml = whole ? g.prefix_ml : g.part_ml;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int row = r + 8 * j;
            if (row >= live) break;
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
                *reinterpret_cast<float2 *>(po + (at + row) * D + 8 * i + c) = make_float2(o[i][2 * j], o[i][2 * j + 1]);
            if ((lane & 3) == 0) pml[at + row] = make_float2(m[j], l[j]);
        }
    };

    if (f0 < f1) begin_item();
    for (; f < f1; ++f) {
        if (!stuck) slice();                            // the records of items stay whole
        if (here.i + 1 == here.s.slices) end_item();
        if (f + 1 < f1) {
            advance(here);
            if (here.i == 0) begin_item();
        }
    }
    if (stuck && lane == 0) atomicOr(g.status, 2);

    // ---- what the runs' ends cut: `here` is each warp's last slice
    const bool tail = f0 < f1 && here.i + 1 < here.s.slices;
    if (tail) sum_rows();
    if (lane == 0) {                                    // an item that begins here and is cut, for the kernel that joins it
        const int64_t i0 = (int64_t)before[here.t] * H + (int64_t)here.h * here.s.slices;
        const bool begins = tail && i0 >= f0;
        CutItem item = {-1, 0, 0, 0};
        if (begins) item = {here.t, here.h, (int)(((i0 + 1) * C - 1) / W), (int)(((i0 + here.s.slices) * C - 1) / W)};
        if (!g.line.blocks) g.cut[me] = item;
        else if (begins) g.cut[here.t * H + here.h] = item;
    }
    if (lane == 0) cut[warp] = tail ? (int64_t)before[here.t] * H + (int64_t)here.h * here.s.slices : -1;
    if (tail && (lane & 3) == 0) {
        stats[warp * 16 + r] = make_float2(m[0], l[0]);
        stats[warp * 16 + r + 8] = make_float2(m[1], l[1]);
    }
    __syncthreads();
    float *join = reinterpret_cast<float *>(smem);                                   // [kWarps][16][kJoinRow]
    int lead = warp, last = warp;                       // the neighbours that cut the same item
    if (tail) {
        while (lead > 0 && cut[lead - 1] == cut[warp]) --lead;
        while (last + 1 < kWarps && cut[last + 1] == cut[warp]) ++last;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int row = r + 8 * j;
            if (row >= live) break;
            float top = -INFINITY;
            for (int w = lead; w <= last; ++w) top = fmaxf(top, stats[w * 16 + row].x);
            const float fix = ex2(m[j] - (top == -INFINITY ? 0.f : top));
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
                *reinterpret_cast<float2 *>(join + (warp * 16 + row) * S::kJoinRow + 8 * i + c) = make_float2(o[i][2 * j] * fix, o[i][2 * j + 1] * fix);
        }
    }
    __syncthreads();
    // the first of each group of neighbours writes the group's piece
    if (tail && lead == warp) {
        const int64_t at = (me * 2 + 1) * 16;
        for (int x = lane; x < live * (D / 4); x += 32) {
            const int row = x / (D / 4), d = (x % (D / 4)) * 4;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int w = warp; w <= last; ++w) {
                const float4 v = *reinterpret_cast<const float4 *>(join + (w * 16 + row) * S::kJoinRow + d);
                sum.x += v.x;
                sum.y += v.y;
                sum.z += v.z;
                sum.w += v.w;
            }
            *reinterpret_cast<float4 *>(g.part_o + (at + row) * D + d) = sum;
        }
        if (lane < live) {
            float top = -INFINITY, total = 0.f;
            for (int w = warp; w <= last; ++w) top = fmaxf(top, stats[w * 16 + lane].x);
            for (int w = warp; w <= last; ++w) total += stats[w * 16 + lane].y * ex2(stats[w * 16 + lane].x - (top == -INFINITY ? 0.f : top));
            g.part_ml[at + lane] = make_float2(top, total);
        }
    }
    // The kernel after this one also reads the prefix's pieces: this one ends after the prefix's kernel.  One block
    // sees to that, the others leave their SM to those that have not started.
    if (blockIdx.x + 1 == gridDim.x) wait_for_previous();
}

// Joins pieces: of the items that runs' ends cut, a block for the warp in whose run one begins; where a prefix was
// done apart, of all items, a block for each, with the prefix's pieces.
constexpr int kJoinThreads = 128;

template <int D, typename T, int kBatch>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ AttendArgs g) {
    const isjl_kv_attend_args &a = g.a;
    const int n = a.n, parts = (g.group + 15) / 16, hq = g.n_kv_heads * g.group;
    wait_for_previous();
    const CutItem item = g.cut[blockIdx.x];
    if (item.t < 0) return;
    const int t = item.t, h = item.h, first = item.first, last = item.last;
    // An item's pieces: of each block the joined ones of the warps whose runs it fills to the end, and that of the
    // last warp, in whose run it ends; or the one of an item that is a warp's own.
    const int kv = h / parts, from = kv * g.group + (h - kv * parts) * 16, rows = min(16, (kv + 1) * g.group - from);
    const int cut = first == last ? 0 : (last - 1) / kWarps - first / kWarps + 2;
    const int prefix_item = g.line.blocks ? kv * g.line.pairs + t / g.line.tokens_of_tile / 2 : 0;
    const int shared = g.line.blocks && sight(g, t).end > 0 ? g.line.last_block(prefix_item) - g.line.first_block(prefix_item) + 1 : 0;
    const int own = cut ? cut : 1, pieces = own + shared;
    T *out = static_cast<T *>(a.out) + t * a.out_stride[0] + from * a.out_stride[1];
    for (int x = threadIdx.x; x < rows * (D / 4); x += kJoinThreads) {
        const int row = x / (D / 4), d = (x % (D / 4)) * 4;
        float top = -INFINITY, total = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k0 = 0; k0 < pieces; k0 += kBatch) {     // some at a time: their loads are under way together
            float2 ml[kBatch];
            float4 v[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int p = min(k0 + k, pieces - 1);
                const bool from_cut = cut && p < own;
                const int w = max(first, (first / kWarps + p) * kWarps);
                const int64_t at = from_cut ? (p + 1 == own ? last * 2 : w * 2 + 1) * 16 + row
                                            : ((int64_t)(p < own ? g.line.pieces : p - own) * n + t) * hq + from + row;
                ml[k] = (from_cut ? g.part_ml : g.prefix_ml)[at];
                v[k] = *reinterpret_cast<const float4 *>((from_cut ? g.part_o : g.prefix_o) + at * D + d);
            }
            float next = top;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) next = fmaxf(next, ml[k].x);
            const float ref = next == -INFINITY ? 0.f : next, fix = ex2(top - ref);
            top = next;
            total *= fix;
            sum.x *= fix;
            sum.y *= fix;
            sum.z *= fix;
            sum.w *= fix;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (k0 + k >= pieces) break;
                const float w = ex2(ml[k].x - ref);
                total += ml[k].y * w;
                sum.x += v[k].x * w;
                sum.y += v[k].y * w;
                sum.z += v[k].z * w;
                sum.w += v[k].w * w;
            }
        }
        const float inv = inverse(total);
        *reinterpret_cast<uint2 *>(out + row * a.out_stride[1] + d) =
            make_uint2(Half<T>::pack(sum.x * inv, sum.y * inv), Half<T>::pack(sum.z * inv, sum.w * inv));
        if (d == 0 && a.lse) a.lse[(int64_t)t * hq + from + row] = log_of(top, total);
    }
}

template <int D, typename T>
cudaError_t launch_of(const AttendArgs &g, const CUtensorMap &k, const CUtensorMap &v, int grid, cudaStream_t st) {
    const bool apart = g.line.blocks > 0;
    const cudaError_t e = launch_kernel(attend_kernel<D, T>, grid, kThreads, attend_smem(D, g.a.n), st, apart, g, k, v);
    if (e != cudaSuccess) return e;
    const int items = apart ? g.a.n * g.n_kv_heads * ((g.group + 15) / 16) : grid * kWarps;
    // Few pieces of many items: few registers, many blocks at once.  Many pieces of few items: their loads together.
    // Whole calls from a cold L2 with 3 and with 12 at a time: window of 1,024 with 256 queries 140 and 143 us, 512 queries
    // over a prefix of 32,768 482 and 496, 900 over 2,560 46 and 50; 1 query over 3,000 tokens 21.6 and 17.5, 17 over a
    // prefix of 2,048 29.8 and 27.8, 40 over 16,384 54.4 and 52.4; equal with 32 over 8,192.  128 queries over 4,096
    // (5 pieces) are 50 and 53: there the rule takes the slower one.
    const bool few = apart ? g.line.pieces < 4 : items < 4 * g.a.n * g.n_kv_heads;
    if (few) return launch_kernel(join_kernel<D, T, 3>, items, kJoinThreads, 0, st, true, g);
    return launch_kernel(join_kernel<D, T, 12>, items, kJoinThreads, 0, st, true, g);
}

template <int D, typename T>
cudaError_t prepare_of(int *blocks, int *queries) {
    // the limit belongs to the function, not to a handle: always the largest
    cudaError_t e = cudaFuncSetAttribute(attend_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)attend_smem(D, ISJL_KV_MAX_ROWS));
    int lo = 1, hi = ISJL_KV_MAX_ROWS + 1, per = 0;
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(blocks, attend_kernel<D, T>, kThreads, attend_smem(D, 1));
    while (e == cudaSuccess && hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, attend_kernel<D, T>, kThreads, attend_smem(D, mid));
        if (per == *blocks) lo = mid; else hi = mid;
    }
    *queries = lo;
    return e;
}

}  // namespace

size_t attend_smem(int head_dim, int n) {
    const size_t ring = head_dim == 64 ? Shape<64>::kRing : head_dim == 128 ? Shape<128>::kRing : Shape<256>::kRing;
    return ring + kWarps * 16 * sizeof(float2) + (size_t)(n + 1) * sizeof(int32_t);
}

cudaError_t prepare_attend(int head_dim, int type, int *blocks, int *queries) {
    if (type == ISJL_KV_BF16)
        return head_dim == 64 ? prepare_of<64, __nv_bfloat16>(blocks, queries)
             : head_dim == 128 ? prepare_of<128, __nv_bfloat16>(blocks, queries) : prepare_of<256, __nv_bfloat16>(blocks, queries);
    return head_dim == 64 ? prepare_of<64, __half>(blocks, queries)
         : head_dim == 128 ? prepare_of<128, __half>(blocks, queries) : prepare_of<256, __half>(blocks, queries);
}

cudaError_t launch_attend(const AttendArgs &g, void *encoder, int head_dim, int type, int grid, cudaStream_t st) {
    CUtensorMap k, v;
    const int rows = min(1 << g.shift, kSlice);
    if (!encode_cache(encoder, &k, g.cache.k, g.cache.k_stride, rows, head_dim / 64, g.n_blocks, g.shift, g.n_kv_heads, head_dim, type) ||
        !encode_cache(encoder, &v, g.cache.v, g.cache.v_stride, rows, head_dim / 64, g.n_blocks, g.shift, g.n_kv_heads, head_dim, type))
        return cudaErrorInvalidValue;
    if (type == ISJL_KV_BF16)
        return head_dim == 64 ? launch_of<64, __nv_bfloat16>(g, k, v, grid, st)
             : head_dim == 128 ? launch_of<128, __nv_bfloat16>(g, k, v, grid, st) : launch_of<256, __nv_bfloat16>(g, k, v, grid, st);
    return head_dim == 64 ? launch_of<64, __half>(g, k, v, grid, st)
         : head_dim == 128 ? launch_of<128, __half>(g, k, v, grid, st) : launch_of<256, __half>(g, k, v, grid, st);
}

}  // namespace isjl
