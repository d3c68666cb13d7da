// kv_prompt.cuh -- what stands around isjl_kv_prompt's products (kv_prompt.cu): rows of queries and the items that they
// make, the run of items that a block has, values that must not spread, and the kernel that joins pieces of items.
#pragma once

#include "kv_prompt_line.cuh"
#include "kv_tma.cuh"

namespace isjl {
namespace {

constexpr int kColumns = 16;                        // of a row's sums that are written at a time
constexpr int kSpoilt = 32;                         // of a row's sums that values not finite are added to at a time
constexpr int kMostRuns = 1024;                     // blocks that have a run, at most
constexpr int kJoinBlocks = 8, kJoinThreads = 128;  // of the joining kernel, for each SM

// What a block does with an item, or with its run's part of one.
struct Item {
    int32_t count;               // tiles; 0: the run has ended
    int32_t tile0, skipped;      // the first of them in the item, tiles left out between first tokens and windows
    int32_t row, kv, q_head, members;    // key head, first query head and query heads
    int32_t start, tokens;       // its queries
    int32_t place;               // of the first one
    int32_t end, low;            // tokens from `end` on and, but for the first ones, before `low` are not seen by any query
    int32_t from, below;         // tokens from `from` on and, but for the first ones, before `below` are not seen by all
    int32_t kind;                // kWhole: all of its tiles; kFirst: the item begins here; kDead: its queries see nothing
};
enum { kWhole = 1, kFirst = 2, kDead = 4 };

// A row as its places are counted with the prefix; `dead`: it sees nothing.
struct Row : PromptRow {
    int32_t start;               // of its queries
    bool dead;
};

__device__ __forceinline__ Row row_of(const PromptArgs &g, int i, bool tell) {
    const isjl_kv_prompt_args &a = g.a;
    const int32_t s0 = a.starts[i], s1 = a.starts[i + 1], len = a.lens[i];
    Row r;
    r.start = s0;
    r.count = s1 - s0;
    r.first = 0;
    r.dead = false;
    if (s0 < 0 || s1 < s0 || s1 > a.n_tokens) {
        if (tell) report(g.status);
        r.count = 0;
    } else if (r.count > 0 && (len < r.count || ((len - 1) >> g.shift) >= a.table_width)) {
        if (tell) report(g.status);
        r.dead = true;
    } else {
        r.first = (a.n_prefix_blocks << g.shift) + len - r.count;
    }
    return r;
}

// place on the line: tile j of an item
struct Place {
    int32_t row, head, item, j, items;
    Row r;
};

// to the next item's first tile; there is one
__device__ __forceinline__ void next_item(const PromptArgs &g, const PromptShape &s, Place &p) {
    p.j = 0;
    if (++p.item == p.items) {
        p.item = 0;
        if (++p.head == g.n_kv_heads * g.parts) {
            p.head = 0;
            do {
                ++p.row;
                p.r = row_of(g, p.row, false);
                p.items = p.r.items(s);
            } while (p.items == 0);
        }
    }
}

// how a tile's rows hold tokens, each with the query heads of (a part of) a key head
inline void share_rows(PromptArgs &g, int tile_rows) {
    g.rows_of_token = g.group < tile_rows ? g.group : tile_rows;
    g.parts = (g.group + g.rows_of_token - 1) / g.rows_of_token;
    g.tokens_of_tile = tile_rows / g.rows_of_token;
}

// query heads of a key head's part
__device__ __forceinline__ int heads_of(const PromptArgs &g, int head, int *first) {
    const int kv = head / g.parts, part = head - kv * g.parts;
    *first = kv * g.group + part * g.rows_of_token;
    return min(g.rows_of_token, g.group - part * g.rows_of_token);
}

// the cache's block of a token at place y, which is one of row `row`'s or the prefix's
__device__ __forceinline__ int32_t block_at(const PromptArgs &g, int row, int32_t y) {
    const int32_t j = y >> g.shift;
    return j < g.a.n_prefix_blocks ? g.a.prefix[j] : g.a.table[(int64_t)row * g.a.table_width + (j - g.a.n_prefix_blocks)];
}

// the first token of an item's j-th tile in this run
__device__ __forceinline__ int32_t tile_at(const PromptShape &s, const Item &x, int j) { return PromptRow::tile(s, x.skipped, x.tile0 + j) * s.keys; }
// whether some query of the item does not see a token of the tile at y0, and whether that is so for token y
__device__ __forceinline__ bool edge(const PromptShape &s, const Item &x, int32_t y0) {
    return y0 + s.keys > x.from || (y0 < x.below && y0 + s.keys > s.sinks);
}
__device__ __forceinline__ bool edge_token(const PromptShape &s, const Item &x, int32_t y) { return y >= x.from || (y < x.below && y >= s.sinks); }

// whether one of a word's two 16-bit numbers is infinite or undefined: its exponent's bits are all set
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    constexpr uint32_t kExponent = Half<T>::kIsBf16 ? 0x7f807f80u : 0x7c007c00u, kLowest = Half<T>::kIsBf16 ? 0x00800080u : 0x04000400u;
    return ((w & kExponent) + kLowest) & 0x80008000u;
}

// Of the values that the sums left out because they are not finite: what they make of kSpoilt columns' sums, a bit each
// (infinite, the other sign's, undefined).  Rare and slow: the row's weights are computed again from the cache.
struct Spoilt {
    uint32_t plus, minus, none;
};
template <int D, typename T>
__device__ __forceinline__ Spoilt spoilt(const PromptArgs &g, const PromptShape &s, const Item &x, int32_t token, int32_t q_head, int column, float top,
                                         float scale) {
    Spoilt out = {0, 0, 0};
    const int32_t place = x.place + token, low = PromptRow::low(s, place);
    for (int32_t j = 0; j < x.count; ++j) {
        const int32_t y0 = tile_at(s, x, j);
        if (!edge(s, x, y0)) continue;
        for (int32_t y = y0; y < min(y0 + s.keys, place + 1); ++y) {
            if (!edge_token(s, x, y) || (y < low && y >= s.sinks)) continue;
            const int32_t block = block_at(g, x.row, y), slot = y & ((1 << g.shift) - 1);
            if ((uint32_t)block >= (uint32_t)g.n_blocks) continue;
            const T *v = static_cast<const T *>(g.cache.v) + block * g.cache.v_stride[0] + slot * g.cache.v_stride[1] + x.kv * g.cache.v_stride[2] + column;
            bool any = false;
#pragma unroll 1
            for (int i = 0; i < kSpoilt / 2; ++i) any = any || not_finite<T>(reinterpret_cast<const uint32_t *>(v)[i]);
            if (!any) continue;
            const T *k = static_cast<const T *>(g.cache.k) + block * g.cache.k_stride[0] + slot * g.cache.k_stride[1] + x.kv * g.cache.k_stride[2];
            const T *q = static_cast<const T *>(g.a.q) + (int64_t)(x.start + token) * g.a.q_stride[0] + (int64_t)q_head * g.a.q_stride[1];
            float dot = 0.f;
#pragma unroll 1
            for (int i = 0; i < D / 2; ++i) {
                const float2 a = Half<T>::unpack(reinterpret_cast<const uint32_t *>(q)[i]), b = Half<T>::unpack(reinterpret_cast<const uint32_t *>(k)[i]);
                dot += a.x * b.x + a.y * b.y;
            }
            const bool counts = ex2(dot * scale - (top == -INFINITY ? 0.f : top)) > 0.f;       // 0 times infinity is undefined
#pragma unroll 1
            for (int i = 0; i < kSpoilt; ++i) {
                const float z = Half<T>::unpack(reinterpret_cast<const uint16_t *>(v)[i]).x;
                if (z - z == 0.f) continue;
                if (!counts || z != z) out.none |= 1u << i;
                else (z > 0.f ? out.plus : out.minus) |= 1u << i;
            }
        }
    }
    return out;
}

// a / b of numbers that are mostly small: 64 bits take a few hundred cycles
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return (a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// A block's run of the line: places f .. f1 - 1, of which `here` is the first.  An item's tiles have some places before them
// that stand for its beginning and end, so that runs of many items have fewer tiles.
struct Run {
    int64_t tiles, blocks;       // places of the line; blocks with a run
    int64_t f, f1;
    Place here;
};

struct RunWords {
    int64_t sums[32], rest, each;        // of the row that the run begins in: tiles before it in the row, and of each head
    int32_t row;
};

// Finds this block's run; all threads of the block.  Whoever needs `here` asks for it with `begin_run`, a whole warp.
template <int kThreads>
__device__ __forceinline__ Run find_run(const PromptArgs &g, const PromptShape &s, RunWords &words) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, H = g.n_kv_heads * g.parts;
    const int per = (g.a.n_rows + kThreads - 1) / kThreads;
    const int begin = min(g.a.n_rows, (int)threadIdx.x * per), end = min(g.a.n_rows, begin + per);
    auto work = [&](int i, bool tell) {
        const Row r = row_of(g, i, tell);
        return r.before(s, r.items(s));
    };
    int64_t sum = 0;             // this thread's rows
    for (int i = begin; i < end; ++i) sum += H * work(i, blockIdx.x == 0);
    __syncwarp();                // the threads come from loops of different lengths
    int64_t before = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t p = __shfl_up_sync(~0u, before, d);
        if (lane >= d) before += p;
    }
    if (lane == 31) words.sums[warp] = before;
    __syncthreads();
    before -= sum;
    Run run = {};
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += words.sums[w];
        run.tiles += words.sums[w];
    }
    run.blocks = min((int64_t)gridDim.x, run.tiles);
    run.f = blockIdx.x < run.blocks ? quotient(run.tiles * blockIdx.x, run.blocks) : run.tiles;
    run.f1 = blockIdx.x < run.blocks ? quotient(run.tiles * (blockIdx.x + 1), run.blocks) : run.tiles;
    if (run.f < run.f1 && before <= run.f && run.f < before + sum)
        for (int i = begin; i < end; ++i) {
            const int64_t each = end - begin == 1 ? quotient(sum, H) : work(i, false);
            if (run.f < before + H * each) {
                words.row = i;
                words.rest = run.f - before;
                words.each = each;
                break;
            }
            before += H * each;
        }
    __syncthreads();
    return run;
}

__device__ __forceinline__ void begin_run(const PromptArgs &g, const PromptShape &s, const RunWords &words, Run &run) {
    if (run.f == run.f1) return;
    const int lane = threadIdx.x & 31;
    Place &p = run.here;
    p.row = words.row;
    p.r = row_of(g, p.row, false);
    p.items = p.r.items(s);
    p.head = (int)quotient(words.rest, words.each);
    const int64_t rest = words.rest - p.head * words.each;
    // the last item that begins at `rest` or before it: 32 places looked at together
    int lo = 0, hi = p.items;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step;
        const uint32_t past = __ballot_sync(~0u, at >= hi || p.r.before(s, at) > rest);
        const int k = past ? __ffs(past) - 1 : 32;
        hi = min(hi, lo + (k + 1) * step);
        lo += k * step;
    }
    p.item = lo;
    p.j = (int)(lo ? rest - p.r.before(s, lo) : rest);
}

// The run's next item, count 0 when there is none.  `writes`: this thread notes the item that the run's end cuts; it
// has to note that there is none before the first call.
__device__ __forceinline__ Item take_item(const PromptArgs &g, const PromptShape &s, Run &run, bool writes) {
    Item x = {};
    if (run.f == run.f1) return x;
    Place &p = run.here;
    const int32_t tiles = p.r.tiles(s, p.item), first = p.item * s.step, last = p.r.end(s, p.item) - 1;
    const int32_t places = (int32_t)min((int64_t)s.extra + tiles - p.j, run.f1 - run.f);
    x.tile0 = max(0, p.j - s.extra);
    x.count = max(0, p.j + places - s.extra) - x.tile0;
    if (x.count == 0) {                                  // the run ends before the item's first tile
        run.f = run.f1;
        return x;
    }
    x.skipped = p.r.skip(s, p.item);
    x.row = p.row;
    x.kv = p.head / g.parts;
    x.members = heads_of(g, p.head, &x.q_head);
    x.start = p.r.start + first;
    x.tokens = min(p.r.count - first, s.step);
    x.place = p.r.first + first;
    x.end = last + 1;
    x.low = PromptRow::low(s, x.place);
    x.from = p.r.dead ? 0 : x.place + 1;
    x.below = PromptRow::low(s, last);
    x.kind = (x.count == tiles ? kWhole : 0) | (x.tile0 == 0 ? kFirst : 0) | (p.r.dead ? kDead : 0);
    if (writes && x.count < tiles && x.tile0 == 0)       // its pieces are those of the blocks from here on
        g.cut[blockIdx.x] = {p.row, p.head, p.item, (int)quotient((run.f - p.j + s.extra + tiles) * run.blocks - 1, run.tiles)};
    run.f += places;
    if (run.f < run.f1) next_item(g, s, p);
    return x;
}

// Joins the pieces of the items that runs' ends cut.  The blocks share the cut items' rows, a few at a time, and a thread
// has four values of a row.  An item has kRows rows in tiles of kTileRows.
template <int D, typename T, int kRows, int kTileRows, int kKeys>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ PromptArgs g, int runs) {
    constexpr int kSlice = kJoinThreads / (D / 4), kSlices = kRows / kSlice;    // rows at a time, such parts of an item
    __shared__ uint32_t masks[kMostRuns / 32];            // blocks in whose runs a cut item begins
    const int lane = threadIdx.x & 31;
    const PromptShape shape = {kKeys, kRows / kTileRows * g.tokens_of_tile, g.a.window, g.a.sinks};
    const int hq = g.n_kv_heads * g.group;
    wait_for_previous();
    for (int b = threadIdx.x; b < kMostRuns; b += kJoinThreads) {
        const uint32_t mine = __ballot_sync(~0u, b < runs && g.cut[b].row >= 0);
        if (lane == 0) masks[b / 32] = mine;
    }
    __syncthreads();
    int count = 0, word = 0;                              // cut items in the words before `word`
    for (int unit = blockIdx.x;; unit += gridDim.x) {
        const int which = unit / kSlices;
        while (word < kMostRuns / 32 && count + __popc(masks[word]) <= which) count += __popc(masks[word++]);
        if (word == kMostRuns / 32) break;
        const int begin = 32 * word + (int)__fns(masks[word], 0, which - count + 1);
        const PromptCut item = g.cut[begin];
        const Row r = row_of(g, item.row, false);
        int first_head;
        const int members = heads_of(g, item.head, &first_head);
        const int at = unit % kSlices * kSlice + threadIdx.x / (D / 4), row = at % kTileRows, d = (threadIdx.x % (D / 4)) * 4;
        const int32_t token = item.item * shape.step + at / kTileRows * g.tokens_of_tile + row / g.rows_of_token;
        const int member = row % g.rows_of_token;
        if (row >= g.tokens_of_tile * g.rows_of_token || member >= members || token >= r.count) continue;
        float top = -INFINITY, total = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int kBatch = 8;                         // their loads are under way together
        for (int b0 = begin; b0 <= item.last; b0 += kBatch) {
            float2 ml[kBatch];
            float4 v[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int b = min(b0 + k, item.last);
                const int64_t from = (int64_t)(2 * b + (b == begin)) * kRows + at;
                ml[k] = g.part_ml[from];
                v[k] = *reinterpret_cast<const float4 *>(g.part_o + from * D + d);
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
                if (b0 + k > item.last) break;
                const float w = ex2(ml[k].x - ref);
                total += ml[k].y * w;
                sum.x += v[k].x * w;
                sum.y += v[k].y * w;
                sum.z += v[k].z * w;
                sum.w += v[k].w * w;
            }
        }
        const float inv = inverse(total);
        const int64_t query = r.start + token;
        *reinterpret_cast<uint2 *>(static_cast<T *>(g.a.out) + query * g.a.out_stride[0] + (first_head + member) * g.a.out_stride[1] + d) =
            make_uint2(Half<T>::pack(sum.x * inv, sum.y * inv), Half<T>::pack(sum.z * inv, sum.w * inv));
        if (d == 0 && g.a.lse)
            g.a.lse[query * hq + first_head + member] = log_of(top, total);
    }
}

}  // namespace
}  // namespace isjl
