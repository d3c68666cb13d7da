// kv_prompt.cu -- causal attention of packed prompts over the paged cache (isjl_kv_prompt).
//
// The queries of a row's tokens, times the `group` query heads of a key head, are the rows of a matrix: S = Q K^T,
// O = softmax(S) V, 4 D operations for each row and visible token, on the fifth-generation tensor cores.  An item is
// two tiles of 128 rows (one with heads of 256 values, whose sums fill half of TMEM) of one key head: a run of
// neighbouring tokens, each with all of its query heads, so that a tile of keys and values is used by all of them.
// An item's tiles of 128 tokens (64) end with the tokens that its last query sees.
//
// Keys and values come by TMA from the cache's blocks through a ring each, one thread issues the products, and each
// row of a tile is one thread of a group of four warps that takes the row's maximum, exponentials and sum.  Scores
// lie in TMEM, their weights take the scores' place as the second product's left operand, and the two row tiles
// alternate: while the tensor cores work for one, the other's group is at its exponentials.  The sums O stay in TMEM
// for the whole run and are rescaled only when a row's maximum has grown by more than 2^8 (fp16: 2^4) since the last
// time; rounding weights to 16 bits is as exact as with the true maximum.
//
// What a query does not see must not reach its sums, and a weight of 0 does not silence an infinite or undefined
// value.  In the tiles of which some of the item's queries see a part only, one warp makes zeros of the values that no
// query sees and of those that are not finite; where it found one of the latter, the rows that see it get it at the
// end, from the cache.
//
// The work is a line of (row, key head, item, tile): every block has an equal run of it, wherever prompts end, and one
// long prompt, many short ones or a few queries over a long cache all keep every SM busy to the end.  Items cut by the
// runs' ends leave pieces (sum, maximum and total of each row), which a second kernel joins in their order.
#include "kv_prompt_line.cuh"
#include "kv_tensor.cuh"

namespace isjl {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kRows = 128;                          // of a row tile
constexpr int kJoinThreads = 128, kJoinSlices = 8;  // blocks of a cut item

template <int D>
struct Shape {
    static constexpr int kGroups = D == 256 ? 1 : 2;             // row tiles of an item, each with its four warps
    static constexpr int kKeys = D == 256 ? 64 : 128;            // of a token tile
    static constexpr int kLoadWarp = 4 * kGroups, kIssueWarp = kLoadWarp + 2, kCleanWarp = kLoadWarp + 3;
    static constexpr int kThreads = 32 * (kLoadWarp + 4);
    static constexpr int kHalves = D / 64;                       // rows of 128 bytes hold 64 values
    static constexpr int kRowHalf = kRows * 128, kKeyHalf = kKeys * 128;
    static constexpr int kRowBytes = kHalves * kRowHalf, kTileBytes = kHalves * kKeyHalf;
    static constexpr int kKeyStages = D == 128 ? 3 : D == 64 ? 4 : 2, kValueStages = D == 128 ? 2 : D == 64 ? 4 : 3;
    static constexpr int kSmem = kGroups * kRowBytes + (kKeyStages + kValueStages) * kTileBytes + 1024;
    static constexpr int kSums = D == 256 ? 256 : 2 * kKeys;     // TMEM: scores from 0, sums from here
    static constexpr int kParts = kKeys / 64;                    // of a tile's weights, handed over one after another
};

// barriers, in 8-byte words
enum { kKeyFull = 0, kValueFull = 8, kFree = 4 /* after a stage's full one */, kClean = 16, kScores = 20, kWeights = 22, kRest = 24, kSumsDone = 26,
       kQueries = 28, kDrain = 30, kBars = 31 };
constexpr int kFlags = 8;        // items whose flags are kept: more than there are stages of values

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

// place on the line: tile j of an item, and how many tiles the item has
struct Place {
    int32_t row, head, item, j, tiles, skipped;
    Row r;
    int32_t items;
};

__device__ __forceinline__ void settle(const PromptShape &s, Place &p) {
    p.tiles = p.r.tiles(s, p.item);
    p.skipped = p.r.skip(s, p.item);
}
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
    settle(s, p);
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

// Which tokens of the tile at y0 some query of an item does not see: they end with those from `from` on, and begin
// with those in [sinks, below).
struct Edge {
    int32_t from, below;
    __device__ __forceinline__ Edge(const PromptShape &s, const Place &p) {
        const int32_t first = p.r.first + p.item * s.step, last = p.r.end(s, p.item) - 1;
        from = p.r.dead ? 0 : first + 1;
        below = p.r.low(s, last);
    }
    __device__ __forceinline__ bool any(const PromptShape &s, int32_t y0) const { return y0 + s.keys > from || (y0 < below && y0 + s.keys > s.sinks); }
    __device__ __forceinline__ bool in(const PromptShape &s, int32_t y) const { return y >= from || (y < below && y >= s.sinks); }
};

// whether one of a word's two 16-bit numbers is infinite or undefined: its exponent's bits are all set
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    constexpr uint32_t kExponent = Half<T>::kIsBf16 ? 0x7f807f80u : 0x7c007c00u, kLowest = Half<T>::kIsBf16 ? 0x00800080u : 0x04000400u;
    return ((w & kExponent) + kLowest) & 0x80008000u;
}

// Of the values that the sums left out because they are not finite: what they make of 32 columns' sums, a bit each
// (infinite, the other sign's, undefined).  Rare and slow: the row's weights are computed again from the cache.
struct Spoilt {
    uint32_t plus, minus, none;
};
template <int D, typename T>
__device__ __noinline__ Spoilt spoilt(const PromptArgs &g, const PromptShape &s, const Place &p, int32_t j0, int32_t j1, int32_t token, int32_t q_head,
                                      int column, float top, float scale) {
    Spoilt out = {0, 0, 0};
    const Edge edge(s, p);
    const int32_t place = p.r.first + token, low = p.r.low(s, place);
    const int kv = p.head / g.parts;
    for (int32_t j = j0; j < j1; ++j) {
        const int32_t y0 = PromptRow::tile(s, p.skipped, j) * s.keys;
        if (!edge.any(s, y0)) continue;
        for (int32_t y = y0; y < min(y0 + s.keys, place + 1); ++y) {
            if (!edge.in(s, y) || (y < low && y >= s.sinks)) continue;
            const int32_t block = block_at(g, p.row, y), slot = y & ((1 << g.shift) - 1);
            if ((uint32_t)block >= (uint32_t)g.n_blocks) continue;
            const T *v = static_cast<const T *>(g.cache.v) + block * g.cache.v_stride[0] + slot * g.cache.v_stride[1] + kv * g.cache.v_stride[2];
            bool any = false;
            for (int i = 0; i < 16; ++i) any = any || not_finite<T>(reinterpret_cast<const uint32_t *>(v + column)[i]);
            if (!any) continue;
            const T *k = static_cast<const T *>(g.cache.k) + block * g.cache.k_stride[0] + slot * g.cache.k_stride[1] + kv * g.cache.k_stride[2];
            const T *q = static_cast<const T *>(g.a.q) + (int64_t)(p.r.start + token) * g.a.q_stride[0] + (int64_t)q_head * g.a.q_stride[1];
            float dot = 0.f;
            for (int i = 0; i < D / 2; ++i) {
                const float2 x = Half<T>::unpack(reinterpret_cast<const uint32_t *>(q)[i]), z = Half<T>::unpack(reinterpret_cast<const uint32_t *>(k)[i]);
                dot += x.x * z.x + x.y * z.y;
            }
            const bool counts = ex2(dot * scale - (top == -INFINITY ? 0.f : top)) > 0.f;       // 0 times infinity is undefined
            for (int i = 0; i < 32; ++i) {
                const float x = Half<T>::unpack(reinterpret_cast<const uint16_t *>(v + column)[i]).x;
                if (x - x == 0.f) continue;
                if (!counts || x != x) out.none |= 1u << i;
                else (x > 0.f ? out.plus : out.minus) |= 1u << i;
            }
        }
    }
    return out;
}

template <int D, typename T>
__global__ void __launch_bounds__(Shape<D>::kThreads, 1)
prompt_kernel(const __grid_constant__ PromptArgs g, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
    using S = Shape<D>;
    constexpr bool kBf16 = Half<T>::kIsBf16;
    constexpr int kKeys = S::kKeys, kChunks = kKeys / 32;
    // operand types, 32-bit sums, 128 rows; the first product has a column for each token and both operands along D, the
    // second D columns and its right operand (values, tokens outermost) across
    constexpr uint32_t kTypes = (1u << 4) | (kBf16 ? (1u << 7) | (1u << 10) : 0u) | ((kRows / 16) << 24);
    constexpr uint32_t kFirst = kTypes | ((kKeys / 8) << 17), kSecond = kTypes | ((D / 8) << 17) | (1u << 16);
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ int64_t warp_sum[S::kThreads / 32];
    __shared__ int64_t found_rest;
    __shared__ int32_t found_row;
    __shared__ uint32_t tmem_base;
    __shared__ int32_t failed_word;
    __shared__ int32_t flag_word[kFlags];           // an item's number on this block, plus one, if the clean warp left out a value
    volatile int32_t *failed = &failed_word, *flags = flag_word;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
    const uint32_t q_at = base, ring = base + S::kGroups * S::kRowBytes;
    const uint32_t bar0 = smem_addr(bars);
    auto bar = [&](int i) { return bar0 + 8 * i; };
    const PromptShape shape = {kKeys, S::kGroups * g.tokens_of_tile, g.a.window, g.a.sinks};
    const int H = g.n_kv_heads * g.parts;

    start_next();
    if (threadIdx.x == 0) {
        tma_prefetch(&kmap);
        tma_prefetch(&vmap);
        failed_word = 0;
        found_row = -1;
        for (int i = 0; i < kFlags; ++i) flag_word[i] = 0;
        for (int i = 0; i < 20; ++i) bar_init(bar(i), 1);
        for (int i = 0; i < 2; ++i) {
            bar_init(bar(kScores + i), 1);
            bar_init(bar(kWeights + i), 128);
            bar_init(bar(kRest + i), 128);
            bar_init(bar(kSumsDone + i), 1);
            bar_init(bar(kQueries + i), 128);
        }
        bar_init(bar(kDrain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == S::kIssueWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }

    // ---- the line: tiles of each row, and where this block's run begins
    int64_t W, f0, f1, C;
    {
        const int per = (g.a.n_rows + S::kThreads - 1) / S::kThreads;
        const int begin = min(g.a.n_rows, (int)threadIdx.x * per), end = min(g.a.n_rows, begin + per);
        auto work = [&](int i, bool tell) {
            const Row r = row_of(g, i, tell);
            return H * r.before(shape, r.items(shape));
        };
        int64_t sum = 0;
        for (int i = begin; i < end; ++i) sum += work(i, blockIdx.x == 0);
        __syncwarp();                // the threads come from loops of different lengths
        int64_t inc = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t p = __shfl_up_sync(~0u, inc, d);
            if (lane >= d) inc += p;
        }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        int64_t at = inc - sum;
        W = 0;
        for (int w = 0; w < S::kThreads / 32; ++w) {
            if (w < warp) at += warp_sum[w];
            W += warp_sum[w];
        }
        C = min((int64_t)gridDim.x, W);
        f0 = blockIdx.x < C ? W * blockIdx.x / C : W;
        f1 = blockIdx.x < C ? W * (blockIdx.x + 1) / C : W;
        if (f0 < f1 && at <= f0 && f0 < at + sum)
            for (int i = begin; i < end; ++i) {
                const int64_t k = work(i, false);
                if (f0 < at + k) {
                    found_row = i;
                    found_rest = f0 - at;
                    break;
                }
                at += k;
            }
        __syncthreads();
    }
    Place here = {};
    if (f0 < f1) {
        here.row = found_row;
        here.r = row_of(g, here.row, false);
        here.items = here.r.items(shape);
        const int64_t each = here.r.before(shape, here.items);
        here.head = (int)(found_rest / each);
        const int64_t rest = found_rest - here.head * each;
        // the last item that begins at `rest` or before it: 32 places looked at together
        int lo = 0, hi = here.items;
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step;
            const uint32_t past = __ballot_sync(~0u, at >= hi || here.r.before(shape, at) > rest);
            const int k = past ? __ffs(past) - 1 : 32;
            hi = min(hi, lo + (k + 1) * step);
            lo += k * step;
        }
        here.item = lo;
        here.j = (int)(rest - here.r.before(shape, lo));
        settle(shape, here);
    }
    fence_after();
    const uint32_t tmem = tmem_base;

    // Registers at launch: 384 x 168.  A row's thread holds 128 scores beside its weights, the third group
    // needs few: 256 x 216 + 128 x 72 are the same sum.  With one row tile there are enough for all.
    if (warp < S::kLoadWarp) {
        if constexpr (S::kGroups == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ---- the rows of one tile, a thread each
        const int group = warp >> 2, row = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;         // this warp's quarter of the TMEM lanes
        const uint32_t s_at = tmem + group * kKeys + lanes, o_at = tmem + S::kSums + group * D + lanes;
        const float scale = g.a.scale * kLog2e;
        uint32_t step = 0;
        int item_no = 0;                           // of this group
        int32_t number = 0;                        // of the block
        int key_stage = 0, value_stage = 0;        // of the keys and values that are freed next
        auto next = [](int &at, int by, int stages) { at = (at + by) % stages; };
        bool ok = true;
        if (threadIdx.x == 0) g.cut[blockIdx.x].row = -1;
        for (int64_t f = f0; f < f1 && ok; ++number) {
            const int count = (int)min((int64_t)here.tiles - here.j, f1 - f);
            const int64_t item_at = f - here.j;
            f += count;
            const bool two = S::kGroups == 2 && here.item * shape.step + g.tokens_of_tile < here.r.count;
            const bool whole = count == here.tiles;
            if (threadIdx.x == 0 && !whole && here.j == 0)
                g.cut[blockIdx.x] = {here.row, here.head, here.item, (int)(((item_at + here.tiles) * C - 1) / W)};
            if (group == 1 && !two) {
                next(key_stage, count, S::kKeyStages);
                next(value_stage, count, S::kValueStages);
                if (f < f1) next_item(g, shape, here);
                continue;
            }
            // The last group to use a tile frees its stages: when it sees its scores, the products of the keys are
            // done, and those of the tile before's values, which were issued earlier.
            const bool frees = (group == 1) == two && (threadIdx.x & 127) == 0;
            int q_head;
            const int members = heads_of(g, here.head, &q_head);
            const int32_t token = here.item * shape.step + group * g.tokens_of_tile + row / g.rows_of_token;
            q_head += row % g.rows_of_token;
            const bool live = row < g.tokens_of_tile * g.rows_of_token && row % g.rows_of_token < members && token < here.r.count;
            const int32_t place = here.r.first + token, seen_end = here.r.dead ? 0 : place + 1, low = here.r.low(shape, place);
            {   // this thread's row of queries, swizzled as the tensor cores read it
                const T *from = static_cast<const T *>(g.a.q) + (int64_t)(here.r.start + token) * g.a.q_stride[0] + (int64_t)q_head * g.a.q_stride[1];
                const uint32_t to = q_at + group * S::kRowBytes + row * 128;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 w = live ? *reinterpret_cast<const uint4 *>(from + 8 * c) : make_uint4(0, 0, 0, 0);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (c / 8) * S::kRowHalf + (((c % 8) ^ (row & 7)) << 4)),
                                 "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                fence_before();
                bar_arrive(bar(kQueries + group));
            }
            float top = -INFINITY, total = 0.f;       // top: what the weights are relative to, times scale
            for (int j = 0; j < count; ++j, ++step) {
                ok = __all_sync(~0u, bar_wait(bar(kScores + group), step & 1, failed));
                if (!ok) break;
                fence_after();
                if (frees) {
                    bar_arrive(bar(kKeyFull + kFree + key_stage));
                    if (j > 0) bar_arrive(bar(kValueFull + kFree + value_stage));
                }
                next(key_stage, 1, S::kKeyStages);
                if (j > 0) next(value_stage, 1, S::kValueStages);
                __syncwarp();                     // lanes come from the wait one by one, loads from TMEM are the warp's
                uint32_t s[kChunks][32];
#pragma unroll
                for (int c = 0; c < kChunks; ++c) tmem_load(s[c], s_at + 32 * c);
                tmem_load_wait();
                const int32_t y0 = PromptRow::tile(shape, here.skipped, here.j + j) * kKeys;
                const int left = seen_end - y0;
                if (left < kKeys) {
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (32 * c + i >= left) s[c][i] = __float_as_uint(-INFINITY);
                }
                if (y0 < low) {
                    const int below = low - y0, kept = shape.sinks - y0;
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (32 * c + i < below && 32 * c + i >= kept) s[c][i] = __float_as_uint(-INFINITY);
                }
                float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 32; ++i)
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) most[c] = fmaxf(most[c], __uint_as_float(s[c][i]));
                const float high = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * scale - Grow<T>::kTop;
                if (j == 0) {
                    top = high;
                } else if (__any_sync(~0u, high > top + Grow<T>::kPass)) {
                    const float next = high > top + Grow<T>::kPass ? high : top;
                    const float fix = top == next ? 1.f : ex2(top - next);      // of -infinity too: another row's maximum grew
                    top = next;
                    total *= fix;
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t o[32];
                        tmem_load(o, o_at + 32 * c);
                        tmem_load_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * fix);
                        tmem_store(o_at + 32 * c, o);
                    }
                }
                const float ref = top == -INFINITY ? 0.f : top;
                float2 part[2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
                for (int h = 0; h < S::kParts; ++h) {
                    uint32_t p[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int c = 2 * h + i / 16, e = 2 * (i % 16);
                        const float2 z = fma2(__uint_as_float(s[c][e]), __uint_as_float(s[c][e + 1]), scale, -ref);
                        const float x = ex2(z.x), y = ex2(z.y);
                        add2(part[i & 1], x, y);
                        p[i] = Half<T>::pack(x, y);
                    }
                    tmem_store(s_at + 32 * h, p);
                    tmem_store_wait();
                    fence_before();
                    bar_arrive(bar((h ? kRest : kWeights) + group));      // the product starts with the first part
                }
                total += (part[0].x + part[0].y) + (part[1].x + part[1].y);
            }
            ok = ok && __all_sync(~0u, bar_wait(bar(kSumsDone + group), item_no & 1, failed));
            if (!ok) break;
            fence_after();
            ++item_no;
            if (frees) bar_arrive(bar(kValueFull + kFree + value_stage));
            next(value_stage, 1, S::kValueStages);
            const bool mended = flags[number % kFlags] == number + 1;
            const float inv = total > 0.f || total != total ? 1.f / total : 0.f;
            // an item's result, or a piece: the item's first one in the block's second place
            T *out = static_cast<T *>(g.a.out) + (int64_t)(here.r.start + token) * g.a.out_stride[0] + (int64_t)q_head * g.a.out_stride[1];
            const int64_t at = ((int64_t)(2 * blockIdx.x + (here.j == 0)) * S::kGroups + group) * kRows + row;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                __syncwarp();
                tmem_load(o, o_at + 32 * c);
                tmem_load_wait();
                if (!live) continue;
                if (mended) {
                    const Spoilt x = spoilt<D, T>(g, shape, here, here.j, here.j + count, token, q_head, 32 * c, top, scale);
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float y = __uint_as_float(o[i]);
                        if (x.plus >> i & 1) y += INFINITY;
                        if (x.minus >> i & 1) y -= INFINITY;
                        if (x.none >> i & 1) y = NAN;
                        o[i] = __float_as_uint(y);
                    }
                }
                if (whole) {
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) w[k] = Half<T>::pack(__uint_as_float(o[i + 2 * k]) * inv, __uint_as_float(o[i + 2 * k + 1]) * inv);
                        *reinterpret_cast<uint4 *>(out + 32 * c + i) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        *reinterpret_cast<uint4 *>(g.part_o + at * D + 32 * c + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                }
            }
            if (live && !whole) g.part_ml[at] = make_float2(top, total);
            if (live && whole && g.a.lse)
                g.a.lse[(int64_t)(here.r.start + token) * (g.n_kv_heads * g.group) + q_head] = total > 0.f || total != total ? (top + log2f(total)) * kLn2 : -INFINITY;
            fence_before();       // the next item's first product overwrites these sums only after its weights
            if (f < f1) next_item(g, shape, here);
        }
    } else {
        if constexpr (S::kGroups == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == S::kLoadWarp || warp == S::kLoadWarp + 1) {
            // ---- keys by one warp, values by the other: one copy for each cache block (or part of one) of a tile and 64 of its values
            const int rows = min(1 << g.shift, kKeys), pieces = kKeys / rows;      // pieces: 1 .. 16
            const uint32_t piece_bytes = rows * 128;
            // this lane's part of a tile: piece lane % pieces, and every 32 / pieces-th half
            const int piece = lane % pieces;
            constexpr int32_t kNone = INT32_MIN;
            // the block's number, if any of the item's queries sees some of its part; -1 - kNone.. are the cache's errors
            auto block_of = [&](const Place &p) {
                const int32_t y = PromptRow::tile(shape, p.skipped, p.j) * kKeys + piece * rows;
                if (p.r.dead || y >= p.r.end(shape, p.item)) return kNone;
                if (y + rows <= p.r.low(shape, p.r.first + p.item * shape.step) && y >= shape.sinks) return kNone;
                return block_at(g, p.row, y);
            };
            // A ring for each: a stage's turns are one warp's, which cannot be two turns ahead of itself.
            const bool values = warp != S::kLoadWarp;
            const int stages = values ? S::kValueStages : S::kKeyStages, full = values ? kValueFull : kKeyFull;
            const uint32_t to = ring + (values ? S::kKeyStages * S::kTileBytes : 0);
            const CUtensorMap *map = values ? &vmap : &kmap;
            int64_t load = 0;
            int stage = 0;
            uint32_t turn = 0;
            bool ok = true;
            int32_t coming = f0 < f1 ? block_of(here) : kNone;             // asked for one tile ahead
            for (int64_t f = f0; f < f1 && ok; ++f) {
                int32_t block = coming;
                const int head = here.head / g.parts;
                const int slot = (PromptRow::tile(shape, here.skipped, here.j) * kKeys + piece * rows) & ((1 << g.shift) - 1);
                if (f + 1 < f1) {
                    if (++here.j == here.tiles) next_item(g, shape, here);
                    coming = block_of(here);
                }
                if ((uint32_t)block >= (uint32_t)g.n_blocks) {             // not seen, or beyond the cache: zeros
                    if (block != kNone) report(g.status);
                    block = g.n_blocks;
                }
                ok = __all_sync(~0u, load < stages || bar_wait(bar(full + kFree + stage), turn ^ 1, failed));
                if (!ok) break;
                if (lane == 0) bar_expect(bar(full + stage), S::kTileBytes);
                __syncwarp();
                for (int half = lane / pieces; half < S::kHalves; half += 32 / pieces)
                    tma_load(to + stage * S::kTileBytes + half * S::kKeyHalf + piece * piece_bytes, map, bar(full + stage), slot, half, head, block);
                ++load;
                if (++stage == stages) { stage = 0; turn ^= 1; }
            }
            // nothing is left in flight, also after a failure
            for (int64_t i = max((int64_t)0, load - stages); i < load; ++i) bar_wait(bar(full + (int)(i % stages)), (uint32_t)(i / stages) & 1, nullptr);
        } else if (warp == S::kCleanWarp) {
            // ---- values that some query of the item does not see
            bool ok = true;
            int stage = 0;
            uint32_t turn = 0;
            int32_t number = 0;
            for (int64_t f = f0; f < f1 && ok; ++f) {
                ok = __all_sync(~0u, bar_wait(bar(kValueFull + stage), turn, failed));
                if (!ok) break;
                const int32_t y0 = PromptRow::tile(shape, here.skipped, here.j) * kKeys, end = here.r.end(shape, here.item);
                const Edge edge(shape, here);
                if (edge.any(shape, y0)) {
                    const uint32_t tile = ring + (S::kKeyStages + stage) * S::kTileBytes;
                    bool found = false;
                    for (int i = lane; i < S::kTileBytes / 16; i += 32) {
                        const int32_t y = y0 + i / 8 % kKeys;
                        if (!edge.in(shape, y)) continue;
                        uint32_t w[4];
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(tile + 16 * i) : "memory");
                        const bool beyond = y >= end;
                        uint32_t bad = 0;
#pragma unroll
                        for (int k = 0; k < 4; ++k) bad |= not_finite<T>(w[k]);
                        if (!beyond && !bad) continue;
                        found = found || !beyond;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t n = not_finite<T>(w[k]);                // bits 15 and 31
                            w[k] = beyond ? 0u : w[k] & ~((n >> 15) * 0xffffu);
                        }
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(tile + 16 * i), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                    }
                    if (found) flags[number % kFlags] = number + 1;
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                __syncwarp();
                if (lane == 0) bar_arrive(bar(kClean + stage));
                if (++stage == S::kValueStages) { stage = 0; turn ^= 1; }
                if (f + 1 < f1 && ++here.j == here.tiles) {
                    next_item(g, shape, here);
                    ++number;
                }
            }
        } else if (warp == S::kIssueWarp) {
            // The whole warp runs this loop, so that addresses stay uniform, and one thread of it issues: with the
            // products of 64 cycles each, their issue has to take less.
            const bool one = elect_one();
            uint32_t step[2] = {0, 0}, begun[2] = {0, 0};       // weights taken, items begun so far of each row tile
            bool ok = tmem_base == 0;                            // all columns are ours: they begin at 0
            // operands differ in their address field alone: low word plus 16-byte steps
            const uint32_t q_lo = (uint32_t)operand(q_at, 16, 1024), k_lo = (uint32_t)operand(ring, 16, 1024);
            const uint32_t v_lo = (uint32_t)operand(ring + S::kKeyStages * S::kTileBytes, S::kKeyHalf, 1024);
            constexpr uint32_t high = (1024 >> 4) | (1u << 14) | (2u << 29);
            auto scores = [&](int i, int stage) {
                const uint32_t a = q_lo + i * (S::kRowBytes >> 4), b = k_lo + stage * (S::kTileBytes >> 4);
                if (one) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t in = (k % 4) * 32;
                        mma_smem(i * kKeys, a + (((k / 4) * S::kRowHalf + in) >> 4), b + (((k / 4) * S::kKeyHalf + in) >> 4), high, kFirst, k > 0);
                    }
                    commit(bar(kScores + i));
                }
            };
            auto sums = [&](int i, int stage, int part, bool add) {
                const uint32_t b = v_lo + stage * (S::kTileBytes >> 4), a = i * kKeys, d = S::kSums + i * D;
                constexpr int kSteps = 4;                        // of 16 tokens
                if (one) {
#pragma unroll
                    for (int k = 0; k < kSteps; ++k)
                        mma_tmem(d, a + (part * kSteps + k) * 8, b + (part * kSteps + k) * (2048 >> 4), high, kSecond, add || part + k > 0);
                }
            };
            auto wait = [&](int b, uint32_t phase) { ok = ok && __all_sync(~0u, bar_wait(bar(b), phase, failed)); };
            int k_at = 0, v_at = 0;                              // stages of the tile's keys and values, and their turns
            uint32_t k_turn = 0, v_turn = 0;
            auto next = [](int &at, uint32_t &turn, int stages) {
                if (++at == stages) { at = 0; turn ^= 1; }
            };
            for (int64_t f = f0; f < f1 && ok;) {
                const int count = (int)min((int64_t)here.tiles - here.j, f1 - f);
                const int groups = S::kGroups == 2 && here.item * shape.step + g.tokens_of_tile < here.r.count ? 2 : 1;
                wait(kKeyFull + k_at, k_turn);
                for (int i = 0; i < groups && ok; ++i) {
                    wait(kQueries + i, begun[i]++ & 1);
                    if (!ok) break;
                    fence_after();
                    scores(i, k_at);
                }
                if (!ok) break;
                next(k_at, k_turn, S::kKeyStages);
                for (int j = 0; j < count && ok; ++j) {
                    const bool more = j + 1 < count;
#pragma unroll
                    for (int i = 0; i < S::kGroups; ++i) {
                        if (i >= groups) break;
                        // one wait for weights and (before the first row tile's) copies: a lane for each barrier
                        const int what = i == 0 ? lane : 0;
                        wait(what == 1 ? kValueFull + v_at : what == 2 ? kClean + v_at : kWeights + i, what == 1 || what == 2 ? v_turn : step[i] & 1);
                        if (!ok) break;
                        fence_after();
                        sums(i, v_at, 0, j > 0);
                        const bool keys = i == 0 && more && (lane == 1 || S::kParts == 1);
                        if (S::kParts > 1 || keys) wait(keys ? kKeyFull + k_at : kRest + i, keys ? k_turn : step[i] & 1);
                        ++step[i];
                        if (!ok) break;
                        fence_after();
                        if (S::kParts > 1) sums(i, v_at, 1, true);
                        if (more) scores(i, k_at);
                        else if (one) commit(bar(kSumsDone + i));
                    }
                    next(v_at, v_turn, S::kValueStages);
                    if (more) next(k_at, k_turn, S::kKeyStages);
                }
                f += count;
                if (f < f1) next_item(g, shape, here);
            }
            if (!ok) {
                // products under way still read shared memory and write TMEM
                *failed = 1;
                if (one) commit(bar(kDrain));
                __syncwarp();
                bar_wait(bar(kDrain), 0);
            }
            __syncwarp();
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && *failed) atomicOr(g.status, 2);
    if (warp == S::kIssueWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// Joins the pieces of the items that runs' ends cut: some blocks for the block in whose run one begins.
template <int D, typename T>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ PromptArgs g) {
    using S = Shape<D>;
    wait_for_previous();
    const PromptCut item = g.cut[blockIdx.x];
    if (item.row < 0) return;
    const PromptShape shape = {S::kKeys, S::kGroups * g.tokens_of_tile, g.a.window, g.a.sinks};
    const Row r = row_of(g, item.row, false);
    int first_head;
    const int members = heads_of(g, item.head, &first_head), hq = g.n_kv_heads * g.group;
    constexpr int kSlice = S::kGroups * kRows / kJoinSlices;
    for (int x = threadIdx.x; x < kSlice * (D / 4); x += kJoinThreads) {
        const int at = blockIdx.y * kSlice + x / (D / 4), row = at % kRows, d = (x % (D / 4)) * 4;
        const int32_t token = item.item * shape.step + at / kRows * g.tokens_of_tile + row / g.rows_of_token;
        const int member = row % g.rows_of_token;
        if (row >= g.tokens_of_tile * g.rows_of_token || member >= members || token >= r.count) continue;
        float top = -INFINITY, total = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int kBatch = 4;                         // their loads are under way together
        for (int b0 = blockIdx.x; b0 <= item.last; b0 += kBatch) {
            float2 ml[kBatch];
            float4 v[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int b = min(b0 + k, item.last);
                const int64_t from = (int64_t)(2 * b + (b == (int)blockIdx.x)) * (S::kGroups * kRows) + at;
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
        const float inv = total > 0.f || total != total ? 1.f / total : 0.f;
        const int64_t query = r.start + token;
        *reinterpret_cast<uint2 *>(static_cast<T *>(g.a.out) + query * g.a.out_stride[0] + (first_head + member) * g.a.out_stride[1] + d) =
            make_uint2(Half<T>::pack(sum.x * inv, sum.y * inv), Half<T>::pack(sum.z * inv, sum.w * inv));
        if (d == 0 && g.a.lse)
            g.a.lse[query * hq + first_head + member] = total > 0.f || total != total ? (top + log2f(total)) * kLn2 : -INFINITY;
    }
}

template <int D, typename T>
cudaError_t launch_of(const PromptArgs &g, const CUtensorMap &k, const CUtensorMap &v, int sms, cudaStream_t st) {
    using S = Shape<D>;
    const cudaError_t e = launch_kernel(prompt_kernel<D, T>, dim3(sms), S::kThreads, S::kSmem, st, false, g, k, v);
    if (e != cudaSuccess) return e;
    return launch_kernel(join_kernel<D, T>, dim3(sms, kJoinSlices), kJoinThreads, 0, st, true, g);
}

template <int D, typename T>
cudaError_t prepare_of() {
    return cudaFuncSetAttribute(prompt_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D>::kSmem);
}

}  // namespace

cudaError_t prepare_prompt(int head_dim, int type) {
    if (type == ISJL_KV_BF16)
        return head_dim == 64 ? prepare_of<64, __nv_bfloat16>() : head_dim == 128 ? prepare_of<128, __nv_bfloat16>() : prepare_of<256, __nv_bfloat16>();
    return head_dim == 64 ? prepare_of<64, __half>() : head_dim == 128 ? prepare_of<128, __half>() : prepare_of<256, __half>();
}

cudaError_t launch_prompt(PromptArgs &g, void *encoder, int head_dim, int type, int sms, cudaStream_t st) {
    CUtensorMap k, v;
    g.rows_of_token = g.group < kRows ? g.group : kRows;
    g.parts = (g.group + g.rows_of_token - 1) / g.rows_of_token;
    g.tokens_of_tile = kRows / g.rows_of_token;
    const int keys = head_dim == 256 ? 64 : 128, rows = 1 << g.shift < keys ? 1 << g.shift : keys;
    if (!encode_cache(encoder, &k, g.cache.k, g.cache.k_stride, rows, 1, g.n_blocks, g.shift, g.n_kv_heads, head_dim, type) ||
        !encode_cache(encoder, &v, g.cache.v, g.cache.v_stride, rows, 1, g.n_blocks, g.shift, g.n_kv_heads, head_dim, type))
        return cudaErrorInvalidValue;
    if (type == ISJL_KV_BF16)
        return head_dim == 64 ? launch_of<64, __nv_bfloat16>(g, k, v, sms, st)
             : head_dim == 128 ? launch_of<128, __nv_bfloat16>(g, k, v, sms, st) : launch_of<256, __nv_bfloat16>(g, k, v, sms, st);
    return head_dim == 64 ? launch_of<64, __half>(g, k, v, sms, st)
         : head_dim == 128 ? launch_of<128, __half>(g, k, v, sms, st) : launch_of<256, __half>(g, k, v, sms, st);
}

}  // namespace isjl
