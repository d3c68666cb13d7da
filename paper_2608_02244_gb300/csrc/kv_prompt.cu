// kv_prompt.cu -- causal attention of packed prompts over the paged cache (isjl_kv_prompt).
//
// The queries of a row's tokens, times the `group` query heads of a key head, are the rows of a matrix: S = Q K^T,
// O = softmax(S) V, 4 D operations for each row and visible token, on the fifth-generation tensor cores.  An item is
// two tiles of 128 rows of one key head: a run of neighbouring tokens, each with all of its query heads, so that a
// tile of keys and values is used by all of them.  An item's tiles of 128 tokens end with the tokens that its last
// query sees.
//
// Keys and values come by TMA from the cache's blocks through a ring each, one thread issues the products, and each
// row of a tile is one thread of a group of four warps that takes the row's maximum, exponentials and sum.  Scores
// lie in TMEM, their weights take the scores' place as the second product's left operand, and the two row tiles
// alternate: while the tensor cores work for one, the other's group is at its exponentials.  The sums O stay in TMEM
// for the whole run and are rescaled only when a row's maximum has grown by more than 2^8 (fp16: 2^4) since the last
// time.  The weights are rounded to 16 bits for the second product, as its instruction takes them, which is as exact as with
// the true maximum; their sum is of the unrounded ones, and scores, maxima, sums and pieces have 32 bits.
//
// Heads of 256 values: one row tile, whose sums take half of TMEM, and tiles of 64 tokens, since 128 rows of queries and
// five tiles of keys and values fill shared memory.  Its scores have two places in turn, and the next ones are issued
// before the weights of these are there, so that the tensor cores have work during the exponentials.
//
// What a query does not see must not reach its sums, and a weight of 0 does not silence an infinite or undefined
// value.  In the tiles of which some of the item's queries see a part only, one warp makes zeros of the values that no
// query sees and of those that are not finite; where it found one of the latter, the rows that see it get it at the
// end, from the cache.  That is slow: one prompt of 16,384 tokens (32 + 8 heads of 128 values) whose values are all undefined
// takes 148 ms.
//
// The work is a line of (row, key head, item, tile): every block has an equal run of it, wherever prompts end, and one
// long prompt, many short ones or a few queries over a long cache all keep every SM busy to the end.  What an item takes
// beside its tiles counts as some tiles more.  Items cut by the
// runs' ends leave pieces (sum, maximum and total of each row), which a second kernel joins in their order.
//
// Measured, 32 + 8 heads of 128 values, bf16: 16,384 tokens 1,205 to 1,225 us (1,800 TFLOP/s; power-limited when it runs
// for long: 1,360 us), 8 requests of 4,096 737 us (1,490), 32 of 1,024 306 us (900), 64 of 256 115 us; 64 values, 16,384 tokens
// 1,047 us (1,050: 128 exponentials a row and tile take the SM 2,048 cycles, the products 1,024); 256 values, 16 + 4 heads,
// 16,384 tokens 1,500 to 1,590 us (1,400; products a warp at a time, 64 rows an item, took 11,700).  Short prompts are bound
// by what an item takes beside its tiles: 4,000 cycles for its results (TMEM loads and stores, during which its rows'
// threads do nothing else), 2,000 until the next item's first weights, 1,200 for the masks of its last tile.
#include "kv_prompt.cuh"
#include "kv_tensor.cuh"

namespace isjl {
namespace {

constexpr int kRows = 128;                          // of a row tile
constexpr int kItems = 8, kAhead = 6;               // planned items kept at a time; planned ahead of the values that are cleaned

template <int D>
struct Shape {
    static constexpr int kGroups = D == 256 ? 1 : 2;             // row tiles of an item, each with its four warps
    static constexpr int kKeys = D == 256 ? 64 : 128;            // of a token tile
    static constexpr int kParts = kKeys / 64;                    // of a tile's weights, handed over one after another
    // An item's first scores, its results and the masks of its last tile, in tiles, which the runs count with them.  With 0, 2,
    // 3 and 4 of them one prompt of 16,384 tokens (128 values) took 1,344, 1,223, 1,226 and 1,232 us, 37 ragged ones (64 values)
    // 172, 135, 145 and 148; with 256 values, 0, 2, 4 and 6: 1,668, 1,555, 1,501 and 1,498 us and, ragged, 161, 122, 111 and 115.
    static constexpr int kExtra = D == 256 ? 4 : 2;
    static constexpr int kLoadWarp = 4 * kGroups, kIssueWarp = kLoadWarp + 2, kPlanWarp = kLoadWarp + 3;     // plans and cleans
    static constexpr int kThreads = 128 * kGroups + 128;
    static constexpr int kSums = 256;                            // TMEM: scores from 0, sums from here
    static constexpr int kHalves = D / 64;                       // rows of 128 bytes hold 64 values
    static constexpr int kQueryHalf = kRows * 128, kQueryBytes = kHalves * kQueryHalf;
    static constexpr int kHalfBytes = kKeys * 128, kTileBytes = kHalves * kHalfBytes;
    static constexpr int kKeyStages = D == 64 ? 4 : 2, kValueStages = D == 64 ? 4 : 3;
    static constexpr int kSmem = kGroups * kQueryBytes + (kKeyStages + kValueStages) * kTileBytes + 1024;
};

__device__ __forceinline__ void store32(void *to, uint4 a, uint4 b) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(to), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}

// What the issuing warp waits for in every tile comes by the block's numbered barriers, which do not lie in shared memory:
// a look at one that does takes some 400 cycles beside products that read shared memory at its full rate.  Weights: one
// barrier for each row tile and part.  Copies that have come and are clean: one of eight, tile after tile, so that two
// more arrivals than the issuing warp has seen are none too many for one.
//
// These waits have no limit, so that they end is up to who arrives.
// Copies: the planning warp, whose waits have one; when it gives up it arrives for this tile and the next.  The issuing
// warp, let go, meets the word that says so before it issues the scores after those, and ends.
// Weights: a row tile's group arrives whenever its scores come, and scores that were issued do come.  It gives up a
// wait for scores only some time after that word was written, when none can be issued any more.
enum { kHandOver = 1 /* + part + 2 row tile */, kCopies = 5 /* + tile % 8 */ };
constexpr int kHandOverThreads = 128 + 32, kCopiesThreads = 64;
constexpr uint64_t kGrace = 50000000ull;        // nanoseconds
template <int kThreads>
__device__ __forceinline__ void numbered_arrive(int id) {
    asm volatile("barrier.cta.arrive %0, %1;" ::"r"(id), "n"(kThreads) : "memory");
}
template <int kThreads>
__device__ __forceinline__ void numbered_sync(int id) {
    asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "n"(kThreads) : "memory");
}

// barriers, in 8-byte words
enum { kKeyFull = 0, kValueFull = 8, kFree = 4 /* after a stage's full one */, kScores = 16, kSumsDone = 18, kQueries = 20, kDrain = 22,
       kItemFull = 23, kItemFree = kItemFull + kItems, kBars = kItemFree + kItems };

template <int D, typename T>
__global__ void __launch_bounds__(Shape<D>::kThreads, 1)
prompt_kernel(const __grid_constant__ PromptArgs g, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
              const __grid_constant__ CUtensorMap vmap) {
    using S = Shape<D>;
    constexpr bool kBf16 = Half<T>::kIsBf16;
    constexpr int kGroups = S::kGroups, kKeys = S::kKeys, kParts = S::kParts, kSums = S::kSums, kThreads = S::kThreads;
    constexpr int kLoadWarp = S::kLoadWarp, kIssueWarp = S::kIssueWarp, kPlanWarp = S::kPlanWarp, kChunks = kKeys / 32;
    constexpr bool kTwo = kGroups == 2;
    // operand types, 32-bit sums, 128 rows; the first product has a column for each token and both operands along D, the
    // second D columns and its right operand (values, tokens outermost) across
    constexpr uint32_t kTypes = (1u << 4) | (kBf16 ? (1u << 7) | (1u << 10) : 0u) | ((kRows / 16) << 24);
    constexpr uint32_t kFirstWhat = kTypes | ((kKeys / 8) << 17), kSecondWhat = kTypes | ((D / 8) << 17) | (1u << 16);
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ Item items[kItems];
    __shared__ RunWords words;
    __shared__ uint32_t tmem_base;
    __shared__ int32_t failed_word;
    __shared__ int32_t flag_word[kItems];           // an item's number in the block, plus one, if a value of it was left out
    volatile int32_t *flags = flag_word;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
    const uint32_t q_at = base, ring = base + kGroups * S::kQueryBytes;
    const uint32_t bar0 = smem_addr(bars);
    auto bar = [&](int i) { return bar0 + 8 * i; };
    const PromptShape shape = {kKeys, kGroups * g.tokens_of_tile, g.a.window, g.a.sinks, S::kExtra};

    start_next();
    if (threadIdx.x == 0) {
        tma_prefetch(&qmap);
        tma_prefetch(&kmap);
        tma_prefetch(&vmap);
        failed_word = 0;
        for (int i = 0; i < kItems; ++i) {
            flag_word[i] = 0;
            bar_init(bar(kItemFull + i), 1);
            bar_init(bar(kItemFree + i), kPlanWarp);        // the warps that read it
        }
        for (int i = 0; i < kScores; ++i) bar_init(bar(i), 1);
        for (int i = 0; i < 2; ++i) {
            bar_init(bar(kScores + i), 1);
            bar_init(bar(kSumsDone + i), 1);
            bar_init(bar(kQueries + i), 1);
        }
        bar_init(bar(kDrain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssueWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }

    Run run = find_run<kThreads>(g, shape, words);
    fence_after();
    const uint32_t tmem = tmem_base;
    // A wait: false if it, or another, gave up.  The clock, which takes a few hundred cycles to read, is looked at once in
    // a while only.
    const uint32_t failed_at = smem_addr(&failed_word);
    auto look_failed = [&]() {
        uint32_t w;
        asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(w) : "r"(failed_at) : "memory");
        return w;
    };
    auto wait_lane = [&](int b, uint32_t phase) {
        uint64_t begin = 0, told = 0;
        for (;;) {
#pragma unroll 1
            for (int i = 0; i < 16; ++i)
                if (bar_try(bar(b), phase)) return true;
            const uint64_t t = now();
            if (begin == 0) begin = t;
            if (t - begin > kLimit) asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(failed_at), "r"(1) : "memory");
            if (look_failed()) {
                if (told == 0) told = t;
                if (warp >= kLoadWarp || t - told > kGrace) return false;
            }
        }
    };
    // of a warp: its threads look together, which costs less than one's look that the others wait for
    auto wait = [&](int b, uint32_t phase) {
        const bool done = __all_sync(~0u, wait_lane(b, phase));
        __syncwarp();
        return done;
    };
    // item `n` of this block's run, when it has been planned
    auto item_of = [&](int n) -> const Item & { return items[n % kItems]; };
    auto wait_item = [&](int n) { return wait(kItemFull + n % kItems, (uint32_t)(n / kItems) & 1); };
    auto done_item = [&](int n) {
        __syncwarp();
        if (lane == 0) bar_arrive(bar(kItemFree + n % kItems));
    };

    // Registers at launch: 384 x 168.  A row's thread holds 128 scores beside its weights, the third group
    // needs few: 256 x 216 + 128 x 72 are the same sum.
    if (warp < kLoadWarp) {
        if (kTwo) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ---- the rows of one tile, a thread each
        const int group = warp >> 2, row = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;         // this warp's quarter of the TMEM lanes
        const uint32_t s_first = tmem + group * kKeys + lanes, o_at = tmem + kSums + group * D + lanes;
        const float scale = g.a.scale * kLog2e;
        const int token = group * g.tokens_of_tile + row / g.rows_of_token, member = row % g.rows_of_token;
        auto two_of = [&](const Item &x) { return x.tokens > g.tokens_of_tile; };
        auto live_of = [&](const Item &x) { return row / g.rows_of_token < g.tokens_of_tile && member < x.members && token < x.tokens; };
        // An item's queries of this row tile: tokens, each with its query heads, are rows one after another.  Rows behind the
        // item's tokens hold other queries or anything: their results are nobody's.  The products with the queries before
        // are done when this group has seen their scores.
        auto load_queries = [&](const Item &x) {
            if ((threadIdx.x & 127) == 0) {
                bar_expect(bar(kQueries + group), S::kHalves * g.tokens_of_tile * g.rows_of_token * 128);
#pragma unroll
                for (int half = 0; half < S::kHalves; ++half)
                    tma_load4(q_at + group * S::kQueryBytes + half * S::kQueryHalf, &qmap, bar(kQueries + group), half, x.q_head,
                              x.start + group * g.tokens_of_tile);
            }
            __syncwarp();
        };
        uint32_t step = 0;
        int item_no = 0;                           // of this group
        // One row tile: a tile's sums, on the barrier that its number in the run says.  Only the last tile's and the one
        // before it are asked for: what the barrier had two tiles earlier was done when the last tile's scores came, and
        // what it has two tiles later waits for weights that are not made yet, so its turn is the one that is meant.
        auto sums_done = [&](uint32_t t) { return wait(kSumsDone + (t & 1), t >> 1 & 1); };
        int key_stage = 0, value_stage = 0;        // of the keys and values that are freed next
        auto next = [](int &at, int by, int stages) { at = (at + by) % stages; };
        bool ok = wait_item(0), loaded = false;
        for (int n = 0; ok && item_of(n).count > 0; ++n) {
            float top = -INFINITY, total = 0.f;       // top: what the weights are relative to, times scale
            {
                const Item &x = item_of(n);
                if (group == 1 && !two_of(x)) {
                    next(key_stage, x.count, S::kKeyStages);
                    next(value_stage, x.count, S::kValueStages);
                    done_item(n);
                    ok = wait_item(n + 1);
                    continue;
                }
                if (!loaded) load_queries(x);
                const int count = x.count, tile0 = x.tile0, skipped = x.skipped;
                // The last group to use a tile frees its stages: when it sees its scores, the products of the keys are
                // done, and those of the values that were issued earlier: of the tile before, or with one row tile of the
                // one before that.
                constexpr int kBehind = kTwo ? 1 : 2;
                bool lost = false;
                const bool frees = (group == 1) == two_of(x) && (threadIdx.x & 127) == 0;
                const int32_t seen_end = x.kind & kDead ? 0 : x.place + token + 1, low = PromptRow::low(shape, x.place + token);
                for (int j = 0; j < count; ++j, ++step) {
                    ok = kTwo ? wait(kScores + group, step & 1) : wait(kScores + (step & 1), step >> 1 & 1);
                    if (!ok) break;
                    fence_after();
                    if (frees) {
                        bar_arrive(bar(kKeyFull + kFree + key_stage));
                        if (j >= kBehind) bar_arrive(bar(kValueFull + kFree + value_stage));
                    }
                    next(key_stage, 1, S::kKeyStages);
                    if (j >= kBehind) next(value_stage, 1, S::kValueStages);
                    const uint32_t s_at = kTwo ? s_first : s_first + (step & 1) * kKeys;
                    __syncwarp();                     // lanes come from the wait one by one, loads from TMEM are the warp's
                    uint32_t s[kChunks][32];
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) tmem_load(s[c], s_at + 32 * c);
                    tmem_load_wait();
                    const int32_t y0 = PromptRow::tile(shape, skipped, tile0 + j) * kKeys;
                    const int left = seen_end - y0;
                    // rows end at different tokens: the whole warp takes a branch that a row of it needs, since what
                    // follows (loads and stores of TMEM) is the warp's
                    if (__any_sync(~0u, left < kKeys)) {
#pragma unroll
                        for (int c = 0; c < kChunks; ++c)
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (32 * c + i >= left) s[c][i] = __float_as_uint(-INFINITY);
                    }
                    if (__any_sync(~0u, y0 < low)) {
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
                        // with one row tile these scores were issued before the last sums
                        if (!kTwo) {
                            lost = !sums_done(step - 1);
                            fence_after();
                        }
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t o[32];
                            __syncwarp();
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
                    for (int h = 0; h < kParts; ++h) {
                        uint32_t p[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const int c = 2 * h + i / 16, e = 2 * (i % 16);
                            const float2 z = fma2(__uint_as_float(s[c][e]), __uint_as_float(s[c][e + 1]), scale, -ref);
                            const float u = ex2(z.x), v = ex2(z.y);
                            add2(part[i & 1], u, v);
                            p[i] = Half<T>::pack(u, v);
                        }
                        __syncwarp();
                        tmem_store(s_at + 32 * h, p);
                        tmem_store_wait();
                        fence_before();
                        // the product starts with the first part
                        numbered_arrive<kHandOverThreads>(kTwo ? kHandOver + h + 2 * group : kHandOver + (step & 1));
                    }
                    if (lost) break;                  // not before the issuing warp is let go
                    total += (part[0].x + part[0].y) + (part[1].x + part[1].y);
                }
                ok = ok && !lost;
                if (!ok) break;
            }
            // The next item's queries come in, and their first product is done, while this one's results are written.
            ok = wait_item(n + 1);
            if (!ok) break;
            const Item &following = item_of(n + 1);
            loaded = following.count > 0 && !(group == 1 && !two_of(following));
            if (loaded) load_queries(following);
            ok = kTwo ? wait(kSumsDone + group, item_no & 1) : sums_done(step - 1);
            if (!ok) break;
            fence_after();
            ++item_no;
            const Item &x = item_of(n);
            for (int i = kTwo ? 1 : min(x.count, 2); i > 0; --i) {
                if ((group == 1) == two_of(x) && (threadIdx.x & 127) == 0) bar_arrive(bar(kValueFull + kFree + value_stage));
                next(value_stage, 1, S::kValueStages);
            }
            const bool left_out = flags[n % kItems] == n + 1, live = live_of(x), whole = x.kind & kWhole;
            const float inv = inverse(total);
            // an item's result, or a piece: the item's first one in the block's second place
            const int64_t query = x.start + token, at = ((int64_t)(2 * blockIdx.x + ((x.kind & kFirst) != 0)) * kGroups + group) * kRows + row;
            const int q_head = x.q_head + member;
            T *out = static_cast<T *>(g.a.out) + query * g.a.out_stride[0] + q_head * g.a.out_stride[1];
            // what was left out, all of it before any result is written: weights are computed from q, which out may be
            if (left_out) {
#pragma unroll 1
                for (int c = 0; c < D / kSpoilt; ++c) {
                    uint32_t o[kSpoilt];
                    __syncwarp();
                    tmem_load(o, o_at + kSpoilt * c);
                    tmem_load_wait();
                    if (live) {
                        const Spoilt y = spoilt<D, T>(g, shape, x, token, q_head, kSpoilt * c, top, scale);
#pragma unroll
                        for (int i = 0; i < kSpoilt; ++i) {
                            float z = __uint_as_float(o[i]);
                            if (y.plus >> i & 1) z += INFINITY;
                            if (y.minus >> i & 1) z -= INFINITY;
                            if (y.none >> i & 1) z = NAN;
                            o[i] = __float_as_uint(z);
                        }
                    }
                    __syncwarp();
                    tmem_store(o_at + kSpoilt * c, o);
                }
                tmem_store_wait();
            }
            // Few columns at a time: with 32, 2 to 3% slower in short items, with all under way together 5%, since this code
            // is fetched anew for each item.
#pragma unroll 1
            for (int c = 0; c < D / kColumns; ++c) {
                uint32_t o[kColumns];
                __syncwarp();
                tmem_load(o, o_at + kColumns * c);
                tmem_load_wait();
                if (live && whole) {
                    uint4 w[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t u[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) u[k] = Half<T>::pack(__uint_as_float(o[8 * i + 2 * k]) * inv, __uint_as_float(o[8 * i + 2 * k + 1]) * inv);
                        w[i] = make_uint4(u[0], u[1], u[2], u[3]);
                    }
                    if (g.out_wide) {
                        store32(out + kColumns * c, w[0], w[1]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i) *reinterpret_cast<uint4 *>(out + kColumns * c + 8 * i) = w[i];
                    }
                } else if (live) {
#pragma unroll
                    for (int i = 0; i < kColumns; i += 8)
                        store32(g.part_o + at * D + kColumns * c + i, make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]), make_uint4(o[i + 4], o[i + 5], o[i + 6], o[i + 7]));
                }
            }
            if (live && !whole) g.part_ml[at] = make_float2(top, total);
            if (live && whole && g.a.lse)
                g.a.lse[query * (g.n_kv_heads * g.group) + q_head] = log_of(top, total);
            fence_before();       // the next item's first weights, after which its products overwrite these sums, come later
            done_item(n);
        }
    } else {
        if (kTwo) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == kLoadWarp || warp == kLoadWarp + 1) {
            // ---- keys by one warp, values by the other: one copy for each cache block (or part of one) of a tile and 64 of
            // its values.  The lanes look up the blocks and one thread issues.
            const int rows = min(1 << g.shift, kKeys), pieces = kKeys / rows;      // pieces: 1 .. 16
            const int piece = lane % pieces;                         // whose block this lane looks up
            const bool one = elect_one();
            // A ring for each: a stage's turns are one warp's, which cannot be two turns ahead of itself.
            const bool values = warp != kLoadWarp;
            const int stages = values ? S::kValueStages : S::kKeyStages, full = values ? kValueFull : kKeyFull;
            const uint32_t to = ring + (values ? S::kKeyStages * S::kTileBytes : 0);
            const CUtensorMap *map = values ? &vmap : &kmap;
            int stage = 0, load = 0, n = 0, j = 0;                   // load: fills so far, counted up to `stages`
            uint32_t turn = 0;
            bool ok = wait_item(0);
            Item x = item_of(0);
            int32_t block = 0, y0 = 0;                               // of the tile that is next
            bool seen = false;
            // the block's number, if any of the item's queries sees some of this part; asked for one tile ahead
            auto look = [&]() {
                y0 = tile_at(shape, x, j);
                const int32_t y = y0 + piece * rows;
                seen = !(x.kind & kDead) && y < x.end && (y + rows > x.low || y < shape.sinks);
                block = seen ? block_at(g, x.row, y) : 0;
            };
            if (ok && x.count > 0) look();
            while (ok && x.count > 0) {
                int32_t from = block;
                const bool real = seen;
                const int kv = x.kv, slot = y0 & ((1 << g.shift) - 1);             // slot: 0 but in blocks larger than a tile
                if (++j == x.count) {
                    done_item(n);
                    ok = wait_item(++n);
                    x = item_of(n);
                    j = 0;
                }
                if (ok && x.count > 0) look();
                if (load == stages) ok = wait(full + kFree + stage, turn ^ 1) && ok;
                if (!ok) break;
                if (!real || (uint32_t)from >= (uint32_t)g.n_blocks) {    // not seen, or beyond the cache: zeros
                    if (real) report(g.status);
                    from = g.n_blocks;
                }
                if (one) bar_expect(bar(full + stage), S::kTileBytes);
                for (int p = 0; p < pieces; ++p) {
                    const int32_t b = __shfl_sync(~0u, from, p);
                    if (one)
#pragma unroll
                        for (int half = 0; half < S::kHalves; ++half)
                            tma_load(to + stage * S::kTileBytes + half * S::kHalfBytes + p * rows * 128, map, bar(full + stage), slot, half, kv, b);
                    __syncwarp();
                }
                if (load < stages) ++load;
                if (++stage == stages) { stage = 0; turn ^= 1; }
            }
            // nothing is left in flight, also after a failure: the last fill of each stage
            for (int i = 0; i < load; ++i) {
                const int s = (stage - 1 - i + 2 * stages) % stages;
                bar_wait(bar(full + s), s < stage ? turn : turn ^ 1, nullptr);
            }
        } else if (warp == kPlanWarp) {
            // ---- the run's items, and values that some query of an item does not see
            begin_run(g, shape, words, run);
            if (lane == 0) g.cut[blockIdx.x].row = -1;
            int planned = 0;
            bool ok = true, ended = false;
            auto plan = [&]() {
                if (ended) return;
                const int at = planned % kItems;
                ok = planned < kItems || wait(kItemFree + at, (uint32_t)(planned / kItems - 1) & 1);
                if (!ok) return;
                const Item x = take_item(g, shape, run, lane == 0);
                ended = x.count == 0;
                __syncwarp();
                if (lane == 0) {
                    items[at] = x;
                    bar_arrive(bar(kItemFull + at));
                }
                __syncwarp();
                ++planned;
            };
            for (int i = 0; i < kAhead && ok; ++i) plan();
            int stage = 0;
            // The tile, of the run, whose keys are waited for; with them the values of the one before are handed over.  All are
            // waited for here, one after another, and given back only after that: no turn of a barrier is taken for another.
            uint32_t turn = 0, tile = 0, handed = 0;
            if (ok && item_of(0).count > 0) {
                ok = wait(kKeyFull, 0);
                if (ok) numbered_arrive<kCopiesThreads>(kCopies + handed++);
            }
            for (int n = 0; ok && item_of(n).count > 0; ++n) {
                plan();
                const Item &x = item_of(n);
                const int count = x.count, end = x.end;
                for (int j = 0; j < count && ok; ++j) {
                    ok = wait(kValueFull + stage, turn);
                    if (!ok) break;
                    const int32_t y0 = tile_at(shape, x, j);
                    if (edge(shape, x, y0)) {
                        const uint32_t tile = ring + (S::kKeyStages + stage) * S::kTileBytes;
                        // 16 bytes in a row's half: rows r0 + lane / 8, + 4, ...; eight of them are under way together
                        auto scan = [&](int r0, int r1) {
                            uint32_t sum[2] = {0, 0};                                  // 0 times a value is 0 if that is finite
                            for (int half = 0; half < S::kHalves; ++half)
                                for (int r = r0 + lane / 8; r < r1; r += 32) {
                                    uint32_t w[8][4];
#pragma unroll
                                    for (int u = 0; u < 8; ++u)                        // the last row more than once
                                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[u][0]), "=r"(w[u][1]), "=r"(w[u][2]), "=r"(w[u][3])
                                                     : "r"(tile + half * S::kHalfBytes + min(r + 4 * u, r1 - 1) * 128 + (lane % 8) * 16) : "memory");
#pragma unroll
                                    for (int u = 0; u < 8; ++u)
#pragma unroll
                                        for (int k = 0; k < 4; ++k) sum[k & 1] = fma2x16<T>(w[u][k], 0, sum[k & 1]);
                                }
                            return __any_sync(~0u, ((sum[0] | sum[1]) & 0x7fff7fffu) != 0);      // -0 may come of it too
                        };
                        auto mend = [&](int r0, int r1) {
                            for (int i = lane; i < (r1 - r0) * S::kHalves * 32; i += 32) {
                                const uint32_t at = tile + i / 32 % S::kHalves * S::kHalfBytes + (r0 + i / 32 / S::kHalves) * 128 + lane * 4;
                                uint32_t w;
                                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
                                w &= ~((not_finite<T>(w) >> 15) * 0xffffu);            // not_finite: bits 15 and 31
                                asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(w) : "memory");
                            }
                        };
                        // rows that some query does not see, a row in both parts once, up to those that none sees
                        const int last = min(max(0, end - y0), kKeys), from = min(max(0, x.from - y0), last);
                        const int first = max(0, shape.sinks - y0), below = min(from, x.below - y0);
                        bool found = false;
                        if (first < below && scan(first, below)) {
                            mend(first, below);
                            found = true;
                        }
                        if (from < last && scan(from, last)) {
                            mend(from, last);
                            found = true;
                        }
                        for (int half = 0; half < S::kHalves; ++half)
                            for (int r = last + lane / 8; r < kKeys; r += 4)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};"
                                             ::"r"(tile + half * S::kHalfBytes + r * 128 + (lane % 8) * 16), "r"(0) : "memory");
                        if (found && lane == 0) flags[n % kItems] = n + 1;
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    __syncwarp();
                    // and the next tile's keys
                    ++tile;
                    if (j + 1 < count || item_of(n + 1).count > 0) ok = wait(kKeyFull + tile % S::kKeyStages, tile / S::kKeyStages & 1);
                    if (!ok) break;
                    numbered_arrive<kCopiesThreads>(kCopies + handed++ % 8);
                    if (++stage == S::kValueStages) { stage = 0; turn ^= 1; }
                }
            }
            if (!ok) {                                           // the issuing warp is let go
                __syncwarp();
                numbered_arrive<kCopiesThreads>(kCopies + handed % 8);
                numbered_arrive<kCopiesThreads>(kCopies + (handed + 1) % 8);
            }
        } else if (warp == kIssueWarp) {
            // The whole warp runs this loop, so that addresses stay uniform, and one thread of it issues: with the
            // products of 64 cycles each, their issue has to take less.  Operands of products and copies are in registers
            // that the warp shares: the others wait for that thread each time (__syncwarp), here and in the loaders.
            const bool one = elect_one();
            uint32_t begun[2] = {0, 0};                          // items begun so far of each row tile
            // operands differ in their address field alone: low word plus 16-byte steps
            const uint32_t q_lo = (uint32_t)operand(q_at, 16, 1024), k_lo = (uint32_t)operand(ring, 16, 1024);
            const uint32_t v_lo = (uint32_t)operand(ring + S::kKeyStages * S::kTileBytes, S::kHalfBytes, 1024);
            constexpr uint32_t high = (1024 >> 4) | (1u << 14) | (2u << 29);
            // of row tile i, into place `to` of two
            auto scores = [&](int i, int to, int stage) {
                const uint32_t a = q_lo + i * (S::kQueryBytes >> 4), b = k_lo + stage * (S::kTileBytes >> 4);
                if (one) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t in = (k % 4) * 32;
                        mma_smem(to * kKeys, a + (((k / 4) * S::kQueryHalf + in) >> 4), b + (((k / 4) * S::kHalfBytes + in) >> 4), high, kFirstWhat, k > 0);
                    }
                    commit(bar(kScores + to));
                }
                __syncwarp();
            };
            auto sums = [&](int i, int from, int stage, int part, bool add) {
                const uint32_t b = v_lo + stage * (S::kTileBytes >> 4), a = from * kKeys, d = kSums + i * D;
                constexpr int kSteps = 4;                        // of 16 tokens
                if (one) {
#pragma unroll
                    for (int k = 0; k < kSteps; ++k)
                        mma_tmem(d, a + (part * kSteps + k) * 8, b + (part * kSteps + k) * (2048 >> 4), high, kSecondWhat, add || part + k > 0);
                }
                __syncwarp();
            };
            int k_at = 0, v_at = 0;                              // stages of the tile's keys and values
            uint32_t taken = 0;                                  // copies handed over so far: the run's first keys, then its tiles
            uint32_t step = 0;                                   // tiles so far
            auto next = [](int &at, int stages) {
                if (++at == stages) at = 0;
            };
            bool ok = tmem_base == 0 && wait_item(0);            // all columns are ours: they begin at 0
            if (ok && item_of(0).count > 0) numbered_sync<kCopiesThreads>(kCopies + taken++);
            for (int n = 0; ok && item_of(n).count > 0; ++n) {
                const int count = item_of(n).count, groups = item_of(n).tokens > g.tokens_of_tile ? 2 : 1;
                done_item(n);
                for (int i = 0; i < groups && ok; ++i) {
                    ok = wait(kQueries + i, begun[i]++ & 1);
                    if (!ok) break;
                    fence_after();
                    scores(i, kTwo ? i : step & 1, k_at);
                }
                if (!ok) break;
                next(k_at, S::kKeyStages);
                for (int j = 0; j < count && ok; ++j) {
                    const bool more = j + 1 < count;
                    const uint32_t others = look_failed();       // used when it has come
                    numbered_sync<kCopiesThreads>(kCopies + taken++ % 8);        // its values, and the next keys
                    if (!kTwo) {
                        // One row tile: the next scores, in the other place, before the weights of these are there.  What lay
                        // in that place were the weights of the tile before, whose product was issued earlier.
                        ok = !__any_sync(~0u, others);
                        if (!ok) break;
                        if (more) scores(0, (step + 1) & 1, k_at);
                        numbered_sync<kHandOverThreads>(kHandOver + (step & 1));
                        fence_after();
                        sums(0, step & 1, v_at, 0, j > 0);
                        if (one) commit(bar(kSumsDone + (step & 1)));
                        __syncwarp();
                        ++step;
                    }
#pragma unroll
                    for (int i = 0; kTwo && i < kGroups; ++i) {
                        if (i >= groups) break;
                        numbered_sync<kHandOverThreads>(kHandOver + 2 * i);
                        fence_after();
                        sums(i, i, v_at, 0, j > 0);
                        numbered_sync<kHandOverThreads>(kHandOver + 1 + 2 * i);
                        fence_after();
                        sums(i, i, v_at, 1, true);
                        if (i == 0) ok = !__any_sync(~0u, others);
                        if (!ok) break;
                        if (more) scores(i, i, k_at);
                        else if (one) commit(bar(kSumsDone + i));
                        __syncwarp();
                    }
                    next(v_at, S::kValueStages);
                    if (more) next(k_at, S::kKeyStages);
                }
                ok = ok && wait_item(n + 1);
            }
            if (!ok) {
                // products under way still read shared memory and write TMEM
                if (lane == 0) asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(failed_at), "r"(1) : "memory");
                if (one) commit(bar(kDrain));
                __syncwarp();
                bar_wait(bar(kDrain), 0);
            }
            __syncwarp();
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && failed_word) atomicOr(g.status, 2);
    if (warp == kIssueWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <int D, typename T>
cudaError_t launch_of(const PromptArgs &g, const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, int sms, cudaStream_t st) {
    const cudaError_t e = launch_kernel(prompt_kernel<D, T>, dim3(sms), Shape<D>::kThreads, Shape<D>::kSmem, st, false, g, q, k, v);
    if (e != cudaSuccess) return e;
    return launch_kernel(join_kernel<D, T, Shape<D>::kGroups * kRows, kRows, Shape<D>::kKeys>, dim3(kJoinBlocks * sms), kJoinThreads, 0, st, true, g, sms);
}

template <int D, typename T>
cudaError_t prepare_of() {
    return cudaFuncSetAttribute(prompt_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D>::kSmem);
}

template <typename T>
cudaError_t prepare_dim(int head_dim) {
    return head_dim == 64 ? prepare_of<64, T>() : head_dim == 128 ? prepare_of<128, T>() : prepare_of<256, T>();
}
template <typename T>
cudaError_t launch_dim(const PromptArgs &g, const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, int head_dim, int sms, cudaStream_t st) {
    return head_dim == 64 ? launch_of<64, T>(g, q, k, v, sms, st) : head_dim == 128 ? launch_of<128, T>(g, q, k, v, sms, st) : launch_of<256, T>(g, q, k, v, sms, st);
}

}  // namespace

cudaError_t prepare_prompt(int head_dim, int type) {
    return type == ISJL_KV_BF16 ? prepare_dim<__nv_bfloat16>(head_dim) : prepare_dim<__half>(head_dim);
}

cudaError_t launch_prompt(PromptArgs &g, void *encoder, int head_dim, int type, int sms, cudaStream_t st) {
    CUtensorMap q, k, v;
    share_rows(g, kRows);
    g.out_wide = reinterpret_cast<uintptr_t>(g.a.out) % 32 == 0 && (g.a.out_stride[0] | g.a.out_stride[1]) % 16 == 0;
    if (sms > kMostRuns) sms = kMostRuns;
    const int keys = head_dim == 256 ? Shape<256>::kKeys : Shape<128>::kKeys, rows = 1 << g.shift < keys ? 1 << g.shift : keys;
    if (!encode_queries(encoder, &q, g.a.q, g.a.q_stride, g.tokens_of_tile, g.rows_of_token, g.a.n_tokens, g.n_kv_heads * g.group, head_dim, type) ||
        !encode_cache(encoder, &k, g.cache.k, g.cache.k_stride, rows, 1, g.n_blocks, g.shift, g.n_kv_heads, head_dim, type) ||
        !encode_cache(encoder, &v, g.cache.v, g.cache.v_stride, rows, 1, g.n_blocks, g.shift, g.n_kv_heads, head_dim, type))
        return cudaErrorInvalidValue;
    return type == ISJL_KV_BF16 ? launch_dim<__nv_bfloat16>(g, q, k, v, head_dim, sms, st) : launch_dim<__half>(g, q, k, v, head_dim, sms, st);
}

}  // namespace isjl
