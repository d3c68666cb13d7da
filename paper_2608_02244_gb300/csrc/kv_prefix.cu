// kv_prefix.cu -- the shared prefix's part of isjl_kv_attend, computed once for the whole batch.
//
// All queries see the same P prefix tokens, so for one key head the queries of the batch (n tokens times the
// `group` query heads of that key head) are the rows of a matrix: S = Q K^T, O = softmax(S) V, 4 D operations
// for each row and token, on the fifth-generation tensor cores.  A block takes two tiles of 128 rows and a
// run of tiles of 128 tokens: keys and values come by TMA from the cache's blocks through a ring each,
// one thread issues the products, and each row of a tile is one thread of a group of four warps that takes
// the row's maximum, exponentials and sum.  Scores lie in TMEM, their weights take the scores' place as the
// second product's left operand, and the two row tiles alternate: while the tensor cores work for one, the
// other's group is at its exponentials.  The sums O stay in TMEM for the whole run; they are rescaled only
// when a row's maximum has grown by more than 2^8 since the last time (fp16: 2^4, from 2^11, so that weights stay
// within 2^15 and small ones keep their bits); rounding weights to 16 bits is as exact as with the true maximum.
//
// The work is a line of (key head, pair of row tiles, token tile); every block has an equal run of it, and
// leaves its piece of each item (sum, maximum and total of each row) for kv_attend.cu to join with the
// requests' own tokens.
//
// 512 queries of 64 + 8 heads of 128 values over 32,768 tokens: 361 us, 1.52 PFLOP/s, on 128 SMs and 421 on 112, 1.4 us
// a step (two tiles of 128 rows by 128 tokens): at 1.93 GHz 2,700 cycles for 2,048 of products, with the tensor cores
// active in 77% of the cycles.  There the step itself is the bound, a row group's way from scores to weights.  On all 152
// SMs the whole call takes 389 us for the first 20 calls and 423 when called for seconds, at 1.64 GHz under the power
// cap (1.36 kW).  Steps of that took it there from 465: one thread's issue with
// uniform addresses (a product takes 64 cycles, its issue took 100), stages freed by the row groups instead of commits,
// weights handed over in halves, waits for copies beside products under way.
//
// Heads of 256 values have no such kernel: two row tiles' scores and sums fill TMEM at 128.
#include "kv_tma.cuh"

namespace isjl {
namespace {

constexpr int kRows = 128, kKeys = 128;        // of a row tile, of a token tile
constexpr int kThreads = 384;                  // two groups of four warps; the loading and the issuing warp's group
constexpr int kLoadWarp = 8, kIssueWarp = 10;
constexpr float kLog2e = 1.4426950408889634f;
// log2 of the growth of a maximum that is let pass, and of the largest weight of the tile that set it
template <typename T>
struct Grow {
    static constexpr float kPass = Half<T>::kIsBf16 ? 8.f : 4.f, kTop = Half<T>::kTop > 0 ? Half<T>::kTop - kPass : 0.f;
};

template <int D>
struct Shape {
    static constexpr int kHalves = D / 64;                       // rows of 128 bytes hold 64 values
    static constexpr int kHalfBytes = 128 * 128;                 // 128 rows of them
    static constexpr int kTileBytes = kHalves * kHalfBytes;
    static constexpr int kKeyStages = D == 128 ? 3 : 4, kValueStages = D == 128 ? 2 : 4;
    static constexpr int kSmem = (2 + kKeyStages + kValueStages) * kTileBytes + 1024;
};

// shared-memory operand with rows of 128 bytes, swizzled by 128 bytes
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t leading, uint32_t stride) {
    return (uint64_t)((at >> 4) & 0x3fff) | ((uint64_t)((leading >> 4) & 0x3fff) << 16) |
           ((uint64_t)((stride >> 4) & 0x3fff) << 32) | (1ull << 46) | (2ull << 61);
}

// operands by the low word and the (common) high word of their descriptors
__device__ __forceinline__ void mma_smem(uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t what, bool add) {
    asm volatile("{\n.reg .pred p;\n.reg .b64 x, y;\nmov.b64 x, {%1, %3};\nmov.b64 y, {%2, %3};\nsetp.ne.b32 p, %5, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, p;\n}"
                 ::"r"(d), "r"(a), "r"(b), "r"(high), "r"(what), "r"((int)add) : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t high, uint32_t what, bool add) {
    asm volatile("{\n.reg .pred p;\n.reg .b64 y;\nmov.b64 y, {%2, %3};\nsetp.ne.b32 p, %5, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n}"
                 ::"r"(d), "r"(a), "r"(b), "r"(high), "r"(what), "r"((int)add) : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t mine;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(mine));
    return mine != 0;
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

#define R8(v, i) "=r"((v)[(i)]), "=r"((v)[(i) + 1]), "=r"((v)[(i) + 2]), "=r"((v)[(i) + 3]), "=r"((v)[(i) + 4]), "=r"((v)[(i) + 5]), "=r"((v)[(i) + 6]), "=r"((v)[(i) + 7])
#define W8(v, i) "r"((v)[(i)]), "r"((v)[(i) + 1]), "r"((v)[(i) + 2]), "r"((v)[(i) + 3]), "r"((v)[(i) + 4]), "r"((v)[(i) + 5]), "r"((v)[(i) + 6]), "r"((v)[(i) + 7])

// two 32-bit operations in one instruction: for the exponents' arguments and sums, 378 -> 361 us with 512 queries of
// 64 + 8 heads over 32,768 tokens
__device__ __forceinline__ float2 fma2(float x, float y, float scale, float offset) {
    float2 z;
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %4};\nmov.b64 c, {%5, %5};\nfma.rn.f32x2 d, a, b, c;\n"
        "mov.b64 {%0, %1}, d;\n}" : "=f"(z.x), "=f"(z.y) : "f"(x), "f"(y), "f"(scale), "f"(offset));
    return z;
}
__device__ __forceinline__ void add2(float2 &sum, float x, float y) {
    asm("{\n.reg .b64 a, b;\nmov.b64 a, {%0, %1};\nmov.b64 b, {%2, %3};\nadd.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
        : "+f"(sum.x), "+f"(sum.y) : "f"(x), "f"(y));
}

// 32 columns of this thread's TMEM lane
__device__ __forceinline__ void tmem_load(uint32_t (&v)[32], uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : R8(v, 0), R8(v, 8), R8(v, 16), R8(v, 24) : "r"(at));
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&v)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(at), W8(v, 0), W8(v, 8), W8(v, 16), W8(v, 24) : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// barriers, in 8-byte words after the tiles
enum { kKeyFull = 0, kValueFull = 8, kFree = 4 /* after a stage's full one */, kScores = 16, kWeights = 18, kSums = 20, kQueries = 22,
       kRest = 24, kDrain = 26, kBars = 27 };

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, 1)
prefix_kernel(const __grid_constant__ PrefixArgs g, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
    using S = Shape<D>;
    constexpr bool kBf16 = sizeof(T) == 2 && Half<T>::kIsBf16;
    // operand types, 32-bit sums, 128 rows; the first product has 128 columns and both operands along D, the
    // second D columns and its right operand (values, tokens outermost) across
    constexpr uint32_t kTypes = (1u << 4) | (kBf16 ? (1u << 7) | (1u << 10) : 0u) | ((kRows / 16) << 24);
    constexpr uint32_t kFirst = kTypes | ((kKeys / 8) << 17), kSecond = kTypes | ((D / 8) << 17) | (1u << 16);
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ uint32_t tmem_base;
    __shared__ int32_t failed_word;
    volatile int32_t *failed = &failed_word;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
    const uint32_t q_at = base, ring = base + 2 * S::kTileBytes;
    const uint32_t bar0 = smem_addr(bars);
    auto bar = [&](int i) { return bar0 + 8 * i; };

    start_next();
    if (threadIdx.x == 0) {
        tma_prefetch(&kmap);
        tma_prefetch(&vmap);
        failed_word = 0;
        for (int i = 0; i < 16; ++i) bar_init(bar(i), 1);
        for (int i = 0; i < 2; ++i) {
            bar_init(bar(kScores + i), 1);
            bar_init(bar(kWeights + i), 128);
            bar_init(bar(kRest + i), 128);
            bar_init(bar(kSums + i), 1);
            bar_init(bar(kQueries + i), 128);
        }
        bar_init(bar(kDrain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssueWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_base;

    // this block's run of the line, item by item: token tiles j0 .. j1 - 1 of item i
    const PrefixLine ln = g.line;
    const int64_t f0 = ln.work() * blockIdx.x / ln.blocks, f1 = ln.work() * (blockIdx.x + 1) / ln.blocks;
    auto two_of = [&](int pair) { return (2 * pair + 1) * ln.tokens_of_tile < g.n; };

    // Registers at launch: 384 x 168.  A row's thread holds 128 scores beside its weights, the third group
    // needs few: 256 x 216 + 128 x 72 are the same sum.
    if (warp < kLoadWarp) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ---- the rows of one tile, a thread each
        const int group = warp >> 2, row = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;         // this warp's quarter of the TMEM lanes
        const uint32_t s_at = tmem + group * 128 + lanes, o_at = tmem + 256 + group * 128 + lanes;
        const float scale = g.scale * kLog2e;
        uint32_t step = 0;
        int item_no = 0;
        int key_stage = 0, value_stage = 0;        // of the keys and values that are freed next
        auto next = [](int &at, int by, int stages) { at = (at + by) % stages; };
        bool ok = true;
        for (int64_t f = f0; f < f1 && ok;) {
            const int item = (int)(f / ln.tiles), j0 = (int)(f - (int64_t)item * ln.tiles);
            const int count = (int)min((int64_t)ln.tiles - j0, f1 - f), head = item / ln.pairs, pair = item % ln.pairs;
            f += count;
            const bool two = two_of(pair);
            if (group == 1 && !two) {
                next(key_stage, count, S::kKeyStages);
                next(value_stage, count, S::kValueStages);
                continue;
            }
            // The last group to use a tile frees its stages: when it sees its scores, the products of the keys are
            // done, and those of the tile before's values, which were issued earlier.
            const bool frees = (group == 1) == two && (threadIdx.x & 127) == 0;
            const int token = (2 * pair + group) * ln.tokens_of_tile + row / g.group, member = row % g.group;
            const bool live = row < ln.tokens_of_tile * g.group && token < g.n;
            const int q_head = head * g.group + member;
            {   // this thread's row of queries, swizzled as the tensor cores read it
                const T *from = static_cast<const T *>(g.q) + (int64_t)token * g.q_stride[0] + (int64_t)q_head * g.q_stride[1];
                const uint32_t to = q_at + group * S::kTileBytes + row * 128;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 w = live ? *reinterpret_cast<const uint4 *>(from + 8 * c) : make_uint4(0, 0, 0, 0);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (c / 8) * S::kHalfBytes + (((c % 8) ^ (row & 7)) << 4)),
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
                uint32_t s[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_load(s[c], s_at + 32 * c);
                tmem_load_wait();
                const int left = g.tokens - (j0 + j) * kKeys;
                if (left < kKeys) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (32 * c + i >= left) s[c][i] = __float_as_uint(-INFINITY);
                }
                float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < 32; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) most[c] = fmaxf(most[c], __uint_as_float(s[c][i]));
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
                for (int h = 0; h < 2; ++h) {
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
                    bar_arrive(bar((h ? kRest : kWeights) + group));      // the product starts with the first half
                }
                total += (part[0].x + part[0].y) + (part[1].x + part[1].y);
            }
            ok = ok && __all_sync(~0u, bar_wait(bar(kSums + group), item_no & 1, failed));
            if (!ok) break;
            fence_after();
            ++item_no;
            if (frees) bar_arrive(bar(kValueFull + kFree + value_stage));
            next(value_stage, 1, S::kValueStages);
            const int64_t at = ((int64_t)(blockIdx.x - ln.first_block(item)) * g.n + token) * (g.n_kv_heads * g.group) + q_head;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                __syncwarp();
                tmem_load(o, o_at + 32 * c);
                tmem_load_wait();
                if (live)
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        *reinterpret_cast<uint4 *>(g.part_o + at * D + 32 * c + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
            }
            if (live) g.part_ml[at] = make_float2(top, total);
            fence_before();       // the next item's first product overwrites these sums only after its weights
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == kLoadWarp || warp == kLoadWarp + 1) {
            // ---- keys by one warp, values by the other: one copy for each cache block (or part of one) of a tile and 64 of its values
            const int rows = min(1 << g.shift, kKeys), pieces = kKeys / rows;      // pieces: 1 .. 16
            const uint32_t piece_bytes = rows * 128;
            // this lane's part of a tile: piece lane % pieces, and every 32 / pieces-th half
            const int piece = lane % pieces;
            constexpr int32_t kNone = INT32_MIN;
            auto block_of = [&](int j) {
                const int token = j * kKeys + piece * rows;
                return token < g.tokens ? g.prefix[token >> g.shift] : kNone;
            };
            // A ring for each: a stage's turns are one warp's, which cannot be two turns ahead of itself.
            const bool values = warp != kLoadWarp;
            const int stages = values ? S::kValueStages : S::kKeyStages, full = values ? kValueFull : kKeyFull;
            const uint32_t to = ring + (values ? S::kKeyStages * S::kTileBytes : 0);
            const CUtensorMap *map = values ? &vmap : &kmap;
            int load = 0, stage = 0;
            uint32_t turn = 0;
            bool ok = true;
            for (int64_t f = f0; f < f1 && ok;) {
                const int item = (int)(f / ln.tiles), j0 = (int)(f - (int64_t)item * ln.tiles), head = item / ln.pairs;
                const int count = (int)min((int64_t)ln.tiles - j0, f1 - f);
                f += count;
                int coming = block_of(j0);                             // asked for one tile ahead
                for (int j = j0; j < j0 + count && ok; ++j) {
                    int block = coming;
                    const int slot = (j * kKeys + piece * rows) & ((1 << g.shift) - 1);
                    if (j + 1 < j0 + count) coming = block_of(j + 1);
                    if ((uint32_t)block >= (uint32_t)g.n_blocks) {                 // beyond the prefix or the cache: zeros
                        if (block != kNone) report(g.status);
                        block = g.n_blocks;
                    }
                    ok = __all_sync(~0u, load < stages || bar_wait(bar(full + kFree + stage), turn ^ 1, failed));
                    if (!ok) break;
                    if (lane == 0) bar_expect(bar(full + stage), S::kTileBytes);
                    __syncwarp();
                    for (int half = lane / pieces; half < S::kHalves; half += 32 / pieces)
                        tma_load(to + stage * S::kTileBytes + half * S::kHalfBytes + piece * piece_bytes, map, bar(full + stage), slot, half,
                                 head, block);
                    ++load;
                    if (++stage == stages) { stage = 0; turn ^= 1; }
                }
            }
            // nothing is left in flight, also after a failure
            for (int i = max(0, load - stages); i < load; ++i) bar_wait(bar(full + i % stages), (i / stages) & 1, nullptr);
        } else if (warp == kIssueWarp) {
            // The whole warp runs this loop, so that addresses stay uniform, and one thread of it issues: with the
            // products of 64 cycles each, their issue has to take less.
            const bool one = elect_one();
            uint32_t step[2] = {0, 0}, begun[2] = {0, 0};       // weights taken, items begun so far of each row tile
            bool ok = tmem_base == 0;                            // all columns are ours: they begin at 0
            // operands differ in their address field alone: low word plus 16-byte steps
            const uint32_t q_lo = (uint32_t)operand(q_at, 16, 1024), k_lo = (uint32_t)operand(ring, 16, 1024);
            const uint32_t v_lo = (uint32_t)operand(ring + S::kKeyStages * S::kTileBytes, S::kHalfBytes, 1024);
            constexpr uint32_t high = (1024 >> 4) | (1u << 14) | (2u << 29);
            auto scores = [&](int i, int stage) {
                const uint32_t a = q_lo + i * (S::kTileBytes >> 4), b = k_lo + stage * (S::kTileBytes >> 4);
                if (one) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = ((k / 4) * S::kHalfBytes + (k % 4) * 32) >> 4;
                        mma_smem(i * 128, a + off, b + off, high, kFirst, k > 0);
                    }
                    commit(bar(kScores + i));
                }
            };
            auto sums = [&](int i, int stage, int half, bool add) {
                const uint32_t b = v_lo + stage * (S::kTileBytes >> 4), a = i * 128, d = 256 + i * 128;
                constexpr int kSteps = kKeys / 32;
                if (one) {
#pragma unroll
                    for (int k = 0; k < kSteps; ++k)
                        mma_tmem(d, a + (half * kSteps + k) * 8, b + (half * kSteps + k) * (2048 >> 4), high, kSecond, add || half + k > 0);
                }
            };
            auto wait = [&](int b, uint32_t phase) { ok = ok && __all_sync(~0u, bar_wait(bar(b), phase, failed)); };
            int k_at = 0, v_at = 0;                              // stages of the tile's keys and values, and their turns
            uint32_t k_turn = 0, v_turn = 0;
            auto next = [](int &at, uint32_t &turn, int stages) {
                if (++at == stages) { at = 0; turn ^= 1; }
            };
            for (int64_t f = f0; f < f1 && ok;) {
                const int item = (int)(f / ln.tiles), j0 = (int)(f - (int64_t)item * ln.tiles);
                const int count = (int)min((int64_t)ln.tiles - j0, f1 - f), groups = two_of(item % ln.pairs) ? 2 : 1;
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
                    for (int i = 0; i < 2; ++i) {
                        if (i >= groups) break;
                        // one wait for weights and (before the first row tile's) copies: a lane for each barrier
                        const bool copies = lane == 1 && i == 0;
                        wait(copies ? kValueFull + v_at : kWeights + i, copies ? v_turn : step[i] & 1);
                        if (!ok) break;
                        fence_after();
                        sums(i, v_at, 0, j > 0);
                        wait(copies && more ? kKeyFull + k_at : kRest + i, copies && more ? k_turn : step[i] & 1);
                        ++step[i];
                        if (!ok) break;
                        fence_after();
                        sums(i, v_at, 1, true);
                        if (more) scores(i, k_at);
                        else if (one) commit(bar(kSums + i));
                    }
                    next(v_at, v_turn, S::kValueStages);
                    if (more) next(k_at, k_turn, S::kKeyStages);
                }
                f += count;
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
    if (warp == kIssueWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <int D, typename T>
cudaError_t launch_of(const PrefixArgs &g, const CUtensorMap &k, const CUtensorMap &v, cudaStream_t st) {
    return launch_kernel(prefix_kernel<D, T>, g.line.blocks, kThreads, Shape<D>::kSmem, st, false, g, k, v);
}

template <int D, typename T>
cudaError_t prepare_of() {
    return cudaFuncSetAttribute(prefix_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D>::kSmem);
}

}  // namespace

cudaError_t prepare_prefix(int head_dim, int type) {
    if (type == ISJL_KV_BF16) return head_dim == 64 ? prepare_of<64, __nv_bfloat16>() : prepare_of<128, __nv_bfloat16>();
    return head_dim == 64 ? prepare_of<64, __half>() : prepare_of<128, __half>();
}

PrefixLine prefix_line(int n, int group, int n_kv_heads, int tokens, int sms) {
    PrefixLine ln;
    ln.tokens_of_tile = kRows / group;
    const int tiles = (n + ln.tokens_of_tile - 1) / ln.tokens_of_tile;
    ln.pairs = (tiles + 1) / 2;
    ln.items = ln.pairs * n_kv_heads;
    ln.tiles = (tokens + kKeys - 1) / kKeys;
    ln.blocks = ln.work() < sms ? (int)ln.work() : sms;
    // most blocks that share an item
    ln.pieces = (int)(((int64_t)ln.tiles * ln.blocks + ln.work() - 1) / ln.work()) + 1;
    return ln;
}

cudaError_t launch_prefix(const PrefixArgs &g, const isjl_kv_cache &cache, void *encoder, int head_dim, int type, cudaStream_t st) {
    CUtensorMap k, v;
    const int rows = g.shift < 7 ? 1 << g.shift : kKeys;
    if (!encode_cache(encoder, &k, cache.k, cache.k_stride, rows, 1, g.n_blocks, g.shift, g.n_kv_heads, head_dim, type) ||
        !encode_cache(encoder, &v, cache.v, cache.v_stride, rows, 1, g.n_blocks, g.shift, g.n_kv_heads, head_dim, type))
        return cudaErrorInvalidValue;
    if (type == ISJL_KV_BF16)
        return head_dim == 64 ? launch_of<64, __nv_bfloat16>(g, k, v, st) : launch_of<128, __nv_bfloat16>(g, k, v, st);
    return head_dim == 64 ? launch_of<64, __half>(g, k, v, st) : launch_of<128, __half>(g, k, v, st);
}

}  // namespace isjl
