// kv_assign.cu -- block tables and slot maps from request lengths (isjl_kv_assign).
//
// Row i of a step holds ceil(len / bs) blocks and needs ceil((len + new) / bs) minus that.  Sums over the
// rows before it say which blocks of the free list are its own and where its tokens lie in the maps, so one
// block of threads takes the sums and everything else is independent: entry t of the maps finds its row by a
// search in `starts`, the k-th new block is the k-th from the top of the free list (or, where that was
// pushed in this very call, an entry of an ended row's table row, found by a search in `first_back`).
// Bound by latency for a step's few hundred tokens, by the 20 bytes a map entry for prompts.
#include "kv_internal.cuh"

namespace isjl {
namespace {

constexpr int kScan = 1024;   // threads of the block that takes the sums
constexpr int kFill = 256;    // threads of the blocks that fill the maps

// exclusive sums of two numbers over the block's threads, and their totals
__device__ __forceinline__ void scan2(int64_t &x, int64_t &y, int64_t &tx, int64_t &ty, int64_t (*sums)[2]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t ix = x, iy = y;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t px = __shfl_up_sync(~0u, ix, d), py = __shfl_up_sync(~0u, iy, d);
        if (lane >= d) { ix += px; iy += py; }
    }
    __syncthreads();
    if (lane == 31) { sums[warp][0] = ix; sums[warp][1] = iy; }
    __syncthreads();
    if (warp == 0) {
        const int64_t vx = sums[lane][0], vy = sums[lane][1];
        int64_t sx = vx, sy = vy;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t px = __shfl_up_sync(~0u, sx, d), py = __shfl_up_sync(~0u, sy, d);
            if (lane >= d) { sx += px; sy += py; }
        }
        sums[lane][0] = sx - vx;
        sums[lane][1] = sy - vy;
        if (lane == 31) { sums[32][0] = sx; sums[32][1] = sy; }
    }
    __syncthreads();
    x = sums[warp][0] + ix - x;
    y = sums[warp][1] + iy - y;
    tx = sums[32][0];
    ty = sums[32][1];
}

struct Row {
    int32_t len, held, back, ask, need;
};

__device__ __forceinline__ Row load_row(const AssignArgs &g, int i) {
    const int bs1 = (1 << g.shift) - 1;
    const int64_t room = (int64_t)g.a.table_width << g.shift;
    Row r;
    r.len = g.a.lens[i];
    const int32_t fresh = g.a.new_tokens[i];
    const bool bad = r.len < 0 || r.len > room;
    if (bad) report(g.status);
    r.held = bad ? 0 : (int32_t)(((int64_t)r.len + bs1) >> g.shift);
    r.back = fresh < 0 ? r.held : 0;
    r.ask = bad || fresh < 0 || (int64_t)r.len + fresh > room ? 0 : fresh;
    r.need = (int32_t)(((int64_t)r.len + r.ask + bs1) >> g.shift) - r.held;
    if (bad) r.need = 0;
    return r;
}

// last i in 0..n-1 with first[i] <= x, for first[0] = 0
__device__ __forceinline__ int find(const int32_t *first, int n, int32_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// entry `index` of the free list after the pushes of this call
__device__ __forceinline__ int32_t free_block(const AssignArgs &g, int32_t n_free, int32_t index) {
    if (index < n_free) return g.a.free_list[index];
    const int32_t k = index - n_free;
    const int i = find(g.first_back, g.a.n_rows, k);
    return g.a.table[(int64_t)i * g.a.table_width + (k - g.first_back[i])];
}

__device__ __forceinline__ int32_t free_count(const AssignArgs &g) {
    const int32_t n = *g.a.n_free;
    if (n < 0 || n > g.n_blocks) report(g.status);
    return min(max(n, 0), g.n_blocks);
}

// n_free and n_free_out may be the same word: what the fill needs of it was put here
struct Head {
    int32_t n_free, avail;
};

// the maps, the new table entries and the pushes, by `count` threads of which this is number `me`
__device__ __forceinline__ void fill(const AssignArgs &g, Head h, int me, int count) {
    const isjl_kv_assign_args &a = g.a;
    const int n = a.n_rows, mask = (1 << g.shift) - 1;
    const int32_t total = n ? a.starts[n] : 0;
    for (int64_t t = me; t < a.max_tokens; t += count) {
        int64_t slot = -1;
        int32_t position = 0, row = -1, visible = 0;
        if (t < total) {
            row = find(a.starts, n, (int32_t)t);
            const int32_t old = a.lens_out[row] - a.granted[row];
            const int32_t at = old + (int32_t)t - a.starts[row];
            const int32_t j = at >> g.shift, held = (old + mask) >> g.shift;
            const int32_t block = j < held ? a.table[(int64_t)row * a.table_width + j]
                                           : free_block(g, h.n_free, h.avail - 1 - (g.first_take[row] + j - held));
            slot = ((int64_t)block << g.shift) + (at & mask);
            position = a.prefix_len + at;
            visible = at + 1;
        }
        a.slots[t] = slot;
        a.positions[t] = position;
        a.rows[t] = row;
        a.visible[t] = visible;
    }
    const int32_t takes = n ? g.first_take[n] : 0, backs = n ? g.first_back[n] : 0;
    for (int32_t k = me; k < takes; k += count) {
        const int i = find(g.first_take, n, k);
        const int32_t old = a.lens_out[i] - a.granted[i];
        const int32_t j = ((old + mask) >> g.shift) + k - g.first_take[i];
        a.table[(int64_t)i * a.table_width + j] = free_block(g, h.n_free, h.avail - 1 - k);
    }
    for (int32_t k = me; k < backs; k += count) {
        if (h.n_free + k >= g.n_blocks) { report(g.status); break; }
        const int i = find(g.first_back, n, k);
        a.free_list[h.n_free + k] = a.table[(int64_t)i * a.table_width + (k - g.first_back[i])];
    }
}

// The sums over the rows.  Each thread takes a run of neighbouring rows, so that one scan over the block is
// enough for any number of them; asked and granted sums take a scan each, since grants depend on the former.
__device__ __forceinline__ Head sums(const AssignArgs &g, int64_t (*smem)[2]) {
    const isjl_kv_assign_args &a = g.a;
    const int n = a.n_rows, per = (n + kScan - 1) / kScan;
    const int begin = min(n, (int)threadIdx.x * per), end = min(n, begin + per);
    const int32_t n_free = free_count(g);
    int64_t need = 0, ask = 0, back = 0, unused = 0, all_need, all_ask, backs, none;
    for (int i = begin; i < end; ++i) {
        const Row r = load_row(g, i);
        need += r.need;
        ask += r.ask;
        back += r.back;
    }
    scan2(need, ask, all_need, all_ask, smem);
    scan2(back, unused, backs, none, smem);
    const int32_t avail = (int32_t)min((int64_t)n_free + backs, (int64_t)g.n_blocks);
    int64_t takes = 0, tokens = 0, total_takes, total_tokens, need_before = need, ask_before = ask;
    for (int i = begin; i < end; ++i) {
        const Row r = load_row(g, i);
        need_before += r.need;
        ask_before += r.ask;
        const bool ok = (r.need == 0 || need_before <= avail) && ask_before <= a.max_tokens;
        takes += ok ? r.need : 0;
        tokens += ok ? r.ask : 0;
    }
    scan2(takes, tokens, total_takes, total_tokens, smem);
    for (int i = begin; i < end; ++i) {
        const Row r = load_row(g, i);
        need += r.need;
        ask += r.ask;
        const bool ok = (r.need == 0 || need <= avail) && ask <= a.max_tokens;
        g.first_back[i] = (int32_t)back;
        g.first_take[i] = (int32_t)takes;
        a.starts[i] = (int32_t)tokens;
        const bool ends = a.new_tokens[i] < 0;
        a.granted[i] = ok ? r.ask : 0;
        back += r.back;
        if (ok) { takes += r.need; tokens += r.ask; }
        a.lens_out[i] = ends ? 0 : r.len + (ok ? r.ask : 0);
    }
    if (threadIdx.x == 0) {
        g.first_back[n] = (int32_t)backs;
        g.first_take[n] = (int32_t)total_takes;
        a.starts[n] = (int32_t)total_tokens;
    }
    __syncthreads();              // all have read n_free
    if (threadIdx.x == 0) *a.n_free_out = avail - (int32_t)total_takes;
    return {n_free, avail};
}

__global__ void __launch_bounds__(kScan) assign_kernel(const __grid_constant__ AssignArgs g) {
    __shared__ int64_t smem[33][2];
    const Head h = sums(g, smem);
    __syncthreads();
    fill(g, h, threadIdx.x, kScan);
}

}  // namespace

cudaError_t launch_assign(const AssignArgs &g, int sms, cudaStream_t st) {
    (void)sms;
    assign_kernel<<<1, kScan, 0, st>>>(g);
    return cudaGetLastError();
}

}  // namespace isjl
