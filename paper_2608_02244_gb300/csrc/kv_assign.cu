// kv_assign.cu -- block tables and slot maps from request lengths (isjl_kv_assign).
//
// Row i of a step holds ceil(len / bs) blocks and needs ceil((len + new) / bs) minus that.  Sums over the
// rows before it say which blocks of the free list are its own and where its tokens lie in the maps, so one
// block of threads takes the sums and everything else is independent: entry t of the maps finds its row by a
// search in `starts`, the k-th new block is the k-th from the top of the free list (or, where that was
// pushed in this very call, an entry of an ended row's table row, found by a search in `back`).
// Bound by latency for a step's few hundred tokens: one kernel does it all from shared memory.  Prompts are
// bound by the 20 bytes a map entry: the block of the sums is followed by a grid that fills the maps.
#include "kv_tma.cuh"

namespace isjl {
namespace {

constexpr int kScan = 1024;   // threads of the block that takes the sums
constexpr int kKeep = 4;      // rows of its threads that stay in registers
constexpr int kFill = 256;    // threads of the blocks that fill the maps, 4 entries each

// inclusive sums of N numbers over the block's threads, and their totals
template <int N>
__device__ __forceinline__ void scan(int64_t (&x)[N], int64_t (&total)[N], int64_t (*sums)[3]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    __syncwarp();                    // the threads come from loops of different lengths
#pragma unroll
    for (int d = 1; d < 32; d <<= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int64_t p = __shfl_up_sync(~0u, x[k], d);
            if (lane >= d) x[k] += p;
        }
    __syncthreads();
    if (lane == 31)
#pragma unroll
        for (int k = 0; k < N; ++k) sums[warp][k] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {       // each warp sums those before it
        int64_t v = lane < warps ? sums[lane][k] : 0, before = lane < warp ? v : 0;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            v += __shfl_xor_sync(~0u, v, d);
            before += __shfl_xor_sync(~0u, before, d);
        }
        x[k] += before;
        total[k] = v;
    }
}

struct Row {
    int32_t len, held, back, ask, need;
    bool ends;
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
    r.ends = fresh < 0;
    r.back = fresh < 0 ? r.held : 0;
    r.ask = bad || fresh < 0 || (int64_t)r.len + fresh > room ? 0 : fresh;
    r.need = (int32_t)(((int64_t)r.len + r.ask + bs1) >> g.shift) - r.held;
    if (bad) r.need = 0;
    return r;
}

// last i in lo..hi-1 with first[i] <= x, for first[lo] <= x
__device__ __forceinline__ int find(const int32_t *first, int lo, int hi, int32_t x) {
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// the same by a whole warp: 32 places looked at together, three loads in a row where the search above takes twelve
__device__ __forceinline__ int find_by_warp(const int32_t *first, int lo, int hi, int32_t x) {
    const int lane = threadIdx.x & 31;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const uint32_t below = __ballot_sync(~0u, at < hi && first[min(at, hi - 1)] <= x);
        lo += (31 - __clz(below)) * step;          // lane 0's place is one of them
        hi = min(hi, lo + step);
    }
    return lo;
}

// the sums, in the block's shared memory or where they were written for a grid
struct Sums {
    const int32_t *starts, *take, *back, *old;      // tokens, blocks taken, blocks given back before each row; its length
    int32_t n_free, avail, tokens, takes, backs;
};

// entry `index` of the free list after the pushes of this call
__device__ __forceinline__ int32_t free_block(const AssignArgs &g, const Sums &h, int32_t index) {
    if (index < h.n_free) return g.a.free_list[index];
    const int32_t k = index - h.n_free;
    const int i = find(h.back, 0, g.a.n_rows, k);
    return g.a.table[(int64_t)i * g.a.table_width + (k - h.back[i])];
}

__device__ __forceinline__ int32_t free_count(const AssignArgs &g) {
    const int32_t n = *g.a.n_free;
    if (n < 0 || n > g.n_blocks) report(g.status);
    return min(max(n, 0), g.n_blocks);
}

// a number that a table or the free list holds for a block, reported if there is no such block
__device__ __forceinline__ int32_t seen(const AssignArgs &g, int32_t block) {
    if ((uint32_t)block >= (uint32_t)g.n_blocks) report(g.status);
    return block;
}

struct Entry {
    int64_t slot;
    int32_t position, row, visible;
};

// entry t of the maps, whose row lies in lo..hi-1; -1 is the slot in a block that is not there, which the caller reports
__device__ __forceinline__ Entry entry_of(const AssignArgs &g, const Sums &h, int32_t t, int lo, int hi) {
    if (t >= h.tokens) return {-1, 0, -1, 0};
    const int mask = (1 << g.shift) - 1;
    const int row = find(h.starts, lo, hi, t);
    const int32_t old = h.old[row], at = old + t - h.starts[row];
    const int32_t j = at >> g.shift, held = (int32_t)(((int64_t)old + mask) >> g.shift);
    const int32_t block = j < held ? g.a.table[(int64_t)row * g.a.table_width + j]
                                   : free_block(g, h, h.avail - 1 - (h.take[row] + j - held));
    const int64_t slot = (uint32_t)block < (uint32_t)g.n_blocks ? ((int64_t)block << g.shift) + (at & mask) : -1;
    return {slot, g.a.prefix_len + at, row, at + 1};
}

// the new table entries and the pushes, by `count` threads of which this is number `me`
__device__ __forceinline__ void move_blocks(const AssignArgs &g, const Sums &h, int me, int count) {
    const isjl_kv_assign_args &a = g.a;
    const int mask = (1 << g.shift) - 1;
    for (int32_t k = me; k < h.takes; k += count) {
        const int i = find(h.take, 0, a.n_rows, k);
        const int32_t j = (int32_t)(((int64_t)h.old[i] + mask) >> g.shift) + k - h.take[i];
        a.table[(int64_t)i * a.table_width + j] = seen(g, free_block(g, h, h.avail - 1 - k));
    }
    for (int32_t k = me; k < h.backs; k += count) {
        const int i = find(h.back, 0, a.n_rows, k);
        a.free_list[h.n_free + k] = seen(g, a.table[(int64_t)i * a.table_width + (k - h.back[i])]);
    }
}

// The sums over the rows, into the given arrays [n_rows + 1] (old: [n_rows]).  Each thread takes a run of
// neighbouring rows, so that one scan over the block is enough for any number of them; a second one is needed
// only where something is refused.
__device__ __forceinline__ Sums sums(const AssignArgs &g, int32_t *starts, int32_t *take, int32_t *back, int32_t *old, int64_t (*smem)[3]) {
    const isjl_kv_assign_args &a = g.a;
    const int n = a.n_rows, per = (n + blockDim.x - 1) / blockDim.x;
    const int begin = min(n, (int)threadIdx.x * per), end = min(n, begin + per);
    const int32_t n_free = free_count(g);
    int64_t x[3] = {0, 0, 0}, total[3], own[3];
    // up to kKeep rows of a thread stay in registers: their loads are under way together
    Row kept[kKeep] = {}, r = {};
    const bool keeps = per <= kKeep;
    if (keeps) {
#pragma unroll
        for (int k = 0; k < kKeep; ++k)
            if (begin + k < end) kept[k] = load_row(g, begin + k);
    }
    auto row_of = [&](int i) {
        Row v = {};
        if (keeps) {
#pragma unroll
            for (int k = 0; k < kKeep; ++k)
                if (i == begin + k) v = kept[k];
        } else {
            v = load_row(g, i);
        }
        return v;
    };
    for (int i = begin; i < end; ++i) {
        r = row_of(i);
        x[0] += r.need;
        x[1] += r.ask;
        x[2] += r.back;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) own[k] = x[k];
    scan(x, total, smem);
    // rows that end with more blocks than there are: only what the list can hold is given back
    const int32_t backs = (int32_t)min(total[2], (int64_t)(g.n_blocks - n_free)), avail = n_free + backs;
    if (total[2] > backs) report(g.status);
    int64_t need = x[0] - own[0], ask = x[1] - own[1], given = x[2] - own[2];          // before this thread's rows
    int64_t y[2] = {need, ask}, got[2] = {total[0], total[1]};
    const bool all = total[0] <= avail && total[1] <= a.max_tokens;
    if (!all) {
        int64_t need_to = need, ask_to = ask;
        y[0] = y[1] = 0;
        for (int i = begin; i < end; ++i) {
            r = row_of(i);
            need_to += r.need;
            ask_to += r.ask;
            const bool ok = (r.need == 0 || need_to <= avail) && ask_to <= a.max_tokens;
            y[0] += ok ? r.need : 0;
            y[1] += ok ? r.ask : 0;
        }
        const int64_t mine[2] = {y[0], y[1]};
        scan(y, got, smem);
        y[0] -= mine[0];
        y[1] -= mine[1];
    }
    for (int i = begin; i < end; ++i) {
        r = row_of(i);
        need += r.need;
        ask += r.ask;
        const bool ok = all || ((r.need == 0 || need <= avail) && ask <= a.max_tokens);
        take[i] = (int32_t)y[0];
        starts[i] = (int32_t)y[1];
        back[i] = (int32_t)min(given, (int64_t)INT32_MAX);
        old[i] = r.len;
        a.granted[i] = ok ? r.ask : 0;
        a.starts[i] = (int32_t)y[1];
        a.lens_out[i] = r.ends ? 0 : r.len + (ok ? r.ask : 0);
        given += r.back;
        if (ok) { y[0] += r.need; y[1] += r.ask; }
    }
    if (threadIdx.x == 0) a.starts[n] = (int32_t)got[1];
    __syncthreads();              // all have read n_free, all sums are written
    if (threadIdx.x == 0) *a.n_free_out = avail - (int32_t)got[0];
    return {starts, take, back, old, n_free, avail, (int32_t)got[1], (int32_t)got[0], backs};
}

// a whole step of at most kScan rows
__global__ void __launch_bounds__(kScan) assign_kernel(const __grid_constant__ AssignArgs g) {
    __shared__ int64_t smem[32][3];
    __shared__ int32_t rows[4][kScan];
    const Sums h = sums(g, rows[0], rows[1], rows[2], rows[3], smem);
    const isjl_kv_assign_args &a = g.a;
    for (int64_t t = threadIdx.x; t < a.max_tokens; t += blockDim.x) {
        const Entry e = entry_of(g, h, (int32_t)t, 0, a.n_rows);
        a.slots[t] = e.slot;
        a.positions[t] = e.position;
        a.rows[t] = e.row;
        a.visible[t] = e.visible;
        if (e.slot < 0 && e.row >= 0) report(g.status);
    }
    move_blocks(g, h, threadIdx.x, blockDim.x);
}

__global__ void __launch_bounds__(kScan) sums_kernel(const __grid_constant__ AssignArgs g) {
    __shared__ int64_t smem[32][3];
    start_next();
    int32_t *w = g.work;
    const int n = g.a.n_rows;
    const Sums h = sums(g, w + 8, w + 8 + n, w + 8 + 2 * n, w + 8 + 3 * n, smem);
    if (threadIdx.x == 0) {
        w[0] = h.n_free;
        w[1] = h.avail;
        w[2] = h.tokens;
        w[3] = h.takes;
        w[4] = h.backs;
    }
}

__global__ void __launch_bounds__(kFill) fill_kernel(const __grid_constant__ AssignArgs g) {
    wait_for_previous();
    const isjl_kv_assign_args &a = g.a;
    const int n = a.n_rows;
    const int32_t *w = g.work;
    const Sums h = {w + 8, w + 8 + n, w + 8 + 2 * n, w + 8 + 3 * n, w[0], w[1], w[2], w[3], w[4]};
    // 4 neighbouring entries a thread, 128 a warp: their rows are between those of the warp's ends
    const int lane = threadIdx.x & 31, warps = gridDim.x * (kFill / 32);
    for (int64_t t0 = 128 * (int64_t)(blockIdx.x * (kFill / 32) + threadIdx.x / 32); t0 < a.max_tokens; t0 += 128 * (int64_t)warps) {
        __syncwarp();                // the searches below are the whole warp's
        int lo = 0, hi = n;
        if (t0 < h.tokens) {
            lo = find_by_warp(h.starts, 0, n, (int32_t)t0);
            hi = find_by_warp(h.starts, lo, n, (int32_t)min(t0 + 127, (int64_t)h.tokens - 1)) + 1;
        }
        const int64_t t = t0 + 4 * lane;
        if (t >= a.max_tokens) continue;
        Entry e[4];
        e[0] = entry_of(g, h, (int32_t)t, lo, hi);
        const int mask = (1 << g.shift) - 1;
        const bool one_block = t + 3 < h.tokens && e[0].slot >= 0 && (e[0].slot & mask) + 3 <= mask && (e[0].row + 1 == n || t + 3 < h.starts[e[0].row + 1]);
#pragma unroll
        for (int k = 1; k < 4; ++k) {
            if (one_block) e[k] = {e[0].slot + k, e[0].position + k, e[0].row, e[0].visible + k};
            else e[k] = entry_of(g, h, (int32_t)min(t + k, (int64_t)INT32_MAX), lo, hi);
        }
        if (t + 3 < a.max_tokens && g.aligned) {
            reinterpret_cast<longlong2 *>(a.slots + t)[0] = make_longlong2(e[0].slot, e[1].slot);
            reinterpret_cast<longlong2 *>(a.slots + t)[1] = make_longlong2(e[2].slot, e[3].slot);
            *reinterpret_cast<int4 *>(a.positions + t) = make_int4(e[0].position, e[1].position, e[2].position, e[3].position);
            *reinterpret_cast<int4 *>(a.rows + t) = make_int4(e[0].row, e[1].row, e[2].row, e[3].row);
            *reinterpret_cast<int4 *>(a.visible + t) = make_int4(e[0].visible, e[1].visible, e[2].visible, e[3].visible);
        } else {
            for (int k = 0; k < 4 && t + k < a.max_tokens; ++k) {
                a.slots[t + k] = e[k].slot;
                a.positions[t + k] = e[k].position;
                a.rows[t + k] = e[k].row;
                a.visible[t + k] = e[k].visible;
            }
        }
    }
    const int me = blockIdx.x * kFill + threadIdx.x, count = gridDim.x * kFill;
    move_blocks(g, h, me, count);
    // The block that a row had begun is looked at once a row: at every entry that took 2,999 rows with 3.3 million entries
    // from 30.5 to 33.1 us, here to 31.1.  Blocks taken and given back are looked at where they move.
    for (int i = me; i < n; i += count) {
        const int32_t end = i + 1 < n ? h.starts[i + 1] : h.tokens;
        if (h.starts[i] < end && (h.old[i] & ((1 << g.shift) - 1))) seen(g, a.table[(int64_t)i * a.table_width + (h.old[i] >> g.shift)]);
    }
}

}  // namespace

// One kernel's block fills 1,024 entries in about 0.5 us; the grid's sums pass through memory and a second kernel's
// start.  Measured, one kernel against two: 256 rows with 1,024 entries 5.0 and 8.4 us, 4,096 7.9 and 8.1, 8,192 11.4
// and 8.1; 32 rows 7.2 and 7.4 at 4,096; 1,000 rows 8.9 and 9.8 at 4,096, 12.8 and 9.6 at 8,192.
constexpr int kOneKernel = 4096;

cudaError_t launch_assign(const AssignArgs &args, int sms, cudaStream_t st) {
    AssignArgs g = args;
    if (g.a.n_rows <= kScan && g.a.max_tokens <= kOneKernel) {
        const int most = g.a.n_rows > g.a.max_tokens ? g.a.n_rows : g.a.max_tokens;
        const int threads = most >= kScan ? kScan : most <= 128 ? 128 : (most + 31) / 32 * 32;
        return launch_kernel(assign_kernel, 1, threads, 0, st, false, g);
    }
    g.aligned = ((reinterpret_cast<uintptr_t>(g.a.slots) | reinterpret_cast<uintptr_t>(g.a.positions) |
                  reinterpret_cast<uintptr_t>(g.a.rows) | reinterpret_cast<uintptr_t>(g.a.visible)) & 15u) == 0;
    const cudaError_t e = launch_kernel(sums_kernel, 1, kScan, 0, st, false, g);
    if (e != cudaSuccess) return e;
    const int64_t blocks = ((int64_t)g.a.max_tokens + 4 * kFill - 1) / (4 * kFill);
    return launch_kernel(fill_kernel, (int)(blocks < 8 * sms ? blocks : 8 * sms), kFill, 0, st, true, g);
}

}  // namespace isjl
