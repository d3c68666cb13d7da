// kv_prompt_line.cuh -- the line of work of kv_prompt.cu: for each row of queries, each key head (or part of its query
// heads) and each of the row's items in order, the tiles of tokens that the item's queries see.  No device code: it
// compiles for the host as well.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define ISJL_LINE __host__ __device__ __forceinline__
#else
#define ISJL_LINE inline
#endif

namespace isjl {

// The sum of floor((a i + b) / m) over i < n.  What a and b have of whole m's comes out at once; the rest counts the
// points under a line, column by column, which is as many as row by row: y rows, of which row j has the columns from
// ceil((m (j + 1) - b) / a) on.  The roles of a and m change as in Euclid's algorithm.  a (n - 1) + b + m < 2^32.
ISJL_LINE int64_t line_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b) {
    int64_t sum = 0, sign = 1;
    while (n > 0) {
        sum += sign * ((int64_t)n * (n - 1) / 2 * (a / m) + (int64_t)n * (b / m));
        a %= m;
        b %= m;
        const uint32_t y = (a * (n - 1) + b) / m;
        if (y == 0) break;
        sum += sign * (int64_t)n * y;
        sign = -sign;
        const uint32_t old = m;
        b = m - b + a - 1;
        m = a;
        a = old;
        n = y;
    }
    return sum;
}

// what is the same for all rows of a call
struct PromptShape {
    int32_t keys;              // tokens of a tile
    int32_t step;              // queries of an item
    int32_t window, sinks;     // window 0: all
    int32_t extra;             // what an item takes beside its tiles, in tiles: places of the line in front of them
    ISJL_LINE int32_t sink_tiles() const { return sinks / keys + (sinks % keys != 0); }
};

// A row's `count` queries lie at places first, first + 1, ...; a query sees the tokens up to its own place.
struct PromptRow {
    int32_t count, first;
    ISJL_LINE int32_t items(const PromptShape &s) const { return (int32_t)(((uint32_t)count + (uint32_t)s.step - 1) / (uint32_t)s.step); }
    // one more than the last place that item p's queries see
    ISJL_LINE int32_t end(const PromptShape &s, int32_t p) const {
        const int64_t last = ((int64_t)p + 1) * s.step;
        return first + (int32_t)(last < count ? last : count);
    }
    // the first place of a query's window
    static ISJL_LINE int32_t low(const PromptShape &s, int32_t place) { return s.window && place >= s.window ? place + 1 - s.window : 0; }
    // tiles between the first tokens' and the window's that none of item p's queries sees
    ISJL_LINE int32_t skip(const PromptShape &s, int32_t p) const {
        const int32_t t = low(s, first + p * s.step) / s.keys - s.sink_tiles();
        return t > 0 ? t : 0;
    }
    ISJL_LINE int32_t tiles(const PromptShape &s, int32_t p) const {
        const int32_t e = end(s, p);
        return e / s.keys + (e % s.keys != 0) - skip(s, p);
    }
    // which tile of tokens is an item's j-th
    static ISJL_LINE int32_t tile(const PromptShape &s, int32_t skipped, int32_t j) { return j < s.sink_tiles() ? j : j + skipped; }
    // places of the line of the items before p, p <= items
    ISJL_LINE int64_t before(const PromptShape &s, int32_t p) const {
        const bool all = p > 0 && p == items(s);           // the last item may be a shorter one
        const int32_t n = all ? p - 1 : p;
        int64_t sum = (int64_t)p * s.extra + line_sum((uint32_t)n, (uint32_t)s.keys, (uint32_t)s.step, (uint32_t)first + (uint32_t)s.step + (uint32_t)s.keys - 1);
        if (s.window) {
            // skipped tiles begin with the item whose window begins `sink_tiles` tiles on
            const int64_t off = (int64_t)first + 1 - s.window - (int64_t)s.sink_tiles() * s.keys;
            const int64_t from = off >= 0 ? 0 : off < -(int64_t)n * s.step ? n : (uint32_t)(-off + s.step - 1) / (uint32_t)s.step;
            if (from < n) sum -= line_sum((uint32_t)(n - from), (uint32_t)s.keys, (uint32_t)s.step, (uint32_t)(off + from * s.step));
        }
        return all ? sum + tiles(s, n) : sum;
    }
};

}  // namespace isjl
