// kv_sight.cuh -- the line of work of the attentions of single queries (kv_attend.cu, kv_attend4.cu): for each query, each
// key head (or part of its query heads), the slices of tokens that it sees.
#pragma once

#include "kv_internal.cuh"

namespace isjl {
namespace {

// what a query sees: tokens end - window .. end - 1 and 0 .. sinks - 1, counted from the first token that
// this kernel reads (the prefix's, or the own ones' where the prefix is done elsewhere)
struct Sight {
    int32_t end, lo, head;     // head: slices with first tokens that lie before the window's first slice
    int32_t slices;            // at least 1: an item without tokens still has a result
    int32_t row;
};

// prefix: tokens of it that are read before the own ones
template <int kSlice>
__device__ __forceinline__ Sight sight_of(const isjl_kv_attend_args &a, int shift, int32_t prefix, int32_t *status, int t) {
    Sight s;
    const int32_t x = a.lens[t];
    s.row = a.rows ? a.rows[t] : t;
    const bool bad = x > 0 && s.row >= 0 && (s.row >= a.n_table_rows || ((x - 1) >> shift) >= a.table_width);
    if (bad) report(status);
    s.end = x <= 0 || s.row < 0 || bad ? 0 : x + prefix;
    s.lo = a.window && s.end > a.window ? s.end - a.window : 0;
    s.head = min((min(a.sinks, s.lo) + kSlice - 1) / kSlice, s.lo / kSlice);
    s.slices = max(1, s.head + (s.end + kSlice - 1) / kSlice - s.lo / kSlice);
    return s;
}

// first token of a query's slice
template <int kSlice>
__device__ __forceinline__ int32_t slice_start(const Sight &s, int i) {
    return (i < s.head ? i : s.lo / kSlice + i - s.head) * kSlice;
}

// place on the line of slices
struct Place {
    int t, h, i;
    Sight s;
};

}  // namespace
}  // namespace isjl
