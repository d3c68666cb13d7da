// kv_ring.cuh -- a place in a ring of stages that copies fill in turn (kv_attend.cu).  No device code: it compiles for
// the host as well.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define ISJL_HOST_DEVICE __host__ __device__
#else
#define ISJL_HOST_DEVICE
#endif

namespace isjl {

// The stage that is taken next and its barrier's phase; each barrier turns once a fill.  Stages 0 .. kStages - 2 are
// filled first; from then on the one before the place is filled, just before the place's own is waited for.
template <int kStages>
struct RingPlace {
    int stage = 0;
    uint32_t phase = 0;
    ISJL_HOST_DEVICE int before() const { return stage == 0 ? kStages - 1 : stage - 1; }
    // stages filled and not taken, from the place on, while it is waited for with `left` fills not taken (filled or not)
    ISJL_HOST_DEVICE int under_way(int64_t left) const { return left < kStages ? (int)left : kStages; }
    ISJL_HOST_DEVICE void take() {
        if (++stage == kStages) { stage = 0; phase ^= 1; }
    }
};

}  // namespace isjl
