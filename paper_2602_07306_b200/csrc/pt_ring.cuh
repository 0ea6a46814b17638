// What a kernel whose wait has given up does before it ends: copies that it has started may still be writing to its shared
// memory, which belongs to another block as soon as this one is gone.
#pragma once
#include "pt_tc.h"
#include "pt_ptx.cuh"

namespace pt {

// Stages of a ring, `n` of them from stage s on, get a bounded time to land.  Of a barrier's two parities one is always that of its
// last complete phase, for which a poll says yes at once; copies under way complete the phase of the other.  (A stage without any
// takes the whole time.  To count those under way costs two of the decode kernels registers in their loops, 3 to 8 % of their time:
// they drain all.)
__device__ __forceinline__ void drain_ring(uint64_t* bars, int stages, int s, int n) {
    for (int i = 0; i < stages && i < n; ++i) {
        WaitClock clock;
        const uint32_t flying = mbar_try(&bars[s], 1) ? 0u : 1u;
        for (uint32_t spin = 0; spin < (1u << 16) && !mbar_try(&bars[s], flying); ++spin)
            if ((spin & 63) == 63 && clock.expired(100000000ull)) break;
        if (++s == stages) s = 0;
    }
}

// The same where copies, and products that read what they brought, belong to several warps: whatever is under way gets 100 ms.
__device__ __forceinline__ void settle_copies() {
    WaitClock clock;
    for (uint32_t i = 0; i < (1u << 20) && !clock.expired(100000000ull); ++i) __nanosleep(1000);
}

}  // namespace pt
