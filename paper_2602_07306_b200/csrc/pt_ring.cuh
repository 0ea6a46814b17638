// What a kernel whose wait has given up does before it ends: copies that it has started may still be writing to its shared
// memory, which belongs to another block as soon as this one is gone.
#pragma once
#include "pt_tc.h"
#include "pt_ptx.cuh"

namespace pt {

// Each of the `pending` stages of a ring that were filled and not yet consumed gets a bounded time to land: they are those from
// stage `slot` on, whose copies complete its phase `parity` (stages before `slot`: the next phase).  The other parity of a stage
// says nothing, it is that of a phase long complete.
__device__ __forceinline__ void drain_ring(uint64_t* bars, int stages, int slot, uint32_t parity, int pending) {
    for (int i = 0; i < stages && i < pending; ++i) {
        WaitClock clock;
        for (uint32_t spin = 0; spin < (1u << 20) && !mbar_try(&bars[slot], parity); ++spin)
            if ((spin & 63) == 63 && clock.expired(100000000ull)) break;
        if (++slot == stages) { slot = 0; parity ^= 1u; }
    }
}

}  // namespace pt
