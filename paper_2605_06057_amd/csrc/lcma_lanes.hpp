// What the lanes of one wave do together, for the 8-bit-integer product and the sort of tokens.
#pragma once
#include <hip/hip_runtime.h>

#include "lcma_device.hpp"

namespace lcma {

// What a wave's lanes wrote to LDS is there for the reads of its other lanes behind this.  For the compiler: the LDS works in order, but without the barrier (which may
// not be moved into a branch) a lane's reads can end up in front of what lanes on the other side of a branch write.
LCMA_DEV void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Sum over the lanes up to and with this one (all 64 lanes at work).
LCMA_DEV int lanes_upto(int v) {
#define LCMA_FROM_LANES(CTRL, ROWS) v += __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 15, false)
    LCMA_FROM_LANES(0x111, 15); // 1, 2, 4, 8 lanes below, inside the rows of 16
    LCMA_FROM_LANES(0x112, 15);
    LCMA_FROM_LANES(0x114, 15);
    LCMA_FROM_LANES(0x118, 15);
    LCMA_FROM_LANES(0x142, 10); // the last lane of the row below, in rows 1 and 3; of the half below, in the upper half
    LCMA_FROM_LANES(0x143, 12);
#undef LCMA_FROM_LANES
    return v;
}

} // namespace lcma
