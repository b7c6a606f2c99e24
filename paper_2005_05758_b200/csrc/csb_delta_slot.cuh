// Which state a sequence of a call has.
#pragma once

#include "csb_delta.hpp"

namespace csb {

// The slot of sequence i, or -1 where the call leaves it alone: a negative or too large slot, or one that an earlier
// sequence of the call has.  All threads of the block take part.
__device__ __forceinline__ long long delta_slot(const DeltaArgs& a, int i) {
    if (!a.slot) return i < a.slots ? i : -1;
    const int mine = a.slot[i];
    int taken = 0;
    for (int j = threadIdx.x; j < i; j += blockDim.x) taken |= a.slot[j] == mine;
    if (__syncthreads_or(taken) || mine < 0 || mine >= a.slots) return -1;
    return mine;
}

}  // namespace csb
