// After an aborted wait: bounded waits until a ring's copies have landed, so that shared memory is not handed back under them.  (Uses
// mbar_try_wait and kWaitBudgetCycles of score_tma.cuh.)
#pragma once

namespace prhs {

// The barriers bar, bar + 8, ... of `slots` slots, filled in turn, `fills` times in all (one phase a fill).  A barrier says of a parity whether the
// latest phase of that parity is complete, and of the parity that is not under way it always says so: only the parity of a slot's
// latest fill tells of its copies.
__device__ __forceinline__ void mbar_drain_ring(uint32_t bar, int slots, int fills) {
  for (int s = 0; s < slots && s < fills; ++s) {
    const uint32_t parity = (uint32_t)((fills - 1 - s) / slots) & 1u;
    const long long t0 = clock64();
    while (!mbar_try_wait(bar + 8 * s, parity))
      if (clock64() - t0 > kWaitBudgetCycles / 8) break;
  }
}

}  // namespace prhs
