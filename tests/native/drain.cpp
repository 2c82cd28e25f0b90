// The drain after an aborted wait, against a model of a ring's barriers whose copies land late, or never.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#define __device__
#define __forceinline__ inline
static long long now = 0;
static long long clock64() { return now += 100; }
// A slot's barrier: phases that are complete, and when its latest fill lands (the fills before it have)
struct Bar {
  int fills = 0;
  long long lands = 0;
};
static std::vector<Bar> bars;
static bool in_range = true;
namespace prhs {
constexpr long long kWaitBudgetCycles = 4000000;
static uint32_t mbar_try_wait(uint32_t bar, uint32_t parity) {
  now += 20;
  const uint32_t i = (bar - 64) / 8;
  if (i >= bars.size()) {
    in_range = false;
    return 1;
  }
  const Bar& b = bars[i];
  const int complete = b.fills == 0 ? 0 : now >= b.lands ? b.fills : b.fills - 1;     // the phase under way is number `complete`
  return (uint32_t)((complete & 1) != (int)parity);
}
}  // namespace prhs
#include "mbar_drain.cuh"

int main() {
  for (int slots = 1; slots <= 8; ++slots)
    for (int fills = 0; fills <= 40; ++fills)
      for (int late = 0; late <= slots; ++late)
        for (int never = 0; never < 2; ++never) {
          now = 0;
          bars.assign(slots, Bar());
          long long last = 0;
          for (int j = 0; j < fills; ++j) {
            Bar& b = bars[j % slots];
            ++b.fills;
            b.lands = j % slots == late ? (never ? 1ll << 60 : 200000) : 1000 * (j % slots);
          }
          for (const Bar& b : bars)
            if (b.fills && b.lands < (1ll << 60)) last = last > b.lands ? last : b.lands;
          prhs::mbar_drain_ring(64, slots, fills);
          const bool waits = !never || late >= slots || late >= fills;
          if (!in_range || (waits && now < last) || now > 10000000) {
            fprintf(stderr, "FAILED: %d slots, %d fills, slot %d late: %lld of %lld\n", slots, fills, late, now, last);
            return 1;
          }
        }
  return 0;
}
