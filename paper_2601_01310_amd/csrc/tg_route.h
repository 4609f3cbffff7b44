// The expert routing table's look-up.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tg {

// Slot of a pair of expert e: the first live ERT candidate of e.
// REPLAY: -1 also when the first pass's slot pr is still alive (its result
// stands). *unserved: the expert lists a local candidate, none alive.
template <bool REPLAY>
__device__ __forceinline__ int resolve_expert(int e, int pr, const int32_t* __restrict__ ert,
                                              int E, int R, const uint8_t* __restrict__ alive,
                                              int S, bool* unserved) {
  int slot = -1;
  bool listed = false;
  if (e >= 0 && e < E) {
    for (int r = 0; r < R; ++r) {
      const int c = ert[(size_t)e * R + r];
      if (c >= 0 && c < S) {
        listed = true;
        if (alive[c]) {
          slot = c;
          break;
        }
      }
    }
  }
  *unserved = slot < 0 && listed;
  if (REPLAY && pr >= 0 && pr < S && alive[pr]) slot = -1;  // first-pass result stands
  return slot;
}

}  // namespace tg
