// Which positions a row of a drafted tree sees.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tg {

// Bits of the positions p0 .. p0 + 31, of those that are `there`, that node
// `node` sees of a request with L committed tokens and n nodes (the first at
// position L). `row`: the node's `words` mask words, or null for a chain
// (Words: a pointer to uint64_t, or what can be indexed like one).
template <class Words>
__device__ __forceinline__ uint32_t seen_bits(Words row, int words, int node, int n, int L, int p0,
                                              uint32_t there) {
  const int j0 = p0 - L;  // node at the first position
  if (j0 <= -32) return there;
  if (j0 >= n) return 0;  // past the last node, where the row may have no word
  const int ctx = max(0, -j0), n0 = max(0, j0);
  uint32_t own;
  if (row) {
    const int at = n0 / 64, sh = n0 % 64;
    uint64_t v = row[at] >> sh;
    if (sh > 32 && at + 1 < words) v |= row[at + 1] << (64 - sh);
    own = (uint32_t)v;
  } else {
    const int k = node - n0 + 1;
    own = k >= 32 ? ~0u : k > 0 ? (1u << k) - 1 : 0u;
  }
  if (n - n0 < 32) own &= (1u << (n - n0)) - 1;
  return there & (ctx ? own << ctx | ((1u << ctx) - 1) : own);
}

}  // namespace tg
