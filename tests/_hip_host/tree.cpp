// The positions that a row of a drafted tree sees, on the CPU, with every mask
// word that is read checked.
#include "tg_tree.h"

namespace {

struct Row {
  const uint64_t* at;
  int words;
  int* outside;
  explicit operator bool() const { return at != nullptr; }
  uint64_t operator[](int i) const {
    if (i >= 0 && i < words) return at[i];
    ++*outside;
    return ~0ull;
  }
};

}  // namespace

extern "C" {

// Over the positions [0, end of the tiles of `unit`) of a request: bits[p] is
// whether the node sees position p. Returns the reads outside the row.
int seen(const uint64_t* row, int words, int node, int n, int L, int unit, uint8_t* bits) {
  int outside = 0;
  const int end = L + n;
  for (int p0 = 0; p0 < (end + unit - 1) / unit * unit; p0 += 32) {
    const int left = end - p0;
    const uint32_t there = left >= 32 ? ~0u : left > 0 ? (1u << left) - 1 : 0u;
    const uint32_t m = tg::seen_bits(Row{row, words, &outside}, words, node, n, L, p0, there);
    for (int i = 0; i < 32; ++i) bits[p0 + i] = m >> i & 1;
  }
  return outside;
}

}  // extern "C"
