// How conf_kv_constrain cuts a row of V logits into the ranges of its workgroups (plain arithmetic, no GPU needed).
// Logits are counted from the 16-byte boundary of the result at or ahead of the row's first one, `off` places ahead: range j
// is the logits of j range - off .. (j + 1) range - off - 1 that the row has.
#pragma once
#include <stdint.h>

namespace confkv {

constexpr int con_off(uintptr_t row) { return (int)((row >> 2) & 3); }
// Ranges that a row needs.  V is at most 2^27.
constexpr int con_ranges(int V, int off, int range) { return (V + off + range - 1) / range; }
// Ranges that the grid has: the most any of B rows needs, the first of which lies at `out`; whole: every row lies on a boundary.
constexpr int con_grid_ranges(uintptr_t out, int B, int V, int range, bool whole) {
  int most = con_ranges(V, 0, range);
  for (int b = 0; b < B && b < 4 && !whole; ++b) {       // (offsets repeat every four rows)
    const int n = con_ranges(V, con_off(out + (uintptr_t)b * V * 4), range);
    most = n > most ? n : most;
  }
  return most;
}
constexpr int con_first(int j, int off, int range) { return j * range - off; }
// A row that needs fewer ranges than the grid has none in the last of them: its workgroup must not count there, where the size
// below is not positive.
constexpr bool con_empty(int first, int V) { return first >= V; }
// Places of a range that begins at logit `first`, those ahead of the row included.
constexpr int con_size(int first, int V, int range) { return range < V - first ? range : V - first; }

}  // namespace confkv
