// How paged attention calls are cut into work items (csrc/paged_cut.h) for the host
// tests.
#include "paged_cut.h"

extern "C" void paged_cut_of(int units, int waves, long long blocks, int* o) {
  const snap::PagedCut c = snap::paged_cut(units, waves, blocks);
  o[0] = c.target;
  o[1] = c.max_items;
}

// The blocks an item of a call of n sequences with nb[i] blocks each.
extern "C" int paged_chunk_of(int waves, int target, int n, int heads, const int* nb) {
  long long total = 0;
  for (int i = 0; i < n; ++i) total += nb[i];
  return snap::paged_chunk(waves, target, n, heads, total, [&](int c) {
    int items = 0;
    for (int i = 0; i < n; ++i) items += c > 0 ? (nb[i] + c - 1) / c : 0;
    return items;
  });
}
