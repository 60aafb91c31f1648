// paged_cut.h -- into how many work items the rows of a paged attention call are
// cut.  Host and device code, no HIP header needed.
#pragma once
#include <stdint.h>

#ifndef SNAP_HD
#ifdef __HIPCC__
#define SNAP_HD __host__ __device__ inline
#else
#define SNAP_HD inline
#endif
#endif

namespace snap {

struct PagedCut {
  int waves;      // items that the card holds at once
  int target;     // items that the rows are cut into, besides one per unit at most
  int max_items;  // items at most
};

// blocks: of all units' rows at most
inline PagedCut paged_cut(int units, int waves, int64_t blocks) {
  PagedCut c;
  c.waves = waves;
  c.target = units < waves / 2 ? waves - units : waves / 2;
  // ceil(blocks / C) a unit, C >= blocks / target: at most target + units items,
  // and no more than there are blocks
  c.max_items = (int)(blocks < c.target + units ? blocks : c.target + units);
  return c;
}

// Blocks an item, C, for units of `total` blocks in all heads' turn (n sequences x
// heads units): as few as keep the items within `waves`.  total / waves of them may
// give more (a unit's last item is short), total / target never does; up to 64
// sequences some between are tried.  items(C): items of one head's units at C.
template <typename Items>
SNAP_HD int paged_chunk(int waves, int target, int n, int heads, int64_t total, Items items) {
  const int64_t t64 = total * heads;
  int64_t c64 = (t64 + target - 1) / target;
  if (n <= 64) {
    const int64_t least = (t64 + waves - 1) / waves, step = (c64 - least) / 4 + 1;
    for (int64_t c = least; c < c64; c += step) {
      if ((int64_t)heads * items((int)c) <= waves) {
        c64 = c;
        break;
      }
    }
  }
  return c64 < 1 ? 1 : (int)c64;
}

}  // namespace snap
