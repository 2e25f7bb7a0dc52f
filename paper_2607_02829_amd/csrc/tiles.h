// Order in which the workgroups of a GEMM take the tiles of its output.
#pragma once
#include "common.h"

namespace sr {

// Workgroups are handed to the eight XCDs round-robin by linear id.  Renumber them so that each
// XCD owns a contiguous range of tiles, and walk tiles in groups of GM tile rows (column by
// column within a group), so the tiles that one XCD runs together share A rows and B columns in
// its L2.  Split-K index outermost.
constexpr int GM = 8;
SR_DEV void tile_coords(int bid, int nwg, int tiles_m, int tiles_n, int& tm, int& tn, int& split) {
  const int x = bid & 7, q = nwg >> 3, rem = nwg & 7;
  const int t = x * q + min(x, rem) + (bid >> 3);
  const int per = tiles_m * tiles_n;
  split = t / per;
  const int u = t - split * per;
  const int grp = u / (GM * tiles_n);
  const int first = grp * GM;
  const int gm = min(GM, tiles_m - first);
  const int v = u - first * tiles_n;
  tm = first + v % gm;
  tn = v / gm;
}

}  // namespace sr
