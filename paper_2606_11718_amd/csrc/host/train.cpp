#include "train.hpp"

#include <algorithm>

namespace ccl {

namespace {

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups of `tiles` dealt to the 8 XCDs in runs of `chunk`.
int64_t dealt(int64_t tiles, int64_t chunk) { return 8 * chunk * up(tiles, 8 * chunk); }

}  // namespace

GroupedForm grouped_form(const GroupedShape& s, int64_t rows, int direction) {
  GroupedForm f;
  f.tile_m = f.tile_n = 128;
  f.chunk = 32;
  int64_t tiles;
  if (direction == GROUPED_WGRAD) {
    f.tiles_m = (int32_t)up(s.out, f.tile_m);
    f.tiles_n = (int32_t)up(s.in, f.tile_n);
    tiles = (int64_t)s.experts * f.tiles_m * f.tiles_n;
  } else {
    f.tiles_n = (int32_t)up(direction == GROUPED_FORWARD ? s.out : s.in, f.tile_n);
    // at most: every expert with rows has one tile that is not whole
    tiles = (rows / f.tile_m + std::min<int64_t>(s.experts, rows)) * f.tiles_n;
  }
  f.workgroups = dealt(tiles, f.chunk);
  return f;
}

}  // namespace ccl
