// Every tile of C exactly once, those with work in the first slots, over a
// range of plans: 0 on success.
#include <cstdio>
#include <vector>

#include "tile_map.hpp"

using namespace ccl;

int main() {
  for (int gr = 1; gr <= 8; gr *= 2)
    for (int gc = 1; gr * gc <= 8; gc *= 2)
      for (int tm : {1, 2, 3, 7, 16})
        for (int tn : {1, 2, 5, 40})
          for (int gm : {1, 4, 8}) {
            const int per = 8 / (gr * gc), rows = tm * gr, cols = tn * gc;
            const TileMap m = make_tile_map(per, gc, tm, tn, (tm * tn + per - 1) / per, gm, 1);
            for (int live = 1; live <= rows; ++live) {
              const LiveMap l = make_live_map(m, gr, live);
              std::vector<int> seen(rows * cols, 0);
              const int64_t grid = 8 * (int64_t)(l.live_per_xcd + l.rest_per_xcd);
              for (int64_t wg = 0; wg < grid; ++wg) {
                int pr, pc, ti, tj;
                if (!live_tile(l, wg, &pr, &pc, &ti, &tj)) continue;
                const bool in = pr >= 0 && pr < gr && pc >= 0 && pc < gc && ti >= 0 && ti < tm && tj >= 0 && tj < tn;
                if (!in || (pr * tm + ti < live) != ((wg >> 3) < l.live_per_xcd)) {
                  std::printf("grid %dx%d tiles %dx%d group %d live %d wg %lld\n", gr, gc, tm, tn, gm, live, (long long)wg);
                  return 1;
                }
                ++seen[(pr * tm + ti) * cols + pc * tn + tj];
              }
              for (int n : seen)
                if (n != 1) {
                  std::printf("grid %dx%d tiles %dx%d group %d live %d: a tile %d times\n", gr, gc, tm, tn, gm, live, n);
                  return 1;
                }
            }
          }
  return 0;
}
