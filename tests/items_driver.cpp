// Walks the wide walk's row tiles and workgroups (pages.h) on the host.
#include <cstdio>
#include <cstdlib>
#include <vector>

#define __host__
#define __device__
#define __forceinline__ inline
#include "pages.h"

using namespace graft;

static void fail(const char *what, long a, long b, long c) {
  std::printf("%s: %ld %ld %ld\n", what, a, b, c);
  std::exit(1);
}

int main() {
  // row tiles of whole waves, at most 128 rows, that cover the rows; the last one has some
  for (int rows = 1; rows < 5000; ++rows) {
    const int n = row_tiles_of(rows), h = height_of(rows);
    if (h % 32 != 0 || h < 32 || h > kWideRows) fail("height", rows, h, n);
    if (n * h < rows || (n - 1) * h >= rows) fail("cover", rows, h, n);
  }
  // every (unit, row tile) has one workgroup, and a unit's are 8 apart where there are eight units
  for (int row_tiles = 1; row_tiles < 12; ++row_tiles)
    for (int units = 1; units < 70; ++units) {
      std::vector<int> seen(units * row_tiles, 0);
      for (int at = 0; at < units * row_tiles; ++at) {
        const Item i = item_at(at, units, row_tiles);
        if (i.unit < 0 || i.unit >= units || i.tile_row < 0 || i.tile_row >= row_tiles) fail("item", at, units, row_tiles);
        if (place_of(i.unit, i.tile_row, units, row_tiles) != at) fail("place", at, units, row_tiles);
        if (seen[i.unit * row_tiles + i.tile_row]++) fail("twice", at, units, row_tiles);
        if (i.tile_row > 0 && i.unit / 8 < units / 8 && at - place_of(i.unit, i.tile_row - 1, units, row_tiles) != 8)
          fail("apart", at, units, row_tiles);
      }
    }
  std::printf("ok\n");
  return 0;
}
