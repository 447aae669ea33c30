// Checks of the attention's tile arithmetic (attend_tiles.h) on the host, and of the two walks'
// steps over it: parts take every tile once, an empty part loads nothing, whatever is loaded has
// keys left, and a buffer reaches neither past the keys nor below zero.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#define __host__
#define __device__
#define __forceinline__ inline
#include "attend_tiles.h"

using namespace graft;

namespace {

struct Case {
  int keys, turns, min_tiles, splits, c[3];
};
long loads = 0, empty_parts = 0;

void need(bool ok, const char *what, const Case &s, int part, int tile) {
  if (ok) return;
  std::printf("%s: keys %d turns %d at least %d splits %d sources %d %d %d part %d tile %d\n", what, s.keys,
              s.turns, s.min_tiles, s.splits, s.c[0], s.c[1], s.c[2], part, tile);
  std::exit(1);
}

// One tile's load at `at`, walked to as tile t.
void load(const Case &s, const Tiles &n, const Spot &at, int part, int t, std::vector<int> &seen) {
  ++loads;
  need(t >= 0 && t < n.all(), "load of no tile", s, part, t);
  const Spot want = spot_of(n, t, s.keys, s.c[0], s.c[1], s.c[2]);
  need(at.source == want.source && at.tile == want.tile && at.left == want.left, "walk left its tiles", s, part, t);
  need(at.left > 0, "load without keys", s, part, t);
  need(at.tile * s.keys + at.left == s.c[at.source], "keys left", s, part, t);
  const int take = at.left < s.keys ? at.left : s.keys;
  for (int row : {1, 32, 256, 1 << 23}) {
    const int last = row == 1 ? 1 : 32;
    const int bytes = extent(at.left, s.keys, row, last);
    need(bytes >= last && bytes == (take - 1) * row + last, "buffer's end", s, part, t);
    // a row behind the last starts past the end, where a load gives zeros
    need(static_cast<int64_t>(take) * row >= bytes, "row behind the last", s, part, t);
  }
  ++seen[t];
}

Spot on(Spot at, int tiles, int keys) {      // as the kernels' advance
  at.tile += tiles;
  at.left -= tiles * keys;
  return at;
}

void wide(const Case &s, const Tiles &n, int part, std::vector<int> &seen) {
  const Part p = part_of(n, part);
  if (!(p.first < p.last)) return;
  Spot at = spot_of(n, p.first, s.keys, s.c[0], s.c[1], s.c[2]);
  load(s, n, at, part, p.first, seen);
  for (int t = p.first; t < p.last; ++t)
    if (t + 1 < p.last) {
      at = at.left > s.keys ? on(at, 1, s.keys) : spot_of(n, t + 1, s.keys, s.c[0], s.c[1], s.c[2]);
      load(s, n, at, part, t + 1, seen);
    }
}

void narrow(const Case &s, const Tiles &n, int part, std::vector<int> &seen) {
  const Part p = part_of(n, part);
  const int prefix = n.n0 + n.n1, t_end = p.last < prefix ? p.last : prefix;
  for (int wave = 0; wave < s.turns; ++wave) {
    int t = p.first + wave, ahead = t;
    Spot at{};
    auto fetch = [&] {
      if (ahead >= t_end) return;
      if (ahead == p.first + wave || at.left <= s.turns * s.keys)
        at = spot_of(n, ahead, s.keys, s.c[0], s.c[1], s.c[2]);
      else
        at = on(at, s.turns, s.keys);
      load(s, n, at, part, ahead, seen);
      ahead += s.turns;
    };
    fetch();
    while (t < t_end) {
      fetch();
      t += s.turns;
    }
    if (t == prefix && t < p.last)
      load(s, n, spot_of(n, t, s.keys, s.c[0], s.c[1], s.c[2]), part, t, seen);
  }
}

}  // namespace

int main() {
  const int sizes[] = {0, 1, 31, 32, 33, 63, 64, 65, 128, 129, 300, 513, 1025};
  for (int left : {0, -1, -64, -4096})
    for (int row : {32, 256, 1 << 23})
      if (extent(left, 64, row, 32) != 0) {
        std::printf("a buffer without keys reaches %d bytes\n", extent(left, 64, row, 32));
        return 1;
      }
  for (int kind = 0; kind < 2; ++kind)
    for (int splits = 1; splits <= 64; splits += splits < 9 ? 1 : 11)
      for (int c0 : sizes)
        for (int c1 : sizes)
          for (int c2 : sizes) {
            if (kind && c2 > 32) continue;      // the narrow walk's blocks fit one tile
            const Case s{kind ? 32 : 64, kind ? 4 : 1, kind ? 1 : 4, splits, {c0, c1, c2}};
            const Tiles n = cut_tiles(c0, c1, c2, s.keys, s.turns, splits, s.min_tiles);
            std::vector<int> seen(n.all(), 0);
            int next = 0;
            for (int part = 0; part < splits; ++part) {
              const Part p = part_of(n, part);
              need(p.first == next && p.last >= p.first && p.last <= n.all(), "parts", s, part, p.first);
              next = p.last;
              empty_parts += p.first == p.last;
              if (kind) narrow(s, n, part, seen);
              else wide(s, n, part, seen);
            }
            need(next == n.all(), "tiles behind the last part", s, splits, next);
            for (int t = 0; t < n.all(); ++t) need(seen[t] == 1, "tile not walked once", s, -1, t);
          }
  std::printf("%ld loads, %ld empty parts\n", loads, empty_parts);
  return empty_parts > 0 ? 0 : 1;
}
