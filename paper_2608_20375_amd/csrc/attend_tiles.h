// attend_tiles.h -- the attention's key tiles: how a sequence's keys are cut into tiles and
// parts, where a tile's keys are, and how far a tile's buffer reaches.  Integers alone, the
// same for the kernels and for a host program that includes this.
#pragma once

namespace graft {

// Tiles of a sequence's keys: the shared prefix's (where it has no pass of its own), the
// cache's, the block's; and how many a part takes.  The walks and the merge agree on it.
struct Tiles {
  int n0, n1, n2, per;
  __host__ __device__ __forceinline__ int all() const { return n0 + n1 + n2; }
};
// c0, c1, c2 keys of the three sources in tiles of `keys`; at most `splits` parts of at least
// min_tiles rounds of `turns` tiles.
__host__ __device__ __forceinline__ Tiles cut_tiles(int c0, int c1, int c2, int keys, int turns, int splits,
                                                    int min_tiles) {
  Tiles t;
  t.n0 = (c0 + keys - 1) / keys;
  t.n1 = (c1 + keys - 1) / keys;
  t.n2 = (c2 + keys - 1) / keys;
  const int rounds = (t.all() + turns - 1) / turns;
  const int per = (rounds + splits - 1) / splits;
  t.per = (per < min_tiles ? min_tiles : per) * turns;
  return t;
}

// Tiles [first, last) of a part.  Parts that a short sequence does not need are empty: first ==
// last, which is then the number of all tiles and no tile's.
struct Part {
  int first, last;
};
__host__ __device__ __forceinline__ Part part_of(const Tiles &t, int part) {
  const int n = t.all();
  Part p;
  p.first = part * t.per < n ? part * t.per : n;
  p.last = p.first + t.per < n ? p.first + t.per : n;
  return p;
}

// Tile t < t.all() of the walk: its source, its number there and the keys from its first on,
// at least one.
struct Spot {
  int source, tile, left;
};
__host__ __device__ __forceinline__ Spot spot_of(const Tiles &n, int t, int keys, int c0, int c1, int c2) {
  Spot s;
  s.source = t < n.n0 ? 0 : t < n.n0 + n.n1 ? 1 : 2;
  s.tile = s.source == 0 ? t : s.source == 1 ? t - n.n0 : t - n.n0 - n.n1;
  s.left = (s.source == 0 ? c0 : s.source == 1 ? c1 : c2) - s.tile * keys;
  return s;
}

// Bytes from a tile's first key to the end of its last: `left` keys, of which a tile takes `keys`,
// `row` bytes apart and `last` long.  0 without keys: a bound below 0 would be one of 4 GB.
__host__ __device__ __forceinline__ int extent(int left, int keys, int row, int last) {
  const int n = left < keys ? left : keys;
  return n > 0 ? (n - 1) * row + last : 0;
}

}  // namespace graft
