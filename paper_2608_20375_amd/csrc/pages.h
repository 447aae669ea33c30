// pages.h -- rows in pages: which page holds a sequence's row, and which keys a tile of rows of
// the paged attention walks.  Integers alone, the same for the kernels and for a host program
// that includes this.
#pragma once

#include <stdint.h>

namespace graft {

// Row r < 2^31 is in entry r / page_rows of its sequence's table.  With 2^(l-1) < page_rows <= 2^l
// the quotient is (r * mul) >> (31 + l), mul = ceil(2^(31 + l) / page_rows) <= 2^32 - 1: the
// product is off by r * e, e < page_rows <= 2^l, so by less than 2^(31 + l).
struct PageMap {
  const int32_t *table;
  int64_t table_stride;
  int32_t table_len, pages, page_rows;
  uint32_t mul;
  int32_t shift;
  __host__ __device__ __forceinline__ int entry(uint32_t r) const {
    return static_cast<int>((static_cast<uint64_t>(r) * mul) >> shift);
  }
  __host__ __device__ __forceinline__ int rows() const { return table_len * page_rows; }
};
inline void set_division(PageMap &m) {
  int l = 0;
  while ((int64_t{1} << l) < m.page_rows) ++l;
  m.shift = 31 + l;
  m.mul = static_cast<uint32_t>(((uint64_t{1} << m.shift) + m.page_rows - 1) / m.page_rows);
}

// The keys that a tile of query rows may see, rows [0, sinks) and [low, end), in tiles of `keys`
// keys that begin at multiples of it: the first n0 tiles, then n1 from tile `first` on.
struct Span {
  int n0, first, n1;
  __host__ __device__ __forceinline__ int all() const { return n0 + n1; }
  __host__ __device__ __forceinline__ int at(int t) const { return t < n0 ? t : first + t - n0; }
};
__host__ __device__ __forceinline__ Span span_of(int low, int sinks, int end, int keys) {
  low = low < 0 ? 0 : low > end ? end : low;
  const int s = sinks < end ? sinks : end;
  const int a = (s + keys - 1) / keys, b = low / keys;
  Span w;
  w.n0 = a < b ? a : 0;
  w.first = a < b ? b : 0;
  w.n1 = (end + keys - 1) / keys - w.first;
  return w;
}

// The first row that a window at position p shows.
__host__ __device__ __forceinline__ int window_low(int p, int window) {
  return window > 0 && p - window + 1 > 0 ? p - window + 1 : 0;
}

// What slots s0 .. s1 of a block of n slots walk, which lies behind `base` rows: the tiles, the rows'
// end, and the rows that every slot sees (those before clear_end that are from clear_low on, or
// among the sinks).  A chain's slot i is at position base + i; a masked one's position is at least
// base - 1 (it may see nothing) and at most base + n - 1.
struct RowTile {
  Span span;
  int end, clear_low, clear_end;
};
__host__ __device__ __forceinline__ RowTile row_tile(int base, int n, int s0, int s1, bool masked, int window,
                                                     int sinks, int keys) {
  RowTile t;
  t.end = masked ? base + n : base + s1 + 1;
  t.span = span_of(window_low(base + (masked ? -1 : s0), window), window > 0 ? sinks : 0, t.end, keys);
  t.clear_low = window_low(base + (masked ? n - 1 : s1), window);
  t.clear_end = masked ? base : base + s0 + 1;
  return t;
}

constexpr int kWideRows = 128;      // most rows of a row tile of the wide walk
// The row tiles of a sequence's query rows of a key head: the narrow walk's one; of the wide one's as few
// as 128 rows each allow, all of one size in whole waves (260 rows are three tiles of three waves, not two
// of four and a rest).
__host__ __device__ __forceinline__ int row_tiles_of(int rows) { return (rows + kWideRows - 1) / kWideRows; }
__host__ __device__ __forceinline__ int height_of(int rows) {
  const int waves = 32 * row_tiles_of(rows);
  return (rows + waves - 1) / waves * 32;
}
// A sequence's workgroups in the wide walk, units (pieces of key heads) x row tiles: a unit's row tiles
// follow each other on one XCD (workgroups go round all 8), whose L2 then holds the keys that they share.
// Eights of units, and what is left in the same way.
struct Item {
  int unit, tile_row;
};
__host__ __device__ __forceinline__ Item item_at(int at, int units, int row_tiles) {
  const int eight = at / (8 * row_tiles), base = 8 * eight, wide = (units - base < 8 ? units - base : 8), x = at - base * row_tiles;
  const int r = x / wide;
  return Item{base + x - r * wide, r};
}
__host__ __device__ __forceinline__ int place_of(int unit, int tile_row, int units, int row_tiles) {
  const int base = unit & ~7, wide = (units - base < 8 ? units - base : 8);
  return base * row_tiles + tile_row * wide + unit - base;
}

// Where piece p of `pieces` begins among a row tile's n tiles.
__host__ __device__ __forceinline__ int cut_at(int n, int pieces, int p) {
  return static_cast<int>(static_cast<int64_t>(n) * p / pieces);
}

// How the wide walk's workgroups share the rounds of all walks (a walk: a row tile's over the keys of its
// sequence and key head): one of more than `per` rounds is cut into ceil(rounds / per) even pieces.  per is the
// least of kCutTries between lo and hi for which all walks and pieces run at once, in `groups` workgroups; or hi.
//   lo: what a workgroup has to do if nothing were rounded up; a join holds kMaxPieces pieces.
//   hi: what fits into the workgroups that are not needed for walks, whatever is rounded up.  Where these are
//       less than a quarter hi would be large, and the longest walks would be walked alone: then twice an even share,
//       and not all run at once.
// Walks of more than twice an even share are less than groups / 2, and so are the pieces added to
// them: there are at most max(groups, walks + groups / 2) workgroups, and at most `groups` pieces of cut walks.
constexpr int kMaxPieces = 128;                   // of a row's keys: four a lane of the merge
constexpr int kCutTries = 4;
struct Cut {
  int lo, hi;
  __host__ __device__ __forceinline__ int at(int k) const { return lo + (hi - lo) * k / (kCutTries - 1); }
};
__host__ __device__ __forceinline__ int pieces_of(int rounds, int per) { return (rounds + per - 1) / per; }
// all: rounds of all walks; most: of the longest
__host__ __device__ __forceinline__ Cut cut_of(int all, int walks, int most, int groups) {
  const int share = pieces_of(all, groups), join = pieces_of(most, kMaxPieces), spare = groups - walks;
  Cut c;
  c.lo = share > join ? share : join;
  c.lo = c.lo > 1 ? c.lo : 1;
  c.hi = 4 * spare >= groups ? pieces_of(all, spare) : 2 * share;
  c.hi = c.hi < most ? c.hi : most;
  c.hi = c.hi > c.lo ? c.hi : c.lo;
  return c;
}

// Whether every slot of the tile sees all rows j .. j + keys - 1.
__host__ __device__ __forceinline__ bool is_clear(const RowTile &t, int j, int keys, int sinks) {
  return j + keys <= t.clear_end && (j >= t.clear_low || j + keys <= sinks);
}

// The lowest n of 64 bits.
__host__ __device__ __forceinline__ uint64_t low_bits(int n) {
  return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1;
}

}  // namespace graft
