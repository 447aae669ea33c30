// Walks pages.h on the host: the division by a page's rows, and the tiles of a span against the
// rows that have to be in them.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

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
  // every page size at borders of pages, and around the largest rows
  for (int d = 1; d <= (1 << 20); d = d < 5000 ? d + 1 : d + 4999) {
    PageMap m{};
    m.page_rows = d;
    set_division(m);
    auto check = [&](uint32_t r) {
      if (m.entry(r) != static_cast<int>(r / d)) fail("division", r, d, m.entry(r));
    };
    for (uint32_t k = 0; k < 40; ++k)
      for (int e = -1; e <= 1; ++e) {
        const int64_t near = static_cast<int64_t>(k) * d + e, far = (0x7FFFFFFFll / d - k) * d + e;
        if (near >= 0 && near <= 0x7FFFFFFFll) check(static_cast<uint32_t>(near));
        if (far >= 0 && far <= 0x7FFFFFFFll) check(static_cast<uint32_t>(far));
      }
    check(0x7FFFFFFFu);
    for (uint32_t i = 0; i < 200; ++i) check((i * 2654435761u) >> 1);
  }
  // all spans of short sequences: the tiles ascend, hold every row that is seen, and no tile but for one
  for (int keys : {32, 64})
    for (int end = 0; end <= 300; end += end < 70 ? 1 : 7)
      for (int low = -3; low <= end + 3; low += low < 70 ? 1 : 5)
        for (int sinks : {0, 1, 4, 31, 32, 33, 64, 65, 100, 299, 300, 1000, 0x7FFFFFFF}) {
          const Span s = span_of(low, sinks, end, keys);
          static bool in[2000];
          for (bool &x : in) x = false;
          int before = -1;
          for (int t = 0; t < s.all(); ++t) {
            const int at = s.at(t);
            if (at <= before || at * keys >= end) fail("tile", end, low, sinks);
            before = at;
            bool used = false;
            for (int r = at * keys; r < (at + 1) * keys; ++r) {
              in[r] = true;
              used |= r < end && (r < sinks || r >= low);
            }
            // between the first rows and the window lies a tile that neither needs only where the two
            // touch it from both sides
            if (!used && s.n0 != 0 && low < end) fail("idle tile", end, low, sinks);
          }
          for (int r = 0; r < end; ++r)
            if ((r < sinks || r >= low) && !in[r]) fail("missing", r, low, sinks);
        }
  // a row tile's tiles against each of its slots' rows: all in, and in a clear tile all seen by all
  for (int base = 0; base <= 200; base += 9)
    for (int n : {1, 2, 7, 40, 70})
      for (int s0 = 0; s0 < n; s0 += 1 + n / 3)
        for (int s1 = s0; s1 < n; s1 += 1 + n / 4)
          for (int window : {0, 1, 5, 64, 100, 0x7FFFFFFF})
            for (int sinks : {0, 3, 40, 0x7FFFFFFF})
              for (bool masked : {false, true})
                for (int keys : {32, 64}) {
                  const RowTile t = row_tile(base, n, s0, s1, masked, window, sinks, keys);
                  auto holds = [&](int r) {
                    for (int i = 0; i < t.span.all(); ++i)
                      if (r / keys == t.span.at(i)) return true;
                    return false;
                  };
                  for (int slot = s0; slot <= s1; ++slot)
                    // a masked slot's position: any from base - 1 to base + slot
                    for (int place = masked ? -1 : slot; place <= slot; ++place)
                      for (int r = 0; r < base + n; ++r) {
                        const bool near = window == 0 || r > static_cast<int64_t>(base) + place - window || r < sinks;
                        const bool sees = r < base ? near : !masked && r <= base + slot && near;
                        if (sees && !holds(r)) fail("row not walked", base, slot, r);
                        const int j = r / keys * keys;
                        if (!sees && is_clear(t, j, keys, window > 0 ? sinks : 0) && place <= n - 1)
                          fail("tile not clear", base, slot, r);
                      }
                  if (masked)
                    for (int r = base; r < base + n; ++r)
                      if (!holds(r)) fail("slot not walked", base, n, r);
                }
  // pieces are in order, without gaps, and as even as whole tiles allow
  for (int n = 0; n <= 300; n += 7)
    for (int pieces = 1; pieces <= 128; ++pieces) {
      if (cut_at(n, pieces, 0) != 0 || cut_at(n, pieces, pieces) != n) fail("ends", n, pieces, 0);
      for (int p = 0; p < pieces; ++p) {
        const int d = cut_at(n, pieces, p + 1) - cut_at(n, pieces, p);
        if (d < n / pieces || d > (n + pieces - 1) / pieces) fail("piece", n, pieces, p);
      }
    }
  if (cut_at(1 << 25, 128, 127) != (1 << 25) / 128 * 127) fail("cut_at", 0, 0, 0);
  if (low_bits(-5) != 0 || low_bits(0) != 0 || low_bits(1) != 1 || low_bits(63) != ~0ull >> 1 ||
      low_bits(64) != ~0ull || low_bits(1000) != ~0ull)
    fail("low_bits", 0, 0, 0);
  if (window_low(10, 0) != 0 || window_low(10, 4) != 7 || window_low(3, 4) != 0 || window_low(3, 0x7FFFFFFF) != 0 ||
      window_low(1 << 30, 1) != 1 << 30)
    fail("window_low", 0, 0, 0);
  std::printf("ok\n");
  return 0;
}
