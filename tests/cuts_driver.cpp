// How the wide walk's rounds are cut (pages.h), on the host: batches of walks of any lengths.
#include <algorithm>
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

struct Seq {
  int rounds, walks;
};

static unsigned state = 1;
static int random(int n) { return static_cast<int>((state = state * 1664525u + 1013904223u) >> 8) % n; }

// A call's choice, as the kernel makes it.
static void check(const std::vector<Seq> &seqs, int groups) {
  int all = 0, walks = 0, most = 0;
  for (const Seq &s : seqs) {
    all += s.rounds * s.walks;
    walks += s.rounds > 0 ? s.walks : 0;
    most = std::max(most, s.rounds);
  }
  const Cut c = cut_of(all, walks, most, groups);
  if (c.at(0) != c.lo || c.at(kCutTries - 1) != c.hi || c.lo < 1 || c.hi < c.lo) fail("order", c.lo, c.hi, groups);
  int per = c.hi;
  for (int k = kCutTries - 2; k >= 0; --k) {
    int n = 0;
    for (const Seq &s : seqs) n += pieces_of(s.rounds, c.at(k)) * s.walks;
    if (n <= groups) per = c.at(k);
  }
  int workgroups = 0, parts = 0;
  for (const Seq &s : seqs) {
    const int p = pieces_of(s.rounds, per);
    if (p > kMaxPieces) fail("pieces of a walk", p, s.rounds, per);
    workgroups += p * s.walks;
    parts += p > 1 ? p * s.walks : 0;
  }
  if (workgroups > std::max(groups, walks + groups / 2)) fail("workgroups", workgroups, walks, groups);
  if (parts > groups) fail("parts", parts, walks, groups);
  // nobody has far more to do than an even share
  const int share = (all + groups - 1) / groups, longest = (most + kMaxPieces - 1) / kMaxPieces;
  if (per > std::max(std::max(5 * share, longest), 1)) fail("longest piece", per, share, most);
}

int main() {
  for (int groups : {2, 3, 7, 60, 511, 512}) {
    // one long sequence among short ones, in any number
    for (int n = 1; n <= 300; ++n)
      for (int walks : {1, 2, 8, 24, 64}) {
        for (int longest : {1, 2, 65, 1024, 16000})
          for (int others : {0, 1, 8, 64}) {
            std::vector<Seq> seqs(n, Seq{others, walks});
            seqs[n / 2].rounds = longest;
            int most = 0, all = 0;
            for (const Seq &s : seqs) most += s.rounds > 0 ? s.walks : 0, all += s.rounds * s.walks;
            // a call that is cut has a workgroup a walk and half of all that run at once more, or one a round
            if (groups == 512 || all <= groups) check(seqs, groups);
          }
      }
    // anything
    for (int i = 0; i < 20000 && groups == 512; ++i) {
      std::vector<Seq> seqs(1 + random(200));
      const int heads = 1 + random(16), far = 1 + random(i % 3 ? 2000 : 40);
      for (Seq &s : seqs) s = Seq{random(far + 1), heads * (1 + random(1 + random(8)))};
      check(seqs, groups);
    }
  }
  std::printf("ok\n");
  return 0;
}
