// k_paged_attend.hip -- attention of a block over a cache in pages, the block's own rows among
// them, with a sliding window and first rows that stay visible.
//
//   o_i = sum_j p_ij v_j / l_i,  p_ij = exp2(c (s_ij - m_i)),  s_ij = q_i . k_j,
//   m_i = max_j s_ij,  l_i = sum_j p_ij,  c = scale log2 e,
// in one pass over the rows that a tile of query rows may see, with a running maximum and sum.
// Rows, products, the second product's operand and the reference of the probabilities are as in
// k_attend.hip: the query heads of a key head are rows beside each other (row = slot * group +
// head of the group), S^T = K Q^T puts a query into a lane, O^T = V^T P^T takes its own
// probabilities as they are and V^T by the transposing LDS read.
//
// Pages.  A lane looks up the page of a key of its own, a tile ahead, and the others' come by lane
// exchanges, so pages of any length work and may end inside a tile.  Addresses are 64 bits, an
// offset inside a page 32.  Rows past a tile's end are loaded from its last row again, rows of
// pages that the pool does not have from page 0: both are hidden.  Tiles also hold rows that no
// query sees (next to a window, behind the first rows), whose pages may be gone: a page is reported
// where a query sees a row of it.
//
// Two walks.  Up to 16 rows a key head (single tokens, short chains) keys are read once and a
// wave's own: narrow_part, bound by memory.  More rows share keys through LDS: wide_part, bound by
// matrix, vector, LDS and load work that two waves a SIMD do not quite overlap.  Rounds of the narrow
// walk are shared evenly over the chip, of the wide one the longest walks are cut, as the lengths on
// the device say, and merge_pages_kernel joins what was cut.
// Measured (in a graph, clocks settled, 32/8 heads of 128, the join included): 64 tokens over up to 8192 e4m3
// rows 109 us for 584 MB (5.4 TB/s), over bf16 rows 195 us for 1158 MB (5.9 TB/s); 32 windows of 4096 over up
// to 16384 rows 93 us for 504 MB (5.4 TB/s; plain reads of as large pieces reach 5.8, 6.6 non-temporal); 16
// trees of up to 64 nodes over up to 4096 rows 80 us for 30 GFLOP and 167 MB; 8 pieces of 1024 prompt
// rows, windows of 2048, 331 us for 257 GFLOP (774 TFLOP/s); one token over 700 rows 13 us, two launches
// and their dependent loads.
//
// Hidden keys.  A tile whose keys all query rows see (most of them) takes no masks.  In the others
// a score that a row does not see becomes -inf, and infinite and NaN values are stored as 0, since
// 0 times them is NaN; where there were any, what the rows that see them get is added after.
#include <algorithm>
#include <type_traits>

#include "attend_device.h"
#include "graft_internal.h"
#include "pages.h"

namespace graft {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kWideKeys = 64;                     // wide_part
constexpr int kFewRows = 16, kFewKeys = 32;       // narrow_part; keys of one wave's tile
constexpr int kWideBlocks = 512;                  // two a CU
constexpr int kLongRounds = 64;                   // of a walk that is left whole where row tiles fill the chip
constexpr int kMergeBlocks = 4096;                // of a merge of twice as much and more, which mostly finds nothing to do

struct Pool {                 // keys or values of one layer; bytes
  const char *p;
  const uint8_t *s;
  int64_t page, head, s_page, s_head;
  uint32_t row, s_row;
};

struct PagedArgs {
  Pool k, v;
  PageMap pages;
  const char *q;
  char *out;
  int64_t q_batch, q_slot, q_head, o_batch, o_slot, o_head;   // bytes
  const int32_t *n_nodes, *cache_len;
  const uint64_t *mask;
  float *lse;
  float *part_o;          // [parts][batch * slots * q_heads][head_dim], unnormalised
  f32x2 *part_ml;         // [parts][batch * slots * q_heads] reference, sum
  uint32_t *error_flag;
  int32_t batch, slots, root, q_heads, kv_heads, group, dim;
  int32_t n_max, words, window, sinks;
  int32_t joins;          // rows of cut walks and others, in the merge's workgroups
  int32_t tile_rows, row_tiles;   // rows of the narrow walk's tile; most row tiles of a sequence and key head
  int32_t cut;            // wide: walks may be cut; 0: a workgroup for each row tile's whole walk
  int32_t *share;         // rounds of a workgroup (0: nothing is to be joined), then [batch] each sequence's first
                          // round or workgroup
  float c;
};

// The arguments, read again where they are used: what a loop does not use would otherwise be kept over
// it in scalar registers, which spill into vector ones, lane by lane.
typedef const __attribute__((address_space(4))) PagedArgs Late;
__device__ __forceinline__ const PagedArgs &late() {
  Late *p = (Late *)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const PagedArgs *)p;
}

// Slots and cache length of sequence b as the kernels use them.
struct Sizes {
  int n, len;
  bool bad;
};
__device__ __forceinline__ Sizes sizes_of(const PagedArgs &a, int b) {
  Sizes s;
  const int most = a.slots - a.root, n = a.n_nodes ? a.n_nodes[b] : most, len = a.cache_len[b];
  s.n = (n < 0 ? 0 : n > most ? most : n) + a.root;
  const int cap = a.pages.rows() - s.n;
  s.len = len < 0 ? 0 : len > cap ? cap : len;
  s.bad = n < 0 || n > most || len < 0 || len > cap;
  return s;
}

// Slots 64 * word .. + 63 of the block that a slot sees under the mask.
__device__ __forceinline__ uint64_t mask_word(const PagedArgs &a, int b, int slot, int word, int n) {
  const int node = slot - a.root;
  uint64_t w;
  if (node < 0) {
    w = word == 0 ? 1 : 0;
  } else {
    const uint64_t *m = a.mask + (static_cast<int64_t>(b) * a.n_max + node) * a.words;
    w = word < a.words ? m[word] : 0;
    if (a.root) w = (w << 1) | (word == 0 ? 1 : word <= a.words ? m[word - 1] >> 63 : 0);
  }
  return w & low_bits(n - word * 64);
}

// A query row's view: rows before `end`, from `low` on or among the sinks, and what its mask shows.
struct View {
  int slot, low, end;
};
__device__ __forceinline__ View view_of(const PagedArgs &a, int b, int slot, int len, int n) {
  View v;
  v.slot = slot;
  int place = slot;
  if (a.mask && a.window > 0) {
    place = -1;
    for (int w = 0; w * 64 < n; ++w) place += __popcll(mask_word(a, b, slot, w, n));
  }
  v.low = window_low(len + place, a.window);
  v.end = a.mask ? len : len + slot + 1;
  return v;
}
// Of keys j .. j + 63 those that the row sees.
__device__ __forceinline__ uint64_t seen_bits(const PagedArgs &a, int b, const View &v, int j, int len, int n) {
  uint64_t w = low_bits(v.end - j) & (low_bits(a.sinks - j) | ~low_bits(v.low - j));
  const int s = j - len;
  if (a.mask && s > -64 && s < n) {
    if (s < 0) {
      w |= mask_word(a, b, v.slot, 0, n) << -s;
    } else {
      w |= mask_word(a, b, v.slot, s >> 6, n) >> (s & 63);
      if (s & 63) w |= mask_word(a, b, v.slot, (s >> 6) + 1, n) << (64 - (s & 63));
    }
  }
  return w;
}

// Where a lane's key is.
struct Spot {
  int page;         // one of the pool's
  uint32_t off;     // row in it
  bool bad;         // the table names none of the pool's
};
__device__ __forceinline__ int entry_at(const PagedArgs &a, const int32_t *table, int j, int end) {
  return table[a.pages.entry(static_cast<uint32_t>(j < end ? j : end - 1))];
}
__device__ __forceinline__ Spot spot_at(const PagedArgs &a, int page, int j, int end) {
  const int r = j < end ? j : end - 1;
  Spot s;
  s.off = static_cast<uint32_t>(r - a.pages.entry(static_cast<uint32_t>(r)) * a.pages.page_rows);
  s.bad = static_cast<uint32_t>(page) >= static_cast<uint32_t>(a.pages.pages);
  s.page = s.bad ? 0 : page;
  return s;
}
// Bytes from a head's first row in page 0.
__device__ __forceinline__ int64_t row_at(const Pool &p, const Spot &s) {
  return s.page * p.page + static_cast<uint64_t>(s.off * p.row);
}
__device__ __forceinline__ int64_t scale_at(const Pool &p, const Spot &s) {
  return s.page * p.s_page + static_cast<uint64_t>(s.off * p.s_row);
}
__device__ __forceinline__ u32x4 take16(const char *p) { return *reinterpret_cast<const u32x4 *>(p); }
__device__ __forceinline__ u32x4 stream16(const char *p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
}

__device__ __forceinline__ int64_t read_lane64(int64_t x, int lane) {
  const uint64_t u = static_cast<uint64_t>(x);
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(u), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(u >> 32), lane);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// Both 16-lane rows' values of a lane's column: x of lane col (+ 32) and of lane col + 16 (+ 32).
__device__ __forceinline__ u32x2 both_rows(uint32_t x) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x, x, false, false));
}
// Lanes 8 .. 15 of every 16 get y of lanes 0 .. 7, the others keep x; and the other way round.
__device__ __forceinline__ uint32_t upper_from(uint32_t x, uint32_t y) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(static_cast<int>(x), static_cast<int>(y), 0x128, 0xF, 0xC, false));
}
__device__ __forceinline__ uint32_t lower_from(uint32_t x, uint32_t y) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(static_cast<int>(x), static_cast<int>(y), 0x128, 0xF, 0x3, false));
}
// The x of keys 8 u + lane % 8, u < 4, where lane l holds key l % 32's.
__device__ __forceinline__ u32x4 of_eights(uint32_t x) {
  const u32x2 r = both_rows(x);
  return u32x4{upper_from(r.x, r.x), lower_from(r.x, r.x), upper_from(r.y, r.y), lower_from(r.y, r.y)};
}

// Waits for all memory operations.  With a store in flight the compiler takes loads to come back in any
// order, and every wait for one of them to be a wait for all: a loop that keeps loads in flight begins without.
__device__ __forceinline__ void drain() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// Four numbers of the values' row of key j, for rows that see infinite or NaN ones.
template <typename T, bool Q8>
__device__ __forceinline__ u32x2 four_at(const PagedArgs &a, const char *v_head, const uint8_t *vs_head, const Spot &s, int x) {
  const char *p = v_head + row_at(a.v, s);
  if (!Q8) return *reinterpret_cast<const u32x2 *>(p + 2 * x);
  const uint32_t unit = vs_head[scale_at(a.v, s)];
  return widen(*reinterpret_cast<const uint32_t *>(p + x), unit_of(unit));
}

// Rows of a row in the outputs.
__device__ __forceinline__ void finish(const PagedArgs &a, int64_t all, float m, float l, float at) {
  a.lse[all] = l == 0.0f ? -INFINITY : (m * a.c + (__log2f(l) - at)) * 0.69314718055994531f;
}

// Up to 16 rows, all of a sequence's and key head's, over tiles t0 .. t1 - 1: every wave walks 32-key tiles of
// its own, keys from memory straight into fragments, values through a stretch of LDS of the wave's
// own, no barriers; the waves' sums are joined at the end.  A tile is in flight while the one before it is
// worked on.  The loads alone, with nothing done to what they bring, take 107 of 125 us of 64
// tokens over e4m3 rows and 90 of 97 of the windows (before the clocks settle); two tiles in flight and 3
// or 4 waves a SIMD gained
// nothing.
// part: where in the workspace the sums go, or -1: they are all there is.
template <typename T, bool Q8, bool HOT, int DP>
__device__ __forceinline__ void narrow_part(const PagedArgs &a, int b, int kvh, int live, int len, const RowTile &tile, int t0,
                                            int t1, int part, u32x4 *lds) {
  constexpr int C = DP / 8, kSteps = DP / 32, kDTiles = DP / 16;
  constexpr int kLoads = Q8 ? DP / 64 : kSteps;         // 16-byte loads of a lane and 16 keys
  constexpr int kBytes = Q8 ? 1 : 2;
  constexpr int kPad = DP + 4;                          // floats of a row when the waves are joined
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));     // a piece's own: what follows from it is not kept over all pieces
  const int lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int quarter = lane >> 4, col = lane & 15;
  u32x4 *s_v = lds + wave * kFewKeys * C;

  // slot and query head of row i
  auto place = [&](const PagedArgs &z, int i, int *slot, int *head) {
    const int rows = live * z.group, row = i < rows ? i : rows - 1;
    *slot = row / z.group;
    *head = kvh * z.group + row - *slot * z.group;
    return i < rows;
  };

  // Contracted entries 8 of a step are chunk k_chunk(step) of a row: the 16 codes that one
  // load brings are two steps' 8.
  auto k_chunk = [&](int s) { return Q8 ? 2 * (4 * (s / 2) + quarter) + s % 2 : 4 * s + quarter; };
  u32x4 rq[kSteps];
  {
    const PagedArgs &z = late();
    int slot, head;
    place(z, col, &slot, &head);
    const char *qp = z.q + b * z.q_batch + slot * z.q_slot + head * z.q_head;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      rq[s] = HOT || k_chunk(s) * 8 < z.dim ? take16(qp + k_chunk(s) * 16) : u32x4{0, 0, 0, 0};
  }

  const int32_t *table = a.pages.table + b * a.pages.table_stride;
  const char *k_head = a.k.p + kvh * a.k.head, *v_head = a.v.p + kvh * a.v.head;
  const uint8_t *ks_head = a.k.s + kvh * a.k.s_head, *vs_head = a.v.s + kvh * a.v.s_head;
  const int mine = lane & 31;                           // the key of a tile whose page this lane looks up

  // Loads of a tile.  A cache line is 128 bytes, and a load of 16 rows of 64 would bring each line
  // for one half of it, the other coming 16 loads later: so a load takes whole lines of 8 rows, lane
  // (quarter, col) chunk quarter + 4 (col / 8) of row 8 u + col % 8 (the windows 103 -> 96 us).  The
  // values go to LDS as they come; two loads' keys change halves (col's and col + 8's) to be rows col
  // of chunks quarter and quarter + 4.  Rows of 64 bytes are taken 16 at a time.  Keys are read once:
  // the loads are non-temporal (random 4 KB pieces are read at 6.6 TB/s so, at 5.8 without).
  constexpr bool kLines = kLoads > 1;
  constexpr int kSets = kLines ? 4 : 2, kEach = kLines ? kLoads / 2 : 1;   // rows of a lane, loads of a row
  const int mine_ch = kLines ? quarter + (col >> 3) * 4 : quarter, mine_row = kLines ? col & 7 : col;
  struct Held {                                         // a tile on its way
    u32x4 rk[kSets][kEach], rv[kSets][kEach];
    uint32_t sk[2], sv[2];                              // scales of rows col and 16 + col
    int j;                                              // first key
    uint32_t bad;                                       // keys on pages that there are none of
  };
  // The loads are made in every step, past the end of the last tile's again: a load that is only made
  // sometimes would have to be waited for with all those before it.
  //
  // HOT: pages of 16 rows or a multiple, so that a tile's halves lie in a page each, and keys and values
  // at the same places of their pools.  Lanes 0 .. 31 work out where the first half begins, the others the
  // second; a lane's own rows are at offsets that never change.
  uint32_t lane_off[2] = {0, 0}, scale_off = 0;
  if (HOT) {
#pragma unroll
    for (int s = 0; s < 2; ++s) lane_off[s] = (8 * s + mine_row) * a.k.row + mine_ch * 16;
    scale_off = col * a.k.s_row;
  }
  const int64_t to_v = v_head - k_head, to_vs = vs_head - ks_head;
  int ahead = t0 + wave;                                // the tile to load next
  int next = 0;                                         // this lane's page of it
  uint32_t next_off = 0;                                // and row there
  auto tile_at = [&](int t) { return tile.span.at(t < t1 ? t : t1 - 1) * kFewKeys; };
  auto look_up = [&](int t) {
    const int j = tile_at(t);
    if (HOT) {
      const uint32_t r = lane < 32 || j + 16 >= tile.end ? j : j + 16;
      const int e = a.pages.entry(r);
      next_off = r - e * a.pages.page_rows;
      next = table[e];
    } else {
      next = entry_at(a, table, j + mine, tile.end);
    }
  };
  look_up(ahead);
  // where the next tile's rows are: worked out before the last loads are waited for
  struct Where {
    const char *k[2];
    const uint8_t *s[2];
    int64_t at;
    int64_t s_at;
    int j;
    uint32_t bad;
  };
  auto find = [&](Where &w) {
    w.j = tile_at(ahead);
    if (HOT) {
      Spot s;
      s.bad = static_cast<uint32_t>(next) >= static_cast<uint32_t>(a.pages.pages);
      s.page = s.bad ? 0 : next;
      s.off = next_off;
      const uint64_t bad = __ballot(s.bad);
      w.bad = (bad & 1 ? 0xFFFFu : 0u) | (bad >> 63 ? 0xFFFF0000u : 0u);
      const int64_t at = row_at(a.k, s), s_at = Q8 ? scale_at(a.k, s) : 0;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        w.k[kt] = k_head + read_lane64(at, 32 * kt);
        w.s[kt] = Q8 ? ks_head + read_lane64(s_at, 32 * kt) : nullptr;
      }
    } else {
      const Spot s = spot_at(a, next, w.j + mine, tile.end);
      w.bad = static_cast<uint32_t>(__ballot(s.bad));
      w.k[0] = k_head + row_at(a.k, s);                 // this lane's
      w.at = row_at(a.v, s);
      if (Q8) {
        w.s[0] = ks_head + scale_at(a.k, s);
        w.s_at = scale_at(a.v, s);
      }
    }
    look_up(ahead + kWaves);
    ahead += kWaves;
  };
  // a side's loads: `p` is where key `mine` lies
  auto side = [&](const char *p, u32x4 (&r)[kSets][kEach]) {
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = static_cast<uint32_t>(at), hi = static_cast<uint32_t>(at >> 32);
    u32x4 l4, h4;
    if (kLines) {
      l4 = of_eights(lo);
      h4 = of_eights(hi);
    } else {
      const u32x2 l2 = both_rows(lo), h2 = both_rows(hi);
      l4 = u32x4{l2.x, l2.y, 0, 0};
      h4 = u32x4{h2.x, h2.y, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
      const char *q = reinterpret_cast<const char *>(static_cast<uint64_t>(h4[u]) << 32 | l4[u]);
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int c0 = (8 * i + mine_ch) * 16;
        r[u][i] = stream16(q + (c0 < kBytes * a.dim ? c0 : 0));
      }
    }
  };
  // The next tile's keys, and then its values, into the registers that are free of the last ones.
  auto fetch_keys = [&](Held &x, const Where &w) {
    x.j = w.j;
    x.bad = w.bad;
    if (HOT) {
#pragma unroll
      for (int kt = 0; kt < 2 && Q8; ++kt) {
        x.sk[kt] = w.s[kt][scale_off];
        x.sv[kt] = (w.s[kt] + to_vs)[scale_off];
      }
#pragma unroll
      for (int u = 0; u < kSets; ++u)
#pragma unroll
        for (int i = 0; i < kEach; ++i) x.rk[u][i] = stream16(w.k[kLines ? u / 2 : u] + lane_off[kLines ? u % 2 : 0] + 128 * i);
    } else {
      if (Q8) {
        x.sk[0] = *w.s[0];                              // of row `mine`
        x.sv[0] = vs_head[w.s_at];
      }
      side(w.k[0], x.rk);
    }
  };
  auto fetch_values = [&](Held &x, const Where &w) {
    if (HOT) {
#pragma unroll
      for (int u = 0; u < kSets; ++u)
#pragma unroll
        for (int i = 0; i < kEach; ++i)
          x.rv[u][i] = stream16(w.k[kLines ? u / 2 : u] + to_v + lane_off[kLines ? u % 2 : 0] + 128 * i);
    } else {
      side(v_head + w.at, x.rv);
    }
  };

  f32x4 o[kDTiles];
  float m, l;
  Ref ref;                      // of m
  m = -INFINITY;
  l = 0.0f;
  ref = ref_of<T>(m, a.c);
#pragma unroll
  for (int d = 0; d < kDTiles; ++d) o[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  auto step = [&](Held &x) {
    const int j = x.j;
    const uint32_t bad = x.bad;
    const bool clear = bad == 0 && is_clear(tile, j, kFewKeys, a.sinks);
    Where w;
    find(w);
    __builtin_amdgcn_sched_barrier(0);
    uint32_t unit_k[2] = {x.sk[0], x.sk[1]}, unit_v[2] = {x.sv[0], x.sv[1]};
    if (Q8 && !HOT) {
      const u32x2 sk = both_rows(x.sk[0]), sv = both_rows(x.sv[0]);
      unit_k[0] = sk.x;
      unit_k[1] = sk.y;
      unit_v[0] = sv.x;
      unit_v[1] = sv.y;
    }
    f32x4 s[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const float uk = Q8 ? unit_of(unit_k[kt]) : 0.0f;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        u32x4 r = x.rk[kt][0];
        if (kLines) {
          const u32x4 &lo = x.rk[2 * kt][i / 2], &hi = x.rk[2 * kt + 1][i / 2];
#pragma unroll
          for (int y = 0; y < 4; ++y) r[y] = i % 2 == 0 ? upper_from(lo[y], hi[y]) : lower_from(hi[y], lo[y]);
        }
        u32x4 f[2];
        if (Q8) {
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const u32x2 z = widen(r[y], uk);
            f[y / 2][2 * (y % 2)] = z.x;
            f[y / 2][2 * (y % 2) + 1] = z.y;
          }
        } else {
          f[0] = r;
        }
        // past the head's numbers the queries hold zeros, which an infinite key would not leave so
        if (!HOT && (4 * i + quarter) * 16 >= kBytes * a.dim) f[0] = f[1] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int y = 0; y < (Q8 ? 2 : 1); ++y)
          s[kt] = T::mfma(f[y], rq[Q8 ? 2 * i + y : i], s[kt]);
      }
    }
    fetch_keys(x, w);
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
      const int r = (kLines ? 8 : 16) * u + mine_row;
      float uv = 0.0f;
      if (Q8) {
        const uint32_t z = unit_v[kLines ? u / 2 : u];
        uv = unit_of(!kLines ? z : u % 2 == 0 ? upper_from(z, z) : lower_from(z, z));
      }
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int c0 = 8 * i + mine_ch;
        if (Q8) {
          u32x4 f[2];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const u32x2 z = widen(x.rv[u][i][y], uv);
            f[y / 2][2 * (y % 2)] = z.x;
            f[y / 2][2 * (y % 2) + 1] = z.y;
          }
          s_v[v_at<C>(r, 2 * c0)] = f[0];
          s_v[v_at<C>(r, 2 * c0 + 1)] = f[1];
        } else {
          s_v[v_at<C>(r, c0)] = x.rv[u][i];
        }
      }
    }
    // before the next tile's loads take their registers
    bool odd = false;
    uint32_t seen = 0;
    if (__builtin_expect(!clear, 0)) {
      const PagedArgs &z = late();
#pragma unroll 1
      for (int i = lane; i < kFewKeys * C; i += kWave) {
        u32x4 w = s_v[i];
        if (tame<T>(w)) {
          s_v[i] = w;
          odd = true;
        }
      }
      int slot, head;
      place(z, col, &slot, &head);
      seen = static_cast<uint32_t>(seen_bits(z, b, view_of(z, b, slot, len, live), j, len, live));
      if ((seen & bad) != 0) atomicOr(z.error_flag, kErrPage);
      seen &= ~bad;
      const uint32_t bits = seen >> (4 * quarter);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        s[i / 4][i % 4] = (bits >> (16 * (i / 4) + i % 4)) & 1u ? s[i / 4][i % 4] : -INFINITY;
      drain();
    }
    fetch_values(x, w);
    // The tile's scores into the running sums, its values being in LDS.  The wave's LDS
    // operations are done in order.
    float mx = s[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[i / 4][i % 4]);
    mx = quarter_max(mx);
    const bool up = __builtin_fmaf(mx, ref.c, ref.off) > T::kLift + T::kSlack;   // as in softmax_step
    if (__ballot(up) != 0) {
      const Ref now = ref_of<T>(up ? mx : m, a.c);
      const float alpha = up ? factor(m, ref.at, mx, now, a.c) : 1.0f;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < kDTiles; ++d) o[d] *= alpha;
      m = up ? mx : m;
      ref = now;
    }
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][i % 4], ref.c, ref.off));
    l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
    const u32x4 p = u32x4{T::pack(e[0], e[1]), T::pack(e[2], e[3]), T::pack(e[4], e[5]), T::pack(e[6], e[7])};
    __builtin_amdgcn_wave_barrier();
    const int vr = 4 * quarter + (col >> 2);
#pragma unroll
    for (int d = 0; d < kDTiles; ++d) {
      typedef __attribute__((address_space(3))) s16x4 *at;
      const char *vp = reinterpret_cast<const char *>(s_v + v_at<C>(vr, 2 * d + ((col & 3) >> 1))) + (col & 1) * 8;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(vp)));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(vp + 16 * C * 16)));
      o[d] = T::mfma(u32x4{lo.x, lo.y, hi.x, hi.y}, p, o[d]);
    }
    __builtin_amdgcn_wave_barrier();
    if (__builtin_expect(__ballot(odd) != 0, 0)) {
      const PagedArgs &z = late();
      const char *v_at0 = z.v.p + kvh * z.v.head;
      const uint8_t *vs_at0 = z.v.s + kvh * z.v.s_head;
#pragma unroll 1
      for (int y = 0; y < kFewKeys && j + y < tile.end; ++y) {
        const Spot sp = spot_at(z, entry_at(z, z.pages.table + b * z.pages.table_stride, j + y, tile.end), j + y, tile.end);
#pragma unroll
        for (int d = 0; d < kDTiles; ++d) {
          const int c0 = d * 16 + 4 * quarter;
          u32x2 w{0, 0};
          if (((seen >> y) & 1) && c0 < z.dim) w = four_at<T, Q8>(z, v_at0, vs_at0, sp, c0);
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const uint16_t n = static_cast<uint16_t>(w[h / 2] >> (16 * (h & 1)));
            o[d][h] += (n & T::kExp) == T::kExp ? T::number(n) : 0.0f;
          }
        }
      }
    }
  };
  Held x;
  drain();
  {
    Where w;
    find(w);
    fetch_keys(x, w);
    fetch_values(x, w);
  }
  for (int t = t0 + wave; t < t1; t += kWaves) step(x);

  // The four waves' rows: each leaves its own with its maximum and sum, then every thread
  // joins 4 numbers of a row, the waves in order.
  const PagedArgs &z = late();
  float *s_o = reinterpret_cast<float *>(lds);
  float *s_m = s_o + kWaves * 16 * kPad, *s_l = s_m + kWaves * 16;
  __syncthreads();
  l = quarter_sum(l);
  if (quarter == 0) {
    s_m[wave * 16 + col] = m;
    s_l[wave * 16 + col] = l;
  }
#pragma unroll
  for (int d = 0; d < kDTiles; ++d)
    *reinterpret_cast<f32x4 *>(s_o + (wave * 16 + col) * kPad + d * 16 + 4 * quarter) = o[d];
  __syncthreads();
  for (int u = tid; u < 16 * (DP / 4); u += kThreads) {
    const int r = u / (DP / 4), c0 = (u % (DP / 4)) * 4;
    int slot, head;
    if (!place(z, r, &slot, &head) || c0 >= z.dim) continue;
    float top = s_m[r];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) top = fmaxf(top, s_m[i * 16 + r]);
    const Ref now = ref_of<T>(top, z.c);
    f32x4 sum{0.0f, 0.0f, 0.0f, 0.0f};
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const float mi = s_m[i * 16 + r];
      const float f = mi == top ? 1.0f : factor(mi, ref_of<T>(mi, z.c).at, top, now, z.c);
      total += s_l[i * 16 + r] * f;
      sum += *reinterpret_cast<const f32x4 *>(s_o + (i * 16 + r) * kPad + c0) * f;
    }
    const int64_t all = (static_cast<int64_t>(b) * z.slots + slot) * z.q_heads + head;
    if (part >= 0) {
      const int64_t at = part * static_cast<int64_t>(kFewRows) + r;
      if (c0 == 0) z.part_ml[at] = f32x2{top, total};
      *reinterpret_cast<f32x4 *>(z.part_o + at * z.dim + c0) = sum;
    } else {
      const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
      *reinterpret_cast<u32x2 *>(z.out + b * z.o_batch + slot * z.o_slot + head * z.o_head + 2 * c0) =
          u32x2{T::pack(sum.x * inv, sum.y * inv), T::pack(sum.z * inv, sum.w * inv)};
      if (z.lse && c0 == 0) finish(z, all, top, total, now.at);
    }
  }
}

// A sequence's row tile.
template <bool WIDE>
__device__ __forceinline__ RowTile tile_of(const PagedArgs &a, int n, int len, int tile_row) {
  const int rows = n * a.group, height = WIDE ? height_of(rows) : 0, first = tile_row * height;
  return row_tile(len, n, WIDE ? first / a.group : 0, WIDE ? (std::min(first + height, rows) - 1) / a.group : n - 1,
                  a.mask != nullptr, a.window, a.sinks, WIDE ? kWideKeys : kFewKeys);
}
// The rounds that it takes for each of its key heads: of four 32-key tiles in the narrow walk, of a
// 64-key tile of the last row tile in the wide one.
template <bool WIDE>
__device__ __forceinline__ int rounds_of(const PagedArgs &a, int n, int len) {
  if (n == 0) return 0;
  const int tiles = tile_of<WIDE>(a, n, len, WIDE ? row_tiles_of(n * a.group) - 1 : 0).span.all();
  return WIDE ? tiles : (tiles + kWaves - 1) / kWaves;
}
// How all rounds are shared.  A thread's sequences are c of them from tid * c on; sums over the workgroup.
template <int N>
struct Sum {
  int before[N], all[N], most;      // in front of the thread's, all, and the largest of `most`
};
// each_wave: all waves have all sequences, and none waits for another.
template <int N>
__device__ __forceinline__ Sum<N> sum_over(const int (&mine)[N], int most, int *s_sum, bool each_wave = false) {
  const int wave = threadIdx.x / kWave;
  Sum<N> s;
#pragma unroll
  for (int i = 0; i < N; ++i) s.before[i] = wave_incl_scan(mine[i]);
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) most = std::max(most, static_cast<int>(xor_lane(static_cast<uint32_t>(most), k)));
  if (each_wave) {
    s.most = __builtin_amdgcn_readfirstlane(most);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s.all[i] = static_cast<int>(__builtin_amdgcn_readlane(static_cast<uint32_t>(s.before[i]), kWave - 1));
      s.before[i] -= mine[i];
    }
    return s;
  }
  __syncthreads();
  if (lane_id() == kWave - 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) s_sum[wave * (N + 1) + i] = s.before[i];
    s_sum[wave * (N + 1) + N] = most;
  }
  __syncthreads();
  s.most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    s.before[i] -= mine[i];
    s.all[i] = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int x = s_sum[w * (N + 1) + i];
      s.before[i] += w < wave ? x : 0;
      s.all[i] += x;
    }
    // the same in all threads: scalars, so that the walk's tables stay scalar
    s.all[i] = __builtin_amdgcn_readfirstlane(s.all[i]);
  }
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s.most = std::max(s.most, s_sum[w * (N + 1) + N]);
  s.most = __builtin_amdgcn_readfirstlane(s.most);
  __syncthreads();
  return s;
}
// A sequence's share: slots, length, rounds of a walk, and walks (key heads and, in the wide walk, row tiles).
struct Share {
  int n, len, rounds, walks;
};
template <bool WIDE>
__device__ __forceinline__ Share share_of(const PagedArgs &a, int b) {
  const Sizes s = sizes_of(a, b);
  if (s.bad && blockIdx.x == 0) atomicOr(a.error_flag, kErrBlockSizes);
  return Share{s.n, s.len, rounds_of<WIDE>(a, s.n, s.len), a.kv_heads * (WIDE ? row_tiles_of(s.n * a.group) : 1)};
}
// of(b, share) for the thread's sequences; the first of them, and up to 256 the only one, is `first`.
template <bool WIDE, typename Of>
__device__ __forceinline__ void each_share(const PagedArgs &a, int b0, int b1, const Share &first, Of of) {
  if (b0 < b1) of(b0, first);
  for (int b = b0 + 1; b < b1; ++b) of(b, share_of<WIDE>(a, b));
}

// The narrow walk's workgroups share all rounds of (sequence, key head, round) evenly, in that order,
// whatever the sequences' lengths: the chip is full until the end.  A workgroup's first piece may be the
// end of a (sequence, key head), its last one a begin: these two go to the workspace, whole ones to the
// outputs.  Every workgroup adds up the rounds in front of its own.
template <typename Piece>
__device__ __forceinline__ void share_rounds(const PagedArgs &a, int *s_sum, Piece piece) {
  const int tid = threadIdx.x, group = blockIdx.x, groups = gridDim.x;
  const int c = (a.batch + kThreads - 1) / kThreads, b0 = tid * c, b1 = std::min(b0 + c, a.batch);
  const Share mine = b0 < b1 ? share_of<false>(a, b0) : Share{0, 0, 0, 0};
  int rounds[1] = {0}, most = 0;
  each_share<false>(a, b0, b1, mine, [&](int, const Share &s) {
    rounds[0] += s.rounds * s.walks;
    most = std::max(most, s.rounds);
  });
  const Sum<1> sum = sum_over(rounds, most, s_sum);
  const int per = std::max((sum.all[0] + groups - 1) / groups, (sum.most + kMaxPieces - 2) / (kMaxPieces - 1));
  const int first = group * per, last = std::min(first + per, sum.all[0]);
  // where the workgroup's first round is, and for the merge where each sequence begins
  int next = sum.before[0];
  each_share<false>(a, b0, b1, mine, [&](int b, const Share &s) {
    if (group == 0) a.share[1 + b] = next;
    if (first >= next && first < next + s.rounds * s.walks) {
      s_sum[0] = b;
      s_sum[1] = next;
      s_sum[2] = s.n;
      s_sum[3] = s.len;
    }
    next += s.rounds * s.walks;
  });
  if (group == 0 && tid == 0) a.share[0] = per;
  __syncthreads();
  if (first >= last) return;
  int b = __builtin_amdgcn_readfirstlane(s_sum[0]), begin = __builtin_amdgcn_readfirstlane(s_sum[1]);
  int n = __builtin_amdgcn_readfirstlane(s_sum[2]), len = __builtin_amdgcn_readfirstlane(s_sum[3]);
  for (int at = first;;) {
    const int r = rounds_of<false>(a, n, len), end = begin + r * a.kv_heads;
    const RowTile tile = tile_of<false>(a, n, len, 0);
    while (at < last && at < end) {
      const int kvh = (at - begin) / r, unit = begin + kvh * r, stop = std::min(unit + r, last);
      const bool whole = unit >= first && unit + r <= last;
      const int part = whole ? -1 : 2 * group + (unit >= first ? 1 : 0);
      __syncthreads();
      piece(b, kvh, n, len, tile, (at - unit) * kWaves, std::min((stop - unit) * kWaves, tile.span.all()), part);
      at = stop;
    }
    if (at >= last) return;
    begin = end;
    ++b;
    const Sizes s = sizes_of(a, b);
    n = __builtin_amdgcn_readfirstlane(s.n);
    len = __builtin_amdgcn_readfirstlane(s.len);
  }
}

// In the wide walk a (sequence, key head) of r rounds is cut into ceil(r / per) even pieces, each a unit
// with a workgroup for every row tile; a row tile's own tiles are cut in that proportion.  A lone piece
// goes to the outputs, the others' sums to the workspace, one place behind the other.  cut_of has what per is.
// Where not all workgroups run at once those of what is cut come first: they are the longest (64 trees of
// up to 64 nodes, the last of them over 65,536 rows and the others over 500: 188 us, 240 in order; but three
// pieces of 400 prompt rows, which all run at once, 102 in order and 113).  (Shared as in the narrow walk, two
// pieces a workgroup begin and end there, and a begin costs three latencies.)
struct Wide {             // what a workgroup of the wide walk does, if t0 < t1
  int b, kvh, n, len, tile_row, t0, t1, part;
  RowTile tile;
};
__device__ __forceinline__ Wide cut_rounds(const PagedArgs &a, int *s_sum) {
  const int tid = threadIdx.x, me = blockIdx.x, groups = std::min<int>(gridDim.x, kWideBlocks);
  const bool each_wave = a.batch <= kWave;
  const int c = (a.batch + kThreads - 1) / kThreads, b0 = each_wave ? std::min(lane_id(), a.batch) : tid * c,
            b1 = std::min(b0 + c, a.batch);
  const Share mine = b0 < b1 ? share_of<true>(a, b0) : Share{0, 0, 0, 0};
  int work[2] = {0, 0}, most = 0;
  each_share<true>(a, b0, b1, mine, [&](int, const Share &s) {
    work[0] += s.rounds * s.walks;
    work[1] += s.walks;
    most = std::max(most, s.rounds);
  });
  const Sum<2> sum = sum_over(work, most, s_sum, each_wave);
  const Cut cut = cut_of(sum.all[0], sum.all[1], sum.most, groups);
  int tried[kCutTries] = {};
  each_share<true>(a, b0, b1, mine, [&](int, const Share &s) {
#pragma unroll
    for (int k = 0; k < kCutTries; ++k) tried[k] += pieces_of(s.rounds, cut.at(k)) * s.walks;
  });
  const Sum<kCutTries> counts = sum_over(tried, 0, s_sum, each_wave);
  int per = cut.hi;
#pragma unroll
  for (int k = kCutTries - 2; k >= 0; --k) per = counts.all[k] <= groups ? cut.at(k) : per;
  int sizes[2] = {0, 0};                                      // workgroups, and those of what is cut
  each_share<true>(a, b0, b1, mine, [&](int, const Share &s) {
    const int p = pieces_of(s.rounds, per) * s.walks;
    sizes[0] += p;
    sizes[1] += s.rounds > per ? p : 0;
  });
  const Sum<2> units = sum_over(sizes, 0, s_sum, each_wave);
  const bool crowded = units.all[0] > groups;
  int next = units.before[0], place = units.before[1];
  each_share<true>(a, b0, b1, mine, [&](int b, const Share &s) {
    const int size = pieces_of(s.rounds, per) * s.walks, from = !crowded ? next : s.rounds > per ? place : units.all[1] + next - place;
    if (me == 0) a.share[1 + b] = place;
    if (me >= from && me < from + size) {
      s_sum[0] = b;
      s_sum[1] = from;
      s_sum[2] = s.n;
      s_sum[3] = s.len;
      s_sum[4] = s.rounds > per ? place : -1;
    }
    next += size;
    place += s.rounds > per ? size : 0;
  });
  if (me == 0 && tid == 0) a.share[0] = units.all[1] > 0 ? per : 0;
  Wide w;
  w.t0 = w.t1 = 0;
  if (me >= units.all[0]) return w;
  __syncthreads();
  w.b = __builtin_amdgcn_readfirstlane(s_sum[0]);
  w.n = __builtin_amdgcn_readfirstlane(s_sum[2]);
  w.len = __builtin_amdgcn_readfirstlane(s_sum[3]);
  const int from = __builtin_amdgcn_readfirstlane(s_sum[1]), part = __builtin_amdgcn_readfirstlane(s_sum[4]);
  const int pieces = pieces_of(rounds_of<true>(a, w.n, w.len), per);
  const Item item = item_at(me - from, pieces * a.kv_heads, row_tiles_of(w.n * a.group));
  const int p = item.unit % pieces;
  w.kvh = item.unit / pieces;
  w.tile_row = item.tile_row;
  w.tile = tile_of<true>(a, w.n, w.len, item.tile_row);
  const int all = w.tile.span.all();
  w.t0 = cut_at(all, pieces, p);
  w.t1 = cut_at(all, pieces, p + 1);
  w.part = part < 0 ? -1 : part + me - from;
  __syncthreads();
  return w;
}
// A workgroup for each row tile's whole walk.
__device__ __forceinline__ Wide whole_walk(const PagedArgs &a) {
  const Item item = item_at(blockIdx.x, a.batch * a.kv_heads, a.row_tiles);
  Wide w;
  w.t0 = w.t1 = 0;
  w.tile_row = item.tile_row;
  w.b = item.unit / a.kv_heads;
  w.kvh = item.unit - w.b * a.kv_heads;
  const Sizes s = sizes_of(a, w.b);
  if (s.bad && item.tile_row == 0 && w.kvh == 0 && threadIdx.x == 0) atomicOr(a.error_flag, kErrBlockSizes);
  w.n = __builtin_amdgcn_readfirstlane(s.n);
  w.len = __builtin_amdgcn_readfirstlane(s.len);
  if (item.tile_row >= row_tiles_of(w.n * a.group)) return w;
  w.tile = tile_of<true>(a, w.n, w.len, item.tile_row);
  w.t1 = w.tile.span.all();
  w.part = -1;
  return w;
}

// N products whose fragments are read kAhead products before they are used.  Left to itself the compiler
// reads a fragment right in front of its product, and the wave waits for LDS every time (8 pieces of 1024
// slots 355 us; 370, 348, 343, 344 and 346 with fragments 1, 2, 3, 4 and 6 products ahead).
constexpr int kAhead = 3;
template <int N, typename Read, typename Product>
__device__ __forceinline__ void pipelined(Read read, Product product) {
  u32x4 f[kAhead];
#pragma unroll
  for (int n = 0; n < kAhead; ++n) f[n] = read(n);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    product(n, f[n % kAhead]);
    if (n + kAhead < N) f[n % kAhead] = read(n + kAhead);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// 128 rows a workgroup, 32 a wave; 64-key tiles in LDS for all four waves, the next tile's loads
// in flight in registers meanwhile, two LDS buffers, one barrier a tile.  A step of two waves a SIMD is 2050
// cycles of matrix work in 4280 (8 pieces of 1024 slots); 1300 of them go by while a wave issues its eight
// loads behind the barrier, where all waves issue theirs.  Loads straight to LDS, and the next tile's
// products beside this tile's exponentials, came to the same time within 1%.
template <typename T, bool Q8, bool HOT, int DP>
__device__ __forceinline__ void wide_part(const PagedArgs &a, int b, int kvh, int live, int len, int tile_row, const RowTile &tile,
                                          int t0, int t1, int part, u32x4 *lds) {
  constexpr int C = DP / 8;                             // 16-byte chunks of a row in LDS
  constexpr int kSteps = DP / 16, kDTiles = DP / 32;
  constexpr int kBuf = kWideKeys * C;                   // a buffer of keys, or of values
  constexpr int kBytes = Q8 ? 1 : 2;
  constexpr int kPer = C * kBytes / 2;                  // threads of a key
  constexpr int kStep = kThreads / kPer, kUnits = kWideKeys / kStep;
  u32x4 *s_k = lds, *s_v = lds + 2 * kBuf;

  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));     // a piece's own, as in narrow_part
  const int lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int h = lane >> 5, col = lane & 31;

  const int rows = live * a.group, local = wave * 32 + col, height = height_of(rows), first = tile_row * height;
  const bool valid = local < height && first + local < rows;
  const int row = valid ? first + local : rows - 1;
  const int slot = row / a.group, head = kvh * a.group + row - slot * a.group;
  const bool busy = __ballot(valid) != 0;

  const int32_t *table = a.pages.table + b * a.pages.table_stride;
  const char *k_head = a.k.p + kvh * a.k.head, *v_head = a.v.p + kvh * a.v.head;
  const uint8_t *ks_head = a.k.s + kvh * a.k.s_head, *vs_head = a.v.s + kvh * a.v.s_head;

  // A thread's share of a tile: 16 bytes of rows r0, r0 + kStep, ...  Lane l works out where key l lies.
  // HOT: a wave's rows of a unit lie in one page, in 16 rows from a multiple of 16 on; in the last tile
  // they may be the page's rows behind the end, or 16 rows with the last one again.
  const int r0 = tid / kPer, ch = tid % kPer;
  const int at16 = HOT || ch * 16 < kBytes * a.dim ? ch * 16 : 0;
  constexpr int kWaveRows = kWave / kPer;
  const uint32_t lane_off = (lane / kPer + (wave * kWaveRows & 15)) * a.k.row + ch * 16;
  const int64_t to_v = v_head - k_head, to_vs = vs_head - ks_head;
  u32x4 rk[kUnits], rv[kUnits];
  uint32_t sk = 0, sv = 0;                              // scales of key `lane`
  int held_j = 0, next = 0;
  uint32_t next_off = 0;
  uint64_t held_bad = 0;
  auto look_up = [&](int t) {
    const int j = tile.span.at(t) * kWideKeys + lane;
    const uint32_t r = j < tile.end ? j : HOT ? (tile.end - 1) & ~15 : tile.end - 1;
    const int e = a.pages.entry(r);
    next_off = r - e * a.pages.page_rows;
    next = table[e];
  };
  look_up(t0);
  auto load = [&](int t) {
    held_j = tile.span.at(t) * kWideKeys;
    Spot s;
    s.bad = static_cast<uint32_t>(next) >= static_cast<uint32_t>(a.pages.pages);
    s.page = s.bad ? 0 : next;
    s.off = next_off;
    held_bad = __ballot(s.bad);
    if (HOT) {
      const int64_t at = row_at(a.k, s);
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const char *p = k_head + read_lane64(at, (wave * kWaveRows & ~15) + i * kStep);
        rk[i] = take16(p + lane_off);
        rv[i] = take16(p + to_v + lane_off);
      }
      if (Q8) {
        const uint8_t *p = ks_head + scale_at(a.k, s);
        sk = *p;
        sv = p[to_vs];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int from = 4 * (r0 + i * kStep);
        Spot r;
        r.page = __builtin_amdgcn_ds_bpermute(from, s.page);
        r.off = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(from, static_cast<int>(s.off)));
        rk[i] = take16(k_head + row_at(a.k, r) + at16);
        rv[i] = take16(v_head + row_at(a.v, r) + at16);
      }
      if (Q8) {
        sk = ks_head[scale_at(a.k, s)];
        sv = vs_head[scale_at(a.v, s)];
      }
    }
    look_up(t + 1 < t1 ? t + 1 : t);
  };
  // Stores the share; true if a value is infinite or NaN where not all rows see the keys (stored
  // as 0 then).
  auto store = [&](int buf, bool clear) {
    bool odd = false;
    u32x4 *k = s_k + buf * kBuf, *v = s_v + buf * kBuf;
    const bool past = !HOT && ch * 16 >= kBytes * a.dim;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int r = r0 + i * kStep;
      if (Q8) {
        const float uk = unit_of(static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(4 * r, static_cast<int>(sk))));
        const float uv = unit_of(static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(4 * r, static_cast<int>(sv))));
        u32x4 f[2];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const u32x2 z = widen(rk[i][y], uk);
          f[y / 2][2 * (y % 2)] = z.x;
          f[y / 2][2 * (y % 2) + 1] = z.y;
        }
        if (past) f[0] = f[1] = u32x4{0, 0, 0, 0};
        k[k_at<C>(r, 2 * ch)] = f[0];
        k[k_at<C>(r, 2 * ch + 1)] = f[1];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const u32x2 z = widen(rv[i][y], uv);
          f[y / 2][2 * (y % 2)] = z.x;
          f[y / 2][2 * (y % 2) + 1] = z.y;
        }
        v[v_at<C>(r, 2 * ch)] = f[0];
        v[v_at<C>(r, 2 * ch + 1)] = f[1];
      } else {
        if (past) rk[i] = u32x4{0, 0, 0, 0};
        k[k_at<C>(r, ch)] = rk[i];
        v[v_at<C>(r, ch)] = rv[i];
      }
    }
    if (__builtin_expect(!clear, 0)) {
#pragma unroll 1
      for (int i = 0; i < kUnits * (Q8 ? 2 : 1); ++i) {
        u32x4 *at = v + (Q8 ? v_at<C>(r0 + i / 2 * kStep, 2 * ch + i % 2) : v_at<C>(r0 + i * kStep, ch));
        u32x4 w = *at;
        if (tame<T>(w)) {
          *at = w;
          odd = true;
        }
      }
    }
    return odd;
  };

  // the queries: the right operand of S^T = K Q^T
  u32x4 rq[kSteps];
  const char *qp = late().q + b * late().q_batch + slot * late().q_slot + head * late().q_head;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) rq[s] = s * 16 < a.dim ? take16(qp + s * 32 + h * 16) : u32x4{0, 0, 0, 0};
  load(t0);
#pragma unroll
  for (int s = 0; s < kSteps; ++s) settle(rq[s]);

  Sums<DP> st;
  st.clear(a.c);
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1, j = held_j;
    const uint64_t bad = held_bad;
    const bool clear = bad == 0 && is_clear(tile, j, kWideKeys, a.sinks);
    const bool odd = store(buf, clear);
    if (t + 1 < t1) load(t + 1);
    bool any_odd = false;
    if (!clear) any_odd = __syncthreads_or(odd);
    else __syncthreads();
    if (!busy) continue;
    const u32x4 *k = s_k + buf * kBuf, *v = s_v + buf * kBuf;
    f32x16 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] = 0.0f;
    // products go first, so that the other wave of the SIMD does its vector work in their time (with the
    // sum made early: 8 pieces of 1024 slots 341 -> 334 us, 16 trees of up to 64 nodes 91 -> 85)
    __builtin_amdgcn_s_setprio(1);
    pipelined<2 * kSteps>([&](int n) { return k[k_at<C>(n % 2 * 32 + col, n / 2 * 2 + h)]; },
                          [&](int n, const u32x4 &f) { s[n % 2] = T::mfma(f, rq[n / 2], s[n % 2]); });
    __builtin_amdgcn_s_setprio(0);
    uint64_t seen = ~0ull;
    if (__builtin_expect(!clear, 0)) {
      const PagedArgs &z = late();
      seen = seen_bits(z, b, view_of(z, b, slot, len, live), j, len, live);
      if ((seen & bad) != 0) atomicOr(z.error_flag, kErrPage);
      seen &= ~bad;
      const uint64_t bits = seen >> (4 * h);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const uint32_t x = static_cast<uint32_t>(bits >> (32 * kt));
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kt][i] = (x >> (8 * (i / 4) + i % 4)) & 1u ? s[kt][i] : -INFINITY;
      }
    }
    u32x4 p[4];
    softmax_step<T, 2>(st, s, p, a.c);
    // the sum is made here: made where it is next needed, 32 probabilities would be kept over the products
    asm volatile("" : "+v"(st.l));
    __builtin_amdgcn_s_setprio(1);
    // four tiles of columns in turn: a product does not wait for the one before it
    pipelined<4 * kDTiles>([&](int n) { return v_fragment<C>(v, n % kDTiles, n / kDTiles, lane); },
                           [&](int n, const u32x4 &f) { st.o[n % kDTiles] = T::mfma(f, p[n / kDTiles], st.o[n % kDTiles]); });
    __builtin_amdgcn_s_setprio(0);
    if (__builtin_expect(any_odd, 0)) {
      const PagedArgs &z = late();
      const char *v_at0 = z.v.p + kvh * z.v.head;
      const uint8_t *vs_at0 = z.v.s + kvh * z.v.s_head;
#pragma unroll 1
      for (int y = 0; y < kWideKeys && j + y < tile.end; ++y) {
        const Spot sp = spot_at(z, entry_at(z, z.pages.table + b * z.pages.table_stride, j + y, tile.end), j + y, tile.end);
#pragma unroll
        for (int d = 0; d < kDTiles; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int c0 = d * 32 + 8 * i + 4 * h;
            u32x2 w{0, 0};
            if (((seen >> y) & 1) && c0 < z.dim) w = four_at<T, Q8>(z, v_at0, vs_at0, sp, c0);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const uint16_t n = static_cast<uint16_t>(w[x / 2] >> (16 * (x & 1)));
              st.o[d][4 * i + x] += (n & T::kExp) == T::kExp ? T::number(n) : 0.0f;
            }
          }
      }
    }
  }

  st.l = half_sum(st.l);
  if (!valid) return;
  const PagedArgs &z = late();
  const int64_t all = (static_cast<int64_t>(b) * z.slots + slot) * z.q_heads + head;
  if (part >= 0) {
    const int64_t at = part * static_cast<int64_t>(kWideRows) + local;
    if (h == 0) z.part_ml[at] = f32x2{st.m, st.l};
    float *po = z.part_o + at * z.dim;
#pragma unroll
    for (int d = 0; d < kDTiles; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int x = d * 32 + 8 * i + 4 * h;
        if (x < z.dim)
          *reinterpret_cast<f32x4 *>(po + x) =
              f32x4{st.o[d][4 * i], st.o[d][4 * i + 1], st.o[d][4 * i + 2], st.o[d][4 * i + 3]};
      }
    return;
  }
  const float inv = st.l > 0.0f || st.l != st.l ? 1.0f / st.l : 0.0f;
  char *op = z.out + b * z.o_batch + slot * z.o_slot + head * z.o_head;
#pragma unroll
  for (int d = 0; d < kDTiles; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = d * 32 + 8 * i + 4 * h;
      if (x < z.dim)
        *reinterpret_cast<u32x2 *>(op + 2 * x) =
            u32x2{T::pack(st.o[d][4 * i] * inv, st.o[d][4 * i + 1] * inv),
                  T::pack(st.o[d][4 * i + 2] * inv, st.o[d][4 * i + 3] * inv)};
    }
  if (z.lse && h == 0) finish(z, all, st.m, st.l, ref_of<T>(st.m, z.c).at);
}

// HOT: heads of DP numbers and
// pages of 16 rows or a multiple.  Others' loads past a head's end go to its begin, and every row
// has an address of its own: more registers and vector work.
template <typename T, bool Q8, bool HOT, int DP, bool WIDE>
__global__ void __launch_bounds__(kThreads, 2)
paged_attend_kernel(PagedArgs a) {
  constexpr int kNarrow = (kWaves * 16 * (DP + 4) + 2 * kWaves * 16 + 3) / 4;   // joining the waves
  constexpr int kValues = kWaves * kFewKeys * (DP / 8);
  __shared__ __align__(16) u32x4 lds[WIDE ? 4 * kWideKeys * (DP / 8) : (kNarrow > kValues ? kNarrow : kValues)];
  int *s_sum = reinterpret_cast<int *>(lds);
  if constexpr (!WIDE) {
    share_rounds(a, s_sum, [&](int b, int kvh, int n, int len, const RowTile &tile, int t0, int t1, int part) {
      narrow_part<T, Q8, HOT, DP>(a, b, kvh, n, len, tile, t0, t1, part, lds);
    });
  } else {
    const Wide w = a.cut ? cut_rounds(a, s_sum) : whole_walk(a);
    if (w.t0 < w.t1) wide_part<T, Q8, HOT, DP>(a, w.b, w.kvh, w.n, w.len, w.tile_row, w.tile, w.t0, w.t1, w.part, lds);
  }
}

// Joins the pieces of a row: 32 lanes each, four pieces a lane for the statistics, four numbers a lane
// for the row.  A workgroup has rows of one slot, so that sizes and shares are scalars (16 trees of up to 64
// nodes, rows of two or three pieces: 16.3 -> 13.4 us).  The rows' first pieces loaded beside the statistics
// gained 0.1 us for one token and cost the trees 1.
template <typename T, bool WIDE>
__device__ __forceinline__ void join_rows(const PagedArgs &a, int block, int per) {
  constexpr int kHeads = kThreads / 32;
  const int lane = lane_id(), l32 = lane & 31;
  const int head_blocks = (a.q_heads + kHeads - 1) / kHeads, bs = block / head_blocks;
  const int b = bs / a.slots, slot = bs - b * a.slots;
  const Sizes sz = sizes_of(a, b);
  if (slot >= sz.n) return;
  const int head = (block - bs * head_blocks) * kHeads + threadIdx.x / 32;
  if (head >= a.q_heads) return;
  const int64_t r = static_cast<int64_t>(bs) * a.q_heads + head;
  const int kvh = head / a.group, row = slot * a.group + head - kvh * a.group;
  const int height = WIDE ? height_of(sz.n * a.group) : a.tile_rows, tile_row = row / height, local = row - tile_row * height;
  const int row_tiles = row_tiles_of(sz.n * a.group);
  const int rounds = rounds_of<WIDE>(a, sz.n, sz.len);
  int g0, pieces;
  if (WIDE) {
    pieces = pieces_of(rounds, per);
    g0 = kvh * pieces;                                        // the first unit
  } else {
    const int unit = a.share[1 + b] + kvh * rounds;
    g0 = unit / per;
    pieces = (unit + rounds - 1) / per - g0 + 1;
  }
  if (pieces == 1) return;                                  // the only one wrote the row
  const int tiles = WIDE ? tile_of<true>(a, sz.n, sz.len, tile_row).span.all() : 0;
  // where piece p's sums are; narrow: the first one is its group's last piece, the others are first ones
  auto at = [&](int p) {
    return WIDE ? static_cast<int64_t>(a.share[1 + b] + place_of(g0 + p, tile_row, pieces * a.kv_heads, row_tiles)) * kWideRows + local
                : static_cast<int64_t>(2 * (g0 + p) + (p == 0 ? 1 : 0)) * a.tile_rows + local;
  };
  // a piece that cut_at leaves nothing, there being fewer tiles than pieces, was not written
  auto some = [&](int p) { return p < pieces && (!WIDE || tiles >= pieces || cut_at(tiles, pieces, p) < cut_at(tiles, pieces, p + 1)); };
  f32x2 ml[4];
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int p = l32 + 32 * k;
    ml[k] = 32 * k < pieces && some(p) ? a.part_ml[at(p)] : f32x2{-INFINITY, 0.0f};
    top = fmaxf(top, ml[k].x);
  }
#pragma unroll
  for (int k = 1; k < 32; k <<= 1) top = fmaxf(top, __uint_as_float(xor_lane(__float_as_uint(top), k)));
  // 0 for a piece without keys that the row sees
  const Ref now = ref_of<T>(top, a.c);
  float w[4], l = 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    w[k] = ml[k].x == top && top != -INFINITY ? 1.0f : factor(ml[k].x, ref_of<T>(ml[k].x, a.c).at, top, now, a.c);
    l += w[k] * ml[k].y;
  }
#pragma unroll
  for (int k = 1; k < 32; k <<= 1) l += __uint_as_float(xor_lane(__float_as_uint(l), k));
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  f32x4 x{0.0f, 0.0f, 0.0f, 0.0f};
  const bool mine = l32 * 4 < a.dim;
  const float *o = a.part_o + (mine ? l32 * 4 : 0);
  for (int p0 = 0; p0 < pieces; p0 += 4) {
    f32x4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const f32x4 *>(o + at(std::min(p0 + k, pieces - 1)) * a.dim);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int p = p0 + k;
      const float f = __shfl(p < 32 ? w[0] : p < 64 ? w[1] : p < 96 ? w[2] : w[3], (lane & 32) + (p & 31));
      if (p < pieces && f != 0.0f) x += v[k] * f;           // what was not written has no weight
    }
  }
  if (mine)
    *reinterpret_cast<u32x2 *>(a.out + b * a.o_batch + slot * a.o_slot + head * a.o_head + l32 * 8) =
        u32x2{T::pack(x.x * inv, x.y * inv), T::pack(x.z * inv, x.w * inv)};
  if (a.lse && l32 == 0) finish(a, r, top, l, now.at);
}
// MANY: of calls with many row tiles, which mostly cut none.
template <typename T, bool WIDE, bool MANY>
__global__ void __launch_bounds__(kThreads)
merge_pages_kernel(PagedArgs a) {
  const int per = a.share[0];
  if (per == 0) return;
  if constexpr (MANY) {
    for (int block = blockIdx.x; block < a.joins; block += gridDim.x) join_rows<T, WIDE>(a, block, per);
  } else {
    join_rows<T, WIDE>(a, blockIdx.x, per);
  }
}

Pool pool_of(const graft_rows &r, int bytes) {
  Pool p;
  p.p = static_cast<const char *>(r.data);
  p.page = r.batch_stride * bytes;
  p.row = static_cast<uint32_t>(r.row_stride * bytes);
  p.head = r.head_stride * bytes;
  p.s = r.scale;
  p.s_page = r.scale_batch_stride;
  p.s_row = static_cast<uint32_t>(r.scale_row_stride);
  p.s_head = r.scale_head_stride;
  return p;
}

}  // namespace

PagedPlan paged_plan(const graft_paged_attention_desc &a) {
  PagedPlan p{};
  const int group = a.q_heads / a.kv_heads;
  const int64_t rows = static_cast<int64_t>(a.slots) * group, outer = static_cast<int64_t>(a.batch) * a.kv_heads;
  // with 17 to 32 rows the wide walk, although three of its four waves have none (8, 16 and 64 trees of up to 7
  // nodes over up to 4096 rows: 31, 49 and 142 us, and 42.7, 55 and 167 with two tiles of 16 rows a wave in
  // the narrow one; only 64 chains of 8 over e4m3 rows lose, 102 and 108)
  p.few = rows <= kFewRows;
  p.row_tiles = p.few ? 1 : static_cast<int>((rows + kWideRows - 1) / kWideRows);
  p.tile_rows = p.few ? kFewRows : kWideRows;
  // keys of a round: of the narrow walk's four waves, or a tile of the wide one
  const int keys = p.few ? kFewKeys * kWaves : kWideKeys;
  int64_t most = static_cast<int64_t>(a.pages.table_len) * a.pages.page_rows;
  if (a.window > 0) most = std::min<int64_t>(most, static_cast<int64_t>(a.window) + a.sinks + a.slots + 2 * keys);
  const int64_t rounds = (most + keys - 1) / keys, tiles = outer * p.row_tiles;
  p.fits = tiles * rounds < (int64_t{1} << 31) - 1024;       // sums are rounded up to workgroups
  if (p.few) {
    // as many as the registers let run at once, of e4m3 rows three a CU (the windows: 95, 94 and 97 us with 256,
    // 512 and 1024 workgroups; e4m3 rows with 512 and 768: 64 tokens over 8192 113 and 111, 128 over 2000 83 and 75,
    // 64 over 500 30 and 26, chains of 4 82 and 76, heads of 64 72 and 65; but 16 tokens over 8192 40 and
    // 44, one over 65,536 39 and 45, and the general form, two a CU, 118 and 136)
    p.blocks = std::min<int64_t>(outer * rounds, a.cache_dtype == GRAFT_E4M3 ? 768 : 512);
  } else if (rounds > 1 && (tiles < kWideBlocks || (rounds > kLongRounds && p.fits && tiles + kWideBlocks <= kMaxBlocks))) {
    // kWideBlocks is what registers and LDS let run at once (16 trees of up to 64 nodes: 91, 106, 112 and 111 us with
    // 512, 640, 768 and 1024 pieces); with more row tiles the longest walks are cut, since one long sequence
    // among short ones would leave the chip to a workgroup for each of its row tiles: over 65,536 rows beside 63 over
    // 500, trees of up to 7 nodes 104 us, whole 1292, trees of up to 64 nodes 184 and 1434; 64 trees of up to
    // 32 nodes over up to 4096 rows, half of whose row tiles are empty, 155 and 210.  Where little is cut that
    // costs the second launch: 64 trees of up to 7 nodes 141 and 136, 8 pieces of 1024 prompt rows 478 and 470.
    // Walks of up to kLongRounds are short enough to be left whole (one over 4096 rows beside 63 over 500:
    // 106 cut and 107 whole; 64 trees of up to 7 nodes over up to 300 rows 22.4 and 18.6).
    p.blocks = std::min(tiles * rounds, std::max<int64_t>(kWideBlocks, tiles + kWideBlocks / 2));
  } else {
    p.fits = true;
    p.blocks = tiles;
    return p;
  }
  constexpr int kHeads = kThreads / 32;                     // of a workgroup of the merge
  p.joins = rounds > 1 ? static_cast<int64_t>(a.batch) * a.slots * ((a.q_heads + int64_t{kHeads} - 1) / kHeads) : 0;
  p.many = !p.few && p.joins > 2 * kMergeBlocks;
  p.merge_blocks = p.many ? std::min<int64_t>(p.joins, kMergeBlocks) : p.joins;
  p.part_rows = p.few ? p.blocks * 2 * p.tile_rows : std::min<int64_t>(p.blocks, kWideBlocks) * kWideRows;
  p.share_at = p.part_rows * (a.head_dim * int64_t{4} + 8);
  p.bytes = p.share_at + (a.batch + int64_t{1}) * 4;
  return p;
}

hipError_t launch_paged_attend(graft_ctx *ctx, const graft_paged_attention_desc &d, const PagedPlan &p,
                               hipStream_t stream) {
  const bool q8 = d.cache_dtype == GRAFT_E4M3;
  PagedArgs a{};
  a.k = pool_of(d.cache_k, q8 ? 1 : 2);
  a.v = pool_of(d.cache_v, q8 ? 1 : 2);
  a.pages = page_map(d.pages);
  a.q = static_cast<const char *>(d.q.data);
  a.q_batch = d.q.batch_stride * 2;
  a.q_slot = d.q.row_stride * 2;
  a.q_head = d.q.head_stride * 2;
  a.out = static_cast<char *>(d.out.data);
  a.o_batch = d.out.batch_stride * 2;
  a.o_slot = d.out.row_stride * 2;
  a.o_head = d.out.head_stride * 2;
  a.n_nodes = d.n_nodes;
  a.cache_len = d.cache_len;
  a.mask = d.mask;
  a.lse = d.lse;
  a.error_flag = ctx->error_flag;
  a.part_o = static_cast<float *>(d.workspace);
  a.part_ml = p.bytes > 0 ? reinterpret_cast<f32x2 *>(a.part_o + p.part_rows * d.head_dim) : nullptr;
  a.share = p.bytes > 0 ? reinterpret_cast<int32_t *>(static_cast<char *>(d.workspace) + p.share_at) : nullptr;
  a.batch = d.batch;
  a.slots = d.slots;
  a.root = d.with_root ? 1 : 0;
  a.q_heads = d.q_heads;
  a.kv_heads = d.kv_heads;
  a.group = d.q_heads / d.kv_heads;
  a.dim = d.head_dim;
  a.n_max = ctx->dims.max_nodes;
  a.words = (ctx->dims.max_nodes + 63) / 64;
  a.window = d.window;
  a.sinks = d.window > 0 ? d.sinks : 0;
  a.tile_rows = p.tile_rows;
  a.row_tiles = p.row_tiles;
  a.cut = !p.few && p.bytes > 0 ? 1 : 0;
  a.joins = static_cast<int32_t>(p.joins);
  a.c = d.scale * 1.4426950408889634f;
  const dim3 grid(static_cast<unsigned>(p.blocks)), block(kThreads);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
  auto pick = [&](auto wide, auto dp, auto full) {
    constexpr bool W = decltype(wide)::value;
    constexpr int D = decltype(dp)::value;
    constexpr bool A = decltype(full)::value;
    if (d.dtype == GRAFT_F16) run(paged_attend_kernel<F16, false, A, D, W>);
    else if (q8) run(paged_attend_kernel<Bf16, true, A, D, W>);
    else run(paged_attend_kernel<Bf16, false, A, D, W>);
  };
  // heads of other sizes run as 64 or 128 columns
  auto width = [&](auto wide) {
    constexpr std::integral_constant<int, 64> k64{};
    constexpr std::integral_constant<int, 128> k128{};
    const bool even = d.pages.page_rows % 16 == 0 && a.k.page == a.v.page && a.k.row == a.v.row && a.k.head == a.v.head &&
                      (!q8 || (a.k.s_page == a.v.s_page && a.k.s_row == a.v.s_row && a.k.s_head == a.v.s_head));
    if (d.head_dim == 128 && even) pick(wide, k128, std::true_type{});
    else if (d.head_dim > 64) pick(wide, k128, std::false_type{});
    else if (d.head_dim == 64 && even) pick(wide, k64, std::true_type{});
    else pick(wide, k64, std::false_type{});
  };
  if (p.few) width(std::false_type{});
  else width(std::true_type{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.merge_blocks == 0) return e;
  const dim3 mgrid(static_cast<unsigned>(p.merge_blocks));
  auto merge = [&](auto kernel) { hipLaunchKernelGGL(kernel, mgrid, block, 0, stream, a); };
  auto join = [&](auto type) {
    using T = decltype(type);
    if (p.few) merge(merge_pages_kernel<T, false, false>);
    else if (p.many) merge(merge_pages_kernel<T, true, true>);
    else merge(merge_pages_kernel<T, true, false>);
  };
  if (d.dtype == GRAFT_F16) join(F16{});
  else join(Bf16{});
  return hipGetLastError();
}

}  // namespace graft
