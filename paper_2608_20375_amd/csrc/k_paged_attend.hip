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
// pages that the pool does not have from page 0: both are hidden.
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
constexpr int kWideRows = 128, kWideKeys = 64;    // wide_part
constexpr int kFewRows = 32, kFewKeys = 32;       // narrow_part; keys of one wave's tile
constexpr int kMaxParts = 64;                     // one a lane of the merge

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
  int64_t rows_all;       // batch * slots * q_heads
  int32_t batch, slots, root, q_heads, kv_heads, group, dim;
  int32_t n_max, words, window, sinks;
  int32_t row_tiles, splits, min_rounds;
  float c;
};

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
__device__ __forceinline__ const char *row_at(const char *head, int64_t page_bytes, uint32_t row_bytes, int page, uint32_t off) {
  return head + page * page_bytes + static_cast<uint64_t>(off * row_bytes);
}
__device__ __forceinline__ u32x4 take16(const char *p) { return *reinterpret_cast<const u32x4 *>(p); }

// Both 16-lane rows' values of a lane's column: x of lane col (+ 32) and of lane col + 16 (+ 32).
__device__ __forceinline__ u32x2 both_rows(uint32_t x) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x, x, false, false));
}

// Four numbers of the values' row of key j, for rows that see infinite or NaN ones.
template <typename T, bool Q8>
__device__ __forceinline__ u32x2 four_at(const PagedArgs &a, const char *v_head, const uint8_t *vs_head, const Spot &s, int x) {
  const char *p = row_at(v_head, a.v.page, a.v.row, s.page, s.off);
  if (!Q8) return *reinterpret_cast<const u32x2 *>(p + 2 * x);
  const uint32_t unit = vs_head[s.page * a.v.s_page + static_cast<uint64_t>(s.off * a.v.s_row)];
  return widen(*reinterpret_cast<const uint32_t *>(p + x), unit_of(unit));
}

struct Item {
  int b, kvh, tile_row, part;
};

// Rows of a row in the outputs.
__device__ __forceinline__ void finish(const PagedArgs &a, int64_t all, float m, float l, float at) {
  a.lse[all] = l == 0.0f ? -INFINITY : (m * a.c + (__log2f(l) - at)) * 0.69314718055994531f;
}

// 16 or 32 rows a workgroup, all of a sequence's and key head's: every wave walks 32-key tiles of
// its own, keys from memory straight into fragments, values through a stretch of LDS of the wave's
// own, no barriers; the waves' sums are joined at the end.
template <typename T, bool Q8, bool FULL, int DP, int QT>
__device__ __forceinline__ void narrow_part(const PagedArgs &a, const Item &it, u32x4 *lds) {
  constexpr int C = DP / 8, kSteps = DP / 32, kDTiles = DP / 16;
  constexpr int kLoads = Q8 ? DP / 64 : kSteps;         // 16-byte loads of a lane and 16 keys
  constexpr int kBytes = Q8 ? 1 : 2;
  constexpr int kPad = DP + 4;                          // floats of a row when the waves are joined
  const int tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int quarter = lane >> 4, col = lane & 15;
  const int b = it.b, kvh = it.kvh;
  u32x4 *s_v = lds + wave * kFewKeys * C;

  const Sizes sz = sizes_of(a, b);
  const int live = __builtin_amdgcn_readfirstlane(sz.n), len = __builtin_amdgcn_readfirstlane(sz.len);
  if (sz.bad && it.part == 0 && kvh == 0 && tid == 0) atomicOr(a.error_flag, kErrBlockSizes);
  if (live == 0) return;
  const RowTile tile = row_tile(len, live, 0, live - 1, a.mask != nullptr, a.window, a.sinks, kFewKeys, kWaves, a.splits, a.min_rounds);
  if (it.part >= tile.parts) return;
  const bool alone = tile.parts == 1;
  const int t0 = it.part * tile.per, t1 = std::min(t0 + tile.per, tile.span.all());

  // slot and query head of row i
  const int rows = live * a.group;
  auto place = [&](int i, int *slot, int *head) {
    const int row = i < rows ? i : rows - 1;
    *slot = row / a.group;
    *head = kvh * a.group + row - *slot * a.group;
    return i < rows;
  };

  // Contracted entries 8 of a step are chunk k_chunk(step) of a row: the 16 codes that one
  // load brings are two steps' 8.
  auto k_chunk = [&](int s) { return Q8 ? 2 * (4 * (s / 2) + quarter) + s % 2 : 4 * s + quarter; };
  u32x4 rq[QT][kSteps];
  View view[QT];
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    int slot, head;
    place(q * 16 + col, &slot, &head);
    view[q] = view_of(a, b, slot, len, live);
    const char *qp = a.q + b * a.q_batch + slot * a.q_slot + head * a.q_head;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      rq[q][s] = k_chunk(s) * 8 < a.dim ? take16(qp + k_chunk(s) * 16) : u32x4{0, 0, 0, 0};
  }

  const int32_t *table = a.pages.table + b * a.pages.table_stride;
  const char *k_head = a.k.p + kvh * a.k.head, *v_head = a.v.p + kvh * a.v.head;
  const uint8_t *ks_head = a.k.s + kvh * a.k.s_head, *vs_head = a.v.s + kvh * a.v.s_head;
  const int mine = lane & 31;                           // the key of a tile whose page this lane looks up

  struct Held {                                         // a tile on its way
    u32x4 rk[2][kLoads], rv[2][kLoads];                 // rows col and 16 + col
    uint32_t sk, sv;                                    // scales of row `mine`
    int j;                                              // first key
    uint32_t bad;                                       // keys on pages that there are none of
  } x;
  int ahead = t0 + wave, next = 0;                      // the tile to load next, this lane's page of it
  if (ahead < t1) next = entry_at(a, table, tile.span.at(ahead) * kFewKeys + mine, tile.end);
  auto fetch = [&]() {
    if (ahead >= t1) return;
    x.j = tile.span.at(ahead) * kFewKeys;
    const Spot s = spot_at(a, next, x.j + mine, tile.end);
    x.bad = static_cast<uint32_t>(__ballot(s.bad));
    const u32x2 page = both_rows(static_cast<uint32_t>(s.page)), off = both_rows(s.off);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const char *p = row_at(k_head, a.k.page, a.k.row, static_cast<int>(page[kt]), off[kt]);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = (4 * i + quarter) * 16;
        x.rk[kt][i] = take16(p + (FULL || at < kBytes * a.dim ? at : 0));
      }
    }
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const char *p = row_at(v_head, a.v.page, a.v.row, static_cast<int>(page[kt]), off[kt]);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = (4 * i + quarter) * 16;
        x.rv[kt][i] = take16(p + (FULL || at < kBytes * a.dim ? at : 0));
      }
    }
    if (Q8) {
      x.sk = ks_head[s.page * a.k.s_page + static_cast<uint64_t>(s.off * a.k.s_row)];
      x.sv = vs_head[s.page * a.v.s_page + static_cast<uint64_t>(s.off * a.v.s_row)];
    }
    ahead += kWaves;
    if (ahead < t1) next = entry_at(a, table, tile.span.at(ahead) * kFewKeys + mine, tile.end);
  };

  f32x4 o[QT][kDTiles];
  float m[QT], l[QT];
  Ref ref[QT];                  // of m
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    m[q] = -INFINITY;
    l[q] = 0.0f;
    ref[q] = ref_of<T>(m[q], a.c);
#pragma unroll
    for (int d = 0; d < kDTiles; ++d) o[q][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  fetch();
  for (int t = t0 + wave; t < t1; t += kWaves) {
    const int j = x.j;
    const uint32_t bad = x.bad;
    const bool clear = bad == 0 && is_clear(tile, j, kFewKeys, a.sinks);
    if (bad != 0 && lane == 0) atomicOr(a.error_flag, kErrPage);
    f32x4 s[QT][2];
#pragma unroll
    for (int q = 0; q < QT; ++q) s[q][0] = s[q][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const u32x2 sk = Q8 ? both_rows(x.sk) : u32x2{0, 0}, sv = Q8 ? both_rows(x.sv) : u32x2{0, 0};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const float uk = unit_of(sk[kt]);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        u32x4 f[2];
        if (Q8) {
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const u32x2 z = widen(x.rk[kt][i][y], uk);
            f[y / 2][2 * (y % 2)] = z.x;
            f[y / 2][2 * (y % 2) + 1] = z.y;
          }
        } else {
          f[0] = x.rk[kt][i];
        }
        // past the head's numbers the queries hold zeros, which an infinite key would not leave so
        if (!FULL && (4 * i + quarter) * 16 >= kBytes * a.dim) f[0] = f[1] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int y = 0; y < (Q8 ? 2 : 1); ++y)
#pragma unroll
          for (int q = 0; q < QT; ++q) s[q][kt] = T::mfma(f[y], rq[q][Q8 ? 2 * i + y : i], s[q][kt]);
      }
    }
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const int r = 16 * kt + col;
      const float uv = unit_of(sv[kt]);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        if (Q8) {
          u32x4 f[2];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const u32x2 z = widen(x.rv[kt][i][y], uv);
            f[y / 2][2 * (y % 2)] = z.x;
            f[y / 2][2 * (y % 2) + 1] = z.y;
          }
          s_v[v_at<C>(r, 2 * (4 * i + quarter))] = f[0];
          s_v[v_at<C>(r, 2 * (4 * i + quarter) + 1)] = f[1];
        } else {
          s_v[v_at<C>(r, 4 * i + quarter)] = x.rv[kt][i];
        }
      }
    }
    // before the next tile's loads take their registers
    bool odd = false;
    uint32_t seen[QT];
    if (__builtin_expect(!clear, 0)) {
#pragma unroll 1
      for (int i = lane; i < kFewKeys * C; i += kWave) {
        u32x4 w = s_v[i];
        if (tame<T>(w)) {
          s_v[i] = w;
          odd = true;
        }
      }
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        seen[q] = static_cast<uint32_t>(seen_bits(a, b, view[q], j, len, live)) & ~bad;
        const uint32_t bits = seen[q] >> (4 * quarter);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          s[q][i / 4][i % 4] = (bits >> (16 * (i / 4) + i % 4)) & 1u ? s[q][i / 4][i % 4] : -INFINITY;
      }
    }
    fetch();
    // The tile's scores into the running sums, its values being in LDS.  The wave's LDS
    // operations are done in order.
    u32x4 p[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      float mx = s[q][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[q][i / 4][i % 4]);
      mx = quarter_max(mx);
      const bool up = __builtin_fmaf(mx, ref[q].c, ref[q].off) > T::kLift + T::kSlack;   // as in softmax_step
      if (__ballot(up) != 0) {
        const Ref now = ref_of<T>(up ? mx : m[q], a.c);
        const float alpha = up ? factor(m[q], ref[q].at, mx, now, a.c) : 1.0f;
        l[q] *= alpha;
#pragma unroll
        for (int d = 0; d < kDTiles; ++d) o[q][d] *= alpha;
        m[q] = up ? mx : m[q];
        ref[q] = now;
      }
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[q][i / 4][i % 4], ref[q].c, ref[q].off));
      l[q] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      p[q] = u32x4{T::pack(e[0], e[1]), T::pack(e[2], e[3]), T::pack(e[4], e[5]), T::pack(e[6], e[7])};
    }
    __builtin_amdgcn_wave_barrier();
    const int vr = 4 * quarter + (col >> 2);
#pragma unroll
    for (int d = 0; d < kDTiles; ++d) {
      typedef __attribute__((address_space(3))) s16x4 *at;
      const char *vp = reinterpret_cast<const char *>(s_v + v_at<C>(vr, 2 * d + ((col & 3) >> 1))) + (col & 1) * 8;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(vp)));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(vp + 16 * C * 16)));
#pragma unroll
      for (int q = 0; q < QT; ++q) o[q][d] = T::mfma(u32x4{lo.x, lo.y, hi.x, hi.y}, p[q], o[q][d]);
    }
    __builtin_amdgcn_wave_barrier();
    if (__builtin_expect(__ballot(odd) != 0, 0)) {
#pragma unroll 1
      for (int y = 0; y < kFewKeys && j + y < tile.end; ++y) {
        const Spot sp = spot_at(a, entry_at(a, table, j + y, tile.end), j + y, tile.end);
#pragma unroll
        for (int q = 0; q < QT; ++q)
#pragma unroll
          for (int d = 0; d < kDTiles; ++d) {
            const int c0 = d * 16 + 4 * quarter;
            u32x2 w{0, 0};
            if (((seen[q] >> y) & 1) && c0 < a.dim) w = four_at<T, Q8>(a, v_head, vs_head, sp, c0);
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              const uint16_t n = static_cast<uint16_t>(w[z / 2] >> (16 * (z & 1)));
              o[q][d][z] += (n & T::kExp) == T::kExp ? T::number(n) : 0.0f;
            }
          }
      }
    }
  }

  // The four waves' rows: each leaves its own with its maximum and sum, then every thread
  // joins 4 numbers of a row, the waves in order.
  float *s_o = reinterpret_cast<float *>(lds);
  float *s_m = s_o + kWaves * 16 * kPad, *s_l = s_m + kWaves * 16;
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    __syncthreads();
    l[q] = quarter_sum(l[q]);
    if (quarter == 0) {
      s_m[wave * 16 + col] = m[q];
      s_l[wave * 16 + col] = l[q];
    }
#pragma unroll
    for (int d = 0; d < kDTiles; ++d)
      *reinterpret_cast<f32x4 *>(s_o + (wave * 16 + col) * kPad + d * 16 + 4 * quarter) = o[q][d];
    __syncthreads();
    for (int u = tid; u < 16 * (DP / 4); u += kThreads) {
      const int r = u / (DP / 4), c0 = (u % (DP / 4)) * 4;
      int slot, head;
      if (!place(q * 16 + r, &slot, &head) || c0 >= a.dim) continue;
      float top = s_m[r];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) top = fmaxf(top, s_m[i * 16 + r]);
      const Ref now = ref_of<T>(top, a.c);
      f32x4 sum{0.0f, 0.0f, 0.0f, 0.0f};
      float total = 0.0f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float mi = s_m[i * 16 + r];
        const float f = mi == top ? 1.0f : factor(mi, ref_of<T>(mi, a.c).at, top, now, a.c);
        total += s_l[i * 16 + r] * f;
        sum += *reinterpret_cast<const f32x4 *>(s_o + (i * 16 + r) * kPad + c0) * f;
      }
      const int64_t all = (static_cast<int64_t>(b) * a.slots + slot) * a.q_heads + head;
      if (!alone) {
        const int64_t at = it.part * a.rows_all + all;
        if (c0 == 0) a.part_ml[at] = f32x2{top, total};
        *reinterpret_cast<f32x4 *>(a.part_o + at * a.dim + c0) = sum;
      } else {
        const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
        *reinterpret_cast<u32x2 *>(a.out + b * a.o_batch + slot * a.o_slot + head * a.o_head + 2 * c0) =
            u32x2{T::pack(sum.x * inv, sum.y * inv), T::pack(sum.z * inv, sum.w * inv)};
        if (a.lse && c0 == 0) finish(a, all, top, total, now.at);
      }
    }
  }
}

// 128 rows a workgroup, 32 a wave; 64-key tiles in LDS for all four waves, the next tile's loads
// in flight in registers meanwhile, two LDS buffers, one barrier a tile.
template <typename T, bool Q8, bool FULL, int DP>
__device__ __forceinline__ void wide_part(const PagedArgs &a, const Item &it, u32x4 *lds) {
  constexpr int C = DP / 8;                             // 16-byte chunks of a row in LDS
  constexpr int kSteps = DP / 16, kDTiles = DP / 32;
  constexpr int kBuf = kWideKeys * C;                   // a buffer of keys, or of values
  constexpr int kBytes = Q8 ? 1 : 2;
  constexpr int kPer = C * kBytes / 2;                  // threads of a key
  constexpr int kStep = kThreads / kPer, kUnits = kWideKeys / kStep;
  u32x4 *s_k = lds, *s_v = lds + 2 * kBuf;

  const int tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int h = lane >> 5, col = lane & 31;
  const int b = it.b, kvh = it.kvh;

  const Sizes sz = sizes_of(a, b);
  const int live = __builtin_amdgcn_readfirstlane(sz.n), len = __builtin_amdgcn_readfirstlane(sz.len);
  if (sz.bad && it.tile_row == 0 && it.part == 0 && kvh == 0 && tid == 0) atomicOr(a.error_flag, kErrBlockSizes);
  const int rows = live * a.group, first = it.tile_row * kWideRows;
  if (first >= rows) return;
  const RowTile tile = row_tile(len, live, first / a.group, (std::min(first + kWideRows, rows) - 1) / a.group, a.mask != nullptr,
                                a.window, a.sinks, kWideKeys, 1, a.splits, a.min_rounds);
  if (it.part >= tile.parts) return;
  const bool alone = tile.parts == 1;
  const int t0 = it.part * tile.per, t1 = std::min(t0 + tile.per, tile.span.all());

  const bool valid = first + wave * 32 + col < rows;
  const int row = valid ? first + wave * 32 + col : rows - 1;
  const int slot = row / a.group, head = kvh * a.group + row - slot * a.group;
  const bool busy = __ballot(valid) != 0;
  const View view = view_of(a, b, slot, len, live);

  const int32_t *table = a.pages.table + b * a.pages.table_stride;
  const char *k_head = a.k.p + kvh * a.k.head, *v_head = a.v.p + kvh * a.v.head;
  const uint8_t *ks_head = a.k.s + kvh * a.k.s_head, *vs_head = a.v.s + kvh * a.v.s_head;

  // a thread's share of a tile: 16 bytes of rows r0, r0 + kStep, ...
  const int r0 = tid / kPer, ch = tid % kPer;
  const int at16 = FULL || ch * 16 < kBytes * a.dim ? ch * 16 : 0;
  u32x4 rk[kUnits], rv[kUnits];
  uint32_t sk = 0, sv = 0;                              // scales of key `lane`
  int held_j = 0, next = entry_at(a, table, tile.span.at(t0) * kWideKeys + lane, tile.end);
  uint64_t held_bad = 0;
  auto load = [&](int t) {
    held_j = tile.span.at(t) * kWideKeys;
    const Spot s = spot_at(a, next, held_j + lane, tile.end);
    held_bad = __ballot(s.bad);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int from = 4 * (r0 + i * kStep);
      const int page = __builtin_amdgcn_ds_bpermute(from, s.page);
      const uint32_t off = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(from, static_cast<int>(s.off)));
      rk[i] = take16(row_at(k_head, a.k.page, a.k.row, page, off) + at16);
      rv[i] = take16(row_at(v_head, a.v.page, a.v.row, page, off) + at16);
    }
    if (Q8) {
      sk = ks_head[s.page * a.k.s_page + static_cast<uint64_t>(s.off * a.k.s_row)];
      sv = vs_head[s.page * a.v.s_page + static_cast<uint64_t>(s.off * a.v.s_row)];
    }
    if (t + 1 < t1) next = entry_at(a, table, tile.span.at(t + 1) * kWideKeys + lane, tile.end);
  };
  // Stores the share; true if a value is infinite or NaN where not all rows see the keys (stored
  // as 0 then).
  auto store = [&](int buf, bool clear) {
    bool odd = false;
    u32x4 *k = s_k + buf * kBuf, *v = s_v + buf * kBuf;
    const bool past = !FULL && ch * 16 >= kBytes * a.dim;
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
  const char *qp = a.q + b * a.q_batch + slot * a.q_slot + head * a.q_head;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) rq[s] = s * 16 < a.dim ? take16(qp + s * 32 + h * 16) : u32x4{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < kSteps; ++s) settle(rq[s]);

  Sums<DP> st;
  st.clear(a.c);
  load(t0);
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1, j = held_j;
    const uint64_t bad = held_bad;
    const bool clear = bad == 0 && is_clear(tile, j, kWideKeys, a.sinks);
    if (bad != 0 && tid == 0) atomicOr(a.error_flag, kErrPage);
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
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
        s[kt] = T::mfma(k[k_at<C>(kt * 32 + col, 2 * i + h)], rq[i], s[kt]);
    uint64_t seen = ~0ull;
    if (__builtin_expect(!clear, 0)) {
      seen = seen_bits(a, b, view, j, len, live) & ~bad;
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
#pragma unroll
    for (int d = 0; d < kDTiles; ++d) {
#pragma unroll
      for (int g = 0; g < 4; ++g) st.o[d] = T::mfma(v_fragment<C>(v, d, g, lane), p[g], st.o[d]);
    }
    if (__builtin_expect(any_odd, 0)) {
#pragma unroll 1
      for (int y = 0; y < kWideKeys && j + y < tile.end; ++y) {
        const Spot sp = spot_at(a, entry_at(a, table, j + y, tile.end), j + y, tile.end);
#pragma unroll
        for (int d = 0; d < kDTiles; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int c0 = d * 32 + 8 * i + 4 * h;
            u32x2 w{0, 0};
            if (((seen >> y) & 1) && c0 < a.dim) w = four_at<T, Q8>(a, v_head, vs_head, sp, c0);
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              const uint16_t n = static_cast<uint16_t>(w[z / 2] >> (16 * (z & 1)));
              st.o[d][4 * i + z] += (n & T::kExp) == T::kExp ? T::number(n) : 0.0f;
            }
          }
      }
    }
  }

  st.l = half_sum(st.l);
  if (!valid) return;
  const int64_t all = (static_cast<int64_t>(b) * a.slots + slot) * a.q_heads + head;
  if (!alone) {
    const int64_t at = it.part * a.rows_all + all;
    if (h == 0) a.part_ml[at] = f32x2{st.m, st.l};
    float *po = a.part_o + at * a.dim;
#pragma unroll
    for (int d = 0; d < kDTiles; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int x = d * 32 + 8 * i + 4 * h;
        if (x < a.dim)
          *reinterpret_cast<f32x4 *>(po + x) =
              f32x4{st.o[d][4 * i], st.o[d][4 * i + 1], st.o[d][4 * i + 2], st.o[d][4 * i + 3]};
      }
    return;
  }
  const float inv = st.l > 0.0f || st.l != st.l ? 1.0f / st.l : 0.0f;
  char *op = a.out + b * a.o_batch + slot * a.o_slot + head * a.o_head;
#pragma unroll
  for (int d = 0; d < kDTiles; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = d * 32 + 8 * i + 4 * h;
      if (x < a.dim)
        *reinterpret_cast<u32x2 *>(op + 2 * x) =
            u32x2{T::pack(st.o[d][4 * i] * inv, st.o[d][4 * i + 1] * inv),
                  T::pack(st.o[d][4 * i + 2] * inv, st.o[d][4 * i + 3] * inv)};
    }
  if (a.lse && h == 0) finish(a, all, st.m, st.l, ref_of<T>(st.m, a.c).at);
}

// QT = 0: the wide walk; else the narrow one, 16 QT rows.  FULL: heads of DP numbers; the others' loads
// past a head's end go to its begin, which takes addresses of their own and registers.
template <typename T, bool Q8, bool FULL, int DP, int QT>
__global__ void __launch_bounds__(kThreads, QT == 1 || (QT == 2 && DP == 64) ? 3 : 2)
paged_attend_kernel(PagedArgs a) {
  constexpr int kNarrow = (kWaves * 16 * (DP + 4) + 2 * kWaves * 16 + 3) / 4;   // joining the waves
  constexpr int kValues = kWaves * kFewKeys * (DP / 8);
  __shared__ __align__(16) u32x4 lds[QT == 0 ? 4 * kWideKeys * (DP / 8) : (kNarrow > kValues ? kNarrow : kValues)];
  // Workgroups go round the 8 XCDs.  Wide: the row tiles of a (part, sequence, key head) follow each
  // other on one, whose L2 then holds their keys.  The others go by an odd number (one may be empty),
  // so that a sequence's parts fall on all XCDs; parts that short sequences leave empty come last.
  const int i = blockIdx.x, outer = a.batch * a.kv_heads, odd = outer | 1;
  Item it;
  int g = i;
  it.tile_row = 0;
  if (QT == 0) {
    const int j = i >> 3;
    g = (j / a.row_tiles) * 8 + (i & 7);
    it.tile_row = j % a.row_tiles;
  }
  it.part = g / odd;
  const int o = g - it.part * odd;
  it.b = o / a.kv_heads;
  it.kvh = o - it.b * a.kv_heads;
  if (it.part >= a.splits || o >= outer) return;
  if (QT == 0) wide_part<T, Q8, FULL, DP>(a, it, lds);
  else narrow_part<T, Q8, FULL, DP, QT == 0 ? 1 : QT>(a, it, lds);
}

// Joins the parts of a row: a wave each, one part a lane for the statistics, two
// numbers a lane for the row.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads)
merge_pages_kernel(PagedArgs a) {
  const int lane = lane_id();
  const int64_t r = static_cast<int64_t>(blockIdx.x) * kWaves + threadIdx.x / kWave;
  if (r >= a.rows_all) return;
  const int64_t bs = r / a.q_heads;
  const int head = static_cast<int>(r - bs * a.q_heads);
  const int b = static_cast<int>(bs / a.slots), slot = static_cast<int>(bs - static_cast<int64_t>(b) * a.slots);
  const Sizes sz = sizes_of(a, b);
  if (slot >= sz.n) return;
  int s0 = 0, s1 = sz.n - 1;
  if (WIDE) {
    const int rows = sz.n * a.group, first = (slot * a.group + head % a.group) / kWideRows * kWideRows;
    s0 = first / a.group;
    s1 = (std::min(first + kWideRows, rows) - 1) / a.group;
  }
  const RowTile tile = row_tile(sz.len, sz.n, s0, s1, a.mask != nullptr, a.window, a.sinks, WIDE ? kWideKeys : kFewKeys,
                                WIDE ? 1 : kWaves, a.splits, a.min_rounds);
  if (tile.parts == 1) return;                             // its only part wrote the row
  const f32x2 ml = lane < tile.parts ? a.part_ml[lane * a.rows_all + r] : f32x2{-INFINITY, 0.0f};
  float top = ml.x;
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) top = fmaxf(top, __uint_as_float(xor_lane(__float_as_uint(top), k)));
  // 0 for a part without keys that the row sees
  const Ref now = ref_of<T>(top, a.c);
  const float w = ml.x == top && top != -INFINITY ? 1.0f : factor(ml.x, ref_of<T>(ml.x, a.c).at, top, now, a.c);
  float l = w * ml.y;
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) l += __uint_as_float(xor_lane(__float_as_uint(l), k));
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  float x = 0.0f, y = 0.0f;
  if (lane * 2 < a.dim) {
    for (int p = 0; p < tile.parts; ++p) {
      const f32x2 v = *reinterpret_cast<const f32x2 *>(a.part_o + (p * a.rows_all + r) * a.dim + lane * 2);
      const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), p));
      x = __builtin_fmaf(f, v.x, x);
      y = __builtin_fmaf(f, v.y, y);
    }
    *reinterpret_cast<uint32_t *>(a.out + b * a.o_batch + slot * a.o_slot + head * a.o_head + lane * 4) =
        T::pack(x * inv, y * inv);
  }
  if (a.lse && lane == 0) finish(a, r, top, l, now.at);
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
  const int64_t rows = static_cast<int64_t>(a.slots) * group;
  p.few = rows <= 16 ? 1 : rows <= kFewRows ? 2 : 0;
  p.row_tiles = p.few ? 1 : static_cast<int>((rows + kWideRows - 1) / kWideRows);
  const int64_t outer = static_cast<int64_t>(a.batch) * a.kv_heads, units = outer * p.row_tiles;
  // keys of a round: of the narrow walk's four waves, or a tile of the wide one
  const int keys = p.few ? kFewKeys * kWaves : kWideKeys;
  int64_t most = static_cast<int64_t>(a.pages.table_len) * a.pages.page_rows;
  if (a.window > 0) most = std::min<int64_t>(most, static_cast<int64_t>(a.window) + a.sinks + a.slots + 2 * keys);
  const int64_t rounds = (most + keys - 1) / keys;
  p.min_rounds = p.few ? 1 : 4;
  int64_t s = ((p.few ? 4096 : 1024) + units - 1) / units;
  s = std::min(s, (rounds + p.min_rounds - 1) / p.min_rounds);
  p.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(s, kMaxParts)));
  const int64_t all = static_cast<int64_t>(a.batch) * a.slots * a.q_heads;
  p.blocks = ((outer | 1) * p.splits + 7) / 8 * 8 * p.row_tiles;
  p.merge_blocks = p.splits > 1 ? (all + kWaves - 1) / kWaves : 0;
  p.bytes = p.splits > 1 ? p.splits * all * (a.head_dim * int64_t{4} + 8) : 0;
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
  a.rows_all = static_cast<int64_t>(d.batch) * d.slots * d.q_heads;
  a.part_o = static_cast<float *>(d.workspace);
  a.part_ml = p.splits > 1 ? reinterpret_cast<f32x2 *>(a.part_o + p.splits * a.rows_all * d.head_dim) : nullptr;
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
  a.row_tiles = p.row_tiles;
  a.splits = p.splits;
  a.min_rounds = p.min_rounds;
  a.c = d.scale * 1.4426950408889634f;
  const dim3 grid(static_cast<unsigned>(p.blocks)), block(kThreads);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
  auto pick = [&](auto few, auto dp, auto full) {
    constexpr int F = decltype(few)::value;
    constexpr int D = decltype(dp)::value;
    constexpr bool A = decltype(full)::value;
    if (d.dtype == GRAFT_F16) run(paged_attend_kernel<F16, false, A, D, F>);
    else if (q8) run(paged_attend_kernel<Bf16, true, A, D, F>);
    else run(paged_attend_kernel<Bf16, false, A, D, F>);
  };
  // heads of other sizes run as 64 or 128 columns
  auto width = [&](auto few) {
    constexpr std::integral_constant<int, 64> k64{};
    constexpr std::integral_constant<int, 128> k128{};
    if (d.head_dim == 128) pick(few, k128, std::true_type{});
    else if (d.head_dim > 64) pick(few, k128, std::false_type{});
    else if (d.head_dim == 64) pick(few, k64, std::true_type{});
    else pick(few, k64, std::false_type{});
  };
  if (p.few == 1) width(std::integral_constant<int, 1>{});
  else if (p.few == 2) width(std::integral_constant<int, 2>{});
  else width(std::integral_constant<int, 0>{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits <= 1) return e;
  const dim3 mgrid(static_cast<unsigned>(p.merge_blocks));
  auto merge = [&](auto kernel) { hipLaunchKernelGGL(kernel, mgrid, block, 0, stream, a); };
  if (d.dtype == GRAFT_F16) {
    if (p.few) merge(merge_pages_kernel<F16, false>);
    else merge(merge_pages_kernel<F16, true>);
  } else {
    if (p.few) merge(merge_pages_kernel<Bf16, false>);
    else merge(merge_pages_kernel<Bf16, true>);
  }
  return hipGetLastError();
}

}  // namespace graft
