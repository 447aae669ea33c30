// k_attend.hip -- attention of a draft block: the queries of the root and of the
// tree's nodes over a prefix that the whole batch shares, the sequence's own cache
// and the block itself under the ancestor mask (the paper's Preliminaries: the target
// verifies the tree in one pass under a tree-attention mask).
//
//   o_i = sum_j p_ij v_j / l_i,  p_ij = exp2(c (s_ij - m_i)),  s_ij = q_i . k_j,
//   m_i = max_j s_ij,  l_i = sum_j p_ij,  c = scale log2 e,
// in one pass over the keys with a running maximum and sum.
//
// Layout.  The query heads of a key head are rows beside each other: row = slot *
// group + head of the group, so a single token of eight query heads is eight rows of
// one tile and a key is loaded once for all of them.
//
// Products.  v_mfma_f32_32x32x16: lane l gives row (or column) l % 32 and 8 of the 16
// contracted entries from 8 (l / 32) on; of the 32 x 32 result it holds column l % 32,
// rows 8 (i / 4) + 4 (l / 32) + i % 4, i < 16.  S^T = K Q^T puts a query into a lane: its
// maximum and sum are taken in the lane, with one exchange with the other half of
// the wave.  O^T = V^T P^T then wants P^T as its right operand: any order of the
// contracted keys will do as long as V^T's is the same, so a lane's own 8 numbers of a
// 16-key group are used where they are, keys 4 h + {0..3, 8..11} of the group in lane
// half h; V^T's fragments come out of row-major LDS by the transposing read
// ds_read_b64_tr_b16 (of 16 lanes, each giving the address of 4 numbers of row s / 4,
// columns 4 (s % 4).., lane i gets column i of the 4 rows).
//
// wide_part: 128 rows a workgroup, 32 a wave; 64-key tiles in LDS for all four waves, the
// next tile's loads in flight in registers meanwhile, two LDS buffers, one barrier a
// tile.  For blocks with many rows: a wave's tile is 1024 cycles of matrix products, about
// 1500 of vector work (the exponentials 512 of them) and 320 of LDS reads, the registers
// (248 of 256 at 128 columns, all of them for codes) leave two waves a SIMD to overlap them, and
// 5000 to 5800 cycles pass for the two.  64 trees of up to 512 nodes over 4096 e4m3 rows and 1024
// shared ones: 1400 us, 858 TFLOP/s; 16 of up to 256 nodes over 4096 bf16 rows: 176 us, 648 TFLOP/s
// (fp16: 184); chains instead of trees the same.  Short runs, at lower clocks, take a tenth longer.
// One LDS buffer and two barriers for a third wave would spill 300 to 400 bytes; sequences in
// the order of their work, or the long ones in parts of an even length, change nothing (short
// runs in turn: 1566 against 1531 us, 210 against 200): the chip is full until near the end.
// narrow_part: 16 or 32 rows a workgroup; every wave walks 32-key tiles of its own (four
// waves, four times the keys in flight), keys from memory straight into fragments, the
// values through a stretch of LDS of the wave's own, no barriers; the four waves' sums
// are joined at the end.  For single tokens and small blocks: bound by the cache's bytes, 64
// tokens of 32 query and 8 key heads over 8192 e4m3 rows and 4096 shared ones 142 us for 593 MB,
// 4.2 TB/s (a head's 128-byte pieces of 1 KB rows are read at 5.4 TB/s at most by any load, whole
// rows at 6.3); a launch's latency at one token over 700 rows, 11.4 us with the merge.
//
// The keys of a sequence (tiles of the shared prefix, of its cache, of its block) are
// split into parts where rows alone do not fill the chip; every part leaves its sums,
// maximum and unnormalised rows in the workspace and merge_parts_kernel joins them.
// When a sequence has fewer rows than a tile, the shared prefix is walked by workgroups
// of their own whose rows come from all sequences: it is read once for a tile of rows
// instead of once for every sequence.
//
// A row's running maximum is only moved when its new maximum is more than 2^8 (fp16: 2^3)
// above it: the sums and rows are fp32 and the probabilities, then up to 2^8, keep their
// relative precision in 16 bits, while rescaling a row's numbers every time would cost a
// fifth of the vector work.  fp16 has few exponents: probabilities are lifted by 2^12 there, so
// that they keep their precision down to 2^-26 of the reference and an absolute 2^-37 below
// (unlifted, keys at 2^-25 would be counted in the sum and lost from the product).  Each row
// decides by itself: were a wave's rows to move together, a row's roundings would depend on
// keys that only its neighbours see.
#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "attend_device.h"
#include "attend_tiles.h"
#include "graft_internal.h"

namespace graft {
namespace {

constexpr int kAttThreads = 256;
constexpr int kAttWaves = kAttThreads / kWave;
constexpr int kRowTile = 128, kKeyTile = 64;      // wide_part
constexpr int kFewRows = 32, kFewKeys = 32;       // narrow_part; keys of one wave's tile
constexpr int kMaxParts = 64;                     // one a lane of the merge
constexpr int kOutside = 0x40000000;              // an offset past every buffer's end
static_assert(kFewKeys * kAttWaves == 2 * kKeyTile, "tiles of both kinds are counted in the plan");

// A side (keys or values) of a source of rows; strides in bytes.
struct Side {
  const char *p;
  const uint8_t *s;
  int64_t batch, head, s_batch, s_head;
  int32_t row, s_row;
};
struct Source {
  Side k, v;
};

struct AttendArgs {
  Source src[3];          // shared prefix, cache, block
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
  int32_t n_max, words, cache_rows, shared_len;
  int32_t tile_keys, turns;   // keys of a tile, tiles that a workgroup's waves take at a time
  int32_t row_tiles, splits, min_tiles, shared_tiles, shared_splits, parts;
  int32_t shared_items;   // workgroups of the shared prefix's own pass
  float c;
};

// Sizes of sequence b as the kernels use them.
__device__ __forceinline__ int slots_of(const AttendArgs &a, int b, bool *bad) {
  const int n = a.n_nodes[b], most = a.slots - a.root;
  *bad = n < 0 || n > most;
  return (n < 0 ? 0 : (n > most ? most : n)) + a.root;
}

__device__ __forceinline__ Tiles tiles_of(const AttendArgs &a, bool packed, int len, int live) {
  const int shared = packed || a.shared_items == 0 ? a.shared_len : 0;
  return cut_tiles(shared, len, live, a.tile_keys, a.turns, packed ? a.shared_splits : a.splits, a.min_tiles);
}
__device__ __forceinline__ int len_of(const AttendArgs &a, int b, bool *bad) {
  if (a.cache_rows == 0) return 0;
  const int n = a.cache_len[b];
  *bad |= n < 0 || n > a.cache_rows;
  return n < 0 ? 0 : (n > a.cache_rows ? a.cache_rows : n);
}

// The walk over the keys of one (sequence, key head): tiles of KEYS keys of each
// source in turn.  All of it is the same for every lane of a wave.
struct Walk {
  const char *k, *v;            // first row of the tile
  const uint8_t *ks, *vs;
  int k_row, v_row, ks_row, vs_row;
  int source, left, tile;       // keys from the tile's first on; tile's number in the source
};

// To tile t of the walk; b's cache has c1 rows, its block c2 slots.
__device__ __forceinline__ void seek(Walk &w, const Tiles &n, int t, int keys, int c0, int c1, int c2, int b,
                                     int kvh) {
  const Spot at = spot_of(n, t, keys, c0, c1, c2);
  // Read from the kernel's argument memory where it is needed (sources come first there):
  // kept in registers over the walk's loop, the three would push out what the loop uses.
  typedef const __attribute__((address_space(4))) Source *Arguments;
  static_assert(offsetof(AttendArgs, src) == 0, "the sources are the first argument");
  Arguments s = (Arguments)__builtin_amdgcn_kernarg_segment_ptr() + at.source;
  asm volatile("" : "+s"(s));
  const int64_t base = at.source == 0 ? 0 : b, first = static_cast<int64_t>(at.tile) * keys;
  w.source = at.source;
  w.tile = at.tile;
  w.left = at.left;
  w.k_row = s->k.row;
  w.v_row = s->v.row;
  w.ks_row = s->k.s_row;
  w.vs_row = s->v.s_row;
  w.k = s->k.p + base * s->k.batch + kvh * s->k.head + first * s->k.row;
  w.v = s->v.p + base * s->v.batch + kvh * s->v.head + first * s->v.row;
  w.ks = s->k.s + base * s->k.s_batch + kvh * s->k.s_head + first * s->k.s_row;
  w.vs = s->v.s + base * s->v.s_batch + kvh * s->v.s_head + first * s->v.s_row;
}
// n tiles on in the same source.
__device__ __forceinline__ void advance(Walk &w, int n, int keys) {
  const int64_t rows = static_cast<int64_t>(n) * keys;
  w.k += rows * w.k_row;
  w.v += rows * w.v_row;
  w.ks += rows * w.ks_row;
  w.vs += rows * w.vs_row;
  w.left -= n * keys;
  w.tile += n;
}

// The slots 64 * word .. + 63 of the block that row (rb, slot) sees.
__device__ __forceinline__ uint64_t seen_word(const AttendArgs &a, int rb, int slot, int word, int live) {
  uint64_t w;
  if (a.mask) {
    const int node = slot - a.root;
    if (node < 0) {
      w = word == 0 ? 1 : 0;
    } else {
      const uint64_t *m = a.mask + (static_cast<int64_t>(rb) * a.n_max + node) * a.words;
      w = word < a.words ? m[word] : 0;
      if (a.root) w = (w << 1) | (word > 0 ? m[word - 1] >> 63 : 1);
    }
  } else {
    const int n = slot - word * 64 + 1;
    w = n <= 0 ? 0 : (n >= 64 ? ~0ull : (1ull << n) - 1);
  }
  const int have = live - word * 64;
  return have < 64 ? w & ((1ull << (have < 0 ? 0 : have)) - 1) : w;
}

// Infinite and NaN values of the `count` slots of a block tile that a row sees (bits of
// seen): they were stored as 0.  Not reached but for such values.
template <typename T, int DP>
__device__ __forceinline__ void add_odd(const char *v, int v_row, int count, uint64_t seen, int h, int dim,
                                        Sums<DP> &st) {
#pragma unroll 1
  for (int j = 0; j < count; ++j) {
    const bool on = (seen >> j) & 1;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = d * 32 + 8 * i + 4 * h;
        u32x2 w{0, 0};
        if (on && at < dim) w = *reinterpret_cast<const u32x2 *>(v + static_cast<int64_t>(j) * v_row + 2 * at);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint16_t n = static_cast<uint16_t>(w[x / 2] >> (16 * (x & 1)));
          st.o[d][4 * i + x] += (n & T::kExp) == T::kExp ? T::number(n) : 0.0f;
        }
      }
  }
}

// What a workgroup works on, whichever way it walks.
struct Item {
  int b, kvh, tile_row, part;
  bool packed;
};

template <typename T, bool Q8, int DP>
__device__ __forceinline__ void wide_part(const AttendArgs &a, const Item &it, u32x4 *lds) {
  constexpr int C = DP / 8;                             // 16-byte chunks of a row in LDS
  constexpr int kSteps = DP / 16, kDTiles = DP / 32;
  constexpr int kBuf = kKeyTile * C;                    // a buffer of keys, or of values
  constexpr int kUnits = kBuf / kAttThreads, kStep = kAttThreads / C;
  u32x4 *s_k = lds, *s_v = lds + 2 * kBuf;

  const int tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);   // uniform: the walk's tables stay scalar
  const int h = lane >> 5, col = lane & 31;
  const int b = it.b, kvh = it.kvh;
  const bool packed = it.packed;

  bool bad = false, unused;
  const int per_seq = a.slots * a.group;
  const int live = packed ? 0 : __builtin_amdgcn_readfirstlane(slots_of(a, b, &bad));
  const int len = packed ? 0 : __builtin_amdgcn_readfirstlane(len_of(a, b, &bad));
  if (bad && it.tile_row == 0 && it.part == 0 && kvh == 0 && tid == 0) atomicOr(a.error_flag, kErrBlockSizes);
  if (!packed && it.tile_row * kRowTile >= live * a.group) return;
  int row = it.tile_row * kRowTile + wave * 32 + col;
  int rb = b;
  if (packed) {
    rb = row < a.batch * per_seq ? row / per_seq : a.batch - 1;
    row -= rb * per_seq;
  }
  const int rlive = packed ? slots_of(a, rb, &unused) : live;
  const bool valid = row < rlive * a.group;
  row = row < per_seq ? row : per_seq - 1;
  const int slot = row / a.group, head = kvh * a.group + row - slot * a.group;
  if (packed && !__syncthreads_or(valid)) return;
  const bool busy = __ballot(valid) != 0;

  const Tiles n = tiles_of(a, packed, len, live);
  const Part part = part_of(n, it.part);
  const int t0 = part.first, t1 = part.last;
  const bool alone = a.shared_items == 0 && n.per >= n.all();   // the only part: no merge
  if (alone && it.part > 0) return;

  // a thread's share of a tile: chunk ch of rows r0, r0 + kStep, ...; of codes, 16 of rows
  // q0, q0 + 2 kStep, ...
  const int r0 = tid / C, ch = tid % C, q0 = tid / (C / 2), qc = tid % (C / 2);
  const int at16 = ch * 8 < a.dim ? ch * 16 : kOutside, at8 = qc * 16 < a.dim ? qc * 16 : kOutside;
  u32x4 rk[kUnits], rv[kUnits];
  uint32_t sk[kUnits / 2], sv[kUnits / 2];
  auto load = [&](const Walk &w) {
    if (Q8 && w.source != 2) {
      const auto bk = buffer(w.k, extent(w.left, kKeyTile, w.k_row, a.dim));
      const auto bv = buffer(w.v, extent(w.left, kKeyTile, w.v_row, a.dim));
      const auto bks = buffer(w.ks, extent(w.left, kKeyTile, w.ks_row, 1));
      const auto bvs = buffer(w.vs, extent(w.left, kKeyTile, w.vs_row, 1));
#pragma unroll
      for (int i = 0; i < kUnits / 2; ++i) {
        const int r = q0 + i * 2 * kStep;
        rk[i] = load16(bk, r * w.k_row + at8);
        sk[i] = __builtin_amdgcn_raw_buffer_load_b8(bks, r * w.ks_row, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < kUnits / 2; ++i) {
        const int r = q0 + i * 2 * kStep;
        rv[i] = load16(bv, r * w.v_row + at8);
        sv[i] = __builtin_amdgcn_raw_buffer_load_b8(bvs, r * w.vs_row, 0, 0);
      }
    } else {
      const auto bk = buffer(w.k, extent(w.left, kKeyTile, w.k_row, 2 * a.dim));
      const auto bv = buffer(w.v, extent(w.left, kKeyTile, w.v_row, 2 * a.dim));
#pragma unroll
      for (int i = 0; i < kUnits; ++i) rk[i] = load16(bk, (r0 + i * kStep) * w.k_row + at16);
#pragma unroll
      for (int i = 0; i < kUnits; ++i) rv[i] = load16(bv, (r0 + i * kStep) * w.v_row + at16);
    }
  };
  // Stores the share; true if a block's value is infinite or NaN (stored as 0 then: a zero
  // probability of a hidden slot must not meet it).
  auto store = [&](int source, int buf) {
    bool odd = false;
    u32x4 *k = s_k + buf * kBuf, *v = s_v + buf * kBuf;
    if (Q8 && source != 2) {
#pragma unroll
      for (int i = 0; i < kUnits / 2; ++i) {
        const int r = q0 + i * 2 * kStep;
        const float uk = unit_of(sk[i]), uv = unit_of(sv[i]);
        u32x2 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = widen(rk[i][j], uk);
        k[k_at<C>(r, 2 * qc)] = u32x4{x[0].x, x[0].y, x[1].x, x[1].y};
        k[k_at<C>(r, 2 * qc + 1)] = u32x4{x[2].x, x[2].y, x[3].x, x[3].y};
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = widen(rv[i][j], uv);
        v[v_at<C>(r, 2 * qc)] = u32x4{x[0].x, x[0].y, x[1].x, x[1].y};
        v[v_at<C>(r, 2 * qc + 1)] = u32x4{x[2].x, x[2].y, x[3].x, x[3].y};
      }
    } else {
      if (source == 2) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) odd |= tame<T>(rv[i]);
      }
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int r = r0 + i * kStep;
        k[k_at<C>(r, ch)] = rk[i];
        v[v_at<C>(r, ch)] = rv[i];
      }
    }
    return odd;
  };

  // the queries: the right operand of S^T = K Q^T
  u32x4 rq[kSteps];
  const char *qp = a.q + rb * a.q_batch + slot * a.q_slot + head * a.q_head;
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
    rq[s] = s * 16 < a.dim ? *reinterpret_cast<const u32x4 *>(qp + s * 32 + h * 16) : u32x4{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < kSteps; ++s) settle(rq[s]);

  Sums<DP> st;
  st.clear(a.c);
  Walk w{};
  uint64_t seen_next = 0;
  if (t0 < t1) {
    seek(w, n, t0, kKeyTile, a.shared_len, len, live, b, kvh);
    load(w);
    if (w.source == 2) seen_next = seen_word(a, rb, slot, w.tile, live);
  }
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    const int source = w.source, left = w.left;
    const char *v_rows = w.v;
    const int v_row = w.v_row;
    const uint64_t seen = seen_next;
    const bool odd = store(source, buf);
    if (t + 1 < t1) {
      if (w.left > kKeyTile) advance(w, 1, kKeyTile);
      else seek(w, n, t + 1, kKeyTile, a.shared_len, len, live, b, kvh);
      load(w);
      if (w.source == 2) seen_next = seen_word(a, rb, slot, w.tile, live);
    }
    bool any_odd = false;
    if (source == 2) any_odd = __syncthreads_or(odd);
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
    if (source == 2 || left < kKeyTile) {
      const uint64_t bits = (source == 2 ? seen : (1ull << left) - 1) >> (4 * h);
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
    if (any_odd) {
      add_odd<T, DP>(v_rows, v_row, left < kKeyTile ? left : kKeyTile, seen, h, a.dim, st);
    }
  }

  st.l = half_sum(st.l);
  if (!valid) return;
  if (!alone) {
    const int at_part = packed ? a.splits + it.part : it.part;
    const int64_t r = (static_cast<int64_t>(rb) * a.slots + slot) * a.q_heads + head;
    const int64_t at = at_part * a.rows_all + r;
    if (h == 0) a.part_ml[at] = f32x2{t0 < t1 ? st.m : -INFINITY, st.l};
    if (t0 >= t1) return;
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
  char *op = a.out + rb * a.o_batch + slot * a.o_slot + head * a.o_head;
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
  if (a.lse && h == 0)
    a.lse[(static_cast<int64_t>(rb) * a.slots + slot) * a.q_heads + head] =
        st.l == 0.0f ? -INFINITY : (st.m * a.c + (__log2f(st.l) - ref_of<T>(st.m, a.c).at)) * 0.69314718055994531f;
}

// Infinite and NaN values as in add_odd, for the narrow walk's rows.
template <typename T, int DP>
__device__ __forceinline__ void add_odd(const char *v, int v_row, int count, uint32_t seen, int quarter, int dim,
                                        f32x4 (&o)[DP / 16]) {
#pragma unroll 1
  for (int j = 0; j < count; ++j) {
    const bool on = (seen >> j) & 1;
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) {
      const int at = d * 16 + 4 * quarter;
      u32x2 w{0, 0};
      if (on && at < dim) w = *reinterpret_cast<const u32x2 *>(v + static_cast<int64_t>(j) * v_row + 2 * at);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint16_t n = static_cast<uint16_t>(w[x / 2] >> (16 * (x & 1)));
        o[d][x] += (n & T::kExp) == T::kExp ? T::number(n) : 0.0f;
      }
    }
  }
}

// Rows of the narrow walk, 16 QT of them, on v_mfma_f32_16x16x32: lane l gives row (or
// column) l % 16 and 8 of the 32 contracted entries from 8 (l / 16) on; of the 16 x 16
// result it holds column l % 16, rows 4 (l / 16) + i.  The same forms as the wide walk's:
// scores transposed, a lane's 8 of a 32-key tile (keys 4 c + i and 16 + 4 c + i in
// quarter c) used as they are.
template <typename T, bool Q8, int DP, int QT>
__device__ __forceinline__ void narrow_part(const AttendArgs &a, const Item &it, u32x4 *lds) {
  constexpr int C = DP / 8, kSteps = DP / 32, kDTiles = DP / 16, kRows = 16 * QT;
  constexpr int kLoads = Q8 ? DP / 64 : kSteps;         // 16-byte loads of a lane and 16 keys
  constexpr int kPad = DP + 4;                          // floats of a row when the waves are joined
  const int tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);   // uniform: the walk's tables stay scalar
  const int quarter = lane >> 4, col = lane & 15;
  const int b = it.b, kvh = it.kvh;
  const bool packed = it.packed;
  u32x4 *s_v = lds + wave * kFewKeys * C;

  bool bad = false, unused;
  const int per_seq = a.slots * a.group;
  const int live = packed ? 0 : __builtin_amdgcn_readfirstlane(slots_of(a, b, &bad));
  const int len = packed ? 0 : __builtin_amdgcn_readfirstlane(len_of(a, b, &bad));
  if (bad && it.tile_row == 0 && it.part == 0 && kvh == 0 && tid == 0) atomicOr(a.error_flag, kErrBlockSizes);
  if (!packed && it.tile_row * kRows >= live * a.group) return;

  // sequence, slot and query head of row i of the workgroup's tile
  auto place = [&](int i, int *rb, int *slot, int *head) {
    int row = it.tile_row * kRows + i;
    *rb = b;
    if (packed) {
      *rb = row < a.batch * per_seq ? row / per_seq : a.batch - 1;
      row -= *rb * per_seq;
    }
    const int rlive = packed ? slots_of(a, *rb, &unused) : live;
    const bool valid = row < rlive * a.group;
    row = row < per_seq ? row : per_seq - 1;
    *slot = row / a.group;
    *head = kvh * a.group + row - *slot * a.group;
    return valid;
  };

  // a part's tiles, in rounds of one tile a wave
  const Tiles n = tiles_of(a, packed, len, live);
  const Part part = part_of(n, it.part);
  const int t0 = part.first, t1 = part.last;
  const bool alone = a.shared_items == 0 && n.per >= n.all();   // the only part: no merge
  if (alone && it.part > 0) return;

  // Contracted entries 8 of a step are chunk k_chunk(step) of a row: the 16 codes that one
  // load brings are two steps' 8.
  auto k_chunk = [&](int s) { return Q8 ? 2 * (4 * (s / 2) + quarter) + s % 2 : 4 * s + quarter; };
  u32x4 rq[QT][kSteps];
  int slots[QT];
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    int rb, head;
    place(q * 16 + col, &rb, &slots[q], &head);
    const char *qp = a.q + rb * a.q_batch + slots[q] * a.q_slot + head * a.q_head;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      rq[q][s] = k_chunk(s) * 8 < a.dim ? *reinterpret_cast<const u32x4 *>(qp + k_chunk(s) * 16) : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int q = 0; q < QT; ++q)
#pragma unroll
    for (int s = 0; s < kSteps; ++s) settle(rq[q][s]);

  const int r0 = lane / C, ch = lane % C, q0 = lane / (C / 2), qc = lane % (C / 2);
  const int at16 = ch * 8 < a.dim ? ch * 16 : kOutside, at8 = qc * 16 < a.dim ? qc * 16 : kOutside;
  constexpr int kVLoads = Q8 ? C / 4 : C / 2, kVStep = Q8 ? 2 * kWave / C : kWave / C;
  struct Held {                                         // a tile on its way
    u32x4 rk[2][kLoads], rv[kVLoads];
    uint32_t sk, sv;                                    // scales of row lane % 32
    int left;
  };
  auto load = [&](Held &x, const Walk &w) {
    x.left = w.left;
    constexpr int kBytes = Q8 ? 1 : 2;
    const auto bk = buffer(w.k, extent(w.left, kFewKeys, w.k_row, kBytes * a.dim));
    const auto bv = buffer(w.v, extent(w.left, kFewKeys, w.v_row, kBytes * a.dim));
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = (4 * i + quarter) * 16;
        x.rk[kt][i] = load16(bk, (16 * kt + col) * w.k_row + (at < kBytes * a.dim ? at : kOutside));
      }
#pragma unroll
    for (int i = 0; i < kVLoads; ++i) {
      const int r = (Q8 ? q0 : r0) + i * kVStep;
      x.rv[i] = load16(bv, r * w.v_row + (Q8 ? at8 : at16));
    }
    if (Q8) {
      const auto bks = buffer(w.ks, extent(w.left, kFewKeys, w.ks_row, 1));
      const auto bvs = buffer(w.vs, extent(w.left, kFewKeys, w.vs_row, 1));
      x.sk = __builtin_amdgcn_raw_buffer_load_b8(bks, (lane & 31) * w.ks_row, 0, 0);
      x.sv = __builtin_amdgcn_raw_buffer_load_b8(bvs, (lane & 31) * w.vs_row, 0, 0);
    }
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
  // A tile's scores into the running sums, its values being in LDS.  The wave's LDS
  // operations are done in order.
  auto take = [&](f32x4 (&s)[QT][2]) {
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
  };
  auto hide = [&](f32x4 (&s)[2], uint32_t seen) {
    const uint32_t bits = seen >> (4 * quarter);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i / 4][i % 4] = (bits >> (16 * (i / 4) + i % 4)) & 1u ? s[i / 4][i % 4] : -INFINITY;
  };

  // the prefix's tiles, the next one on its way (two: no faster, and 60 to 90 registers more)
  Walk w{};
  int t = t0 + wave;
  const int prefix = n.n0 + n.n1, t_end = t1 < prefix ? t1 : prefix;
  int ahead = t;                                        // the walk's tile
  auto fetch = [&](Held &x) {
    if (ahead >= t_end) return;
    if (ahead == t0 + wave || w.left <= kAttWaves * kFewKeys)
      seek(w, n, ahead, kFewKeys, a.shared_len, len, live, b, kvh);
    else
      advance(w, kAttWaves, kFewKeys);
    load(x, w);
    ahead += kAttWaves;
  };
  auto step = [&](Held &x) {
    const int left = x.left;
    // row 16 kt + col's scale: lanes col and col + 16 of each half hold both
    const u32x2 pair = Q8 ? __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x.sk, x.sk, false, false)) : u32x2{0, 0};
    f32x4 s[QT][2];
#pragma unroll
    for (int q = 0; q < QT; ++q) s[q][0] = s[q][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const float uk = unit_of(kt == 0 ? pair.x : pair.y);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        u32x4 f[2];
        if (Q8) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u32x2 y = widen(x.rk[kt][i][j], uk);
            f[j / 2][2 * (j % 2)] = y.x;
            f[j / 2][2 * (j % 2) + 1] = y.y;
          }
        } else {
          f[0] = x.rk[kt][i];
        }
#pragma unroll
        for (int j = 0; j < (Q8 ? 2 : 1); ++j)
#pragma unroll
          for (int q = 0; q < QT; ++q) s[q][kt] = T::mfma(f[j], rq[q][Q8 ? 2 * i + j : i], s[q][kt]);
      }
    }
#pragma unroll
    for (int i = 0; i < kVLoads; ++i) {
      const int r = (Q8 ? q0 : r0) + i * kVStep;
      if (Q8) {
        const float uv = unit_of(__builtin_amdgcn_ds_bpermute(4 * r, static_cast<int>(x.sv)));
        u32x2 y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = widen(x.rv[i][j], uv);
        s_v[v_at<C>(r, 2 * qc)] = u32x4{y[0].x, y[0].y, y[1].x, y[1].y};
        s_v[v_at<C>(r, 2 * qc + 1)] = u32x4{y[2].x, y[2].y, y[3].x, y[3].y};
      } else {
        s_v[v_at<C>(r, ch)] = x.rv[i];
      }
    }
    fetch(x);
    if (left < kFewKeys) {
#pragma unroll
      for (int q = 0; q < QT; ++q) hide(s[q], (1u << left) - 1);
    }
    take(s);
    t += kAttWaves;
  };
  Held held;
  fetch(held);
  while (t < t_end) step(held);
  // the block: at most 32 slots, one tile, by the wave whose turn it is
  if (t == prefix && t < t1) {
    seek(w, n, t, kFewKeys, a.shared_len, len, live, b, kvh);
    const auto bk = buffer(w.k, extent(live, kFewKeys, w.k_row, 2 * a.dim));
    const auto bv = buffer(w.v, extent(live, kFewKeys, w.v_row, 2 * a.dim));
    f32x4 s[QT][2];
#pragma unroll
    for (int q = 0; q < QT; ++q) s[q][0] = s[q][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const u32x4 f = load16(bk, (16 * kt + col) * w.k_row + (k_chunk(i) * 8 < a.dim ? k_chunk(i) * 16 : kOutside));
#pragma unroll
        for (int q = 0; q < QT; ++q) s[q][kt] = T::mfma(f, rq[q][i], s[q][kt]);
      }
    bool odd = false;
#pragma unroll
    for (int i = 0; i < C / 2; ++i) {
      const int r = r0 + i * (kWave / C);
      u32x4 x = load16(bv, r * w.v_row + at16);
      odd |= tame<T>(x);
      s_v[v_at<C>(r, ch)] = x;
    }
    uint32_t seen[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      seen[q] = static_cast<uint32_t>(seen_word(a, b, slots[q], 0, live));
      hide(s[q], seen[q]);
    }
    take(s);
    if (__ballot(odd) != 0) {
#pragma unroll
      for (int q = 0; q < QT; ++q) add_odd<T, DP>(w.v, w.v_row, live, seen[q], quarter, a.dim, o[q]);
    }
  }

  // The four waves' rows: each leaves its own with its maximum and sum, then every thread
  // joins 4 numbers of a row, the waves in order.
  float *s_o = reinterpret_cast<float *>(lds);
  float *s_m = s_o + kAttWaves * 16 * kPad, *s_l = s_m + kAttWaves * 16;
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
    for (int u = tid; u < 16 * (DP / 4); u += kAttThreads) {
      const int r = u / (DP / 4), x = (u % (DP / 4)) * 4;
      int rb, slot, head;
      if (!place(q * 16 + r, &rb, &slot, &head) || x >= a.dim) continue;
      float top = s_m[r];
#pragma unroll
      for (int i = 1; i < kAttWaves; ++i) top = fmaxf(top, s_m[i * 16 + r]);
      const Ref now = ref_of<T>(top, a.c);
      f32x4 sum{0.0f, 0.0f, 0.0f, 0.0f};
      float total = 0.0f;
#pragma unroll
      for (int i = 0; i < kAttWaves; ++i) {
        const float mi = s_m[i * 16 + r];
        const float f = mi == top ? 1.0f : factor(mi, ref_of<T>(mi, a.c).at, top, now, a.c);
        total += s_l[i * 16 + r] * f;
        sum += *reinterpret_cast<const f32x4 *>(s_o + (i * 16 + r) * kPad + x) * f;
      }
      const int64_t all = (static_cast<int64_t>(rb) * a.slots + slot) * a.q_heads + head;
      if (!alone) {
        const int64_t at = (packed ? a.splits + it.part : it.part) * a.rows_all + all;
        if (x == 0) a.part_ml[at] = f32x2{t0 < t1 ? top : -INFINITY, total};
        if (t0 < t1) *reinterpret_cast<f32x4 *>(a.part_o + at * a.dim + x) = sum;
      } else {
        const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
        *reinterpret_cast<u32x2 *>(a.out + rb * a.o_batch + slot * a.o_slot + head * a.o_head + 2 * x) =
            u32x2{T::pack(sum.x * inv, sum.y * inv), T::pack(sum.z * inv, sum.w * inv)};
        if (a.lse && x == 0)
          a.lse[all] =
              total == 0.0f ? -INFINITY : (top * a.c + (__log2f(total) - now.at)) * 0.69314718055994531f;
      }
    }
  }
}

// QT = 0: the wide walk; else the narrow one, 16 QT rows.
template <typename T, bool Q8, int DP, int QT>
__global__ void __launch_bounds__(kAttThreads, QT == 1 || (QT == 2 && DP == 64) ? 3 : 2)
attend_kernel(AttendArgs a) {
  constexpr int kNarrow = (kAttWaves * 16 * (DP + 4) + 2 * kAttWaves * 16 + 3) / 4;   // joining the waves
  constexpr int kValues = kAttWaves * kFewKeys * (DP / 8);
  __shared__ __align__(16) u32x4 lds[QT == 0 ? 4 * kKeyTile * (DP / 8) : (kNarrow > kValues ? kNarrow : kValues)];
  Item it;
  it.packed = static_cast<int>(blockIdx.x) < a.shared_items;
  if (it.packed) {
    int i = blockIdx.x;
    it.part = i % a.shared_splits;
    i /= a.shared_splits;
    it.tile_row = i % a.shared_tiles;
    it.kvh = i / a.shared_tiles;
    it.b = 0;
  } else {
    // Workgroups go round the 8 XCDs.  What reads the same memory follows each other on one:
    // wide, the row tiles of a (part, sequence, key head), whose keys then stay in its L2 (the
    // heads' keys together would not: 1806 against 1380 us for 64 trees of up to 512 nodes);
    // narrow, the key heads of a (part, sequence), whose rows lie side by side.  The groups go by
    // an odd number (one of them may be empty), so that a sequence's parts fall on all XCDs;
    // parts that short sequences leave empty come last.
    const int i = blockIdx.x - a.shared_items;
    const int j = i >> 3, inner = QT == 0 ? a.row_tiles : a.kv_heads * a.row_tiles;
    const int g = (j / inner) * 8 + (i & 7), r = j % inner;
    const int outer = QT == 0 ? a.batch * a.kv_heads : a.batch, odd = outer | 1;
    it.part = g / odd;
    const int o = g - it.part * odd;
    it.b = QT == 0 ? o / a.kv_heads : o;
    it.kvh = QT == 0 ? o - it.b * a.kv_heads : r / a.row_tiles;
    it.tile_row = QT == 0 ? r : r - it.kvh * a.row_tiles;
    if (it.part >= a.splits || o >= outer) return;
  }
  if (QT == 0) wide_part<T, Q8, DP>(a, it, lds);
  else narrow_part<T, Q8, DP, QT == 0 ? 1 : QT>(a, it, lds);
}

// Joins the parts of a row: a wave each, one part a lane for the statistics, two
// numbers a lane for the row.
template <typename T>
__global__ void __launch_bounds__(kAttThreads)
merge_parts_kernel(AttendArgs a) {
  const int lane = lane_id();
  const int64_t r = static_cast<int64_t>(blockIdx.x) * kAttWaves + threadIdx.x / kWave;
  if (r >= a.rows_all) return;
  const int64_t bs = r / a.q_heads;
  const int head = static_cast<int>(r - bs * a.q_heads);
  const int b = static_cast<int>(bs / a.slots), slot = static_cast<int>(bs - static_cast<int64_t>(b) * a.slots);
  bool unused;
  const int live = slots_of(a, b, &unused);
  if (slot >= live) return;
  const Tiles n = tiles_of(a, false, len_of(a, b, &unused), live);
  if (a.shared_items == 0 && n.per >= n.all()) return;     // its only part wrote the row
  const f32x2 ml = lane < a.parts ? a.part_ml[lane * a.rows_all + r] : f32x2{-INFINITY, 0.0f};
  float top = ml.x;
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) top = fmaxf(top, __uint_as_float(xor_lane(__float_as_uint(top), k)));
  // 0 for a part without keys
  const Ref now = ref_of<T>(top, a.c);
  const float w = ml.x == top && top != -INFINITY ? 1.0f : factor(ml.x, ref_of<T>(ml.x, a.c).at, top, now, a.c);
  float l = w * ml.y;
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) l += __uint_as_float(xor_lane(__float_as_uint(l), k));
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  const uint64_t used = __ballot(lane < a.parts && ml.x != -INFINITY);
  float x = 0.0f, y = 0.0f;
  if (lane * 2 < a.dim) {
    for (uint64_t left = used; left; left &= left - 1) {
      const int p = __builtin_ctzll(left);
      const f32x2 v = *reinterpret_cast<const f32x2 *>(a.part_o + (p * a.rows_all + r) * a.dim + lane * 2);
      const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), p));
      x = __builtin_fmaf(f, v.x, x);
      y = __builtin_fmaf(f, v.y, y);
    }
    *reinterpret_cast<uint32_t *>(a.out + b * a.o_batch + slot * a.o_slot + head * a.o_head + lane * 4) =
        T::pack(x * inv, y * inv);
  }
  if (a.lse && lane == 0)
    a.lse[r] = l == 0.0f ? -INFINITY : (top * a.c + (__log2f(l) - now.at)) * 0.69314718055994531f;
}

// rows: extent along the row stride; a stride that one row does not need is the row's own
// length, since the bounds of a tile's buffer are counted with it.
Side side(const graft_rows &r, int bytes, int dim, int rows) {
  Side s;
  s.p = static_cast<const char *>(r.data);
  s.batch = r.batch_stride * bytes;
  s.row = static_cast<int32_t>((rows > 1 ? r.row_stride : dim) * bytes);
  s.head = r.head_stride * bytes;
  s.s = r.scale;
  s.s_batch = r.scale_batch_stride;
  s.s_row = static_cast<int32_t>(rows > 1 ? r.scale_row_stride : 1);
  s.s_head = r.scale_head_stride;
  return s;
}

}  // namespace

// The narrow walk up to 32 rows of a sequence and key head.  us narrow and wide, in a graph, three
// input sets in turn, 8 key heads of 128 over up to 4096 rows:
//   rows                    8          16          24          32
//   1 sequence, bf16     25.4 21.3   26.8 21.4   28.6 21.4   30.1 21.5
//   32 sequences, bf16   79.2 79.1   84.0 80.3  102.8 82.6  108.4 83.1
//   32 sequences, e4m3   57.6 83.3   63.4 84.4   88.1 85.0   93.3 86.1
// One token of 20 and 32 heads a key head over 16384 rows 27.2 28.8 and 30.2 32.1, e4m3 26.2 30.4 and
// 29.6 32.7; over 700 rows 15.2 15.8 and 16.6 16.1, e4m3 14.9 16.8 and 15.8 17.2; 64 trees of 7 nodes
// over up to 4096 e4m3 rows 119 148.  So up to 16 rows the narrow walk wins or is near; from 17 to
// 32 it wins over codes and for single tokens, and trees over bf16 rows would be faster in the wide one.
// 17 to 32 rows are one row tile, in two tiles of columns that share every row read.  Two row tiles of 16
// would read a cache twice: 24 and 32 rows 26.7 and 27.0, 97.5 and 96.5, 72.3 and 72.9 us in the lines
// above, where there are few workgroups or the second read comes from a cache, but 64 trees of 7 nodes of 4
// key heads over up to 16384 bf16 rows 294 instead of 268, and beside 4096 shared rows 205 instead of 153.
AttendPlan attend_plan(const graft_attention &a) {
  AttendPlan p{};
  const int group = a.q_heads / a.kv_heads;
  const int64_t rows = static_cast<int64_t>(a.slots) * group;
  p.column_tiles = rows <= 16 ? 1 : rows <= kFewRows ? 2 : 0;
  const bool few = p.column_tiles > 0;
  const int tile = few ? 16 * p.column_tiles : kRowTile;
  p.row_tiles = static_cast<int>((rows + tile - 1) / tile);
  const int64_t units = static_cast<int64_t>(a.batch) * a.kv_heads * p.row_tiles;
  // keys of a tile of the wide walk, or of a round of the narrow one's four waves
  const int keys = few ? kFewKeys * kAttWaves : kKeyTile;
  auto tiles = [](int64_t n, int k) { return (n + k - 1) / k; };
  // a pass of its own where sequences share a row tile
  const bool own_pass = a.shared_len > 0 && a.batch > 1 && rows * 2 <= kRowTile;
  const int64_t most = (own_pass ? 0 : tiles(a.shared_len, keys)) + tiles(a.cache_rows, keys) + tiles(a.slots, keys);
  // the shortest part: below it a part costs more than it shares (one token over 700 keys
  // 11.4 us, in parts of 4 rounds 12.7; 5 trees of 70 nodes over 1664 keys 24.2 us, in parts of
  // 2 tiles 29.2, of 8 26.8)
  p.min_tiles = few ? 1 : 4;
  auto cut = [&](int64_t n_units, int64_t n_tiles, int64_t want, int64_t cap) {
    int64_t s = (want + n_units - 1) / n_units;
    s = std::min(s, (n_tiles + p.min_tiles - 1) / p.min_tiles);
    return static_cast<int>(std::max<int64_t>(1, std::min(s, cap)));
  };
  if (own_pass) {
    p.shared_tiles = static_cast<int>((a.batch * rows + tile - 1) / tile);
    p.shared_splits = cut(static_cast<int64_t>(a.kv_heads) * p.shared_tiles, tiles(a.shared_len, keys), 256, 32);
  }
  // a wide part leaves 512 bytes for each of its rows, which the merge reads: splitting pays
  // only where the chip is not filled (16 trees of up to 256 nodes: 200 us whole, 240 in 4 parts)
  p.splits = cut(units, most, few ? 4096 : 1024, own_pass ? 32 : kMaxParts);
  p.parts = p.splits + p.shared_splits;
  const int64_t all = static_cast<int64_t>(a.batch) * a.slots * a.q_heads;
  const int64_t outer = few ? a.batch : static_cast<int64_t>(a.batch) * a.kv_heads;
  const int64_t groups = ((outer | 1) * p.splits + 7) / 8 * 8 * (few ? a.kv_heads : 1);
  p.blocks = static_cast<int64_t>(a.kv_heads) * p.shared_tiles * p.shared_splits + groups * p.row_tiles;
  p.merge_blocks = p.parts > 1 ? (all + kAttWaves - 1) / kAttWaves : 0;
  p.bytes = p.parts > 1 ? p.parts * all * (a.head_dim * int64_t{4} + 8) : 0;
  return p;
}

hipError_t launch_attend(graft_ctx *ctx, const graft_attention &d, const AttendPlan &p,
                         hipStream_t stream) {
  const bool q8 = d.cache_dtype == GRAFT_E4M3;
  AttendArgs a{};
  const int w = q8 ? 1 : 2;
  a.src[0] = Source{side(d.shared_k, w, d.head_dim, d.shared_len), side(d.shared_v, w, d.head_dim, d.shared_len)};
  a.src[1] = Source{side(d.cache_k, w, d.head_dim, d.cache_rows), side(d.cache_v, w, d.head_dim, d.cache_rows)};
  a.src[2] = Source{side(d.k, 2, d.head_dim, d.slots), side(d.v, 2, d.head_dim, d.slots)};
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
  a.part_ml = p.parts > 1 ? reinterpret_cast<f32x2 *>(a.part_o + p.parts * a.rows_all * d.head_dim) : nullptr;
  a.batch = d.batch;
  a.slots = d.slots;
  a.root = d.with_root ? 1 : 0;
  a.q_heads = d.q_heads;
  a.kv_heads = d.kv_heads;
  a.group = d.q_heads / d.kv_heads;
  a.dim = d.head_dim;
  a.n_max = ctx->dims.max_nodes;
  a.words = (ctx->dims.max_nodes + 63) / 64;
  a.cache_rows = d.cache_rows;
  a.shared_len = d.shared_len;
  a.tile_keys = p.column_tiles > 0 ? kFewKeys : kKeyTile;
  a.turns = p.column_tiles > 0 ? kAttWaves : 1;
  a.row_tiles = p.row_tiles;
  a.splits = p.splits;
  a.min_tiles = p.min_tiles;
  a.shared_tiles = p.shared_tiles;
  a.shared_splits = p.shared_splits;
  a.parts = p.parts;
  a.shared_items = p.shared_tiles * p.shared_splits * d.kv_heads;
  a.c = d.scale * 1.4426950408889634f;
  const dim3 grid(static_cast<unsigned>(p.blocks)), block(kAttThreads);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
  auto pick = [&](auto tiles, auto dp) {
    constexpr int F = decltype(tiles)::value;
    constexpr int D = decltype(dp)::value;
    if (d.dtype == GRAFT_F16) run(attend_kernel<F16, false, D, F>);
    else if (q8) run(attend_kernel<Bf16, true, D, F>);
    else run(attend_kernel<Bf16, false, D, F>);
  };
  // heads of other sizes run as 64 or 128 columns: 16 trees of up to 256 nodes 109 and 112 us at 32
  // and 64 numbers, 170, 171, 173 and 176 at 80, 96, 112 and 128
  auto width = [&](auto tiles) {
    if (d.head_dim > 64) pick(tiles, std::integral_constant<int, 128>{});
    else pick(tiles, std::integral_constant<int, 64>{});
  };
  if (p.column_tiles == 1) width(std::integral_constant<int, 1>{});
  else if (p.column_tiles == 2) width(std::integral_constant<int, 2>{});
  else width(std::integral_constant<int, 0>{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts <= 1) return e;
  const dim3 mgrid(static_cast<unsigned>(p.merge_blocks));
  if (d.dtype == GRAFT_F16) hipLaunchKernelGGL(merge_parts_kernel<F16>, mgrid, block, 0, stream, a);
  else hipLaunchKernelGGL(merge_parts_kernel<Bf16>, mgrid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace graft
