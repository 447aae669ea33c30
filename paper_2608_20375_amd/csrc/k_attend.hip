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
// one tile and a key is loaded once for all of them.  A workgroup takes 128 rows, 32
// a wave, and walks 64-key tiles staged in LDS, the next tile's loads in flight in
// registers meanwhile, two LDS buffers, one barrier a tile.
//
// Products.  v_mfma_f32_32x32x16: lane l gives row (or column) l % 32 and 8 of the 16
// contracted entries from 8 (l / 32) on; of the 32 x 32 result it holds column l % 32,
// rows 8 (i / 4) + 4 (l / 32) + i % 4, i < 16.  S^T = K Q^T puts a query into a lane: its
// maximum and sum are taken in the lane, with one exchange with the other half of
// the wave.  O^T = V^T P^T then wants P^T as its right operand: any order of the
// contracted keys will do as long as V^T's is the same, so a lane's own 8 numbers of a
// 16-key group are used where they are, keys 4 h + {0..3, 8..11} of the group in lane
// half h, and V is stored transposed in LDS with the keys of each group in that order.
//
// LDS.  K: 16-byte chunk c of key r at chunk c ^ (r % 8 or 16), V^T: row d, 8-byte slot
// p at p ^ 2 ((d ^ d / 8) % 8): a wave's 16-byte reads of 8 rows and its stores of a
// column of chunks then touch different banks.
//
// The keys of a sequence (the shared prefix, its cache, its block: 64-key tiles of each)
// are split into parts where rows alone do not fill the chip; every part leaves its
// sums, maximum and unnormalised row in the workspace and merge_kernel joins them.
// When a sequence has fewer rows than a tile, the shared prefix is walked by
// workgroups of their own whose rows come from all sequences: it is read once for 128
// rows instead of once for every sequence.
#include <algorithm>

#include "graft_internal.h"

namespace graft {
namespace {

constexpr int kAttThreads = 256;
constexpr int kAttWaves = kAttThreads / kWave;
constexpr int kRowTile = 128;
constexpr int kKeyTile = 64;
constexpr int kMaxParts = 64;          // one a lane of the merge

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct Bf16 {
  static constexpr uint32_t kExp = 0x7F80u;      // exponent of infinities and NaN
  static __device__ __forceinline__ f32x16 mfma(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
  }
  static __device__ __forceinline__ float number(uint16_t h) {
    return __uint_as_float(static_cast<uint32_t>(h) << 16);
  }
};
struct F16 {
  static constexpr uint32_t kExp = 0x7C00u;
  static __device__ __forceinline__ f32x16 mfma(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, f16x2));
  }
  static __device__ __forceinline__ float number(uint16_t h) {
    return static_cast<float>(__builtin_bit_cast(_Float16, h));
  }
};

// A side (keys or values) of one source of rows; strides in bytes.
struct Side {
  const char *p;
  int64_t batch, row, head;
  const uint8_t *s;
  int64_t s_batch, s_row, s_head;
};

struct AttendArgs {
  Side block_k, block_v, cache_k, cache_v, shared_k, shared_v;
  const char *q;
  char *out;
  int64_t q_batch, q_slot, q_head, o_batch, o_slot, o_head;   // bytes
  const int32_t *n_nodes, *cache_len;
  const uint64_t *mask;
  float *lse;
  float *part_o;          // [parts][batch * slots * q_heads][head_dim], unnormalised
  f32x2 *part_ml;         // [parts][batch * slots * q_heads] c * maximum, sum
  uint32_t *error_flag;
  int64_t rows_all;       // batch * slots * q_heads
  int32_t batch, slots, root, q_heads, kv_heads, group, dim;
  int32_t n_max, words, cache_rows, shared_len;
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

// One 64-key tile of a source.
struct Tile {
  Side k, v;              // p, s moved to the sequence and key head
  int key0, count;
  bool quant, block;
};

// e4m3 pair -> two numbers of 16 bits with the scale applied; exact in bf16.
__device__ __forceinline__ uint32_t widen(uint32_t w, bool high, float unit) {
  const f32x2 x = high ? __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true)
                       : __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
  return (__float_as_uint(x.x * unit) >> 16) | (__float_as_uint(x.y * unit) & 0xFFFF0000u);
}
__device__ __forceinline__ float unit_of(uint32_t s) {
  return __uint_as_float(s ? s << 23 : 0x00400000u);
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

template <typename T, bool Q8, int DP>
__global__ void __launch_bounds__(kAttThreads, 2)
attend_kernel(AttendArgs a) {
  constexpr int kChunks = DP / 8;                       // 16-byte chunks of a key row in LDS
  constexpr int kSteps = DP / 16, kDTiles = DP / 32;
  constexpr int kKUnits = kKeyTile * kChunks / kAttThreads;
  constexpr int kVThreads = kKeyTile / 4 * kChunks;     // 4 keys x 8 numbers each
  __shared__ __align__(16) u32x4 s_k[2][kKeyTile * kChunks];
  __shared__ __align__(16) u32x2 s_v[2][DP * (kKeyTile / 4)];

  const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
  const int h = lane >> 5, col = lane & 31;

  // which rows and which keys
  const bool packed = static_cast<int>(blockIdx.x) < a.shared_items;
  int b = 0, kvh, tile_row, part;
  if (packed) {
    int i = blockIdx.x;
    part = i % a.shared_splits;
    i /= a.shared_splits;
    tile_row = i % a.shared_tiles;
    kvh = i / a.shared_tiles;
  } else {
    // the row tiles of one (sequence, key head, part) read the same keys: they
    // follow each other on one XCD (workgroups go round the 8 XCDs)
    const int i = blockIdx.x - a.shared_items;
    const int j = i >> 3;
    const int g = (j / a.row_tiles) * 8 + (i & 7);
    tile_row = j % a.row_tiles;
    part = g % a.splits;
    const int bh = g / a.splits;
    b = bh / a.kv_heads;
    kvh = bh - b * a.kv_heads;
    if (b >= a.batch) return;
  }

  bool bad = false;
  const int per_seq = a.slots * a.group;
  const int live = packed ? 0 : slots_of(a, b, &bad);
  if (!packed && tile_row * kRowTile >= live * a.group) {
    if (bad && tile_row == 0 && part == 0 && kvh == 0 && tid == 0) atomicOr(a.error_flag, kErrBlockSizes);
    return;
  }
  int row = tile_row * kRowTile + wave * 32 + col;
  int rb = b;
  if (packed) {
    const int total = a.batch * per_seq;
    rb = row < total ? row / per_seq : a.batch - 1;
    row -= rb * per_seq;
  }
  bool unused;
  const int rlive = packed ? slots_of(a, rb, &unused) : live;
  const bool valid = row < rlive * a.group;
  row = row < per_seq ? row : per_seq - 1;
  const int slot = row / a.group, head = kvh * a.group + row - slot * a.group;
  if (packed && !__syncthreads_or(valid)) return;
  const bool busy = __ballot(valid) != 0;

  int len = 0;
  if (!packed && a.cache_rows > 0) {
    len = a.cache_len[b];
    bad |= len < 0 || len > a.cache_rows;
    len = len < 0 ? 0 : (len > a.cache_rows ? a.cache_rows : len);
  }
  if (bad && tile_row == 0 && part == 0 && kvh == 0 && tid == 0) atomicOr(a.error_flag, kErrBlockSizes);
  const int n_shared = packed || a.shared_items == 0 ? (a.shared_len + kKeyTile - 1) / kKeyTile : 0;
  const int n_cache = packed ? 0 : (len + kKeyTile - 1) / kKeyTile;
  const int n_block = packed ? 0 : (live + kKeyTile - 1) / kKeyTile;
  const int n_tiles = n_shared + n_cache + n_block;
  const int splits = packed ? a.shared_splits : a.splits;
  int per = (n_tiles + splits - 1) / splits;
  per = per < a.min_tiles ? a.min_tiles : per;
  const int t0 = part * per < n_tiles ? part * per : n_tiles;
  const int t1 = t0 + per < n_tiles ? t0 + per : n_tiles;

  auto tile_at = [&](int t) {
    Tile x;
    int64_t base;
    if (t < n_shared) {
      x.k = a.shared_k;
      x.v = a.shared_v;
      x.key0 = t * kKeyTile;
      x.count = a.shared_len - x.key0;
      x.quant = Q8;
      x.block = false;
      base = 0;
    } else if (t < n_shared + n_cache) {
      x.k = a.cache_k;
      x.v = a.cache_v;
      x.key0 = (t - n_shared) * kKeyTile;
      x.count = len - x.key0;
      x.quant = Q8;
      x.block = false;
      base = b;
    } else {
      x.k = a.block_k;
      x.v = a.block_v;
      x.key0 = (t - n_shared - n_cache) * kKeyTile;
      x.count = live - x.key0;
      x.quant = false;
      x.block = true;
      base = b;
    }
    x.count = x.count < kKeyTile ? x.count : kKeyTile;
    x.k.p += base * x.k.batch + kvh * x.k.head;
    x.v.p += base * x.v.batch + kvh * x.v.head;
    if (Q8 && x.quant) {
      x.k.s += base * x.k.s_batch + kvh * x.k.s_head;
      x.v.s += base * x.v.s_batch + kvh * x.v.s_head;
    }
    return x;
  };

  // a thread's share of a tile: kKUnits 16-byte chunks of keys (or half as many of
  // codes), and 4 keys x 8 numbers of the values
  u32x4 rk[kKUnits], rv[4];
  uint32_t sk[kKUnits], sv[4];
  const int vc = tid % kChunks, vg = tid / kChunks;
  const bool v_mine = tid < kVThreads && vc * 8 < a.dim;
  auto load = [&](const Tile &x) {
    if (Q8 && x.quant) {
      constexpr int kQ = kChunks / 2;
#pragma unroll
      for (int i = 0; i < kKUnits / 2; ++i) {
        const int u = tid + i * kAttThreads, r = u / kQ, c = u % kQ;
        rk[i] = u32x4{0, 0, 0, 0};
        sk[i] = 127;
        if (r < x.count && c * 16 < a.dim) {
          const int64_t key = x.key0 + r;
          rk[i] = *reinterpret_cast<const u32x4 *>(x.k.p + key * x.k.row + c * 16);
          sk[i] = x.k.s[key * x.k.s_row];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = vg * 4 + i;
        rv[i] = u32x4{0, 0, 0, 0};
        sv[i] = 127;
        if (v_mine && r < x.count) {
          const int64_t key = x.key0 + r;
          const u32x2 w = *reinterpret_cast<const u32x2 *>(x.v.p + key * x.v.row + vc * 8);
          rv[i] = u32x4{w.x, w.y, 0, 0};
          sv[i] = x.v.s[key * x.v.s_row];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kKUnits; ++i) {
        const int u = tid + i * kAttThreads, r = u / kChunks, c = u % kChunks;
        rk[i] = u32x4{0, 0, 0, 0};
        if (r < x.count && c * 8 < a.dim)
          rk[i] = *reinterpret_cast<const u32x4 *>(x.k.p + static_cast<int64_t>(x.key0 + r) * x.k.row + c * 16);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = vg * 4 + i;
        rv[i] = u32x4{0, 0, 0, 0};
        if (v_mine && r < x.count)
          rv[i] = *reinterpret_cast<const u32x4 *>(x.v.p + static_cast<int64_t>(x.key0 + r) * x.v.row + vc * 16);
      }
    }
  };
  // Stores the share; true if a block's value is infinite or NaN (stored as 0 then:
  // a zero probability of a hidden slot must not meet it).
  auto store = [&](const Tile &x, int buf) {
    bool odd = false;
    if (Q8 && x.quant) {
      constexpr int kQ = kChunks / 2;
#pragma unroll
      for (int i = 0; i < kKUnits / 2; ++i) {
        const int u = tid + i * kAttThreads, r = u / kQ, c = u % kQ;
        const float unit = unit_of(sk[i]);
        u32x4 w0, w1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t lo = widen(rk[i][j], false, unit), hi = widen(rk[i][j], true, unit);
          if (j < 2) { w0[2 * j] = lo; w0[2 * j + 1] = hi; }
          else { w1[2 * j - 4] = lo; w1[2 * j - 3] = hi; }
        }
        const int sw = r & (kChunks - 1);
        s_k[buf][r * kChunks + ((2 * c) ^ sw)] = w0;
        s_k[buf][r * kChunks + ((2 * c + 1) ^ sw)] = w1;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float unit = unit_of(sv[i]);
        const uint32_t x0 = rv[i].x, x1 = rv[i].y;
        rv[i] = u32x4{widen(x0, false, unit), widen(x0, true, unit), widen(x1, false, unit),
                      widen(x1, true, unit)};
      }
    } else {
#pragma unroll
      for (int i = 0; i < kKUnits; ++i) {
        const int u = tid + i * kAttThreads, r = u / kChunks, c = u % kChunks;
        s_k[buf][r * kChunks + (c ^ (r & (kChunks - 1)))] = rk[i];
      }
      if (x.block) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t w = rv[i][j];
            const uint32_t e = T::kExp;
            const bool lo = (w & e) == e, hi = (w & (e << 16)) == e << 16;
            odd |= lo | hi;
            rv[i][j] = w & ~((lo ? 0xFFFFu : 0u) | (hi ? 0xFFFF0000u : 0u));
          }
      }
    }
    if (tid < kVThreads) {
      // keys 4 vg .. + 3 are the low or the high four of half (vg & 1) of group vg / 4
      const int p = (vg >> 2) * 4 + (vg & 1) * 2 + ((vg >> 1) & 1);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int d = vc * 8 + j;
        const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
        u32x2 w;
        w.x = __builtin_amdgcn_perm(rv[1][j / 2], rv[0][j / 2], sel);
        w.y = __builtin_amdgcn_perm(rv[3][j / 2], rv[2][j / 2], sel);
        s_v[buf][d * (kKeyTile / 4) + (p ^ (2 * ((d ^ (d >> 3)) & 7)))] = w;
      }
    }
    return odd;
  };
  // The slots of block tile x that this lane's row sees.
  auto sees = [&](const Tile &x) -> uint64_t {
    const int tb = x.key0 / kKeyTile;
    uint64_t w;
    if (a.mask) {
      const int node = slot - a.root;
      if (node < 0) {
        w = tb == 0 ? 1 : 0;
      } else {
        const uint64_t *m = a.mask + (static_cast<int64_t>(rb) * a.n_max + node) * a.words;
        w = tb < a.words ? m[tb] : 0;
        if (a.root) w = (w << 1) | (tb > 0 ? m[tb - 1] >> 63 : 1);
      }
    } else {
      const int n = slot - x.key0 + 1;
      w = n <= 0 ? 0 : (n >= 64 ? ~0ull : (1ull << n) - 1);
    }
    return x.count < 64 ? w & ((1ull << x.count) - 1) : w;
  };

  // the queries: the right operand of S^T = K Q^T
  u32x4 rq[kSteps];
  const char *qp = a.q + rb * a.q_batch + slot * a.q_slot + head * a.q_head;
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
    rq[s] = s * 16 < a.dim ? *reinterpret_cast<const u32x4 *>(qp + s * 32 + h * 16) : u32x4{0, 0, 0, 0};

  f32x16 o[kDTiles];
#pragma unroll
  for (int d = 0; d < kDTiles; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  Tile cur{}, next{};
  uint64_t seen = 0, seen_next = 0;
  if (t0 < t1) {
    cur = tile_at(t0);
    load(cur);
    if (cur.block) seen = sees(cur);
  }
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    const bool odd = store(cur, buf);
    if (t + 1 < t1) {
      next = tile_at(t + 1);
      load(next);
      if (next.block) seen_next = sees(next);
    }
    bool any_odd = false;
    if (cur.block) any_odd = __syncthreads_or(odd);
    else __syncthreads();
    if (busy) {
      f32x16 s[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kt][i] = 0.0f;
        const int r = kt * 32 + col;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
          if (i * 16 < a.dim)
            s[kt] = T::mfma(s_k[buf][r * kChunks + ((2 * i + h) ^ (r & (kChunks - 1)))], rq[i], s[kt]);
      }
      if (cur.block || cur.count < kKeyTile) {
        const uint64_t w = cur.block ? seen : (1ull << cur.count) - 1;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          const uint32_t bits = static_cast<uint32_t>(w >> (32 * kt)) >> (4 * h);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            s[kt][i] = (bits >> (8 * (i / 4) + i % 4)) & 1u ? s[kt][i] : -INFINITY;
        }
      }
      float mx = m;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kt][i]);
      mx = fmaxf(mx, other_half(mx));
      const float off = mx == -INFINITY ? 0.0f : mx * a.c;
      if (__ballot(mx != m) != 0) {
        const float alpha = __builtin_amdgcn_exp2f(m * a.c - off);
        l *= alpha;
#pragma unroll
        for (int d = 0; d < kDTiles; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
        m = mx;
      }
      u32x4 p[4];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        float e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][i], a.c, -off));
          l += e[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) p[2 * kt + i / 4][i % 4] = T::pack(e[2 * i], e[2 * i + 1]);
      }
#pragma unroll
      for (int d = 0; d < kDTiles; ++d) {
        if (d * 32 >= a.dim) continue;
        const int r = d * 32 + col;
        const int sw = 2 * ((r ^ (r >> 3)) & 7);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const u32x4 v = *reinterpret_cast<const u32x4 *>(
              &s_v[buf][r * (kKeyTile / 4) + ((4 * g + 2 * h) ^ sw)]);
          o[d] = T::mfma(v, p[g], o[d]);
        }
      }
      if (any_odd) {
        // infinite and NaN values of the slots that the row does see
        for (int j = 0; j < cur.count; ++j) {
          const uint16_t *v = reinterpret_cast<const uint16_t *>(
              cur.v.p + static_cast<int64_t>(cur.key0 + j) * cur.v.row);
          if (!((seen >> j) & 1)) continue;
#pragma unroll
          for (int d = 0; d < kDTiles; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int at = d * 32 + 8 * (i / 4) + 4 * h + i % 4;
              if (at < a.dim && (v[at] & T::kExp) == T::kExp) o[d][i] += T::number(v[at]);
            }
        }
      }
    }
    cur = next;
    seen = seen_next;
  }

  l += other_half(l);
  if (!valid) return;
  if (a.parts > 1) {
    const int at_part = packed ? a.splits + part : part;
    const int64_t r = (static_cast<int64_t>(rb) * a.slots + slot) * a.q_heads + head;
    const int64_t at = at_part * a.rows_all + r;
    if (h == 0) a.part_ml[at] = f32x2{t0 < t1 ? m * a.c : -INFINITY, l};
    if (t0 >= t1) return;
    float *po = a.part_o + at * a.dim;
#pragma unroll
    for (int d = 0; d < kDTiles; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int x = d * 32 + 8 * i + 4 * h;
        if (x < a.dim)
          *reinterpret_cast<f32x4 *>(po + x) =
              f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
      }
    return;
  }
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  char *op = a.out + rb * a.o_batch + slot * a.o_slot + head * a.o_head;
#pragma unroll
  for (int d = 0; d < kDTiles; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = d * 32 + 8 * i + 4 * h;
      if (x < a.dim)
        *reinterpret_cast<u32x2 *>(op + 2 * x) =
            u32x2{T::pack(o[d][4 * i] * inv, o[d][4 * i + 1] * inv),
                  T::pack(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
    }
  if (a.lse && h == 0)
    a.lse[(static_cast<int64_t>(rb) * a.slots + slot) * a.q_heads + head] =
        l == 0.0f ? -INFINITY : (m * a.c + __log2f(l)) * 0.69314718055994531f;
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
  if (slot >= slots_of(a, b, &unused)) return;
  const f32x2 ml = lane < a.parts ? a.part_ml[lane * a.rows_all + r] : f32x2{-INFINITY, 0.0f};
  float top = ml.x;
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) top = fmaxf(top, __uint_as_float(xor_lane(__float_as_uint(top), k)));
  const float off = top == -INFINITY ? 0.0f : top;
  const float w = __builtin_amdgcn_exp2f(ml.x - off);      // 0 for a part without keys
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
  if (a.lse && lane == 0) a.lse[r] = l == 0.0f ? -INFINITY : (off + __log2f(l)) * 0.69314718055994531f;
}

Side side(const graft_rows &r, int bytes) {
  Side s;
  s.p = static_cast<const char *>(r.data);
  s.batch = r.batch_stride * bytes;
  s.row = r.row_stride * bytes;
  s.head = r.head_stride * bytes;
  s.s = r.scale;
  s.s_batch = r.scale_batch_stride;
  s.s_row = r.scale_row_stride;
  s.s_head = r.scale_head_stride;
  return s;
}

}  // namespace

AttendPlan attend_plan(const graft_attention &a) {
  AttendPlan p{};
  const int group = a.q_heads / a.kv_heads;
  const int64_t rows = static_cast<int64_t>(a.slots) * group;
  const int root = a.with_root ? 1 : 0;
  p.row_tiles = static_cast<int>((rows + kRowTile - 1) / kRowTile);
  const int64_t units = static_cast<int64_t>(a.batch) * a.kv_heads * p.row_tiles;
  auto tiles = [](int64_t n) { return (n + kKeyTile - 1) / kKeyTile; };
  const int64_t shared = tiles(a.shared_len);
  // a pass of its own where sequences share a row tile
  const bool own_pass = a.shared_len > 0 && a.batch > 1 && rows * 2 <= kRowTile;
  const int64_t most = (own_pass ? 0 : shared) + tiles(a.cache_rows) + tiles(a.slots);
  p.min_tiles = 4;
  auto cut = [&](int64_t n_units, int64_t n_tiles, int64_t want, int64_t cap) {
    int64_t s = (want + n_units - 1) / n_units;
    s = std::min(s, (n_tiles + p.min_tiles - 1) / p.min_tiles);
    return static_cast<int>(std::max<int64_t>(1, std::min(s, cap)));
  };
  (void)root;
  if (own_pass) {
    p.shared_tiles = static_cast<int>((a.batch * rows + kRowTile - 1) / kRowTile);
    p.shared_splits = cut(static_cast<int64_t>(a.kv_heads) * p.shared_tiles, shared, 512, 32);
  }
  p.splits = cut(units, most, 2048, own_pass ? 32 : kMaxParts);
  p.parts = p.splits + p.shared_splits;
  const int64_t all = static_cast<int64_t>(a.batch) * a.slots * a.q_heads;
  p.bytes = p.parts > 1 ? p.parts * all * (a.head_dim * int64_t{4} + 8) : 0;
  return p;
}

hipError_t launch_attend(graft_ctx *ctx, const graft_attention &d, const AttendPlan &p,
                         hipStream_t stream) {
  const bool q8 = d.cache_dtype == GRAFT_E4M3;
  AttendArgs a{};
  a.block_k = side(d.k, 2);
  a.block_v = side(d.v, 2);
  a.cache_k = side(d.cache_k, q8 ? 1 : 2);
  a.cache_v = side(d.cache_v, q8 ? 1 : 2);
  a.shared_k = side(d.shared_k, q8 ? 1 : 2);
  a.shared_v = side(d.shared_v, q8 ? 1 : 2);
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
  a.row_tiles = p.row_tiles;
  a.splits = p.splits;
  a.min_tiles = p.min_tiles;
  a.shared_tiles = p.shared_tiles;
  a.shared_splits = p.shared_splits;
  a.parts = p.parts;
  a.shared_items = p.shared_tiles * p.shared_splits * d.kv_heads;
  a.c = d.scale * 1.4426950408889634f;
  const int64_t groups = (static_cast<int64_t>(d.batch) * d.kv_heads * p.splits + 7) / 8 * 8;
  const dim3 grid(static_cast<unsigned>(a.shared_items + groups * p.row_tiles)), block(kAttThreads);
  const bool wide = d.head_dim > 64;
  if (d.dtype == GRAFT_F16) {
    if (wide) hipLaunchKernelGGL((attend_kernel<F16, false, 128>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((attend_kernel<F16, false, 64>), grid, block, 0, stream, a);
  } else if (q8) {
    if (wide) hipLaunchKernelGGL((attend_kernel<Bf16, true, 128>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((attend_kernel<Bf16, true, 64>), grid, block, 0, stream, a);
  } else {
    if (wide) hipLaunchKernelGGL((attend_kernel<Bf16, false, 128>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((attend_kernel<Bf16, false, 64>), grid, block, 0, stream, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts <= 1) return e;
  const dim3 mgrid(static_cast<unsigned>((a.rows_all + kAttWaves - 1) / kAttWaves));
  if (d.dtype == GRAFT_F16) hipLaunchKernelGGL(merge_parts_kernel<F16>, mgrid, block, 0, stream, a);
  else hipLaunchKernelGGL(merge_parts_kernel<Bf16>, mgrid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace graft
