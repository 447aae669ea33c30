// k_pages.hip -- a key/value cache in pages: a block's queries and keys rotated by their
// positions, keys and values appended (copied, or quantised as in k_cache.hip), and the
// accepted path's rows moved up after the acceptance.
//
// Pair (x, y) of a head becomes (x cos a - y sin a, y cos a + x sin a), a = position * freq.
// A thread owns two 16-byte pieces of a head, one of either half of what is rotated: eight pairs (f, f +
// rot / 2), or four pairs (2f, 2f + 1) in each piece.  A head of D numbers is D / 16 neighbouring lanes
// (rounded up to a power of two, for the exchange of the maximum that a quantised head needs), which read
// and write neighbouring pieces.
//
// Angles: a position is up to 2^31 and an angle of 10^5 radians has 2^-7 as its last bit in
// fp32, so the angle is formed in fp64, taken to revolutions with both parts of the product
// by 1 / 2 pi, and reduced to an eighth of a turn; sine and cosine of what is left are Taylor
// sums in fp32, to y^9 and y^10 (below 2e-9 at pi / 4).  They are made once a row in LDS and
// used by all of its heads.
//
// Both kernels are bound by memory: a number is read once and written once.  Measured (in a graph):
// prompts of up to 2048 rows of 32/8 heads of 128, rotated over three axes, 35 us for 164 MB (4.6 TB/s; a
// large copy 5.1); 64 trees of up to 64 nodes to e4m3 pages 23 us, and 11 for the read back, for 91 MB; one
// token 3.7 us; 64 paths of up to 16 rows in 72 planes 42 us for 199 MB (4.7 TB/s); one path 4.6 us.
#include "graft_internal.h"

#include "pages.h"

namespace graft {
namespace {

constexpr int kPageThreads = 256;
// Rows a thread loads before it stores any: 1, 2 and 4 take 40.6, 36.1 and 38.4 us for the prompts, 37.5, 34.6
// and 40.2 for the trees.
constexpr int kPageRows = 2;
constexpr int kMostThreads = 1024;
// Rows of the path in registers at a time: 4, 8 and 16 take 44.0, 42.8 and 42.3 us for the 64 paths.
constexpr int kPathGroup = 16;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct Place {             // of a tensor's rows: byte strides
  char *p;
  int64_t batch, row, head;
};

struct WriteArgs {
  Place q, q_out, k, v, cache_k, cache_v;   // batch strides of the caches are the pages'
  uint8_t *scale_k, *scale_v;
  int64_t sk_page, sk_row, sk_head, sv_page, sv_row, sv_head;
  PageMap pages;
  const int32_t *n_rows, *start, *positions, *axis;
  const double *freq;
  int32_t batch, slots, q_heads, kv_heads, dim, half, pair_step, axes;   // half: rot_dim / 2
  int32_t lanes, cols;                  // lanes of a head; of a row
  int32_t at_once, threads, col_blocks, row_blocks;
  uint32_t *error_flag;
};

// cos and sin of t radians.
__device__ __forceinline__ f32x2 turn_of(double t) {
  constexpr double kInv = 0.15915494309189533577, kInvLow = -9.8393383e-18;   // 1 / 2 pi
  const double hi = t * kInv;
  const double r = (hi - __builtin_rint(hi)) + __builtin_fma(t, kInvLow, __builtin_fma(t, kInv, -hi));
  const double k = __builtin_rint(4.0 * r);
  const float y = static_cast<float>((r - 0.25 * k) * 6.28318530717958647693);
  const float z = y * y;
  const float s = __builtin_fmaf(y * z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), y);
  const float c = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  const int quarter = static_cast<int>(k) & 3;
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return f32x2{quarter == 1 || quarter == 2 ? -a : a, quarter >= 2 ? -b : b};
}

template <bool HALF>
__device__ __forceinline__ float lower(uint32_t w) {
  return HALF ? static_cast<float>(__builtin_bit_cast(f16x2, w).x) : __uint_as_float(w << 16);
}
template <bool HALF>
__device__ __forceinline__ float upper(uint32_t w) {
  return HALF ? static_cast<float>(__builtin_bit_cast(f16x2, w).y) : __uint_as_float(w & 0xFFFF0000u);
}
template <bool HALF>
__device__ __forceinline__ uint32_t pack(float x, float y) {
  return HALF ? __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, f16x2))
              : __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
}

// Codes of 8 numbers over 2^e, as in k_cache.hip.
__device__ __forceinline__ uint64_t encode(const float *x, int e) {
  const float inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  const float top = e == 120 ? 240.0f : 448.0f;   // 256 * 2^120 is past fp32
  uint32_t out[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    uint32_t code = 0, nan = 0;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y = x[4 * q + i];
      nan |= y != y ? 0x7Fu << (8 * i) : 0u;
      v[i] = fminf(fmaxf(y * inv, -top), top);
    }
    code = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], code, false);
    code = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], code, true);
    out[q] = code | nan;
  }
  return static_cast<uint64_t>(out[1]) << 32 | out[0];
}

// What is read once does not stay in the caches (the prompts 40.2 -> 36.1 us, the paths 50.6 -> 42.3; the
// trees, whose blocks the caches still hold, 32.5 -> 34.6; non-temporal stores too cost the paths 3.9).
__device__ __forceinline__ u32x4 load_once(const char *p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
}

// HALF: fp16 numbers, else bf16.  Q8: e4m3 pages.  A workgroup has whole rows, so that their angles are made
// once (with neighbouring pieces and non-temporal reads the prompts 47 -> 36 us).
template <bool HALF, bool Q8>
__global__ void __launch_bounds__(kMostThreads)
write_kernel(WriteArgs a) {
  extern __shared__ f32x2 turns[];        // [rows of the workgroup][half]
  int blk = blockIdx.x;
  const int cb = blk % a.col_blocks;
  blk /= a.col_blocks;
  const int rb = blk % a.row_blocks, b = blk / a.row_blocks;
  int n = a.n_rows ? a.n_rows[b] : a.slots;
  const int first = a.start ? a.start[b] : 0;
  if ((n < 0 || n > a.slots) && cb == 0 && rb == 0 && threadIdx.x == 0) atomicOr(a.error_flag, kErrBlockSizes);
  n = n < 0 ? 0 : n > a.slots ? a.slots : n;
  const int span = a.at_once * kPageRows, row0 = rb * span;
  if (row0 >= n) return;

  const int sub = a.at_once > 1 ? threadIdx.x / a.cols : 0;
  const int col = a.at_once > 1 ? threadIdx.x - sub * a.cols : cb * blockDim.x + threadIdx.x;
  const int unit = col & (a.lanes - 1), hd = col / a.lanes;
  const bool mine = sub < a.at_once && col < a.cols && unit * 16 < a.dim;
  const bool is_q = hd < a.q_heads, is_k = !is_q && hd < a.q_heads + a.kv_heads;
  const int head = is_q ? hd : is_k ? hd - a.q_heads : hd - a.q_heads - a.kv_heads;
  const bool turned = (is_q || is_k) && unit * 8 < a.half;
  // A thread's eight numbers each at c0.. and c1..: a piece of either half of what is rotated, or of
  // either half of the rest, so that a head's lanes read neighbouring 16 bytes.
  const int part = is_q || is_k ? 2 * a.half : 0, mid = turned ? a.half : (a.dim - part) / 2;
  const int c0 = turned ? unit * 8 : part + (unit - part / 16) * 8, c1 = c0 + mid;
  const char *src = is_q ? a.q.p + b * a.q.batch + head * a.q.head
                         : is_k ? a.k.p + b * a.k.batch + head * a.k.head : a.v.p + b * a.v.batch + head * a.v.head;
  const int64_t src_row = is_q ? a.q.row : is_k ? a.k.row : a.v.row;

  u32x4 lo[kPageRows], hi[kPageRows];
  int page[kPageRows], off[kPageRows];
  bool ok[kPageRows];
#pragma unroll
  for (int x = 0; x < kPageRows; ++x) {
    const int i = row0 + sub + x * a.at_once;
    ok[x] = mine && i < n;
    lo[x] = hi[x] = u32x4{0, 0, 0, 0};
    if (ok[x]) {
      lo[x] = load_once(src + i * src_row + c0 * 2);
      hi[x] = load_once(src + i * src_row + c1 * 2);
    }
  }
#pragma unroll
  for (int x = 0; x < kPageRows; ++x) {
    page[x] = off[x] = 0;
    if (ok[x] && !is_q) {
      const int64_t r = static_cast<int64_t>(first) + row0 + sub + x * a.at_once;
      bool good = r >= 0 && r < a.pages.rows();
      const int entry = a.pages.entry(good ? static_cast<uint32_t>(r) : 0u);
      off[x] = good ? static_cast<int>(r) - entry * a.pages.page_rows : 0;
      page[x] = good ? a.pages.table[b * a.pages.table_stride + entry] : -1;
      good = page[x] >= 0 && page[x] < a.pages.pages;
      if (!good) atomicOr(a.error_flag, kErrPage);
      ok[x] = good;
    }
  }

  if (a.half > 0) {
    const int rows = n - row0 < span ? n - row0 : span;
    for (int u = threadIdx.x; u < rows * a.half; u += blockDim.x) {
      const int r = u / a.half, f = u - r * a.half;
      int64_t pos = static_cast<int64_t>(first) + row0 + r;
      if (a.positions) {
        int ax = a.axis ? a.axis[f] : 0;
        if (ax < 0 || ax >= a.axes) {
          atomicOr(a.error_flag, kErrPage);
          ax = 0;
        }
        pos = a.positions[(static_cast<int64_t>(ax) * a.batch + b) * a.slots + row0 + r];
      }
      turns[u] = turn_of(static_cast<double>(pos) * a.freq[f]);
    }
    __syncthreads();
  }

#pragma unroll
  for (int x = 0; x < kPageRows; ++x) {
    const int r = sub + x * a.at_once, i = row0 + r;
    float u[8], w[8];                     // what goes to c0.. and c1..
    if (turned || (Q8 && !is_q)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u[2 * j] = lower<HALF>(lo[x][j]);
        u[2 * j + 1] = upper<HALF>(lo[x][j]);
        w[2 * j] = lower<HALF>(hi[x][j]);
        w[2 * j + 1] = upper<HALF>(hi[x][j]);
      }
    }
    if (turned && ok[x]) {
      if (a.pair_step == 1) {
        const f32x2 *t = turns + r * a.half + c0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const f32x2 cs = t[j];
          const float p = u[j], s = w[j];
          u[j] = p * cs.x - s * cs.y;
          w[j] = s * cs.x + p * cs.y;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const f32x2 cs = turns[r * a.half + (j < 4 ? c0 : c1) / 2 + j % 4];
          float *z = j < 4 ? u + 2 * j : w + 2 * (j - 4);
          const float p = z[0], s = z[1];
          z[0] = p * cs.x - s * cs.y;
          z[1] = s * cs.x + p * cs.y;
        }
      }
    }
    if (Q8 && !is_q) {
      uint32_t m = 0;                     // the largest finite magnitude's bits
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t p = __float_as_uint(u[j]) & 0x7FFFFFFFu, s = __float_as_uint(w[j]) & 0x7FFFFFFFu;
        m = p > m && p < 0x7F800000u ? p : m;
        m = s > m && s < 0x7F800000u ? s : m;
      }
      // the head's lanes hold the same row; lanes without numbers hold zeros
      for (int y = 1; y < a.lanes; y <<= 1) {
        const uint32_t o = xor_lane(m, y);
        m = o > m ? o : m;
      }
      int e = static_cast<int>(m >> 23) - 135 + ((m & 0x7FFFFFu) > 0x600000u ? 1 : 0);
      e = e < -118 ? -118 : e;
      if (ok[x]) {
        char *d = is_k ? a.cache_k.p + page[x] * a.cache_k.batch + off[x] * a.cache_k.row + head * a.cache_k.head
                       : a.cache_v.p + page[x] * a.cache_v.batch + off[x] * a.cache_v.row + head * a.cache_v.head;
        *reinterpret_cast<uint64_t *>(d + c0) = encode(u, e);
        *reinterpret_cast<uint64_t *>(d + c1) = encode(w, e);
        if (unit == 0) {
          uint8_t *s = is_k ? a.scale_k + page[x] * a.sk_page + off[x] * a.sk_row + head * a.sk_head
                            : a.scale_v + page[x] * a.sv_page + off[x] * a.sv_row + head * a.sv_head;
          *s = static_cast<uint8_t>(e + 127);
        }
      }
    } else if (ok[x]) {
      if (turned) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          lo[x][j] = pack<HALF>(u[2 * j], u[2 * j + 1]);
          hi[x][j] = pack<HALF>(w[2 * j], w[2 * j + 1]);
        }
      }
      char *d = is_q ? a.q_out.p + b * a.q_out.batch + i * a.q_out.row + head * a.q_out.head
                : is_k ? a.cache_k.p + page[x] * a.cache_k.batch + off[x] * a.cache_k.row + head * a.cache_k.head
                       : a.cache_v.p + page[x] * a.cache_v.batch + off[x] * a.cache_v.row + head * a.cache_v.head;
      *reinterpret_cast<u32x4 *>(d + c0 * 2) = lo[x];
      *reinterpret_cast<u32x4 *>(d + c1 * 2) = hi[x];
    }
  }
}

struct PathArgs {
  char *p;
  uint8_t *scale;
  int64_t plane, page, row, head;               // bytes
  int64_t s_plane, s_page, s_row, s_head;
  PageMap pages;
  const int32_t *start, *acc_len, *acc_nodes;
  int32_t heads, chunks, root, most, n_max, blocks_per_seq;
  int64_t total;                                // n_planes * heads * chunks
  uint32_t *error_flag;
};

__device__ __forceinline__ int64_t uniform64(int64_t v, int lane) {
  const uint64_t u = static_cast<uint64_t>(v);
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(u), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(u >> 32), lane);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// A thread owns 16 bytes of a (plane, head) and takes them through the whole path, up to 16 rows
// loaded before any is stored: rows lie 256 bytes and more apart, and loads in flight are what there is to
// gain.  Row i of the block receives row nodes[i] >= i: what a group
// stores to is behind no row that a later group reads, since nodes[j] >= j.
__global__ void __launch_bounds__(kPageThreads)
path_kernel(PathArgs a) {
  const int b = blockIdx.x / a.blocks_per_seq, blk = blockIdx.x - b * a.blocks_per_seq;
  const int lane = lane_id();
  int n = a.acc_len[b];
  n = n < 0 ? 0 : n > a.most ? a.most : n;
  if (n == 0) return;
  // a row of the path a lane (at most 64): where it is and where it goes
  const int node = lane < n ? a.acc_nodes[static_cast<int64_t>(b) * a.most + lane] : lane;
  const int64_t base = (a.start ? a.start[b] : 0) + static_cast<int64_t>(a.root);
  const int64_t from = base + node, to = base + lane;
  bool good = node >= 0 && node < a.n_max && to >= 0 && from >= 0 && from < a.pages.rows() && to < a.pages.rows();
  const int32_t *table = a.pages.table + b * a.pages.table_stride;
  const uint32_t rs = good && lane < n ? static_cast<uint32_t>(from) : 0u, rd = good && lane < n ? static_cast<uint32_t>(to) : 0u;
  const int es = a.pages.entry(rs), ed = a.pages.entry(rd);
  const int ps = table[es], pd = table[ed];
  good = good && ps >= 0 && ps < a.pages.pages && pd >= 0 && pd < a.pages.pages;
  if (blk == 0 && threadIdx.x < kWave && lane < n && !good) atomicOr(a.error_flag, kErrPage);
  const int64_t os = static_cast<int64_t>(rs) - static_cast<int64_t>(es) * a.pages.page_rows;
  const int64_t od = static_cast<int64_t>(rd) - static_cast<int64_t>(ed) * a.pages.page_rows;
  const int64_t at_s = ps * a.page + os * a.row, at_d = pd * a.page + od * a.row;
  const int64_t sc_s = ps * a.s_page + os * a.s_row, sc_d = pd * a.s_page + od * a.s_row;
  const uint64_t moves = __ballot(lane < n && good && node != lane);
  if (moves == 0) return;

  const int64_t t = static_cast<int64_t>(blk) * kPageThreads + threadIdx.x;
  const bool active = t < a.total;
  const int64_t tc = active ? t : 0;
  const int64_t ph = tc / a.chunks;
  const int chunk = static_cast<int>(tc - ph * a.chunks);
  const int64_t plane = ph / a.heads, head = ph - plane * a.heads;
  char *p = a.p + plane * a.plane + head * a.head + chunk * 16;
  uint8_t *s = a.scale + plane * a.s_plane + head * a.s_head;
  const bool scales = a.scale != nullptr && chunk == 0 && active;
  for (int g = 0; g < n; g += kPathGroup) {
    u32x4 v[kPathGroup];
    uint8_t w[kPathGroup];
#pragma unroll
    for (int k = 0; k < kPathGroup; ++k) {
      if (((moves >> g) >> k) & 1) {
        if (active) v[k] = load_once(p + uniform64(at_s, g + k));
        if (scales) w[k] = s[uniform64(sc_s, g + k)];
      }
    }
#pragma unroll
    for (int k = 0; k < kPathGroup; ++k) {
      if (((moves >> g) >> k) & 1) {
        if (active) *reinterpret_cast<u32x4 *>(p + uniform64(at_d, g + k)) = v[k];
        if (scales) s[uniform64(sc_d, g + k)] = w[k];
      }
    }
  }
}

Place place(const graft_rows &r, int bytes) {
  return Place{static_cast<char *>(r.data), r.batch_stride * bytes, r.row_stride * bytes, r.head_stride * bytes};
}

WriteArgs plan_write(const graft_paged_rows &r, int64_t *blocks) {
  const bool q8 = r.cache_dtype == GRAFT_E4M3;
  const int w = q8 ? 1 : 2;
  WriteArgs a{};
  a.q = place(r.q, 2);
  a.q_out = place(r.q_out, 2);
  a.k = place(r.k, 2);
  a.v = place(r.v, 2);
  a.cache_k = place(r.cache_k, w);
  a.cache_v = place(r.cache_v, w);
  a.scale_k = r.cache_k.scale;
  a.scale_v = r.cache_v.scale;
  a.sk_page = r.cache_k.scale_batch_stride;
  a.sk_row = r.cache_k.scale_row_stride;
  a.sk_head = r.cache_k.scale_head_stride;
  a.sv_page = r.cache_v.scale_batch_stride;
  a.sv_row = r.cache_v.scale_row_stride;
  a.sv_head = r.cache_v.scale_head_stride;
  a.pages = page_map(r.pages);
  a.n_rows = r.n_rows;
  a.start = r.start;
  a.positions = r.positions;
  a.axis = r.axis;
  a.freq = r.freq;
  a.batch = r.batch;
  a.slots = r.slots;
  a.q_heads = r.q_heads;
  a.kv_heads = r.kv_heads;
  a.dim = r.head_dim;
  a.half = r.rot_dim / 2;
  a.pair_step = r.interleaved ? 2 : 1;
  a.axes = r.axes;
  a.lanes = 1;
  while (a.lanes < r.head_dim / 16) a.lanes *= 2;
  a.cols = (r.q_heads + 2 * r.kv_heads) * a.lanes;
  // a row's columns in one workgroup, whose angles they share, where they fit: whole waves, or several
  // rows of up to 256 columns
  a.at_once = a.cols <= kPageThreads ? kPageThreads / a.cols : 1;
  a.threads = a.cols <= kPageThreads ? kPageThreads : a.cols <= kMostThreads ? (a.cols + kWave - 1) / kWave * kWave : 512;
  a.col_blocks = (a.cols + a.threads - 1) / a.threads;
  const int span = a.at_once * kPageRows;
  a.row_blocks = (r.slots + span - 1) / span;
  *blocks = static_cast<int64_t>(a.col_blocks) * a.row_blocks * r.batch;
  return a;
}

PathArgs plan_path(const graft_paged_path &d, int64_t *blocks) {
  const int bytes = d.dtype == GRAFT_E4M3 ? 1 : 2;
  PathArgs a{};
  a.p = static_cast<char *>(d.rows.data);
  a.scale = d.dtype == GRAFT_E4M3 ? d.rows.scale : nullptr;
  a.plane = d.rows.plane_stride * bytes;
  a.page = d.rows.batch_stride * bytes;
  a.row = d.rows.row_stride * bytes;
  a.head = d.rows.head_stride * bytes;
  a.s_plane = d.rows.scale_plane_stride;
  a.s_page = d.rows.scale_batch_stride;
  a.s_row = d.rows.scale_row_stride;
  a.s_head = d.rows.scale_head_stride;
  a.pages = page_map(d.pages);
  a.start = d.start;
  a.acc_len = d.acc_len;
  a.acc_nodes = d.acc_nodes;
  a.heads = d.heads;
  a.chunks = d.head_dim * bytes / 16;
  a.root = d.with_root ? 1 : 0;
  a.total = static_cast<int64_t>(d.n_planes) * d.heads * a.chunks;
  const int64_t per_seq = (a.total + kPageThreads - 1) / kPageThreads;
  a.blocks_per_seq = static_cast<int32_t>(per_seq < kMaxBlocks ? per_seq : kMaxBlocks);
  *blocks = per_seq * d.batch;
  return a;
}

}  // namespace

PageMap page_map(const graft_page_table &t) {
  PageMap m{};
  m.table = t.table;
  m.table_stride = t.table_stride;
  m.table_len = t.table_len;
  m.pages = t.pages;
  m.page_rows = t.page_rows;
  set_division(m);
  return m;
}

int64_t paged_write_blocks(const graft_paged_rows &r) {
  int64_t blocks;
  const WriteArgs a = plan_write(r, &blocks);
  return blocks * ((a.threads + 255) / 256);   // a launch counts its threads
}

hipError_t launch_paged_write(graft_ctx *ctx, const graft_paged_rows &r, hipStream_t stream) {
  int64_t blocks;
  WriteArgs a = plan_write(r, &blocks);
  a.error_flag = ctx->error_flag;
  const dim3 grid(static_cast<unsigned>(blocks)), block(static_cast<unsigned>(a.threads));
  const size_t lds = static_cast<size_t>(a.at_once) * kPageRows * a.half * sizeof(f32x2);   // 32 KB at most
  if (r.cache_dtype == GRAFT_E4M3) hipLaunchKernelGGL((write_kernel<false, true>), grid, block, lds, stream, a);
  else if (r.dtype == GRAFT_F16) hipLaunchKernelGGL((write_kernel<true, false>), grid, block, lds, stream, a);
  else hipLaunchKernelGGL((write_kernel<false, false>), grid, block, lds, stream, a);
  return hipGetLastError();
}

int64_t paged_commit_blocks(const graft_paged_path &p) {
  int64_t blocks;
  plan_path(p, &blocks);
  return blocks;
}

hipError_t launch_paged_commit(graft_ctx *ctx, const graft_paged_path &p, hipStream_t stream) {
  int64_t blocks;
  PathArgs a = plan_path(p, &blocks);
  a.most = ctx->dims.num_pos;
  a.n_max = ctx->dims.max_nodes;
  a.error_flag = ctx->error_flag;
  hipLaunchKernelGGL(path_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kPageThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace graft
