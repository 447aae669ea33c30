// k_cache.hip -- the verifier's key/value cache: rows appended at every
// sequence's own length (an accepted path with its root, or a prompt), copied or
// quantised on the way, and quantised rows read back.
//
// A (row, head) of D numbers is stored as e4m3 codes and one scale 2^e, e the
// smallest integer >= -118 with max |x| <= 448 * 2^e.  A power of two costs a
// floating-point code no precision (only the spread of its exponents counts), makes
// x / 2^e exact, so that a code is the one rounding of x that there is, and takes
// one byte.  From max |x| = 1.f * 2^(E - 127) in bf16, e = E - 135, one more where
// 1.f > 1.75 (448 = 1.75 * 2^8).  Below 2^-118 bf16 could not hold the smallest code.
//
// Both kernels are bound by memory.  A thread owns 16 bytes of the wider side, so that a
// wave's accesses there are 1 KB without gaps (32 bytes in two stores of 16 each took 340 us
// where this takes 157); a head's threads are a power of two of neighbouring lanes, so the
// maximum is a lane exchange.  A thread has four rows in flight and no more, so that
// workgroups spread: reading 64 sequences' 512 to 4096 rows of two planes of 8 x 128 back to
// bf16 takes 156, 171, 177 and 179 us with 4, 8, 16 and 32 (919 MB: 5.9 TB/s, past the
// 5.1 of a large copy), to fp32 257 for 1531 MB.  Appending 64 sequences' paths of up to 17 rows to
// 72 planes of 8 x 128 takes 27.7 us quantised and 24.6 as a plain copy, where reading the same
// rows back takes 13.2: a path's rows lie apart in the block, and a row's load waits for its list
// entry's.  4 prompts of up to 2048 rows to 2 planes: 14.7 us quantised (36 MB), 13.9 copied (48 MB).
#include "graft_internal.h"

namespace graft {
namespace {

constexpr int kMoveThreads = 256;
constexpr int kMoveRows = 4;     // rows a thread loads before it stores any
constexpr uint32_t kBf16Inf = 0x7F80u;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

enum class Move { kCopy, kQuantise, kRead16, kRead32 };

struct MoveArgs {
  graft_rows src, dst;
  const int32_t *n_rows, *start, *list;
  int32_t list_len, root;
  int32_t src_rows, dst_rows, most;    // most: rows of a sequence at most
  int32_t heads, chunks, lanes;        // threads that a head needs, and has
  int32_t cols;                        // n_planes * heads * lanes
  int32_t at_once;                     // rows side by side in a workgroup
  int32_t col_blocks, row_blocks;
  uint32_t *error_flag;
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Largest finite magnitude of the 8 numbers, as bf16 bits.
__device__ __forceinline__ uint32_t largest(const u32x4 &a) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = a[i] & 0x7FFFu, hi = (a[i] >> 16) & 0x7FFFu;
    m = lo > m && lo < kBf16Inf ? lo : m;
    m = hi > m && hi < kBf16Inf ? hi : m;
  }
  return m;
}

// Codes of the 8 numbers over 2^e.
__device__ __forceinline__ u32x2 encode(const u32x4 &a, int e) {
  const float inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  // 256 * 2^120 is past fp32
  const float top = e == 120 ? 240.0f : 448.0f;
  u32x2 out;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    uint32_t code = 0, nan = 0;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = a[2 * q + i / 2];
      const float x = i & 1 ? bf16_hi(w) : bf16_lo(w);
      nan |= x != x ? 0x7Fu << (8 * i) : 0u;
      v[i] = fminf(fmaxf(x * inv, -top), top);   // only infinities and e = 120 are cut
    }
    code = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], code, false);
    code = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], code, true);
    out[q] = code | nan;
  }
  return out;
}

// Numbers of a thread: 16 bytes of the wider side.
constexpr int numbers(Move m) { return m == Move::kRead32 ? 4 : 8; }

template <Move MODE>
__global__ void __launch_bounds__(kMoveThreads)
move_kernel(MoveArgs a) {
  constexpr int kNum = numbers(MODE);
  constexpr bool kWrite = MODE == Move::kCopy || MODE == Move::kQuantise;
  int blk = blockIdx.x;
  const int cb = blk % a.col_blocks;
  blk /= a.col_blocks;
  const int rb = blk % a.row_blocks, b = blk / a.row_blocks;
  int n = a.n_rows[b];
  const int first = a.start ? a.start[b] : 0;
  const int cap = kWrite && a.list ? a.list_len : a.most;
  n = (n < 0 ? 0 : (n > cap ? cap : n)) + a.root;
  const int row0 = rb * (a.at_once * kMoveRows);
  if (row0 >= n) return;

  const int sub = a.at_once > 1 ? threadIdx.x / a.cols : 0;
  const int col = a.at_once > 1 ? threadIdx.x - sub * a.cols : cb * kMoveThreads + threadIdx.x;
  const int chunk = col & (a.lanes - 1), ph = col / a.lanes;
  const int plane = ph / a.heads, head = ph - plane * a.heads;
  const bool mine = sub < a.at_once && col < a.cols && chunk < a.chunks;
  const int64_t p = mine ? plane : 0, h = mine ? head : 0, c = mine ? chunk * kNum : 0;
  const int64_t s_at = p * a.src.plane_stride + b * a.src.batch_stride + h * a.src.head_stride + c;
  const int64_t d_at = p * a.dst.plane_stride + b * a.dst.batch_stride + h * a.dst.head_stride + c;
  const graft_rows &q = kWrite ? a.dst : a.src;    // the cache
  uint8_t *scale = MODE == Move::kCopy
                       ? nullptr
                       : q.scale + p * q.scale_plane_stride + b * q.scale_batch_stride +
                             h * q.scale_head_stride;
  const char *src = static_cast<const char *>(a.src.data);
  char *dst = static_cast<char *>(a.dst.data);

  const int base = row0 + sub;
  u32x4 v[kMoveRows];
  int64_t to[kMoveRows];
  uint32_t sc[kMoveRows];
  bool ok[kMoveRows];
#pragma unroll
  for (int k = 0; k < kMoveRows; ++k) {
    const int i = base + k * a.at_once;
    ok[k] = mine && i < n;
    int64_t from = 0;
    to[k] = 0;
    if (ok[k]) {
      if (kWrite) {
        from = i;
        if (a.list)
          from = i < a.root ? 0 : a.list[static_cast<int64_t>(b) * a.list_len + i - a.root] +
                                      static_cast<int64_t>(a.root);
        // a node's entry is at least 0: with a root, row 0 is the root's alone
        const bool good = from >= (a.list && i >= a.root ? a.root : 0) && from < a.src_rows;
        to[k] = static_cast<int64_t>(first) + i;
        ok[k] = good && to[k] >= 0 && to[k] < a.dst_rows;
      } else {
        to[k] = i;
        from = static_cast<int64_t>(first) + i;
        ok[k] = from >= 0 && from < a.src_rows;
      }
      if (!ok[k]) atomicOr(a.error_flag, kErrCacheRow);
    }
    v[k] = u32x4{0, 0, 0, 0};
    sc[k] = 0;
    if (ok[k]) {
      if (kWrite) {
        v[k] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4 *>(src + 2 * (s_at + from * a.src.row_stride)));
      } else {
        const char *at = src + s_at + from * a.src.row_stride;
        if constexpr (kNum == 8) {
          const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(at));
          v[k].x = w.x;
          v[k].y = w.y;
        } else {
          v[k].x = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(at));
        }
        sc[k] = scale[from * a.src.scale_row_stride];
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kMoveRows; ++k) {
    if (MODE == Move::kCopy) {
      if (ok[k]) *reinterpret_cast<u32x4 *>(dst + 2 * (d_at + to[k] * a.dst.row_stride)) = v[k];
    } else if (MODE == Move::kQuantise) {
      uint32_t m = largest(v[k]);
      // the head's lanes hold the same row; the others' zeros change nothing
      for (int x = 1; x < a.lanes; x <<= 1) {
        const uint32_t o = xor_lane(m, x);
        m = o > m ? o : m;
      }
      int e = static_cast<int>(m >> 7) - 135 + ((m & 0x7Fu) > 0x60u ? 1 : 0);
      e = e < -118 ? -118 : e;
      if (ok[k]) {
        *reinterpret_cast<u32x2 *>(dst + d_at + to[k] * a.dst.row_stride) = encode(v[k], e);
        if (chunk == 0) scale[to[k] * a.dst.scale_row_stride] = static_cast<uint8_t>(e + 127);
      }
    } else if (ok[k]) {
      const float unit = __uint_as_float(sc[k] ? sc[k] << 23 : 0x00400000u);
      float x[kNum];
#pragma unroll
      for (int i = 0; i < kNum / 4; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(v[k][i]), false);
        const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(v[k][i]), true);
        x[4 * i] = lo.x * unit;
        x[4 * i + 1] = lo.y * unit;
        x[4 * i + 2] = hi.x * unit;
        x[4 * i + 3] = hi.y * unit;
      }
      u32x4 w;
      if constexpr (kNum == 8) {
        // at most 4 significant bits: the upper half of the fp32 number is the bf16 number
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xFFFF0000u);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
      }
      __builtin_nontemporal_store(
          w, reinterpret_cast<u32x4 *>(dst + (kNum == 8 ? 2 : 4) * (d_at + to[k] * a.dst.row_stride)));
    }
  }
}

Move mode_of(const graft_cache_move &m, bool write) {
  if (write) return m.dst_dtype == GRAFT_E4M3 ? Move::kQuantise : Move::kCopy;
  return m.dst_dtype == GRAFT_F32 ? Move::kRead32 : Move::kRead16;
}
// All of a call's arguments but the context's; blocks: the workgroups of its launch.
MoveArgs plan_move(const graft_cache_move &m, bool write, int64_t *blocks) {
  const Move mode = mode_of(m, write);
  const int most = !write ? m.dst_rows : m.list ? m.list_len + (m.with_root ? 1 : 0) : m.src_rows;
  MoveArgs a{};
  a.src = m.src;
  a.dst = m.dst;
  a.n_rows = m.n_rows;
  a.start = m.start;
  a.list = write ? m.list : nullptr;
  a.list_len = m.list_len;
  a.root = a.list && m.with_root ? 1 : 0;
  a.src_rows = m.src_rows;
  a.dst_rows = m.dst_rows;
  a.most = most;
  a.heads = m.heads;
  a.chunks = m.head_dim / numbers(mode);
  a.lanes = 1;
  while (a.lanes < a.chunks) a.lanes *= 2;
  a.cols = m.n_planes * m.heads * a.lanes;
  a.at_once = a.cols < kMoveThreads ? kMoveThreads / a.cols : 1;
  a.col_blocks = (a.cols + kMoveThreads - 1) / kMoveThreads;
  const int per = a.at_once * kMoveRows;
  a.row_blocks = (most + per - 1) / per;
  *blocks = static_cast<int64_t>(a.col_blocks) * a.row_blocks * m.batch;
  return a;
}

hipError_t launch_move(graft_ctx *ctx, const graft_cache_move &m, bool write, hipStream_t stream) {
  int64_t blocks;
  MoveArgs a = plan_move(m, write, &blocks);
  a.error_flag = ctx->error_flag;
  const dim3 grid(static_cast<unsigned>(blocks)), block(kMoveThreads);
  switch (mode_of(m, write)) {
    case Move::kCopy: hipLaunchKernelGGL(move_kernel<Move::kCopy>, grid, block, 0, stream, a); break;
    case Move::kQuantise: hipLaunchKernelGGL(move_kernel<Move::kQuantise>, grid, block, 0, stream, a); break;
    case Move::kRead16: hipLaunchKernelGGL(move_kernel<Move::kRead16>, grid, block, 0, stream, a); break;
    case Move::kRead32: hipLaunchKernelGGL(move_kernel<Move::kRead32>, grid, block, 0, stream, a); break;
  }
  return hipGetLastError();
}

}  // namespace

int64_t cache_move_blocks(const graft_cache_move &m, bool write) {
  int64_t blocks;
  plan_move(m, write, &blocks);
  return blocks;
}

hipError_t launch_cache_write(graft_ctx *ctx, const graft_cache_move &m, hipStream_t stream) {
  return launch_move(ctx, m, true, stream);
}

hipError_t launch_cache_read(graft_ctx *ctx, const graft_cache_move &m, hipStream_t stream) {
  return launch_move(ctx, m, false, stream);
}

}  // namespace graft
