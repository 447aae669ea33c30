// k_paged_attend.hip -- attention of a block over a cache in pages, with a window and sinks.
//
//   o_i = sum_j p_ij v_j / l_i,  p_ij = exp(s_ij - m_i),  s_ij = scale q_i . k_j,
// a wave a query row, one key after the other.
#include "graft_internal.h"

#include "pages.h"

namespace graft {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct PagedArgs {
  graft_paged_attention_desc d;
  PageMap pages;
  int32_t n_max, words;
  uint32_t *error_flag;
};

__device__ __forceinline__ f32x2 pair_at(const graft_rows &r, int dtype, int64_t at, float unit) {
  if (dtype == GRAFT_E4M3) {
    const uint16_t w = *reinterpret_cast<const uint16_t *>(static_cast<const char *>(r.data) + at);
    const f32x2 v = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    return f32x2{v.x * unit, v.y * unit};
  }
  const uint32_t w = *reinterpret_cast<const uint32_t *>(static_cast<const char *>(r.data) + 2 * at);
  if (dtype == GRAFT_F16) {
    const f16x2 h = __builtin_bit_cast(f16x2, w);
    return f32x2{static_cast<float>(h.x), static_cast<float>(h.y)};
  }
  return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)};
}

__global__ void __launch_bounds__(256)
paged_attend_kernel(PagedArgs a) {
  const graft_paged_attention_desc &d = a.d;
  const int lane = lane_id();
  const int64_t r = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave;
  if (r >= static_cast<int64_t>(d.batch) * d.slots * d.q_heads) return;
  const int64_t bs = r / d.q_heads;
  const int head = static_cast<int>(r - bs * d.q_heads), kvh = head / (d.q_heads / d.kv_heads);
  const int b = static_cast<int>(bs / d.slots), slot = static_cast<int>(bs - static_cast<int64_t>(b) * d.slots);
  const int root = d.with_root ? 1 : 0, most = d.slots - root;
  int n = d.n_nodes ? d.n_nodes[b] : most, len = d.cache_len[b];
  bool bad = n < 0 || n > most;
  n = (n < 0 ? 0 : n > most ? most : n) + root;
  const int cap = a.pages.rows() - n;
  bad |= len < 0 || len > cap;
  len = len < 0 ? 0 : len > cap ? cap : len;
  if (bad && lane == 0) atomicOr(a.error_flag, kErrBlockSizes);
  if (slot >= n) return;
  auto sees = [&](int s) {                      // slot s < n of the block
    if (!d.mask) return s <= slot;
    const int node = slot - root, other = s - root;
    if (other < 0) return true;
    if (node < 0) return false;
    return ((d.mask[(static_cast<int64_t>(b) * a.n_max + node) * a.words + (other >> 6)] >> (other & 63)) & 1) != 0;
  };
  int place = slot;
  if (d.mask) {
    place = -1;
    for (int s = 0; s < n; ++s) place += sees(s) ? 1 : 0;
  }
  const int low = window_low(len + place, d.window), end = d.mask ? len + n : len + slot + 1;
  const int64_t q_at = b * d.q.batch_stride + slot * d.q.row_stride + head * d.q.head_stride + 2 * lane;
  const bool mine = 2 * lane < d.head_dim;
  const f32x2 q = mine ? pair_at(d.q, d.dtype, q_at, 1.0f) : f32x2{0.0f, 0.0f};
  float m = -INFINITY, l = 0.0f;
  f32x2 o{0.0f, 0.0f};
  for (int j = 0; j < end; ++j) {
    if (j < low && j >= d.sinks && (j < len || !d.mask)) continue;
    if (j >= len && !sees(j - len)) continue;
    const int entry = a.pages.entry(j), off = j - entry * a.pages.page_rows;
    const int64_t page = a.pages.table[b * a.pages.table_stride + entry];
    if (page < 0 || page >= a.pages.pages) {
      if (lane == 0) atomicOr(a.error_flag, kErrPage);
      continue;
    }
    auto unit = [&](const graft_rows &x) {
      if (d.cache_dtype != GRAFT_E4M3) return 1.0f;
      const uint32_t s = x.scale[page * x.scale_batch_stride + off * x.scale_row_stride + kvh * x.scale_head_stride];
      return __uint_as_float(s << 23);
    };
    auto at = [&](const graft_rows &x) { return page * x.batch_stride + off * x.row_stride + kvh * x.head_stride + 2 * lane; };
    const f32x2 k = mine ? pair_at(d.cache_k, d.cache_dtype, at(d.cache_k), unit(d.cache_k)) : f32x2{0.0f, 0.0f};
    const f32x2 v = mine ? pair_at(d.cache_v, d.cache_dtype, at(d.cache_v), unit(d.cache_v)) : f32x2{0.0f, 0.0f};
    float s = q.x * k.x + q.y * k.y;
    for (int x = 1; x < kWave; x <<= 1) s += __uint_as_float(xor_lane(__float_as_uint(s), x));
    s *= d.scale;
    const float top = fmaxf(m, s);
    const float f = m == -INFINITY ? 0.0f : __expf(m - top), p = top == -INFINITY ? 0.0f : __expf(s - top);
    l = l * f + p;
    o.x = o.x * f + p * v.x;
    o.y = o.y * f + p * v.y;
    m = top;
  }
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  if (mine) {
    const f32x2 y{o.x * inv, o.y * inv};
    char *out = static_cast<char *>(d.out.data) + 2 * (b * d.out.batch_stride + slot * d.out.row_stride + head * d.out.head_stride + 2 * lane);
    *reinterpret_cast<uint32_t *>(out) = d.dtype == GRAFT_F16
        ? __builtin_bit_cast(uint32_t, __builtin_convertvector(y, f16x2))
        : __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
  }
  if (d.lse && lane == 0) d.lse[r] = l == 0.0f ? -INFINITY : m + __logf(l);
}

}  // namespace

PagedPlan paged_plan(const graft_paged_attention_desc &a) {
  PagedPlan p{};
  p.blocks = (static_cast<int64_t>(a.batch) * a.slots * a.q_heads + 3) / 4;
  return p;
}

hipError_t launch_paged_attend(graft_ctx *ctx, const graft_paged_attention_desc &d, const PagedPlan &p,
                               hipStream_t stream) {
  PagedArgs a{};
  a.d = d;
  a.pages = page_map(d.pages);
  a.n_max = ctx->dims.max_nodes;
  a.words = (ctx->dims.max_nodes + 63) / 64;
  a.error_flag = ctx->error_flag;
  hipLaunchKernelGGL(paged_attend_kernel, dim3(static_cast<unsigned>(p.blocks)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace graft
