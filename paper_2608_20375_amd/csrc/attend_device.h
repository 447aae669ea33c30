// attend_device.h -- what the attention kernels share: the element types' products, the softmax
// with a running reference, LDS places and fragments.
//
// Products.  v_mfma_f32_32x32x16: lane l gives row (or column) l % 32 and 8 of the 16
// contracted entries from 8 (l / 32) on; of the 32 x 32 result it holds column l % 32,
// rows 8 (i / 4) + 4 (l / 32) + i % 4, i < 16.  v_mfma_f32_16x16x32: row l % 16, 8 of 32
// entries from 8 (l / 16) on; column l % 16, rows 4 (l / 16) + i.
#pragma once

#include "graft_internal.h"

namespace graft {
namespace {

constexpr float kFar = 268435456.0f;              // exp2's argument whose last bit is 16
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// kSlack: log2 by which a maximum may be passed.  kLift: log2 of a factor on all
// probabilities and their sums, taken off the lse again.
struct Bf16 {
  static constexpr uint32_t kExp = 0x7F80u;      // exponent of infinities and NaN
  static constexpr float kSlack = 8.0f, kLift = 0.0f;
  static __device__ __forceinline__ f32x16 mfma(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
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
  // 2^15 at most, of 65504.  16 trees of up to 256 nodes: 210 us, unlifted with kSlack 8 205
  // (in turn, short runs).
  static constexpr float kSlack = 3.0f, kLift = 12.0f;
  static __device__ __forceinline__ f32x16 mfma(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, f16x2));
  }
  static __device__ __forceinline__ float number(uint16_t h) {
    return static_cast<float>(__builtin_bit_cast(_Float16, h));
  }
};

__device__ __forceinline__ float half_max(float v) {   // with the other half's lane
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(
      __float_as_uint(v), __float_as_uint(v), false, false));
  return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float half_sum(float v) {
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(
      __float_as_uint(v), __float_as_uint(v), false, false));
  return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// Over the wave's four quarters (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float quarter_max(float v) {
  v = half_max(v);
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(
      __float_as_uint(v), __float_as_uint(v), false, false));
  return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float quarter_sum(float v) {
  v = half_sum(v);
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(
      __float_as_uint(v), __float_as_uint(v), false, false));
  return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// Buffers with the hardware's bounds check: a load past `bytes` gives zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void *p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00020000);
}
__device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t r, int at) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
}

// 4 codes and their scale's byte -> two pairs of bf16, exact.
__device__ __forceinline__ u32x2 widen(uint32_t w, float unit) {
  u32x2 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, unit, false));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, unit, true));
  return r;
}
__device__ __forceinline__ float unit_of(uint32_t s) { return __uint_as_float(s << 23); }

// Infinite and NaN numbers of w to 0; true if there were any.
template <typename T>
__device__ __forceinline__ bool tame(u32x4 &w) {
  bool odd = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bool lo = (w[j] & T::kExp) == T::kExp;
    const bool hi = (w[j] & (T::kExp << 16)) == T::kExp << 16;
    odd |= lo | hi;
    w[j] &= ~((lo ? 0xFFFFu : 0u) | (hi ? 0xFFFF0000u : 0u));
  }
  return odd;
}

// What a row's probabilities are relative to: the score m stands for 2^at, a score s for
// 2^(c s + off), in one multiply-add.  off is rounded, so `at` is not exactly kLift; it is kept
// with the sums wherever two references meet.  A score too far out for that (its last bit is 16
// in exp2's argument) gets a power of two as c: then c m is exact, and whatever is below m
// is nothing beside it, as it is under the true c.
struct Ref {
  float c, off, at;
};
// off without a reference, fp32's largest: any score is above it, -inf gives 0
constexpr float kNoRef = 3.40282347e38f;
template <typename T>
__device__ __forceinline__ Ref ref_of(float m, float c) {
  const float size = fabsf(m * c);
  const uint32_t next = (__float_as_uint(c) + 0x7FFFFFu) & 0xFF800000u;         // c's next power
  const uint32_t e = (__float_as_uint(m) >> 23) & 0xFFu;
  const uint32_t most = (e < 90u ? 254u : 344u - e) << 23;                      // c |m| < 2^91
  Ref r;
  r.c = size >= kFar ? __uint_as_float(next < most ? next : most) : c;
  r.off = __builtin_fmaf(-m, r.c, T::kLift);
  // a large off's last bit counts, and fp16 could overflow: at from below
  const uint32_t below = __float_as_uint(r.off) + (r.off < 0.0f ? 1u : ~0u);
  r.off = __builtin_fmaf(m, r.c, r.off) > T::kLift + 0.25f ? __uint_as_float(below) : r.off;
  r.at = __builtin_fmaf(m, r.c, r.off);
  const bool none = m == -INFINITY;
  r.off = none ? kNoRef : r.off;
  r.at = none ? T::kLift : r.at;
  return r;
}
// Factor that takes sums under the reference `from`, whose `at` is given, to `to`, which is `now`.
__device__ __forceinline__ float factor(float from, float at, float to, const Ref &now, float c) {
  return from == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((from - to) * c + (now.at - at));
}

// Running state of 32 rows in a wave.
template <int DP>
struct Sums {
  f32x16 o[DP / 32];
  float m, l;                   // m: what the probabilities are relative to
  float c, off;                 // its ref_of

  __device__ __forceinline__ void clear(float scale) {
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    m = -INFINITY;
    l = 0.0f;
    off = kNoRef;
    c = scale;
  }
};

// One step of the softmax over KT 32-key score tiles: probabilities, packed as right
// operands of the second product (two 16-key groups a tile).
template <typename T, int KT, int DP>
__device__ __forceinline__ void softmax_step(Sums<DP> &st, f32x16 (&s)[KT], u32x4 (&p)[2 * KT], float c) {
  float mx = s[0][0];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kt][i]);
  mx = half_max(mx);
  const bool up = __builtin_fmaf(mx, st.c, st.off) > T::kLift + T::kSlack;
  if (__ballot(up) != 0) {
    // a row moves by its own maximum alone: the others' factor is 1
    const Ref now = ref_of<T>(up ? mx : st.m, c);
    const float alpha = up ? factor(st.m, __builtin_fmaf(st.m, st.c, st.off), mx, now, c) : 1.0f;
    st.l *= alpha;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.o[d][i] *= alpha;
    st.m = up ? mx : st.m;
    st.c = now.c;
    st.off = now.off;
  }
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    float e[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][i], st.c, st.off));
    float l0 = 0.0f, l1 = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      l0 += e[i];
      l1 += e[i + 1];
      p[2 * kt + i / 8][(i / 2) % 4] = T::pack(e[i], e[i + 1]);
    }
    st.l += l0 + l1;
  }
}

// LDS place of 16-byte chunk c of row r of C chunks (256 or 128 bytes), so that what a read
// touches at a time, 16 lanes of 16 bytes or 32 of 8, falls on all 64 banks: a fragment of the
// keys is one chunk of 16 rows, the transposing reads take 4 chunks of 4 rows (wide) or 2 of 8
// (narrow).  Writes of codes, 8 lanes a row in every other chunk, meet in pairs; dealt over two
// rows they would not, and nothing was faster for it (1377 against 1382 us).
template <int C> __device__ __forceinline__ int k_at(int r, int c) {
  return r * C + (c ^ (C == 16 ? r & 15 : (r >> 1) & 7));
}
template <int C> __device__ __forceinline__ int v_at(int r, int c) {
  const int f = C == 16 ? ((r & 3) << 2) | ((r >> 2) & 1) << 1 | (r & 1)
                        : ((r >> 1) & 1) * 5 | ((r >> 2) & 1) << 1;
  return r * C + (c ^ f);
}

// V^T's fragment: columns 32 d .. + 31 of keys 16 g + 4 h + {0..3, 8..11}; base is the
// lane's row and column of the transposing read, for g = 0.
template <int C>
__device__ __forceinline__ u32x4 v_fragment(const u32x4 *s_v, int d, int g, int lane) {
  typedef __attribute__((address_space(3))) s16x4 *at;
  const int h = lane >> 5, s = lane & 15;
  const int r = 4 * h + (s >> 2), c = 4 * d + 2 * ((lane >> 4) & 1) + ((s & 3) >> 1);
  const char *p = reinterpret_cast<const char *>(s_v + v_at<C>(r, c)) + (s & 1) * 8 + g * 16 * C * 16;
  const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(p)));
  const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(p + 8 * C * 16)));
  return u32x4{lo.x, lo.y, hi.x, hi.y};
}

// Waits for a loaded value here.  Left to its first use inside the walk's loop, the wait would
// be for all loads in every round, the next tile's among them.
__device__ __forceinline__ void settle(u32x4 &x) { asm volatile("" : "+v"(x)); }

}  // namespace
}  // namespace graft
