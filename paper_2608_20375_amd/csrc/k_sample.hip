// k_sample.hip -- the sampled acceptance walk: at every node that the walk reaches
// a token is drawn from the target model's probabilities with a given random
// number, and followed while the tree has it (the paper's Preliminaries: the target
// verifies the tree, the longest accepted path is committed; here for targets that
// sample).
//
// p(v) = e_v / S, e_v = exp((z_v - M) / T), M = max z, S = sum e;
// x = min{v : sum_{w <= v} e_w > u S}.  T = 0: the largest logit, lowest index.
//
// Only the rows on the walk's path are read, but the next row is known only when
// this one's token is.  So a launch takes one level.  A row's 16-byte vectors are cut
// into runs of 64 `rep` (one vector a lane; rep is 1 up to 2^19 words of 16 bits, 2^18 of
// fp32), four runs make a flight, and the flights are dealt to the waves of the
// sequence's workgroups.  A wave leaves its flight's maximum and the four runs' sums of
// exponentials over it.  In the next launch one wave of each workgroup combines the
// level's flights (at most 256, one to four a lane), finds the run that holds u S by a
// scan, reads that run again for the token, looks for the child, and all go on with the
// child's row.  Every workgroup of a sequence does this by itself and arrives at the same
// bits, so there is no flag, counter or wait between workgroups.  (Every wave by itself,
// without a barrier: 64 walks of 128256 words 211 us instead of 198, the vector units
// being busy with it; workgroups of 512 threads: 209; all levels of a walk in one
// workgroup: 85 instead of 71 us at 32000 words.)  Sequences whose walk has ended leave
// at once.  The flights' arrays alternate by level.
//
// Exponentials and sums are fp64: with V borders between tokens on [0, 1), an error
// of 1e-7 in the sums would change one draw in a hundred at V = 150000.
//
// Bounds and times.  A level of few walks is a chain of latencies: 6.5 us, of which 1 is
// the walk's state, 2.5 the draw, 0.6 the child, 2.4 the next row and its sums; a launch
// without walks is 2.8 us.  A level of many walks is bound by the fp64 multiply-adds: 128
// rows of 151936 words 23 us before any walk has ended, of which the instructions alone
// are 11.  The vector registers (190 for 16-bit logits) leave two waves a SIMD; held to
// 168 or 128 they spill: a sixth and a half more time for the 128 walks.
// Whole calls, as far as the walks go: 38 to 60 us for one walk of 32000 words and up to 8 levels, 63
// to 92 for 5 of 70001 fp32 words, 193 to 207 for 64 of 128256 (fp16 as bf16), 365 to 403 for 128 of
// 151936 words and up to 32 levels.
#include "graft_internal.h"

namespace graft {
namespace {

constexpr int kSampThreads = 256;
constexpr int kSampWaves = kSampThreads / kWave;
constexpr int kRuns = 4;                 // runs of a flight: vectors of a lane in flight
constexpr int kGroups = 4;               // flights of a row at most: kGroups a lane
// Waves of a launch, about: the same 128 walks of 151936 words take 341, 316 and 340 us for 4096,
// 8192 and 16384.
constexpr int64_t kSampTarget = 8192;
constexpr int kSampTree = 4;             // tree slots a lane loads ahead
constexpr int kStopped = -2;             // a walk that has ended; -1 is the root
constexpr double kLog2e = 1.4426950408889634;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct Sums {
  double run[kRuns];                     // T = 0: run[0] is the index of the maximum
};

struct SampleArgs {
  const int32_t *n_nodes, *tokens, *parents;
  const void *root, *node;
  int64_t root_stride, node_batch, node_row;
  const float *temperature;
  const double *uniform;
  int32_t *acc_len, *acc_nodes, *bonus;
  float *logp;
  int32_t *ring, *ring_pos;
  int32_t *state;                        // [L + 1][batch] node of each level
  float *tops;                           // [2][batch][flights] maxima
  Sums *sums;                            // [2][batch][flights]
  uint32_t *error_flag;
  int32_t batch, L, V, n_max, node_rows, window, update;
  int32_t splits, flights, rep;          // workgroups and flights of a row; vectors of a lane and run
};

template <typename E> struct Vec;
template <> struct Vec<float> {
  static constexpr int kPer = 4;
  static constexpr uint32_t kNone = 0xFF800000u;          // -inf
  static __device__ __forceinline__ float get(const u32x4 &v, int i) { return __uint_as_float(v[i]); }
};
template <> struct Vec<uint16_t> {
  static constexpr int kPer = 8;
  static constexpr uint32_t kNone = 0xFF80u;
  static __device__ __forceinline__ float get(const u32x4 &v, int i) {
    return __uint_as_float(i & 1 ? v[i / 2] & 0xFFFF0000u : v[i / 2] << 16);
  }
};
template <> struct Vec<_Float16> {
  static constexpr int kPer = 8;
  static constexpr uint32_t kNone = 0xFC00u;
  static __device__ __forceinline__ float get(const u32x4 &v, int i) {
    union { uint32_t u; _Float16 h[2]; } c{v[i / 2]};
    return static_cast<float>(c.h[i & 1]);
  }
};

// A row cut at 16-byte borders: vector j holds tokens j * kPer - off .. + kPer - 1.
template <typename E>
struct Row {
  static constexpr int kPer = Vec<E>::kPer;
  const E *row;
  int off, n_vec, V;
  __device__ __forceinline__ Row(const E *r, int v) : row(r), V(v) {
    off = static_cast<int>((reinterpret_cast<uintptr_t>(r) & 15u) / sizeof(E));
    n_vec = (off + v + kPer - 1) / kPer;
  }
  __device__ __forceinline__ int first(int j) const { return j * kPer - off; }
  // vectors j .. j + n - 1 hold tokens only
  __device__ __forceinline__ bool inside(int j, int n) const {
    return first(j) >= 0 && static_cast<int64_t>(first(j)) + static_cast<int64_t>(n) * kPer <= V;
  }
  __device__ __forceinline__ u32x4 whole(int j) const {
    return *reinterpret_cast<const u32x4 *>(row + first(j));
  }
  // Any vector, -inf where it has no token.  Nothing outside the row is read.
  __device__ __forceinline__ u32x4 any(int j) const {
    constexpr int kBits = 8 * sizeof(E), kIn = 32 / kBits;
    u32x4 raw;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = Vec<E>::kNone | (kIn == 2 ? Vec<E>::kNone << 16 : 0u);
    if (j >= n_vec) return raw;
    if (inside(j, 1)) return whole(j);
    const int t = first(j);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = t + i < 0 ? 0 : (t + i < V ? t + i : V - 1);
      uint32_t w;
      if constexpr (sizeof(E) == 4) w = reinterpret_cast<const uint32_t *>(row)[at];
      else w = reinterpret_cast<const uint16_t *>(row)[at];
      w = at == t + i ? w : Vec<E>::kNone;
      raw[i / kIn] = i % kIn ? (raw[i / kIn] & 0xFFFFu) | w << 16 : w | (kIn == 2 ? raw[i / kIn] & 0xFFFF0000u : 0u);
    }
    return raw;
  }
};

// Exponentials under a maximum: e_v = 2^(c (z_v - M)), c = log2(e) / T.  y = c (z - M) is split
// by adding 1.5 * 2^52, which leaves the nearest whole number in the low word; 2^f of the rest f
// in [-1/2, 1/2] is the polynomial that equals it at the 11 Chebyshev nodes, off by 3e-16 of
// the value at most and 1 at f = 0; the whole number goes to the exponent.  Differences below
// 1100 / c, masked tokens' and NaN among them, give 0.  17 instructions in all.
struct Exp2 {
  static constexpr int kDeg = 10;
  double c, low, round, coef[kDeg];
  __device__ __forceinline__ explicit Exp2(double T) {
    c = kLog2e / T;
    c = c > 1e-300 ? c : 1e-300;
    low = -1100.0 / c;
    round = 6755399441055744.0;
    asm("" : "+s"(round));
    constexpr double k[kDeg] = {0.69314718055995, 0.24022650695910097, 0.05550410866444772,
                                0.009618129107606888, 0.0013333558230164974, 0.0001540353044173605,
                                1.5252657260200837e-05, 1.321544258792169e-06,
                                1.0208690299958306e-07, 7.072585949269223e-09};
#pragma unroll
    for (int i = 0; i < kDeg; ++i) {
      coef[i] = k[i];
      // one scalar operand of a multiply-add, not a move before it
      asm("" : "+s"(coef[i]));
    }
  }
  // N at a time, step by step: a multiply-add's successor waits for it.
  template <int N>
  __device__ __forceinline__ void run(const float (&z)[N], double top, double (&w)[N]) const {
    double f[N];
    int n[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double d = fmax(static_cast<double>(z[i]) - top, low), t = fma(d, c, round);
      f[i] = fma(d, c, round - t);
      n[i] = static_cast<int>(static_cast<uint32_t>(__double_as_longlong(t)));
      w[i] = coef[kDeg - 1];
    }
#pragma unroll
    for (int k = kDeg - 2; k >= -1; --k)
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = fma(w[i], f[i], k < 0 ? 1.0 : coef[k < 0 ? 0 : k]);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = ldexp(w[i], n[i]);
  }
};
// e of a vector's tokens: 1 at the maximum, which may be infinite (a case of its own).
template <typename E>
__device__ __forceinline__ void weights(const u32x4 &raw, float top, const Exp2 &ex,
                                        double (&w)[Vec<E>::kPer]) {
  float z[Vec<E>::kPer];
  if (top == INFINITY) {
#pragma unroll
    for (int i = 0; i < Vec<E>::kPer; ++i) w[i] = Vec<E>::get(raw, i) == INFINITY ? 1.0 : 0.0;
  } else {
#pragma unroll
    for (int i = 0; i < Vec<E>::kPer; ++i) z[i] = Vec<E>::get(raw, i);
    ex.run(z, top, w);
  }
}
// Factor of a sum over the maximum `from` under the maximum `to`.
__device__ __forceinline__ double factor(float from, float to, const Exp2 &ex) {
  if (to == INFINITY) return from == INFINITY ? 1.0 : 0.0;
  const float z[1] = {from};
  double w[1];
  ex.run(z, to, w);
  return w[0];
}
// Largest over the lanes, in scalar registers: the steps of wave_incl_scan, lanes without a
// source keeping their own.
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_max(float v) {
  const int x = static_cast<int>(__float_as_uint(v));
  return fmaxf(v, __uint_as_float(static_cast<uint32_t>(
                      __builtin_amdgcn_update_dpp(x, x, CTRL, ROWS, 0xF, false))));
}
__device__ __forceinline__ float wave_max(float v) {
  v = dpp_max<0x111, 0xF>(v);
  v = dpp_max<0x112, 0xF>(v);
  v = dpp_max<0x114, 0xF>(v);
  v = dpp_max<0x118, 0xF>(v);
  v = dpp_max<0x142, 0xA>(v);
  v = dpp_max<0x143, 0xC>(v);
  return __uint_as_float(static_cast<uint32_t>(
      __builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(v)), kWave - 1)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_f64(double v) {   // lanes without a source: 0
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(v));
  const uint32_t lo = static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(u), CTRL, ROWS, 0xF, false));
  const uint32_t hi = static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), CTRL, ROWS, 0xF, false));
  return __longlong_as_double(static_cast<long long>((static_cast<uint64_t>(hi) << 32) | lo));
}
// Inclusive prefix sums over the lanes, by the steps of wave_incl_scan.
__device__ __forceinline__ double wave_scan(double v) {
  v += dpp_f64<0x111, 0xF>(v);
  v += dpp_f64<0x112, 0xF>(v);
  v += dpp_f64<0x114, 0xF>(v);
  v += dpp_f64<0x118, 0xF>(v);
  v += dpp_f64<0x142, 0xA>(v);
  v += dpp_f64<0x143, 0xC>(v);
  return v;
}
// x over the lanes' pairs (lane, lane ^ M) in the lanes without bit M, y in those with it.
template <int M> __device__ __forceinline__ double swap_add(double x, double y) {
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x)), v = static_cast<uint64_t>(__double_as_longlong(y));
  uint32_t w[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t p = static_cast<uint32_t>(u >> (32 * i)), q = static_cast<uint32_t>(v >> (32 * i));
    const auto r = M == 32 ? __builtin_amdgcn_permlane32_swap(p, q, false, false)
                           : __builtin_amdgcn_permlane16_swap(p, q, false, false);
    w[0][i] = r[0];
    w[1][i] = r[1];
  }
  const auto f64 = [](const uint32_t (&z)[2]) {
    return __longlong_as_double(static_cast<long long>((static_cast<uint64_t>(z[1]) << 32) | z[0]));
  };
  return f64(w[0]) + f64(w[1]);
}
__device__ __forceinline__ double lane_f64(double v, int lane) {   // of a uniform lane
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(v));
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(u), lane));
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(u >> 32), lane));
  return __longlong_as_double(static_cast<long long>((static_cast<uint64_t>(hi) << 32) | lo));
}
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const int o = static_cast<int>(xor_lane(static_cast<uint32_t>(v), m));
    v = o < v ? o : v;
  }
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int first_lane(uint64_t lanes) { return __builtin_ctzll(lanes); }
__device__ __forceinline__ int last_lane(uint64_t lanes) { return 63 - __builtin_clzll(lanes); }

template <typename E>
__device__ __forceinline__ const E *row_of(const SampleArgs &a, int b, int node) {
  return node < 0 ? static_cast<const E *>(a.root) + b * a.root_stride
                  : static_cast<const E *>(a.node) + b * a.node_batch + node * a.node_row;
}

__device__ __forceinline__ double temperature(const SampleArgs &a, int b, bool *bad) {
  const float t = a.temperature ? a.temperature[b] : 1.0f;
  *bad = !(t >= 0.0f);
  return *bad ? 0.0 : static_cast<double>(t);
}

// A level's flights, one to kGroups a lane.
struct Level {
  float top[kGroups];
  Sums sums[kGroups];
};

// A drawn token: -1 if none has a positive probability.  Its logit, the maximum and the
// sum give the log-probability.
struct Draw {
  int token;
  float z, top;
  double total;
  __device__ __forceinline__ float logp(double T) const {
    if (token < 0) return -INFINITY;
    if (T == 0.0) return 0.0f;
    const double d = z == top ? 0.0 : (static_cast<double>(z) - static_cast<double>(top)) / T;
    return static_cast<float>(d - log(total));
  }
};
// The token of a level from its flights, the same in all lanes.
template <typename E>
__device__ __forceinline__ Draw draw_token(const SampleArgs &a, Level &at, const Row<E> &row,
                                          const Exp2 &ex, double T, double u) {
  const int lane = lane_id();
  const int per = kWave * a.rep;                         // vectors of a run
  const int flights = (row.n_vec + kRuns * per - 1) / (kRuns * per);
  float m = -INFINITY;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    if (g * kWave + lane >= flights) {
      at.top[g] = -INFINITY;
      at.sums[g] = Sums{};
    }
    m = fmaxf(m, at.top[g]);
  }
  const float top = wave_max(m);
  if (top == -INFINITY) return Draw{-1, top, top, 0.0};
  if (T == 0.0) {
    int best = INT32_MAX;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int i = static_cast<int>(at.sums[g].run[0]);
      if (at.top[g] == top && i < best) best = i;
    }
    return Draw{wave_min(best), top, top, 1.0};
  }
  double all[kGroups], upto[kGroups], total = 0.0;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    all[g] = 0.0;
    upto[g] = total;
    if (g * kWave >= flights) continue;
    const double f = factor(at.top[g], top, ex);
#pragma unroll
    for (int r = 0; r < kRuns; ++r) {
      at.sums[g].run[r] *= f;
      all[g] += at.sums[g].run[r];
    }
    upto[g] = total + wave_scan(all[g]);
    total = lane_f64(upto[g], kWave - 1);
  }
  const double goal = u * total;
  // the first flight whose sum passes the goal; rounding or u >= 1 may leave none, then the
  // last with a token, and its last token
  uint64_t lanes = 0;
  int group = 0;
#pragma unroll
  for (int g = 0; g < kGroups; ++g)
    if (lanes == 0 && (lanes = __ballot(all[g] > 0.0 && upto[g] > goal)) != 0) group = g;
  bool past = lanes == 0;
  int who = past ? 0 : first_lane(lanes);
  if (past) {
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const uint64_t some = __ballot(all[g] > 0.0);
      if (some != 0) {
        group = g;
        who = last_lane(some);
      }
    }
  }
  double sum[kRuns] = {}, before = 0.0;
#pragma unroll
  for (int g = 0; g < kGroups; ++g)
    if (g == group) {
      before = lane_f64(upto[g] - all[g], who);
#pragma unroll
      for (int r = 0; r < kRuns; ++r) sum[r] = lane_f64(at.sums[g].run[r], who);
    }
  // likewise the run
  int run = -1, last = 0;
  double base = before, last_base = before;
#pragma unroll
  for (int r = 0; r < kRuns; ++r) {
    if (sum[r] > 0.0) {
      last = r;
      last_base = before;
      if (run < 0 && !past && before + sum[r] > goal) {
        run = r;
        base = before;
      }
    }
    before += sum[r];
  }
  if (run < 0) {
    run = last;
    base = last_base;
    past = true;
  }
  // and the token
  const int v0 = ((group * kWave + who) * kRuns + run) * per;
  int tok = -1;
  float z = 0.0f;
  for (int r = 0; r < a.rep; ++r) {
    const int j = v0 + r * kWave + lane;
    const u32x4 raw = row.any(j);
    double w[Vec<E>::kPer], mine = 0.0;
    weights<E>(raw, top, ex, w);
#pragma unroll
    for (int i = 0; i < Vec<E>::kPer; ++i) mine += w[i];
    const double end = base + wave_scan(mine);
    const uint64_t hits = past ? 0 : __ballot(mine > 0.0 && end > goal), some = __ballot(mine > 0.0);
    base = lane_f64(end, kWave - 1);
    if (some == 0) continue;
    // the lane's first token past the goal, its last with a probability where rounding leaves none
    double upto_i = end - mine;
    int hit = -1;
    float hit_z = 0.0f;
    bool found = false;
#pragma unroll
    for (int i = 0; i < Vec<E>::kPer; ++i) {
      upto_i += w[i];
      if (w[i] > 0.0 && !found) {
        hit = row.first(j) + i;
        hit_z = Vec<E>::get(raw, i);
        found = hits != 0 && upto_i > goal;
      }
    }
    const int from = hits != 0 ? first_lane(hits) : last_lane(some);
    tok = __builtin_amdgcn_readlane(hit, from);
    z = __uint_as_float(static_cast<uint32_t>(
        __builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(hit_z)), from)));
    if (hits != 0) break;
  }
  return Draw{tok, z, top, total};   // tok < 0 only if the row changed under the call
}

// Level `level` of every walk: its node from the level before, then this
// wave's flights of the node's row.  level L + 1 ends the walks.
template <typename E>
__global__ void __launch_bounds__(kSampThreads)
sample_kernel(SampleArgs a, int level) {
  __shared__ int s_node;
  __shared__ Draw s_drawn;
  const int splits = level <= a.L ? a.splits : 1;
  const int b = blockIdx.x / splits;
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane((blockIdx.x - b * splits) * kSampWaves + threadIdx.x / kWave);
  const int before = level > 0 ? a.state[(level - 1) * a.batch + b] : -1;
  if (before == kStopped) {
    if (wave == 0 && lane == 0 && level <= a.L) a.state[level * a.batch + b] = kStopped;
    return;
  }
  bool bad_t;
  const double T = temperature(a, b, &bad_t);
  const Exp2 ex(T);
  int node = -1;
  if (level > 0) {
    if (wave % kSampWaves == 0) {
      // the tree's arrays with the flights: one round trip
      int32_t par[kSampTree], tok[kSampTree];
      const int64_t tree = static_cast<int64_t>(b) * a.n_max;
#pragma unroll
      for (int k = 0; k < kSampTree; ++k) {
        const int i = lane + k * kWave;
        par[k] = a.parents[tree + (i < a.n_max ? i : a.n_max - 1)];
        tok[k] = a.tokens[tree + (i < a.n_max ? i : a.n_max - 1)];
      }
      Level left;
      const int64_t at = (static_cast<int64_t>((level - 1) & 1) * a.batch + b) * a.flights;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        const int f = g * kWave + lane;
        if (f < a.flights) {
          left.top[g] = a.tops[at + f];
          left.sums[g] = a.sums[at + f];
        }
      }
      const double u = a.uniform[static_cast<int64_t>(b) * (a.L + 1) + level - 1];
      int n = a.n_nodes[b];
      n = n < 0 ? 0 : (n > a.n_max ? a.n_max : n);
      n = n > a.node_rows ? a.node_rows : n;
      const Draw drawn = draw_token<E>(a, left, Row<E>(row_of<E>(a, b, before), a.V), ex, T, u);
      const int x = drawn.token;
      int child = INT32_MAX;
#pragma unroll
      for (int k = kSampTree - 1; k >= 0; --k) {
        const int i = lane + k * kWave;
        const uint64_t hits = __ballot(i < n && i > before && par[k] == before && tok[k] == x);
        if (hits != 0) child = k * kWave + first_lane(hits);
      }
      for (int k = kSampTree * kWave; k < n && child == INT32_MAX; k += kWave) {
        const int i = k + lane;
        const uint64_t hits = __ballot(i < n && i > before && a.parents[tree + i] == before && a.tokens[tree + i] == x);
        if (hits != 0) child = k + first_lane(hits);
      }
      const bool go = child != INT32_MAX && level <= a.L && x >= 0;
      node = go ? child : kStopped;
      if (wave == 0) {
        const int d = level - 1;                  // nodes accepted before this token
        if (lane == 0) {
          if (level <= a.L) a.state[level * a.batch + b] = node;
          if (!go && a.logp) a.logp[static_cast<int64_t>(b) * (a.L + 1) + d] = drawn.logp(T);
          if (go) a.acc_nodes[static_cast<int64_t>(b) * a.L + d] = child;
          if (x < 0) atomicOr(a.error_flag, kErrTargetRow);
        }
        if (!go) {
          for (int i = d + lane; i < a.L; i += kWave)
            a.acc_nodes[static_cast<int64_t>(b) * a.L + i] = -1;
          if (a.logp)
            for (int i = d + 1 + lane; i <= a.L; i += kWave)
              a.logp[static_cast<int64_t>(b) * (a.L + 1) + i] = 0.0f;
          if (lane == 0) {
            a.acc_len[b] = d;
            a.bonus[b] = x;
            if (a.update) {
              const int p = a.ring_pos[b];
              a.ring[static_cast<int64_t>(b) * a.window + p] = d;
              a.ring_pos[b] = (p + 1) % a.window;
            }
          }
        }
      }
      if (lane == 0) {
        s_node = node;
        s_drawn = drawn;
      }
    }
    __syncthreads();
    node = __builtin_amdgcn_readfirstlane(s_node);
    if (node == kStopped) return;
  } else if (wave == 0 && lane == 0) {
    a.state[b] = -1;
    if (bad_t) atomicOr(a.error_flag, kErrTargetRow);
  }

  // this wave's flights of the row
  const Row<E> row(row_of<E>(a, b, node), a.V);
  const int per = kWave * a.rep;
  const int flights = (row.n_vec + kRuns * per - 1) / (kRuns * per);
  const int64_t at = (static_cast<int64_t>(level & 1) * a.batch + b) * a.flights;
  for (int f = wave; f < flights; f += splits * kSampWaves) {
    float m = -INFINITY;
    int best = INT32_MAX;                         // T = 0: index of this lane's maximum
    double sum[kRuns] = {};
    for (int r = 0; r < a.rep; ++r) {
      const int j0 = f * kRuns * per + r * kWave;
      u32x4 raw[kRuns];
      if (row.inside(j0, 3 * per + kWave)) {
#pragma unroll
        for (int k = 0; k < kRuns; ++k) raw[k] = row.whole(j0 + k * per + lane);
      } else {
#pragma unroll
        for (int k = 0; k < kRuns; ++k) raw[k] = row.any(j0 + k * per + lane);
      }
      float g = m;
#pragma unroll
      for (int k = 0; k < kRuns; ++k)
#pragma unroll
        for (int i = 0; i < Vec<E>::kPer; ++i) g = fmaxf(g, Vec<E>::get(raw[k], i));
      if (T == 0.0) {
#pragma unroll
        for (int k = 0; k < kRuns; ++k)
#pragma unroll
          for (int i = 0; i < Vec<E>::kPer; ++i) {
            const float z = Vec<E>::get(raw[k], i);
            const int t = row.first(j0 + k * per + lane) + i;
            if (z > m || (z == m && m != -INFINITY && t < best)) {
              m = z;
              best = t;
            }
          }
        continue;
      }
      const float all = wave_max(g);
      if (all == -INFINITY) continue;
      if (r > 0) {
        const double scale = factor(m, all, ex);
#pragma unroll
        for (int k = 0; k < kRuns; ++k) sum[k] *= scale;
      }
      m = all;
#pragma unroll
      for (int k = 0; k < kRuns; ++k) {
        double w[Vec<E>::kPer];
        weights<E>(raw[k], all, ex, w);
#pragma unroll
        for (int i = 0; i < Vec<E>::kPer; ++i) sum[k] += w[i];
      }
    }
    if (T == 0.0) {
      const float all = wave_max(m);
      best = wave_min(m == all ? best : INT32_MAX);
      if (lane == 0) {
        a.tops[at + f] = all;
        a.sums[at + f].run[0] = static_cast<double>(best);
      }
      continue;
    }
    // the four sums together: halves of the wave keep two each, then rows of 16 one each
    double t = swap_add<16>(swap_add<32>(sum[0], sum[2]), swap_add<32>(sum[1], sum[3]));
    t += xor_lane_f64(t, 8);
    t += xor_lane_f64(t, 4);
    t += xor_lane_f64(t, 2);
    t += xor_lane_f64(t, 1);
    if ((lane & 15) == 0) a.sums[at + f].run[lane / 16] = t;
    if (lane == 0) a.tops[at + f] = m;
  }
  // the token's log-probability, which nothing waits for
  if (level > 0 && wave == splits * kSampWaves - 1 && lane == 0 && a.logp)
    a.logp[static_cast<int64_t>(b) * (a.L + 1) + level - 1] = s_drawn.logp(T);
}

}  // namespace

SamplePlan sample_plan(const graft_dims &d, int batch, int dtype) {
  SamplePlan p;
  const int64_t once = kRuns * kWave, most = kGroups * kWave;
  // 16-byte vectors of a row, whatever its alignment
  const int words = dtype == GRAFT_F32 ? 4 : 8;
  const int64_t vectors = (static_cast<int64_t>(d.vocab) + 2 * words - 2) / words;
  p.rep = static_cast<int>((vectors + once * most - 1) / (once * most));
  p.flights = static_cast<int>((vectors + once * p.rep - 1) / (once * p.rep));
  const int64_t want = kSampTarget / batch > 1 ? kSampTarget / batch : 1;   // waves a row
  const int64_t each = (p.flights + want - 1) / want;
  p.splits = static_cast<int>((p.flights + each * kSampWaves - 1) / (each * kSampWaves));
  const int64_t n = int64_t{2} * batch * p.flights;
  p.tops_at = (static_cast<int64_t>(d.num_pos + 1) * batch * 4 + 255) & ~int64_t{255};
  p.sums_at = (p.tops_at + n * 4 + 255) & ~int64_t{255};
  p.bytes = p.sums_at + n * static_cast<int64_t>(sizeof(Sums));
  return p;
}

int64_t sample_bytes(const graft_dims &d, int batch) {
  const int64_t wide = sample_plan(d, batch, GRAFT_F32).bytes;
  const int64_t half = sample_plan(d, batch, GRAFT_BF16).bytes;
  return wide > half ? wide : half;
}

hipError_t launch_accept_sampled(graft_ctx *ctx, int batch, const int32_t *n_nodes,
                                 const int32_t *tokens, const int32_t *parents,
                                 const graft_target_logits *t, int32_t *acc_len,
                                 int32_t *acc_nodes, int32_t *bonus, float *logp,
                                 int update_history, void *workspace, hipStream_t stream) {
  const graft_dims &d = ctx->dims;
  const SamplePlan p = sample_plan(d, batch, t->dtype);
  SampleArgs a{};
  a.n_nodes = n_nodes;
  a.tokens = tokens;
  a.parents = parents;
  a.root = t->root;
  a.node = t->node;
  a.root_stride = t->root_stride;
  a.node_batch = t->node_batch_stride;
  a.node_row = t->node_row_stride;
  a.temperature = t->temperature;
  a.uniform = t->uniform;
  a.acc_len = acc_len;
  a.acc_nodes = acc_nodes;
  a.bonus = bonus;
  a.logp = logp;
  a.ring = ctx->hist_ring;
  a.ring_pos = ctx->hist_pos;
  a.state = static_cast<int32_t *>(workspace);
  a.tops = reinterpret_cast<float *>(static_cast<char *>(workspace) + p.tops_at);
  a.sums = reinterpret_cast<Sums *>(static_cast<char *>(workspace) + p.sums_at);
  a.error_flag = ctx->error_flag;
  a.batch = batch;
  a.L = d.num_pos;
  a.V = d.vocab;
  a.n_max = d.max_nodes;
  a.node_rows = t->node_rows;
  a.window = d.hist_window;
  a.update = update_history;
  a.splits = p.splits;
  a.flights = p.flights;
  a.rep = p.rep;
  hipError_t e = hipSuccess;
  for (int level = 0; e == hipSuccess && level <= d.num_pos + 1; ++level) {
    const dim3 grid(static_cast<unsigned>(batch) * (level <= d.num_pos ? a.splits : 1));
    const dim3 block(kSampThreads);
    if (t->dtype == GRAFT_F32)
      hipLaunchKernelGGL(sample_kernel<float>, grid, block, 0, stream, a, level);
    else if (t->dtype == GRAFT_BF16)
      hipLaunchKernelGGL(sample_kernel<uint16_t>, grid, block, 0, stream, a, level);
    else
      hipLaunchKernelGGL(sample_kernel<_Float16>, grid, block, 0, stream, a, level);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace graft
