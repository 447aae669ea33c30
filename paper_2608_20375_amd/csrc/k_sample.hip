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
// this one's token is.  So a launch takes one level: a row's words are dealt to
// `splits` workgroups and their waves, each of which leaves the maximum of its run
// of words and the sum of their exponentials over it.  The next launch's workgroups
// each combine the level's partials (at most 256, one a thread), find the run that
// holds u S by a scan, read that run again for the token, look for the child, and go
// on with the child's row; every workgroup of a sequence does this by itself and
// arrives at the same bits, so no flag, counter or wait between workgroups is
// needed.  Sequences whose walk has ended leave at once.  Row pairs of partials
// alternate by level.
//
// Exponentials and sums are fp64: with V borders between tokens on [0, 1), an error
// of 1e-7 in the sums would change one draw in a hundred at V = 150000.
#include "graft_internal.h"

namespace graft {
namespace {

constexpr int kSampThreads = 256;
constexpr int kSampWaves = kSampThreads / kWave;
constexpr int kSampParts = 256;          // partials of a row at most: one a thread
constexpr int kSampFlight = 4;           // 16-byte vectors of a lane in flight
constexpr int kStopped = -2;             // a walk that has ended; -1 is the root
static_assert(kMaxNodes % kSampThreads == 0, "tree slots a thread");

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct Part {
  double max, sum;                       // T = 0: the sum is the index of the maximum
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
  Part *parts;                           // [2][batch][splits * kSampWaves]
  uint32_t *error_flag;
  int32_t batch, L, V, n_max, node_rows, window, update;
  int32_t splits;
};

__device__ __forceinline__ float value(const float *p) { return *p; }
__device__ __forceinline__ float value(const uint16_t *p) {
  return __uint_as_float(static_cast<uint32_t>(*p) << 16);
}
__device__ __forceinline__ float value(const _Float16 *p) { return static_cast<float>(*p); }

template <typename E> struct Vec;
template <> struct Vec<float> {
  static constexpr int kPer = 4;
  static __device__ __forceinline__ float get(const u32x4 &v, int i) { return __uint_as_float(v[i]); }
};
template <> struct Vec<uint16_t> {
  static constexpr int kPer = 8;
  static __device__ __forceinline__ float get(const u32x4 &v, int i) {
    return __uint_as_float(i & 1 ? v[i / 2] & 0xFFFF0000u : v[i / 2] << 16);
  }
};
template <> struct Vec<_Float16> {
  static constexpr int kPer = 8;
  static __device__ __forceinline__ float get(const u32x4 &v, int i) {
    union { uint32_t u; _Float16 h[2]; } c{v[i / 2]};
    return static_cast<float>(c.h[i & 1]);
  }
};

// A row cut at 16-byte borders: vector j holds tokens j * kPer - off .. + kPer - 1.
template <typename E>
struct Row {
  const E *row;
  int off, n_vec, V;
  __device__ __forceinline__ Row(const E *r, int v) : row(r), V(v) {
    off = static_cast<int>((reinterpret_cast<uintptr_t>(r) & 15u) / sizeof(E));
    n_vec = (off + v + Vec<E>::kPer - 1) / Vec<E>::kPer;
  }
  __device__ __forceinline__ int first(int j) const { return j * Vec<E>::kPer - off; }
  // Vector j as fp32; -inf where it has no token, and for NaN.  Only whole vectors
  // are loaded as such: nothing outside the row is read.
  __device__ __forceinline__ void load(int j, bool on, u32x4 *raw) const {
    const int t = first(j);
    if (on && t >= 0 && t + Vec<E>::kPer <= V)
      *raw = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(row + t));
  }
  __device__ __forceinline__ void take(int j, bool on, const u32x4 &raw,
                                       float (&x)[Vec<E>::kPer]) const {
    const int t = first(j);
    const bool whole = on && t >= 0 && t + Vec<E>::kPer <= V;
#pragma unroll
    for (int i = 0; i < Vec<E>::kPer; ++i) {
      float z = -INFINITY;
      if (whole) z = Vec<E>::get(raw, i);
      else if (on && t + i >= 0 && t + i < V) z = value(row + t + i);
      x[i] = z != z ? -INFINITY : z;
    }
  }
};

// e_v: 1 at the maximum (an infinite one too), 0 for masked tokens.
__device__ __forceinline__ double weight(float z, double max, double inv_t) {
  const double d = static_cast<double>(z);
  if (d == max) return 1.0;
  if (z == -INFINITY || max == INFINITY) return 0.0;
  return exp((d - max) * inv_t);
}
// A part's sum over another maximum.
__device__ __forceinline__ double rescale(double sum, double from, double to, double inv_t) {
  if (from == to) return sum;
  if (from == -INFINITY || to == INFINITY) return 0.0;
  return sum * exp((from - to) * inv_t);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1)
    v = fmaxf(v, __uint_as_float(xor_lane(__float_as_uint(v), m)));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) v += xor_lane_f64(v, m);
  return v;
}
__device__ __forceinline__ double shfl_up_f64(double v, int d) {
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(v));
  const uint32_t lo = __shfl_up(static_cast<uint32_t>(u), d);
  const uint32_t hi = __shfl_up(static_cast<uint32_t>(u >> 32), d);
  return __longlong_as_double(static_cast<long long>((static_cast<uint64_t>(hi) << 32) | lo));
}

// Inclusive prefix sums over the workgroup's threads in thread order.
__device__ __forceinline__ double block_scan(double v, double *s_wave) {
  const int lane = lane_id(), wave = threadIdx.x / kWave;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const double o = shfl_up_f64(v, d);
    if (lane >= d) v += o;
  }
  __syncthreads();
  if (lane == kWave - 1) s_wave[wave] = v;
  __syncthreads();
  double before = 0.0;
  for (int w = 0; w < wave; ++w) before += s_wave[w];
  return before + v;
}
// Smallest and largest of one int a thread.
__device__ __forceinline__ int block_min(int v, int *s_int) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const int o = static_cast<int>(xor_lane(static_cast<uint32_t>(v), m));
    v = o < v ? o : v;
  }
  __syncthreads();
  if (lane_id() == 0) s_int[threadIdx.x / kWave] = v;
  __syncthreads();
  int r = s_int[0];
#pragma unroll
  for (int w = 1; w < kSampWaves; ++w) r = s_int[w] < r ? s_int[w] : r;
  return r;
}

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

// The token of a level from its partials, -1 if no token has a positive
// probability; *lp its log-probability.  Every thread gets both.
template <typename E>
__device__ int draw_token(const SampleArgs &a, const Part &mine, int n_parts, const Row<E> &row,
                          double T, double u, double *s_wave, float *s_max, int *s_int, double *lp) {
  const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
  const double inv_t = 1.0 / T;
  const bool have = tid < n_parts;
  // maxima are fp32 numbers
  const float m = have ? static_cast<float>(mine.max) : -INFINITY;
  const float wm = wave_max(m);
  __syncthreads();
  if (lane == 0) s_max[wave] = wm;
  __syncthreads();
  float top = s_max[0];
#pragma unroll
  for (int w = 1; w < kSampWaves; ++w) top = fmaxf(top, s_max[w]);
  *lp = 0.0;
  if (top == -INFINITY) {
    *lp = -INFINITY;
    return -1;
  }
  if (T == 0.0) return block_min(have && m == top ? static_cast<int>(mine.sum) : INT32_MAX, s_int);
  const double M = static_cast<double>(top);
  const double part = have ? rescale(mine.sum, mine.max, M, inv_t) : 0.0;
  const double upto = block_scan(part, s_wave);
  __syncthreads();
  if (tid == kSampThreads - 1) s_wave[0] = upto;
  __syncthreads();
  const double total = s_wave[0], goal = u * total;
  // the run that holds the goal: the first whose sum passes it; rounding or u >= 1
  // may leave none, then the last with a token
  int run = block_min(have && upto > goal && part > 0.0 ? tid : kSampThreads, s_int);
  const bool past = run == kSampThreads;
  if (past) run = -block_min(have && part > 0.0 ? -tid : 1, s_int);
  __syncthreads();
  if (tid == run) s_wave[0] = upto - part;
  __syncthreads();
  const double before = s_wave[0];
  const int per = (row.n_vec + n_parts - 1) / n_parts;
  const int v0 = run * per, v1 = v0 + per < row.n_vec ? v0 + per : row.n_vec;
  const int each = (per + kSampThreads - 1) / kSampThreads;
  const int a0 = v0 + tid * each < v1 ? v0 + tid * each : v1;
  const int a1 = a0 + each < v1 ? a0 + each : v1;
  double sum = 0.0;
  float x[Vec<E>::kPer];
  for (int j = a0; j < a1; ++j) {
    u32x4 raw{};
    row.load(j, true, &raw);
    row.take(j, true, raw, x);
#pragma unroll
    for (int i = 0; i < Vec<E>::kPer; ++i) sum += weight(x[i], M, inv_t);
  }
  const double end = before + block_scan(sum, s_wave);
  double at = end - sum;
  int hit = INT32_MAX, last = -1;                 // -1: none (and block_min gives 1)
  // this thread's tokens: the first past the goal, and the last with a probability
  for (int j = a0; j < a1; ++j) {
    u32x4 raw{};
    row.load(j, true, &raw);
    row.take(j, true, raw, x);
#pragma unroll
    for (int i = 0; i < Vec<E>::kPer; ++i) {
      const double w = weight(x[i], M, inv_t);
      at += w;
      const int t = row.first(j) + i;
      if (w > 0.0) {
        last = t;
        if (at > goal && hit == INT32_MAX) hit = t;
      }
    }
  }
  int x_tok = past ? INT32_MAX : block_min(hit, s_int);
  if (x_tok == INT32_MAX) x_tok = -block_min(-last, s_int);
  if (x_tok < 0) {   // only if the row changed under the call
    *lp = -INFINITY;
    return -1;
  }
  const float z = value(row.row + x_tok);
  *lp = (static_cast<double>(z) == M ? 0.0 : (static_cast<double>(z) - M) * inv_t) - log(total);
  return x_tok;
}

// Level `level` of every walk: its node from the level before, then this
// workgroup's share of the node's row.  level L + 1 ends the walks.
template <typename E>
__global__ void __launch_bounds__(kSampThreads)
sample_kernel(SampleArgs a, int level) {
  __shared__ double s_wave[kSampWaves];
  __shared__ float s_max[kSampWaves];
  __shared__ int s_int[kSampWaves];
  const int splits = level <= a.L ? a.splits : 1;
  const int b = blockIdx.x / splits, split = blockIdx.x - b * splits;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave;
  const int n_parts = a.splits * kSampWaves;
  bool bad_t;
  const double T = temperature(a, b, &bad_t);
  int node = -1;
  if (level > 0) {
    const int before = a.state[(level - 1) * a.batch + b];
    if (before == kStopped) {
      if (split == 0 && tid == 0 && level <= a.L) a.state[level * a.batch + b] = kStopped;
      return;
    }
    // the tree's arrays with the partials: one round trip
    constexpr int kPer = kMaxNodes / kSampThreads;
    int32_t par[kPer], tok[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = tid + k * kSampThreads;
      const int64_t at = static_cast<int64_t>(b) * a.n_max + (i < a.n_max ? i : a.n_max - 1);
      par[k] = a.parents[at];
      tok[k] = a.tokens[at];
    }
    Part mine{-INFINITY, 0.0};
    if (tid < n_parts)
      mine = a.parts[(static_cast<int64_t>((level - 1) & 1) * a.batch + b) * n_parts + tid];
    const double u = a.uniform[static_cast<int64_t>(b) * (a.L + 1) + level - 1];
    int n = a.n_nodes[b];
    n = n < 0 ? 0 : (n > a.n_max ? a.n_max : n);
    n = n > a.node_rows ? a.node_rows : n;
    double lp;
    const Row<E> row(row_of<E>(a, b, before), a.V);
    const int x = draw_token<E>(a, mine, n_parts, row, T, u, s_wave, s_max, s_int, &lp);
    int child = INT32_MAX;
#pragma unroll
    for (int k = kPer - 1; k >= 0; --k) {
      const int i = tid + k * kSampThreads;
      if (i < n && i > before && par[k] == before && tok[k] == x) child = i;
    }
    child = block_min(child, s_int);
    const bool go = child != INT32_MAX && level <= a.L && x >= 0;
    node = go ? child : kStopped;
    if (split == 0) {
      const int d = level - 1;                  // nodes accepted before this token
      if (tid == 0) {
        if (level <= a.L) a.state[level * a.batch + b] = node;
        if (a.logp) a.logp[static_cast<int64_t>(b) * (a.L + 1) + d] = static_cast<float>(lp);
        if (go) a.acc_nodes[static_cast<int64_t>(b) * a.L + d] = child;
        if (x < 0) atomicOr(a.error_flag, kErrTargetRow);
      }
      if (!go) {
        for (int i = d + tid; i < a.L; i += kSampThreads)
          a.acc_nodes[static_cast<int64_t>(b) * a.L + i] = -1;
        if (a.logp)
          for (int i = d + 1 + tid; i <= a.L; i += kSampThreads)
            a.logp[static_cast<int64_t>(b) * (a.L + 1) + i] = 0.0f;
        if (tid == 0) {
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
    if (!go) return;
  } else if (split == 0 && tid == 0) {
    a.state[b] = -1;
    if (bad_t) atomicOr(a.error_flag, kErrTargetRow);
  }

  // this wave's run of the row's vectors
  const Row<E> row(row_of<E>(a, b, node), a.V);
  const int per = (row.n_vec + n_parts - 1) / n_parts;
  const int run = split * kSampWaves + wave;
  const int v0 = run * per, v1 = v0 + per < row.n_vec ? v0 + per : row.n_vec;
  const double inv_t = 1.0 / T;
  float m = -INFINITY;
  double sum = 0.0;                               // T = 0: the index of m
  for (int j0 = v0; j0 < v1; j0 += kSampFlight * kWave) {
    u32x4 raw[kSampFlight] = {};
#pragma unroll
    for (int k = 0; k < kSampFlight; ++k) {
      const int j = j0 + k * kWave + lane;
      row.load(j, j < v1, &raw[k]);
    }
    float x[kSampFlight][Vec<E>::kPer];
    float g = m;
#pragma unroll
    for (int k = 0; k < kSampFlight; ++k) {
      const int j = j0 + k * kWave + lane;
      row.take(j, j < v1, raw[k], x[k]);
#pragma unroll
      for (int i = 0; i < Vec<E>::kPer; ++i) g = fmaxf(g, x[k][i]);
    }
    if (T == 0.0) {
      // a later equal value never replaces an earlier one of this lane
#pragma unroll
      for (int k = 0; k < kSampFlight; ++k)
#pragma unroll
        for (int i = 0; i < Vec<E>::kPer; ++i)
          if (x[k][i] > m) {
            m = x[k][i];
            sum = static_cast<double>(row.first(j0 + k * kWave + lane) + i);
          }
    } else {
      const float all = wave_max(g);
      if (all == -INFINITY) continue;
      const double M = static_cast<double>(all);
      sum = rescale(sum, static_cast<double>(m), M, inv_t);
      m = all;
#pragma unroll
      for (int k = 0; k < kSampFlight; ++k)
#pragma unroll
        for (int i = 0; i < Vec<E>::kPer; ++i) sum += weight(x[k][i], M, inv_t);
    }
  }
  if (T == 0.0) {
    const float all = wave_max(m);
    double best = m == all ? sum : 4294967296.0;
#pragma unroll
    for (int k = 1; k < kWave; k <<= 1) best = fmin(best, xor_lane_f64(best, k));
    m = all;
    sum = best;
  } else {
    sum = wave_sum(sum);
  }
  if (lane == 0)
    a.parts[(static_cast<int64_t>(level & 1) * a.batch + b) * n_parts + run] =
        Part{static_cast<double>(m), sum};
}

int64_t state_bytes(const graft_dims &d, int batch) {
  return (static_cast<int64_t>(d.num_pos + 1) * batch * 4 + 255) & ~int64_t{255};
}

}  // namespace

// Workgroups of a row: enough to give every CU a few, each wave at least 512
// words, at most kSampParts partials.
int sample_splits(const graft_dims &d, int batch) {
  int s = (1024 + batch - 1) / batch;
  const int most = (d.vocab + 512 * kSampWaves - 1) / (512 * kSampWaves);
  s = s < most ? s : most;
  const int cap = kSampParts / kSampWaves;
  s = s < cap ? s : cap;
  return s < 1 ? 1 : s;
}

int64_t sample_bytes(const graft_dims &d, int batch) {
  return state_bytes(d, batch) +
         int64_t{2} * batch * sample_splits(d, batch) * kSampWaves * sizeof(Part);
}

hipError_t launch_accept_sampled(graft_ctx *ctx, int batch, const int32_t *n_nodes,
                                 const int32_t *tokens, const int32_t *parents,
                                 const graft_target_logits *t, int32_t *acc_len,
                                 int32_t *acc_nodes, int32_t *bonus, float *logp,
                                 int update_history, void *workspace, hipStream_t stream) {
  const graft_dims &d = ctx->dims;
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
  a.parts = reinterpret_cast<Part *>(static_cast<char *>(workspace) + state_bytes(d, batch));
  a.error_flag = ctx->error_flag;
  a.batch = batch;
  a.L = d.num_pos;
  a.V = d.vocab;
  a.n_max = d.max_nodes;
  a.node_rows = t->node_rows;
  a.window = d.hist_window;
  a.update = update_history;
  a.splits = sample_splits(d, batch);
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
