// Sampled acceptance: softmax of logits, walk down the draft tree by random numbers.
#ifndef SV_SAMPLE_H
#define SV_SAMPLE_H

#include "sv_frag.h"

namespace sv {

// ---- probabilities from logits -----------------------------------------------------------------

template <int NT>
__device__ inline float block_reduce(float v, bool maximum, float* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const float o = __shfl_xor(v, off, kWave);
    v = maximum ? fmaxf(v, o) : v + o;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v = maximum ? fmaxf(v, red[w]) : v + red[w];
  return v;
}

// grid = rows, block = NT: maximum, sum, quotients, a pass over the row each.
template <int NT>
__global__ __launch_bounds__(NT) void token_probs_kernel(const float* z, int n, float inv_t, float* p) {
  __shared__ float red[NT / 64];
  const float* src = z + (size_t)blockIdx.x * n;
  float* dst = p + (size_t)blockIdx.x * n;
  float m = -INFINITY;
  bool nan = false;
  for (int i = threadIdx.x; i < n; i += NT) {
    const float v = src[i];
    nan |= v != v;
    m = fmaxf(m, v);
  }
  m = block_reduce<NT>(m, true, red);
  if (m == -INFINITY) m = 0.f;               // nothing but -infinity: every term is zero
  float s = 0.f;
  for (int i = threadIdx.x; i < n; i += NT) s += expf((src[i] - m) * inv_t);
  s = block_reduce<NT>(nan ? NAN : s, false, red);
  const float r = s == 0.f ? 0.f : 1.f / s;
  for (int i = threadIdx.x; i < n; i += NT) dst[i] = expf((src[i] - m) * inv_t) * r;
}

// ---- sampled acceptance ------------------------------------------------------------------------
// One workgroup walks down one tree.  What the tests need of the nodes - parent, token, p and q of the
// token in the parent's row, random number - is fetched for all nodes at once; the walk itself is
// scalar work on LDS values that every wave repeats for itself, so that its branches are uniform over the
// workgroup.  Only sums over whole rows (a second sibling, the final draw) read the rows.
// Sums are float64: the inputs are float32, so that a sum is exact unless its terms span more
// than 2^29, and the choice of a token does not hang on the order of the summation.

struct SampleArgs {
  const int32_t* parent;
  const int32_t* token;
  const float *target, *draft;
  const float *u_accept, *u_draw;
  int T, n_vocab, lo, d_cap;
  uint8_t* accept_mask;
  int32_t *accepted_len, *best_node, *path, *out_tokens, *status;
};

__device__ inline double wave_sum_f64(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  return v;
}

__device__ inline float mass_of(float p) { return p > 0.f ? p : 0.f; }       // (a NaN has none)

// What is left of a row: the part of column i that a draw can still hit.
struct RestOfRow {
  const float *p, *q;        // q: NULL where the children were chosen
  double less;
  const int* refused;        // LDS: columns that do not count
  int n_refused;
  __device__ double at(int i) const {
    const double v = (double)p[i] - (q ? less * (double)mass_of(q[i]) : 0.0);
    if (!(v > 0.0)) return 0.0;                    // (a NaN too)
    for (int r = 0; r < n_refused; ++r)
      if (refused[r] == i) return 0.0;
    return v;
  }
};

// Sums over a row, and the column that a cumulated sum of `goal` falls on.  The columns are cut into one run
// per wave; the run that holds the goal is cut again, until a thread has kLeaf columns.
template <int NT>
struct RowSearch {
  static constexpr int kWaves = NT / 64, kLeaf = 4;
  double part[kWaves];       // LDS: sums of the runs
  int hit, last;

  __device__ void sums(const RestOfRow& row, int begin, int end, int run) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int first = begin + wave * run, stop = min(end, first + run);
    double s = 0.0;
    for (int i = first + lane; i < stop; i += 64) s += row.at(i);
    s = wave_sum_f64(s);
    __syncthreads();
    if (lane == 0) part[wave] = s;
    __syncthreads();
  }
  __device__ static int run_of(int n) { return (n + kWaves - 1) / kWaves; }
  // (leaves the runs' sums in part)
  __device__ double total(const RestOfRow& row, int n) {
    sums(row, 0, n, run_of(n));
    double s = 0.0;
    for (int w = 0; w < kWaves; ++w) s += part[w];
    return s;
  }
  // First column with mass at which the cumulated sum exceeds goal, the last one with mass if there is
  // none.  After total(row, n).
  __device__ int find(const RestOfRow& row, int n, double goal) {
    int begin = 0, end = n;
    double before = 0.0;
    while (end - begin > NT * kLeaf) {
      const int run = run_of(end - begin);
      if (end - begin < n) sums(row, begin, end, run);
      int in = 0;
      double cum = before, at = before;
      for (int w = 0; w < kWaves; ++w) {
        if (part[w] > 0.0) {
          in = w;
          at = cum;
          if (cum + part[w] > goal) break;
        }
        cum += part[w];
      }
      before = at;
      begin += in * run;
      end = min(end, begin + run);
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first = begin + kLeaf * (int)threadIdx.x;
    double v[kLeaf], mine = 0.0;
#pragma unroll
    for (int k = 0; k < kLeaf; ++k) {
      v[k] = first + k < end ? row.at(first + k) : 0.0;
      mine += v[k];
    }
    double upto = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const double o = __shfl_up(upto, off, kWave);
      if (lane >= off) upto += o;
    }
    __syncthreads();
    if (lane == 63) part[wave] = upto;
    if (threadIdx.x == 0) {
      hit = n;
      last = 0;
    }
    __syncthreads();
    double cum = before + (upto - mine);
    for (int w = 0; w < wave; ++w) cum += part[w];
#pragma unroll
    for (int k = 0; k < kLeaf; ++k) {
      if (!(v[k] > 0.0)) continue;
      cum += v[k];
      if (cum > goal) atomicMin(&hit, first + k);
      atomicMax(&last, first + k);
    }
    __syncthreads();
    return hit < n ? hit : last;
  }
};

template <int NT>
__global__ __launch_bounds__(NT) void sampled_accept_kernel(const SampleArgs a) {
  __shared__ RowSearch<NT> search;
  __shared__ int s_parent[SV_MAX_TREE_NODES], s_col[SV_MAX_TREE_NODES], s_refused[SV_MAX_TREE_NODES];
  __shared__ float s_p[SV_MAX_TREE_NODES], s_q[SV_MAX_TREE_NODES], s_u[SV_MAX_TREE_NODES];
  const int b = blockIdx.x, tid = threadIdx.x, T = a.T, n = a.n_vocab;
  const size_t base = (size_t)b * T;
  int32_t* path = a.path + (size_t)b * (a.d_cap + 1);
  int32_t* out = a.out_tokens + (size_t)b * (a.d_cap + 1);
  for (int c = tid; c < T; c += NT) {
    int par = c ? a.parent[base + c] : -1;
    if (par >= c) par = -1;
    const long long col = (long long)a.token[base + c] - a.lo;
    const bool in = par >= 0 && col >= 0 && col < n;
    s_parent[c] = par;
    s_col[c] = in ? (int)col : -1;
    s_u[c] = a.u_accept[base + c];
    s_p[c] = in ? mass_of(a.target[(base + par) * n + col]) : 0.f;
    s_q[c] = in && a.draft ? mass_of(a.draft[(base + par) * n + col]) : 0.f;
    a.accept_mask[base + c] = c == 0;
  }
  for (int i = tid; i <= a.d_cap; i += NT) {
    path[i] = i ? -1 : 0;
    out[i] = -1;
  }
  __syncthreads();

  int node = 0, depth = 0, n_refused = 0;
  double less = 0.0, mass = 1.0;
  bool stale = false;                        // mass is that of before the last refusal
  RestOfRow row{a.target + base * n, a.draft ? a.draft + base * n : nullptr, 0.0, s_refused, 0};
  if (depth < a.d_cap)
    for (int c = 1; c < T; ++c) {
      if (s_parent[c] != node) continue;
      const int x = s_col[c];
      double p = s_p[c];
      bool take;
      if (a.draft) {
        if (stale) mass = search.total(row, n);
        stale = false;
        double left = p - less * (double)s_q[c];
        left = left > 0.0 ? left : 0.0;
        take = (double)s_u[c] * (double)s_q[c] * mass < left;
        if (!take) {
          less += mass;
          stale = true;
          row.less = less;
        }
      } else {
        for (int r = 0; r < n_refused; ++r)
          if (s_refused[r] == x) p = 0.0;
        take = (double)s_u[c] * mass < p;
        if (!take) {
          if (p > 0.0) mass = mass > p ? mass - p : 0.0;
          __syncthreads();
          if (tid == 0) s_refused[n_refused] = x;
          __syncthreads();
          ++n_refused;
        }
      }
      if (!take) continue;
      node = c;
      ++depth;
      less = 0.0; mass = 1.0; stale = false; n_refused = 0;
      row.p = a.target + (base + c) * n;
      row.q = a.draft ? a.draft + (base + c) * n : nullptr;
      row.less = 0.0;
      if (tid == 0) {
        a.accept_mask[base + c] = 1;
        path[depth] = c;
        out[depth - 1] = x + a.lo;
      }
      if (depth >= a.d_cap) break;
    }
  __syncthreads();

  // the draw
  row.n_refused = n_refused;
  double w = search.total(row, n);
  int status = 0;
  if (!(w > 0.0)) {
    status = 1;
    row.q = nullptr;
    row.n_refused = 0;
    w = search.total(row, n);
    if (!(w > 0.0)) status = 3;
  }
  const int col = search.find(row, n, (double)a.u_draw[b] * w);
  if (tid == 0) {
    a.accepted_len[b] = depth;
    a.best_node[b] = node;
    out[depth] = a.lo + (status == 3 ? 0 : col);
    a.status[b] = status;
  }
}

}  // namespace sv
#endif
