// Sampled acceptance: softmax of logits, walk down the draft tree by random numbers.
#ifndef SV_SAMPLE_H
#define SV_SAMPLE_H

#include <type_traits>

#include "sv_frag.h"

namespace sv {

// ---- probabilities from logits -----------------------------------------------------------------

__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

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

// kPast: rows of more than 8192 columns are written past the caches (960 x 32000: 55.6 -> 42.7 us; with the loads past
// them as well 48.3).
template <bool kPast>
__device__ inline void store_prob(float* p, float v) {
  if constexpr (kPast) __builtin_nontemporal_store(v, p);
  else *p = v;
}

constexpr float kProbsUnit = 0x1p-24f;

// grid = (rows, 1 or shares of a row), block = NT.  A row of up to NT * K columns stays in registers, K of them per thread, and is read once;
// a longer one (K = 0) is read twice, first for a running maximum and the sum that goes with it.  Its quotients can be
// dealt to gridDim.y workgroups, each of which goes through the whole row for the sum (a CU fetches some 50 bytes a
// nanosecond: 3 rows of 128000 columns 25.3 us by one workgroup each, 14.8 by eight) - not in place, where one would
// overwrite what another has still to read.
// The exponent is (z - max) log2(e) / temperature, with the factor rounded once, the quotient a product with the sum's rounded
// reciprocal: 2^-24 of x more for an exponent x, half a step more for a quotient, than two divisions for each column.
// kUnits: logits are taken in units of 2^-24, for temperatures above 2^100, where a difference that float32 does not hold
// may be an exponent that it does.
template <int NT, int K, bool kUnits = false>
__global__ __launch_bounds__(NT) void token_probs_kernel(const float* z, int n, float c, float* p) {
  __shared__ float red[NT / 64];
  const float* src = z + (size_t)blockIdx.x * n;
  float* dst = p + (size_t)blockIdx.x * n;
  float m = -INFINITY, s = 0.f;
  bool nan = false;
  auto at = [&](int i) { return kUnits ? src[i] * kProbsUnit : src[i]; };
  if constexpr (K > 0) {
    float v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = at(min(k * NT + (int)threadIdx.x, n - 1));
#pragma unroll
    for (int k = 0; k < K; ++k) {
      nan |= v[k] != v[k];
      m = fmaxf(m, v[k]);
    }
    m = block_reduce<NT>(m, true, red);
    if (m == -INFINITY) m = 0.f;             // nothing but -infinity: every term is zero
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = exp2_of((v[k] - m) * c);
      s += k * NT + (int)threadIdx.x < n ? v[k] : 0.f;
    }
    s = block_reduce<NT>(nan ? NAN : s, false, red);
    const float r = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (k * NT + (int)threadIdx.x < n) store_prob<(K > 8)>(dst + k * NT + threadIdx.x, v[k] * r);
  } else {
    constexpr int kBatch = 16;
    float mine = -INFINITY;
    for (int i0 = 0; i0 < n; i0 += kBatch * NT) {
      float v[kBatch], top = mine;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) v[k] = at(min(i0 + k * NT + (int)threadIdx.x, n - 1));
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        nan |= v[k] != v[k];
        top = fmaxf(top, v[k]);
      }
      const float use = top == -INFINITY ? 0.f : top;
      s *= exp2_of((mine - use) * c);
      mine = top;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) s += i0 + k * NT + (int)threadIdx.x < n ? exp2_of((v[k] - use) * c) : 0.f;
    }
    m = block_reduce<NT>(mine, true, red);
    if (m == -INFINITY) m = 0.f;
    s = block_reduce<NT>(nan ? NAN : s * exp2_of((mine - m) * c), false, red);
    const float r = s == 0.f ? 0.f : 1.f / s;
    const int share = (n + (int)gridDim.y - 1) / (int)gridDim.y, begin = (int)blockIdx.y * share, end = min(n, begin + share);
    for (int i0 = begin; i0 < end; i0 += kBatch * NT) {
      float v[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) v[k] = at(min(i0 + k * NT + (int)threadIdx.x, end - 1));
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int i = i0 + k * NT + (int)threadIdx.x;
        if (i < end) store_prob<true>(dst + i, exp2_of((v[k] - m) * c) * r);
      }
    }
  }
}

// ---- sampled acceptance ------------------------------------------------------------------------
// One workgroup walks down one tree.  What the tests need of the nodes - parent, token, p and q of the
// token in the parent's row, random number - is fetched for all nodes at once; each wave then has all nodes in its
// registers, two a lane, and goes through the walk for itself: children are found by ballot, a child's numbers come
// by readlane, and the branches are uniform over the workgroup.  Only sums over whole rows (before a second
// sibling, and for the draw) read the rows.
// Sums are float64, in an order that the length of a row fixes: results are the same in every run.  They are not exact: p - less q is
// rounded from a node's second refusal on, and a sum where range and number of its terms take more than 29 bits together.
// They go from lane to lane by data-parallel primitives (through LDS, and with every wave adding up all waves' parts by
// itself, 16 trees over 4000 columns, about four children to a node, took 26.6 us, 11.6 this way, 9.7 with rows held).
// Bound for long rows by one CU per tree: chains of two nodes over 33000 - 256000 columns, of which p and q of one row are summed,
// take 9 us and the row's bytes, 42 a nanosecond from memory (128 chains: 5.3 TB/s together) or 53 (32 chains), 45 and 68 from the
// Infinity Cache; 128 over 128259 columns 33 us for 131 MB, where 20 would be the memory's time.  A tree over 256 columns,
// 5.3 us, is a chain of loads: tree, probabilities of the tokens, the last row.

struct SampleArgs {
  const int32_t* parent;
  const int32_t* token;
  const float *target, *draft;
  const float *u_accept, *u_draw;
  int T, n_vocab, lo, d_cap;
  uint8_t* accept_mask;
  int32_t *accepted_len, *best_node, *path, *out_tokens, *status;
};

// The value of another lane by data-parallel primitive, 0 from where there is none.
template <int kCtrl, int kRows>
__device__ inline double dpp_f64(double v) {
  const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
  const u32x2_t r = {(unsigned)__builtin_amdgcn_update_dpp(0, (int)w[0], kCtrl, kRows, 0xf, false),
                     (unsigned)__builtin_amdgcn_update_dpp(0, (int)w[1], kCtrl, kRows, 0xf, false)};
  return __builtin_bit_cast(double, r);
}
// Sums up to each lane: of the first 16 lanes, of all.
__device__ inline double row_scan_f64(double v) {
  v += dpp_f64<0x111, 0xf>(v);               // row_shr:1, 2, 4, 8
  v += dpp_f64<0x112, 0xf>(v);
  v += dpp_f64<0x114, 0xf>(v);
  return v + dpp_f64<0x118, 0xf>(v);
}
__device__ inline double wave_scan_f64(double v) {
  v = row_scan_f64(v);
  v += dpp_f64<0x142, 0xa>(v);               // row_bcast:15 to rows 1 and 3, row_bcast:31 to rows 2 and 3
  return v + dpp_f64<0x143, 0xc>(v);
}
__device__ inline double lane_f64(double v, int lane) {
  const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
  const u32x2_t r = {(unsigned)__builtin_amdgcn_readlane((int)w[0], lane), (unsigned)__builtin_amdgcn_readlane((int)w[1], lane)};
  return __builtin_bit_cast(double, r);
}

__device__ inline float mass_of(float p) { return fmaxf(p, 0.f); }       // (a NaN has none)

// What is left of a row: max(p - less q, 0), or p without the refused columns.
struct RestOfRow {
  const float *p, *q;
  double less;               // 0: q is not read
  const int* refused;        // LDS
  int n_refused;
};

// Of columns i, i + STEP, ..: kFull if all N lie before `end`, else what lies behind counts 0.
template <int N, int STEP, bool kQ, bool kFull>
__device__ inline void rest_at(const RestOfRow& row, int i, int end, double* v) {
  float p[N], q[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int at = kFull ? i + k * STEP : min(i + k * STEP, end - 1);
    p[k] = row.p[at];
    q[k] = kQ ? row.q[at] : 0.f;
  }
  for (int r = 0; r < row.n_refused; ++r) {
    const int x = row.refused[r];
#pragma unroll
    for (int k = 0; k < N; ++k) p[k] = i + k * STEP == x ? 0.f : p[k];
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = kQ ? fmax(fma(-row.less, (double)mass_of(q[k]), (double)p[k]), 0.0) : (double)mass_of(p[k]);
    if (!kFull) v[k] = i + k * STEP < end ? v[k] : 0.0;
  }
}

// A row that its workgroup holds from one sum to the next: a thread's columns of p in registers, those of q in LDS, which
// no other thread reads (both in registers spills).  16 trees of 60 drawn tokens over 1000 / 4000 / 16000 / 32000 columns, about
// three children to a node: 9.4 / 10.7 / 14.8 / 21.0 us with each sum from the caches, 7.7 / 9.3 / 13.4 / 18.1 this way;
// about four, which is more sums: 9.8 / 11.6 / 17.8 / 28.7 and 7.8 / 9.7 / 14.3 / 24.3.
template <int NT>
struct HeldRow {
  static constexpr int kColumns = NT == 64 ? 4 : (NT == 128 ? 8 : (NT == 256 ? 16 : 32));    // (each NT's longest row)
  static constexpr int kBatch = NT == 64 ? 4 : (NT <= 256 ? 8 : 16);
  float p[kColumns];
  // of a wave's columns first .. stop - 1, the sum of a lane's
  __device__ double sum(const RestOfRow& row, float* held_q, int first, int stop, bool fresh) {
    const int lane = threadIdx.x & 63;
    float* my_q = held_q + threadIdx.x;
    double s = 0.0;
#pragma unroll
    for (int b = 0; b < kColumns; b += kBatch) {
      if (first + 64 * b >= stop) continue;
      float q[kBatch];
      if (fresh) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const int i = first + lane + 64 * (b + k), at = min(i, stop - 1);
          p[b + k] = row.p[at];
          q[k] = row.q[at];
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const bool in = first + lane + 64 * (b + k) < stop;
          p[b + k] = in ? p[b + k] : 0.f;
          q[k] = in ? mass_of(q[k]) : 0.f;
          my_q[(b + k) * NT] = q[k];
        }
      } else {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) q[k] = my_q[(b + k) * NT];
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) s += fmax(fma(-row.less, (double)q[k], (double)p[b + k]), 0.0);
    }
    return s;
  }
};

// Sums over a row, and the column that a cumulated sum of `goal` falls on.  The columns are cut into one run
// per wave; the run that holds the goal is cut again, until a thread has kLeaf columns.
template <int NT>
struct RowSearch {
  static constexpr int kWaves = NT / 64, kLeaf = 4, kBatch = NT == 64 ? 4 : 8;
  double part[kWaves];       // LDS: sums of the runs
  int hit, last;

  template <bool kQ>
  __device__ static double lane_sum(const RestOfRow& row, int first, int stop) {
    const int lane = threadIdx.x & 63;
    double s = 0.0, v[kBatch];
    int i = first;
    for (; i + 64 * kBatch <= stop; i += 64 * kBatch) {
      rest_at<kBatch, 64, kQ, true>(row, i + lane, stop, v);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) s += v[k];
    }
    if (i < stop) {
      rest_at<kBatch, 64, kQ, false>(row, i + lane, stop, v);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) s += v[k];
    }
    return s;
  }
  __device__ void sums(const RestOfRow& row, int begin, int end, int run) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int first = begin + wave * run, stop = min(end, first + run);
    const double s = wave_scan_f64(row.less != 0.0 ? lane_sum<true>(row, first, stop) : lane_sum<false>(row, first, stop));
    publish(wave, s);
  }
  // the sum up to lane 63 of each wave -> part
  __device__ void publish(int wave, double upto) {
    __syncthreads();
    if ((threadIdx.x & 63) == 63) part[wave] = upto;
    __syncthreads();
  }
  __device__ static int run_of(int n) { return (n + kWaves - 1) / kWaves; }
  __device__ double my_part() const { return (threadIdx.x & 63) < kWaves ? part[threadIdx.x & 63] : 0.0; }
  // (leaves the runs' sums in part)
  __device__ double total(const RestOfRow& row, int n) {
    sums(row, 0, n, run_of(n));
    return lane_f64(row_scan_f64(my_part()), 15);
  }
  // The same of a row with q that the workgroup holds; fresh: it has to be fetched first.
  __device__ double total(const RestOfRow& row, int n, HeldRow<NT>& held, float* held_q, bool fresh) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), run = run_of(n);
    publish(wave, wave_scan_f64(held.sum(row, held_q, wave * run, min(n, wave * run + run), fresh)));
    return lane_f64(row_scan_f64(my_part()), 15);
  }
  // First column with mass at which the cumulated sum exceeds goal, the last one with mass if there is
  // none.  After total(row, n).
  __device__ int find(const RestOfRow& row, int n, double goal) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    int begin = 0, end = n;
    double before = 0.0;
    while (kWaves > 1 && end - begin > NT * kLeaf) {       // (one wave is for rows of up to 64 kLeaf columns: it could not cut them)
      const int run = run_of(end - begin);
      if (end - begin < n) sums(row, begin, end, run);
      const double mine = my_part(), upto = row_scan_f64(mine);
      const unsigned long long some = __builtin_amdgcn_ballot_w64(mine > 0.0), over = some & __builtin_amdgcn_ballot_w64(before + upto > goal);
      const int in = over ? __builtin_ctzll(over) : (some ? 63 - __builtin_clzll(some) : 0);
      if (in) before += lane_f64(upto, in - 1);
      begin += in * run;
      end = min(end, begin + run);
    }
    const int first = begin + kLeaf * (int)threadIdx.x;
    double v[kLeaf], mine = 0.0;
    if (row.less != 0.0) rest_at<kLeaf, 1, true, false>(row, first, end, v);
    else rest_at<kLeaf, 1, false, false>(row, first, end, v);
#pragma unroll
    for (int k = 0; k < kLeaf; ++k) mine += v[k];
    const double upto = wave_scan_f64(mine);
    if (threadIdx.x == 0) {
      hit = n;
      last = 0;
    }
    publish(wave, upto);
    const double waves = row_scan_f64(my_part());
    double cum = before + (wave ? lane_f64(waves, wave - 1) : 0.0) + (upto - mine);
    int my_hit = n, my_last = -1;
#pragma unroll
    for (int k = 0; k < kLeaf; ++k) {
      cum += v[k];
      const bool some = v[k] > 0.0;
      my_hit = (some & (cum > goal) & (my_hit == n)) ? first + k : my_hit;
      my_last = some ? first + k : my_last;
    }
    // (columns rise with the lanes)
    const unsigned long long hits = __builtin_amdgcn_ballot_w64(my_hit < n), lasts = __builtin_amdgcn_ballot_w64(my_last >= 0);
    if (hits && lane == __builtin_ctzll(hits)) atomicMin(&hit, my_hit);
    if (lasts && lane == 63 - __builtin_clzll(lasts)) atomicMax(&last, my_last);
    __syncthreads();
    return hit < n ? hit : last;
  }
};

// A number per node, two nodes a lane.
template <typename V>
struct Nodes {
  V lo, hi;
  __device__ Nodes(const V* of_all, int lane) : lo(of_all[lane]), hi(of_all[64 + lane]) {}
  __device__ V of(int c) const { return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, c < 64 ? lo : hi), c & 63)); }
};
struct NodeSet {
  unsigned long long lo, hi;
  __device__ bool has(int c) const { return (c < 64 ? lo : hi) >> (c & 63) & 1; }
  __device__ void add(int c) {
    const unsigned long long bit = 1ull << (c & 63);
    lo |= c < 64 ? bit : 0;
    hi |= c < 64 ? 0 : bit;
  }
  __device__ int take_first() {
    const bool low = lo != 0;
    const int c = low ? __builtin_ctzll(lo) : 64 + __builtin_ctzll(hi);
    hi = low ? hi : hi & (hi - 1);
    lo &= lo - 1;            // (0 stays 0)
    return c;
  }
};

template <int NT, bool kDrawn, bool kHeld>
__global__ __launch_bounds__(NT) void sampled_accept_kernel(const SampleArgs a) {
  __shared__ RowSearch<NT> search;
  __shared__ int s_parent[SV_MAX_TREE_NODES], s_col[SV_MAX_TREE_NODES], s_refused[SV_MAX_TREE_NODES];
  __shared__ float s_p[SV_MAX_TREE_NODES], s_q[SV_MAX_TREE_NODES], s_u[SV_MAX_TREE_NODES];
  __shared__ int s_path[SV_MAX_DEPTH + 1];
  __shared__ float s_held[kHeld ? NT * HeldRow<NT>::kColumns : 1];
  HeldRow<NT> held;
  int held_node = -1;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, T = a.T, n = a.n_vocab;
  const size_t base = (size_t)b * T;
  for (int c = tid; c < SV_MAX_TREE_NODES; c += NT) {
    int par = -1;
    if (c > 0 && c < T) {
      par = a.parent[base + c];
      const long long col = (long long)a.token[base + c] - a.lo;
      s_u[c] = a.u_accept[base + c];
      if (par >= c) par = -1;
      const bool in = par >= 0 && col >= 0 && col < n;
      s_col[c] = in ? (int)col : -1;
      s_p[c] = in ? mass_of(a.target[(base + par) * n + col]) : 0.f;
      s_q[c] = in && kDrawn ? mass_of(a.draft[(base + par) * n + col]) : 0.f;
    }
    s_parent[c] = par;
  }
  const double u_draw = a.u_draw[b];
  __syncthreads();
  const Nodes<int> par(s_parent, lane), cols(s_col, lane);
  const Nodes<float> ps(s_p, lane), qs(s_q, lane), us(s_u, lane);

  int node = 0, depth = 0;
  NodeSet taken{1, 0}, kids;
  double less = 0.0;
  RestOfRow row{a.target + base * n, kDrawn ? a.draft + base * n : nullptr, 0.0, s_refused, 0};
  for (;;) {
    kids = NodeSet{0, 0};
    if (depth < a.d_cap) kids = NodeSet{__builtin_amdgcn_ballot_w64(par.lo == node), __builtin_amdgcn_ballot_w64(par.hi == node)};
    NodeSet todo = kids;
    int next = -1;
    double mass = 1.0;
    bool stale = false;                      // mass is that of before the last refusal
    less = 0.0;
    while (todo.lo | todo.hi) {
      const int c = todo.take_first();
      double p = ps.of(c);
      const double u = us.of(c);
      bool take;
      if constexpr (kDrawn) {
        if (stale) {
          row.less = less;
          if constexpr (kHeld) mass = search.total(row, n, held, s_held, held_node != node);
          else mass = search.total(row, n);
          held_node = node;
        }
        const double q = qs.of(c), rest = fmax(fma(-less, q, p), 0.0);
        take = u * q * mass < rest;
        less += take ? 0.0 : mass;
        stale = true;
      } else {
        const int x = cols.of(c);
        // an earlier sibling of the same token has been refused
        if (__builtin_amdgcn_ballot_w64((par.lo == node && cols.lo == x && lane < c) || (par.hi == node && cols.hi == x && 64 + lane < c))) p = 0.0;
        take = u * mass < p;
        if (!take) mass = mass > p ? mass - p : 0.0;
      }
      if (take) {
        next = c;
        break;
      }
    }
    if (next < 0) break;
    node = next;
    ++depth;
    taken.add(node);
    if (tid == 0) s_path[depth] = node;
    row.p = a.target + (base + node) * n;
    if (kDrawn) row.q = a.draft + (base + node) * n;
  }

  // the draw: from what the refused children (all of the last node's) have left
  row.less = less;
  if constexpr (!kDrawn) {
    const unsigned long long before = (1ull << lane) - 1;
    if (tid < 64 && kids.lo >> lane & 1) s_refused[__builtin_popcountll(kids.lo & before)] = cols.lo;
    if (tid < 64 && kids.hi >> lane & 1) s_refused[__builtin_popcountll(kids.lo) + __builtin_popcountll(kids.hi & before)] = cols.hi;
    row.n_refused = __builtin_popcountll(kids.lo) + __builtin_popcountll(kids.hi);
  }
  __syncthreads();
  // (a row that nobody summed before is not needed again: nothing would be gained by holding it)
  double w = kHeld && held_node == node ? search.total(row, n, held, s_held, false) : search.total(row, n);
  int status = 0;
  if (!(w > 0.0)) {
    status = 1;
    row.less = 0.0;
    row.n_refused = 0;
    w = search.total(row, n);
    if (!(w > 0.0)) status = 3;
  }
  const int col = search.find(row, n, u_draw * w);
  for (int c = tid; c < T; c += NT) a.accept_mask[base + c] = taken.has(c);
  if (tid <= a.d_cap) {
    const size_t at = (size_t)b * (a.d_cap + 1) + tid;
    a.path[at] = tid == 0 ? 0 : (tid <= depth ? s_path[tid] : -1);
    a.out_tokens[at] = tid < depth ? s_col[s_path[tid + 1]] + a.lo : (tid > depth ? -1 : a.lo + (status == 3 ? 0 : col));
  }
  if (tid == 0) {
    a.accepted_len[b] = depth;
    a.best_node[b] = node;
    a.status[b] = status;
  }
}

}  // namespace sv
#endif
