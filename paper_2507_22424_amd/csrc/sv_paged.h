// Paged key-value cache: append of rotated keys, attention of one new token per sequence.
#ifndef SV_PAGED_H
#define SV_PAGED_H

#include "sv_frag.h"

namespace sv {

struct PagedCache {
  void *k, *v;
  const int32_t* table;      // [n_seqs][max_pages]
  int n_seqs, max_pages, n_pages, page_size, n_kv, d;
};

__device__ inline void store_row(float* p, float v) { *p = v; }
__device__ inline void store_row(bf16_t* p, float v) { p->bits = (uint16_t)pack_bf16x2(v, v); }

// ---- append ------------------------------------------------------------------------------------

struct AppendArgs {
  PagedCache c;
  const int32_t *seq, *pos;
  const float *q, *k, *v;
  long long q_stride, k_stride, v_stride;
  int n_q;
  double log2_theta;
  float* q_out;
  int32_t* status;
};

// grid = tokens, block = 256.  The rotation's angle is taken in turns and reduced in float64: at position 10^6 a
// float32 angle is off by 0.06.
template <typename T>
__global__ __launch_bounds__(256) void paged_append_kernel(const AppendArgs a) {
  __shared__ float s_cos[SV_MAX_PAGED_HEAD_DIM / 2], s_sin[SV_MAX_PAGED_HEAD_DIM / 2];
  const int t = blockIdx.x, tid = threadIdx.x, d = a.c.d, half = d / 2;
  const int seq = a.seq[t], pos = a.pos[t];
  int status = seq < 0 ? 1 : (seq >= a.c.n_seqs || pos < 0 || pos / a.c.page_size >= a.c.max_pages ? 2 : 0);
  int page = 0;
  if (status == 0) {
    page = a.c.table[(size_t)seq * a.c.max_pages + pos / a.c.page_size];
    if (page < 0 || page >= a.c.n_pages) status = 4;
  }
  if (a.status && tid == 0) a.status[t] = status;
  if (status) return;
  if (tid < half) {
    const double turns = (double)pos * exp2(-2.0 * tid / d * a.log2_theta) * 0.15915494309189533577;
    const float x = (float)(2.0 * (turns - rint(turns)));
    s_cos[tid] = cospif(x);
    s_sin[tid] = sinpif(x);
  }
  __syncthreads();
  const int row = pos % a.c.page_size;
  const float *q = a.q + t * a.q_stride, *k = a.k + t * a.k_stride, *v = a.v + t * a.v_stride;
  for (int i = tid; i < (a.n_q + a.c.n_kv) * half; i += 256) {
    const int h = i / half, e = i - h * half;
    const bool is_q = h < a.n_q;
    const float* src = is_q ? q + h * d : k + (h - a.n_q) * d;
    const float x = src[e], y = src[e + half], c = s_cos[e], s = s_sin[e];
    const float x2 = x * c - y * s, y2 = y * c + x * s;
    if (is_q) {
      float* dst = a.q_out + ((size_t)t * a.n_q + h) * d;
      dst[e] = x2;
      dst[e + half] = y2;
    } else {
      T* dst = (T*)a.c.k + (((size_t)page * a.c.n_kv + h - a.n_q) * a.c.page_size + row) * d;
      store_row(dst + e, x2);
      store_row(dst + e + half, y2);
    }
  }
  for (int i = tid; i < a.c.n_kv * d; i += 256) {
    const int h = i / d, e = i - h * d;
    store_row((T*)a.c.v + (((size_t)page * a.c.n_kv + h) * a.c.page_size + row) * d + e, v[i]);
  }
}

// ---- attention ---------------------------------------------------------------------------------

struct PagedAttnArgs {
  PagedCache c;
  const int32_t* seq_len;
  int max_len, n_q, window, n_sink;
  float scale;
  const float* q;
  float *out, *lse;
  int32_t* status;
};

// grid = (query heads, sequences), block = 256: four waves take the visible rows in turn, a lane holds up to four
// columns; running maximum and sum per wave, joined through LDS.
template <typename T>
__global__ __launch_bounds__(256) void paged_attention_rows(const PagedAttnArgs a) {
  __shared__ float s_m[4], s_l[4], s_o[4][SV_MAX_PAGED_HEAD_DIM];
  __shared__ int s_bad;
  const int h = blockIdx.x, s = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, d = a.c.d;
  const int hk = h / (a.n_q / a.c.n_kv);
  int len = a.seq_len[s];
  len = len < 0 ? 0 : (len > a.max_len ? a.max_len : len);
  int n_sink = 0, first = 0;                 // visible: 0 .. n_sink - 1 and first .. len - 1
  if (a.window > 0 && len > a.window) {
    first = len - a.window;
    n_sink = min(a.n_sink, first);
  }
  const int n_seen = n_sink + len - first;
  const size_t qrow = ((size_t)s * a.n_q + h) * d;
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) q[e] = e * 64 + lane < d ? a.q[qrow + e * 64 + lane] * a.scale : 0.f;
  for (int i = wave; i < n_seen; i += 4) {
    const int j = i < n_sink ? i : first + (i - n_sink);
    const int page = a.c.table[(size_t)s * a.c.max_pages + j / a.c.page_size];
    if (page < 0 || page >= a.c.n_pages) {
      if (lane == 0) s_bad = 1;
      continue;
    }
    const size_t at = (((size_t)page * a.c.n_kv + hk) * a.c.page_size + j % a.c.page_size) * d;
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e * 64 + lane < d) x += q[e] * to_f32(((const T*)a.c.k)[at + e * 64 + lane]);
    x = wave_sum(x);
    const float m2 = fmaxf(m, x), f = m2 == -INFINITY ? 1.f : expf(m - m2), w = m2 == -INFINITY ? 0.f : expf(x - m2);
    m = m2;
    l = l * f + w;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e * 64 + lane < d) o[e] = o[e] * f + w * to_f32(((const T*)a.c.v)[at + e * 64 + lane]);
  }
  if (lane == 0) {
    s_m[wave] = m;
    s_l[wave] = l;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) s_o[wave][e * 64 + lane] = o[e];
  __syncthreads();
  float m_all = -INFINITY, l_all = 0.f, v = 0.f;
  for (int w = 0; w < 4; ++w) m_all = fmaxf(m_all, s_m[w]);
  for (int w = 0; w < 4; ++w) {
    const float f = s_m[w] == -INFINITY ? 0.f : expf(s_m[w] - m_all);
    l_all += f * s_l[w];
    v += f * s_o[w][threadIdx.x];
  }
  if ((int)threadIdx.x < d) a.out[qrow + threadIdx.x] = l_all > 0.f ? v / l_all : (l_all == 0.f ? 0.f : l_all);
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[(size_t)s * a.n_q + h] = l_all == 0.f ? -INFINITY : m_all + logf(l_all);
    if (a.status && h == 0) a.status[s] = s_bad;
  }
}

}  // namespace sv
#endif
