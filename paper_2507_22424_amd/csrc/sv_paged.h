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

__device__ inline void store4(float* p, f32x4_t v) { *(f32x4_t*)p = v; }
__device__ inline void store4(bf16_t* p, f32x4_t v) { *(uint2*)p = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])); }

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
// float32 angle is off by 0.06.  A thread turns four pairs of a head; the values, which need no angle, go first.
template <typename T>
__global__ __launch_bounds__(256) void paged_append_kernel(const AppendArgs a) {
  __shared__ __attribute__((aligned(16))) float s_cos[SV_MAX_PAGED_HEAD_DIM / 2], s_sin[SV_MAX_PAGED_HEAD_DIM / 2];
  const int t = blockIdx.x, tid = threadIdx.x, d = a.c.d, half = d / 2, quads = half / 4;
  const int seq = a.seq[t], pos = a.pos[t], in_seq = pos / a.c.page_size;
  int status = seq < 0 ? 1 : (seq >= a.c.n_seqs || pos < 0 || in_seq >= a.c.max_pages ? 2 : 0);
  int page = 0;
  if (status == 0) {
    page = a.c.table[(size_t)seq * a.c.max_pages + in_seq];
    if (page < 0 || page >= a.c.n_pages) status = 4;
  }
  if (a.status && tid == 0) a.status[t] = status;
  if (status) return;
  const size_t row0 = (size_t)page * a.c.n_kv * a.c.page_size + (pos - in_seq * a.c.page_size);     // of KV head 0
  const float *q = a.q + t * a.q_stride, *k = a.k + t * a.k_stride, *v = a.v + t * a.v_stride;
  for (int i = tid; i < a.c.n_kv * 2 * quads; i += 256) {
    const int h = i / (2 * quads), e = (i - h * 2 * quads) * 4;
    store4((T*)a.c.v + (row0 + (size_t)h * a.c.page_size) * d + e, *(const f32x4_t*)(v + 4 * i));
  }
  if (tid < half) {
    const double turns = (double)pos * exp2(-2.0 * tid / d * a.log2_theta) * 0.15915494309189533577;
    const float x = (float)(2.0 * (turns - rint(turns)));
    s_cos[tid] = cospif(x);
    s_sin[tid] = sinpif(x);
  }
  __syncthreads();
  for (int i = tid; i < (a.n_q + a.c.n_kv) * quads; i += 256) {
    const int h = i / quads, e = (i - h * quads) * 4;
    const bool is_q = h < a.n_q;
    const float* src = (is_q ? q + h * d : k + (h - a.n_q) * d) + e;
    const f32x4_t x = *(const f32x4_t*)src, y = *(const f32x4_t*)(src + half);
    const f32x4_t c = *(const f32x4_t*)(s_cos + e), s = *(const f32x4_t*)(s_sin + e);
    const f32x4_t x2 = x * c - y * s, y2 = y * c + x * s;
    if (is_q) {
      float* dst = a.q_out + ((size_t)t * a.n_q + h) * d + e;
      store4(dst, x2);
      store4(dst + half, y2);
    } else {
      T* dst = (T*)a.c.k + (row0 + (size_t)(h - a.n_q) * a.c.page_size) * d + e;
      store4(dst, x2);
      store4(dst + half, y2);
    }
  }
}

// ---- attention ---------------------------------------------------------------------------------
// Everything is computed transposed, S^T = K Q^T and O^T = V^T P^T, on matrix instructions whose 16 columns are
// the query heads of one KV head.  A lane holds one query column c = lane % 16 and, of a unit of 16 keys,
// the scores of keys 4g .. 4g+3 (g = lane / 16), which are the weights that the second product wants of it: nothing
// moves between lanes.  Of V a lane takes the rows of its own four keys, 16 bytes each, and a register of the V^T operand
// is two halves of registers that it holds already; K rows become operands through LDS, which also holds the queries
// and joins the waves.  Units are 16 rows of a page at a multiple of 16, so that a unit lies in one page.
//
// Bound by the cache's rows from memory.  A wave has the next tile's K under way while it works on a tile, and the next V
// from its end on; three workgroups of four waves, or two of six, share a CU (head_dim 128: 167 registers).  64 sequences of 17 - 8192
// tokens, 32 query and 8 KV heads of 128, bf16: 181 us for 1.08 GB, 5.9 TB/s (a plain streaming read: 6.7); one
// of 131071: 89 us for 537 MB, 6.0 TB/s.  With little to read it is the chain of loads: 281 tokens, 32 heads,
// 7.3 us, of which an empty kernel takes 2.0, the first tile with all that it waits for 3.3, the second 1.6.
// 32-bit sums: queries and weights enter the bf16 products in three parts, which is all of their 24 bits.

struct PagedAttnArgs {
  PagedCache c;
  const int32_t* seq_len;
  int max_len, n_q, window, n_sink;
  int n_blocks;              // blocks of 16 query heads per KV head
  int n_split, split_units;  // workgroups that share a sequence's units, units of each (a multiple of 2)
  float scale;               // with log2(e)
  const float* q;
  float *out, *lse;
  int32_t* status;
  float *part, *part_ml;     // [rows][n_split][d], [rows][n_split][2]
};

// Units of 16 rows that hold a visible row: those of the first rows, then those of the window.
struct VisibleRows {
  int len, first, n_sink;    // visible: 0 .. n_sink - 1 and first .. len - 1
  int sink_units, main_unit, n_units;
  __host__ __device__ VisibleRows(int length, int max_len, int window, int sinks) {
    len = length < 0 ? 0 : (length > max_len ? max_len : length);
    first = n_sink = 0;
    if (window > 0 && len > window) {
      first = len - window;
      n_sink = sinks < first ? sinks : first;
    }
    sink_units = (n_sink + 15) / 16;
    main_unit = first / 16 > sink_units ? first / 16 : sink_units;
    const int end = (len + 15) / 16;
    n_units = sink_units + (end > main_unit ? end - main_unit : 0);
  }
  __device__ int unit(int u) const { return u < sink_units ? u : u - sink_units + main_unit; }
  __device__ bool full(int unit) const {
    return unit * 16 + 16 <= len && (unit * 16 >= first || unit * 16 + 16 <= n_sink);
  }
  // (joined bit by bit: with && and || each of a tile's rows takes a branch of its own)
  __device__ bool sees(int j) const { return (j < len) & ((j >= first) | (j < n_sink)); }
};

__device__ inline f32x4_t mfma_bf16(uint4 a, uint4 b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// x = hi + mid + lo, bf16 each (24 bits: x itself, but for what lies below 2^-24 of it)
__device__ inline void split8_3(const float* v, uint4* part) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = v[e];
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = pack_bf16x2(r[2 * e], r[2 * e + 1]);
      r[2 * e] -= bf16_lo_f32(w[e]);
      r[2 * e + 1] -= bf16_hi_f32(w[e]);
    }
    part[p] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A load of the cache; NT: past the caches.
template <int NT, typename V>
__device__ inline V load_row(const char* p) {
  typedef unsigned words_t __attribute__((ext_vector_type(sizeof(V) / 4)));
  const auto src = (const __attribute__((address_space(1))) words_t*)p;
  if constexpr (NT) return __builtin_bit_cast(V, __builtin_nontemporal_load(src));
  else return __builtin_bit_cast(V, *src);
}

// The K rows of a tile on their way from the cache to the operand: fetched with the 16 bytes of neighbouring lanes next to
// each other, and turned by LDS into a row per lane.  (Fetched as operands, 16 neighbouring lanes touch 16 rows, and the
// cache in front of the L2 looks up 64 lines for an instruction: 64 sequences of up to 8192 tokens 199 us, 189 this way, 40
// query heads to a KV head 73 and 60.)  In LDS the 16-byte pieces of row r change places by an
// exclusive or with r, so that 16 lanes that read the same piece of 16 rows hit different banks.
template <int kUnits, int kRowBytes, int NT>
struct PagedKeys {
  static constexpr int kPieces = kRowBytes / 16, kLoads = kPieces / 4, kMask = (kPieces < 16 ? kPieces : 16) - 1;
  u32x4_t r[kUnits][kLoads];
  // row_bytes: of a row in the cache (pieces behind it: its last one again)
  __device__ void load(int u, const char* base, int row_bytes, int lane) {
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const int i = n * 64 + lane;
      r[u][n] = load_row<NT, u32x4_t>(base + (unsigned)(i / kPieces * row_bytes + min(i % kPieces * 16, row_bytes - 16)));
    }
  }
  __device__ void stage(u32x4_t* lds, int lane) const {
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int n = 0; n < kLoads; ++n) {
        const int i = n * 64 + lane, row = i / kPieces;
        lds[u * 16 * kPieces + row * kPieces + ((i % kPieces) ^ (row & kMask))] = r[u][n];
      }
  }
  static __device__ u32x4_t piece(const u32x4_t* lds, int u, int c, int i) { return lds[u * 16 * kPieces + c * kPieces + (i ^ (c & kMask))]; }
};

// A tile of the cache in registers and its two products.  DP: head_dim rounded up to 64, 128 or 256 (columns
// behind head_dim: q is zero, K and V repeat columns of the row, and the outputs are not stored).
template <typename T, int DP, int NT>
struct PagedTile;

template <int DP, int NT>
struct PagedTile<bf16_t, DP, NT> {
  static constexpr int kUnits = 2, kSteps = DP / 32, kOut = DP / 16;
  static constexpr int kE = DP / 16 < 8 ? DP / 16 : 8, kLoads = DP / 16 / kE;    // V: elements of a load, loads of a row
  static constexpr int kScores = 8;
  typedef PagedKeys<kUnits, DP * 2, NT> Keys;
  Keys k;
  uint32_t v[8][kE / 2 * kLoads];
  typedef uint4 QPart;
  static constexpr int kParts = 3;           // of the query operand of a step

  static __device__ int out_col(int t, int m) { return t / kE * 16 * kE + kE * m + t % kE; }
  static __device__ void load_q(int s, const float* src, bool real, float scale, int d, int g, QPart* part) {
    // (loaded whether wanted or not: a load under a condition is waited for before the next)
    const int col = 32 * s + 8 * g;
    const f32x4_t* at = (const f32x4_t*)(src + min(col, d - 8));
    const f32x4_t a = at[0], b = at[1];
    const bool want = real & (col < d);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = want ? (e < 4 ? a[e & 3] : b[e & 3]) * scale : 0.f;
    split8_3(x, part);
  }
  __device__ void load_v(int u, const char* base, int d, int g, int c) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int l = 0; l < kLoads; ++l) {
        const char* p = base + (unsigned)((4 * g + r) * d + min(128 * l + kE * c, d - kE)) * 2u;
        uint32_t* dst = v[4 * u + r] + l * (kE / 2);
        if constexpr (kE == 8) {
          const uint4 w = load_row<NT, uint4>(p);
          dst[0] = w.x; dst[1] = w.y; dst[2] = w.z; dst[3] = w.w;
        } else {
          const uint2 w = load_row<NT, uint2>(p);
          dst[0] = w.x; dst[1] = w.y;
        }
      }
  }
  __device__ void keep_v(int e, bool seen) {
#pragma unroll
    for (int w = 0; w < kE / 2 * kLoads; ++w) v[e][w] = seen ? v[e][w] : 0;
  }
  // q, keys: LDS, q as [part][64 lanes]
  static __device__ void scores(const QPart (*q)[64], const u32x4_t* keys, int lane, int g, int c, float* x) {
    f32x4_t s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const uint4 k0 = __builtin_bit_cast(uint4, Keys::piece(keys, 0, c, 4 * i + g)), k1 = __builtin_bit_cast(uint4, Keys::piece(keys, 1, c, 4 * i + g));
#pragma unroll
      for (int p = 2; p >= 0; --p) {
        const uint4 w = q[3 * i + p][lane];
        s[0] = mfma_bf16(k0, w, s[0]);
        s[1] = mfma_bf16(k1, w, s[1]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = s[e / 4][e % 4];
  }
  __device__ void add(const float* p, f32x4_t* o) const {
    uint4 w[3];
    split8_3(p, w);
#pragma unroll
    for (int t = 0; t < kOut; ++t) {
      const unsigned sel = t & 1 ? 0x07060302u : 0x05040100u;
      uint4 a;
      a.x = __builtin_amdgcn_perm(v[1][t / 2], v[0][t / 2], sel);
      a.y = __builtin_amdgcn_perm(v[3][t / 2], v[2][t / 2], sel);
      a.z = __builtin_amdgcn_perm(v[5][t / 2], v[4][t / 2], sel);
      a.w = __builtin_amdgcn_perm(v[7][t / 2], v[6][t / 2], sel);
#pragma unroll
      for (int i = 2; i >= 0; --i) o[t] = mfma_bf16(a, w[i], o[t]);
    }
  }
};

template <int DP, int NT>
struct PagedTile<float, DP, NT> {
  static constexpr int kUnits = 1, kSteps = DP / 16, kOut = DP / 16;
  static constexpr int kScores = 4;
  typedef PagedKeys<kUnits, DP * 4, NT> Keys;
  Keys k;
  f32x4_t v[4][DP / 64];
  typedef f32x4_t QPart;
  static constexpr int kParts = 1;

  static __device__ int out_col(int t, int m) { return t / 4 * 64 + 4 * m + t % 4; }
  static __device__ void load_q(int s, const float* src, bool real, float scale, int d, int g, QPart* part) {
    const int col = 16 * s + 4 * g;
    const f32x4_t a = *(const f32x4_t*)(src + min(col, d - 4));
    const bool want = real & (col < d);
#pragma unroll
    for (int e = 0; e < 4; ++e) part[0][e] = want ? a[e] * scale : 0.f;
  }
  __device__ void load_v(int, const char* base, int d, int g, int c) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int l = 0; l < DP / 64; ++l)
        v[r][l] = load_row<NT, f32x4_t>(base + (unsigned)((4 * g + r) * d + min(64 * l + 4 * c, d - 4)) * 4u);
  }
  __device__ void keep_v(int e, bool seen) {
#pragma unroll
    for (int l = 0; l < DP / 64; ++l)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[e][l][i] = seen ? v[e][l][i] : 0.f;
  }
  static __device__ void scores(const QPart (*q)[64], const u32x4_t* keys, int lane, int g, int c, float* x) {
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const f32x4_t k0 = __builtin_bit_cast(f32x4_t, Keys::piece(keys, 0, c, 4 * i + g)), w = q[i][lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k0[e], w[e], s, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = s[r];
  }
  __device__ void add(const float* p, f32x4_t* o) const {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < kOut; ++t) o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][t / 4][t % 4], p[r], o[t], 0, 0, 0);
  }
};

// One workgroup = (sequence, KV head, block of 16 query heads, split); its waves (NW) take tiles in turn.  A lane of a
// wave looks up the page of one of the wave's units, all of them before the first is needed: a split has at most
// kBatchUnits of them per wave.  grid.x = sequences * KV heads * splits, rounded up to a multiple of 8, * blocks.
constexpr int kBatchUnits = 64, kPagedWaves = 4;
template <typename T, int DP, int NT, int NW>
__global__ __launch_bounds__(64 * NW, DP == 256 ? 1 : (DP == 128 && sizeof(T) == 4 ? 2 : 3)) void paged_attention_mfma(const PagedAttnArgs a) {
  using Tile = PagedTile<T, DP, NT>;
  constexpr int kU = Tile::kUnits, kPitch = DP + 4;
  __shared__ float s_m[NW][16], s_l[NW][16];
  // a wave's keys, and in their place its outputs when they are done with
  constexpr size_t kKeyBytes = (size_t)kU * 16 * DP * sizeof(T), kOutBytes = sizeof(float) * 16 * kPitch, kWaveBytes = kKeyBytes > kOutBytes ? kKeyBytes : kOutBytes;
  __shared__ __attribute__((aligned(16))) unsigned char s_raw[NW][kWaveBytes];
  auto s_o = [&](int w) { return reinterpret_cast<float (*)[kPitch]>(s_raw[w]); };
  __shared__ typename Tile::QPart s_q[Tile::kSteps * Tile::kParts][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 4, c = lane & 15, d = a.c.d;
  // Workgroups go to the XCDs in turn.  A layer of them, one per sequence and KV head, takes the same split of all; a layer
  // begins an odd number of XCDs behind the one before, so that the splits of a sequence go round them all.  The last
  // splits, which only long sequences have, come first.  The blocks of a KV head's queries, which read the same
  // rows, go to one XCD, one right after the other.
  const unsigned octet = blockIdx.x / (8 * a.n_blocks), in_octet = blockIdx.x % (8 * a.n_blocks), n_tasks = a.c.n_seqs * a.c.n_kv;
  const int hb = in_octet / 8;
  const unsigned id = octet * 8 + in_octet % 8, layer = id / n_tasks;
  const unsigned task = (id - layer * n_tasks + (n_tasks & 1 ? 0 : layer)) % n_tasks;
  const int split = a.n_split - 1 - (int)layer, seq = task / a.c.n_kv, hk = task - seq * a.c.n_kv;
  if (split < 0) return;                     // (the tasks are rounded up to a multiple of 8)
  const int u_begin = split * a.split_units, u_wave = u_begin + wave * kU;
  const int G = a.n_q / a.c.n_kv, n_heads = min(16, G - 16 * hb);
  const size_t row0 = (size_t)seq * a.n_q + hk * G + 16 * hb;

  // The first loads - length, pages of the units, queries - do not wait for each other: without a window the units
  // are known before the length is (pages of units behind it are looked up too, and not used).
  const VisibleRows rows(a.seq_len[seq], a.max_len, a.window, a.n_sink);
  const int my_unit = u_wave + lane / kU * (NW * kU) + lane % kU;
  const int my_at = a.window ? rows.unit(my_unit) : my_unit, page_units = a.c.page_size / 16, my_page = my_at / page_units;
  const int page = a.c.table[(size_t)seq * a.c.max_pages + min(my_page, a.c.max_pages - 1)];
  const bool in_pool = (unsigned)page < (unsigned)a.c.n_pages;
  const long long my_off = in_pool ? (((long long)page * a.c.n_kv + hk) * a.c.page_size + (my_at - my_page * page_units) * 16) * d * (int)sizeof(T) : 0;
  Tile tile;
  typename Tile::QPart part[Tile::kSteps / NW + 1][Tile::kParts];
#pragma unroll
  for (int s = 0; s * NW < Tile::kSteps; ++s)
    if (s * NW + wave < Tile::kSteps)
      Tile::load_q(s * NW + wave, a.q + (row0 + min(c, n_heads - 1)) * d, c < n_heads, a.scale, d, g, part[s]);
  const unsigned long long pool_units = __builtin_amdgcn_ballot_w64(in_pool);
  auto offset = [&](int i) {                 // bytes of the wave's i-th unit
    return (size_t)(unsigned)__builtin_amdgcn_readlane((int)my_off, i) | (size_t)__builtin_amdgcn_readlane((int)(my_off >> 32), i) << 32;
  };
  auto load_k = [&](int it) {
#pragma unroll
    for (int u = 0; u < kU; ++u) tile.k.load(u, (const char*)a.c.k + offset(it * kU + u), d * (int)sizeof(T), lane);
  };
  auto load_v = [&](int it) {
#pragma unroll
    for (int u = 0; u < kU; ++u) tile.load_v(u, (const char*)a.c.v + offset(it * kU + u), d, g, c);
  };
  load_k(0);
  load_v(0);

#pragma unroll
  for (int s = 0; s * NW < Tile::kSteps; ++s)
    if (s * NW + wave < Tile::kSteps)
#pragma unroll
      for (int p = 0; p < Tile::kParts; ++p) s_q[(s * NW + wave) * Tile::kParts + p][lane] = part[s][p];
  const int u_end = min(rows.n_units, u_begin + a.split_units);
  __syncthreads();
  if (u_begin >= u_end && split > 0) return;
  const int n_it = max(0, u_end - u_wave + NW * kU - 1) / (NW * kU);
  f32x4_t o[Tile::kOut];
#pragma unroll
  for (int t = 0; t < Tile::kOut; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  for (int it = 0; it < n_it; ++it) {
    float x[Tile::kScores];
    u32x4_t* keys = reinterpret_cast<u32x4_t*>(s_raw[wave]);
    tile.k.stage(keys, lane);
    const bool more = it + 1 < n_it;
    if (more) load_k(it + 1);
    int q_lane = lane;
    asm volatile("" : "+v"(q_lane));         // (else the queries are taken out of the loop, into registers)
    Tile::scores(s_q, keys, q_lane, g, c, x);
    const int u0 = u_wave + it * (NW * kU);
    bool full = true;
#pragma unroll
    for (int u = 0; u < kU; ++u)
      full = full & (u0 + u < u_end) & (bool)(pool_units >> (it * kU + u) & 1) & rows.full(rows.unit(u0 + u));
    if (!full) {
#pragma unroll
      for (int e = 0; e < Tile::kScores; ++e) {
        const int u = e / 4;
        const bool seen = rows.sees(rows.unit(u0 + u) * 16 + 4 * g + e % 4) & (u0 + u < u_end) & (bool)(pool_units >> (it * kU + u) & 1);
        x[e] = seen ? x[e] : -INFINITY;
        tile.keep_v(e, seen);
      }
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < Tile::kScores; ++e) top = fmaxf(top, x[e]);
    // the maximum of a query moves in the first tiles and rarely afterwards
    if (__builtin_amdgcn_ballot_w64(top > m) != 0) {
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float m2 = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m2);
      m = m2;
      l *= f;
#pragma unroll
      for (int t = 0; t < Tile::kOut; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[t][r] *= f;
    }
    const float m_use = m == -INFINITY ? 0.f : m;
    float p[Tile::kScores];
#pragma unroll
    for (int e = 0; e < Tile::kScores; ++e) {
      p[e] = __builtin_amdgcn_exp2f(x[e] - m_use);
      l += p[e];
    }
    tile.add(p, o);
    if (more) load_v(it + 1);
  }

  // ---- join the waves ----
  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  if (g == 0) {
    s_m[wave][c] = m;
    s_l[wave][c] = l;
  }
  if (c < n_heads) {
#pragma unroll
    for (int t = 0; t < Tile::kOut; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) s_o(wave)[c][Tile::out_col(t, 4 * g + r)] = o[t][r];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n_heads * (d / 4); i += 64 * NW) {
    const int h = i / (d / 4), e = (i - h * (d / 4)) * 4;
    float m_all = -INFINITY, l_all = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) m_all = fmaxf(m_all, s_m[w][h]);
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = s_m[w][h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][h] - m_all);
      l_all += f * s_l[w][h];
      v += f * *(const f32x4_t*)&s_o(w)[h][e];
    }
    const size_t row = row0 + h;
    if (a.n_split > 1) {
      *(f32x4_t*)(a.part + (row * a.n_split + split) * d + e) = v;
      if (e == 0) {
        a.part_ml[(row * a.n_split + split) * 2] = m_all;
        a.part_ml[(row * a.n_split + split) * 2 + 1] = l_all;
      }
    } else {
      if (l_all != 0.f) v *= 1.f / l_all;
      *(f32x4_t*)(a.out + row * d + e) = v;
      if (e == 0 && a.lse) a.lse[row] = l_all == 0.f ? -INFINITY : (m_all + __builtin_amdgcn_logf(l_all)) * 0.6931471805599453f;
    }
  }
  if (a.status && a.n_split == 1 && hk == 0 && hb == 0) {
    const int any = __syncthreads_or(!in_pool & (my_unit < u_end));
    if (threadIdx.x == 0) a.status[seq] = any;
  }
}

// Joins the splits of a row.  A thread has four columns of it and every J-th split; the J sums are added in order
// through LDS.  J = 1 up to kMost splits, whose loads a thread has under way together.  Behind the workgroups that
// join (grid: ceil(rows * d / 4 / (256 / J))) come one per sequence that look over its pages for the status.
template <int J, int kMost>
__global__ __launch_bounds__(256) void paged_attention_join(const PagedAttnArgs a, unsigned n_join) {
  constexpr int kCols = 256 / J;             // columns (of four) of a workgroup
  __shared__ float s_l[J][kCols];
  __shared__ f32x4_t s_v[J][kCols];
  const int d = a.c.d, tid = threadIdx.x, quads = d / 4;
  if (blockIdx.x >= n_join) {
    const int seq = blockIdx.x - n_join, page_units = a.c.page_size / 16;
    const VisibleRows rows(a.seq_len[seq], a.max_len, a.window, a.n_sink);
    bool bad = false;
#pragma unroll 8                             // (lookups under way together: 131071 rows 94.9 us with one at a time, 92.9)
    for (int u = tid; u < rows.n_units; u += 256)
      bad |= (unsigned)a.c.table[(size_t)seq * a.c.max_pages + rows.unit(u) / page_units] >= (unsigned)a.c.n_pages;
    const int any = __syncthreads_or(bad);
    if (tid == 0) a.status[seq] = any;
    return;
  }
  const unsigned n_rows = (unsigned)a.c.n_seqs * a.n_q;
  const size_t at = (size_t)blockIdx.x * kCols + tid % kCols;
  const unsigned row = min((unsigned)(at / quads), n_rows - 1);
  const int col = (int)(at % quads) * 4, i = tid / kCols;
  const bool real = at < (size_t)n_rows * quads;
  const VisibleRows rows(a.seq_len[row / a.n_q], a.max_len, a.window, a.n_sink);
  const int n = max(1, (rows.n_units + a.split_units - 1) / a.split_units);
  const float2* ml = (const float2*)a.part_ml + (size_t)row * a.n_split;
  const float* part = a.part + (size_t)row * a.n_split * d + col;
  float m = -INFINITY, l = 0.f;
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
  if constexpr (J == 1) {
    float2 e[kMost];
    f32x4_t w[kMost];
#pragma unroll
    for (int s = 0; s < kMost; ++s) {
      e[s] = ml[min(s, n - 1)];
      w[s] = *(const f32x4_t*)(part + (size_t)min(s, n - 1) * d);
      m = fmaxf(m, e[s].x);
    }
#pragma unroll
    for (int s = 0; s < kMost; ++s) {
      const float f = ((s < n) & (e[s].x != -INFINITY)) ? __builtin_amdgcn_exp2f(e[s].x - m) : 0.f;
      l += f * e[s].y;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += f == 0.f ? 0.f : f * w[s][k];
    }
  } else {
#pragma unroll 4
    for (int s = i; s < n; s += J) m = fmaxf(m, ml[s].x);
    s_l[i][tid % kCols] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < J; ++k) m = fmaxf(m, s_l[k][tid % kCols]);
    __syncthreads();
#pragma unroll 4
    for (int s = i; s < n; s += J) {
      const float2 e = ml[s];
      const float f = e.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(e.x - m);
      l += f * e.y;
      v += f * *(const f32x4_t*)(part + (size_t)s * d);
    }
    s_l[i][tid % kCols] = l;
    s_v[i][tid % kCols] = v;
    __syncthreads();
    if (i > 0) return;
#pragma unroll
    for (int k = 1; k < J; ++k) {
      l += s_l[k][tid];
      v += s_v[k][tid];
    }
  }
  if (!real) return;
  if (l != 0.f) v *= 1.f / l;
  *(f32x4_t*)(a.out + (size_t)row * d + col) = v;
  if (col == 0 && a.lse) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

}  // namespace sv
#endif
