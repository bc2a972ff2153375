// C-ABI entry points of the paged key-value cache: argument checks, planning, launches.
#include <cmath>

#include "sv_paged.h"

namespace sv {

static int check_paged(const sv_paged_cache* c) {
  if (!c || !c->k || !c->v || !c->block_table) return SV_ERR_NULL;
  if (c->dtype != SV_F32 && c->dtype != SV_BF16) return SV_ERR_DTYPE;
  if (c->n_seqs < 1 || c->n_seqs > (1 << 15) || c->max_pages < 1 || c->n_pages < 1 || c->page_size < 16 || c->page_size % 16 ||
      (long long)c->max_pages * c->page_size > (1ll << 30) || c->n_kv_heads < 1 || c->n_kv_heads > (1 << 15) ||
      c->head_dim < 8 || c->head_dim % 8 || c->head_dim > SV_MAX_PAGED_HEAD_DIM)
    return SV_ERR_SHAPE;
  if ((uintptr_t)c->k % 16 || (uintptr_t)c->v % 16) return SV_ERR_SHAPE;
  return SV_OK;
}

static PagedCache view(const sv_paged_cache& c) {
  return {c.k, c.v, c.block_table, c.n_seqs, c.max_pages, c.n_pages, c.page_size, c.n_kv_heads, c.head_dim};
}

static int check_heads(const sv_paged_cache& c, int n_q, int max_len) {
  if (n_q < 1 || n_q > (1 << 15) || n_q % c.n_kv_heads || max_len < 0 || max_len > c.max_pages * c.page_size) return SV_ERR_SHAPE;
  // A launch has less than 2^32 threads.  Attention: up to 2^23 pieces (beyond some 3000 workgroups nothing is cut finer than
  // 4096 rows) of 256 threads, of up to 512 where there are no more than kGroupsWide.  Join: 64 threads at most for a query
  // head, 2048 for one of more than 16 pieces, which here means 3000 heads at most, or 65536 rows and up to 2^19 heads.
  const long long pieces = (max_len + 4095ll) / 4096;
  return (long long)c.n_seqs * n_q * (pieces > 1 ? pieces : 1) > (1ll << 23) ? SV_ERR_SHAPE : SV_OK;
}

// How a call is split over the chip, in workgroups' rounds (a tile for each wave).  A workgroup has four waves, or six or
// eight ("wide") where registers leave room for two of these on a CU, if that saves a round and there is a workgroup per CU
// at most, or more than six rounds' work for each (32 and 8 heads of 128, bf16: 281 tokens 8.1 us narrow, 7.3 wide, 48
// sequences of 1028 visible tokens 18.1, 16.4; but 48 of up to 300 tokens 12.6, 14.6, 100 tokens 5.3, 5.6).
// Up to one workgroup per CU a row is cut into pieces of a round, if that saves three rounds (the second launch,
// which joins them, takes 4 us), or two narrow ones, which take longer: 600 tokens, 10.0 us in one piece, 8.4 in four;
// 16 sequences of up to 600, 10.9 in one, 11.6 in two; one of 300 and heads of 256, 12.5 in one, 10.0 in three.
// Whole rows of more than ten wide rounds, and pieces of more than ten narrow ones, are cut further, into pieces of four:
// until as many run as can at a time (three per CU), or four times as many for several sequences, some of which are shorter
// than others (24 float32 sequences of up to 1500 tokens, 11.8 rounds: 17.7 us in two pieces, 15.0 in five; 64 of 17 - 8192 tokens:
// 214 us in 1024 pieces, 202 in three times as many; but 32 of up to 1500, 7.8 rounds: 25.1 us whole, 27.4 in two, and 4
// float32 ones of up to 3000, 18.1 us in eight, 24.0 in eleven).  A piece has a unit of 16 rows at least for each query
// head of a KV head, beside whose rows its results would not be little.  Splits (and with them the scratch) never get
// fewer as max_len grows.
constexpr int kGroupsSmall = 256, kGroupsOne = 768, kGroupsRagged = 4 * kGroupsOne;
constexpr int kGroupsWide = 1 << 21;         // at most, of more than four waves: check_heads
constexpr long long kInfinityCache = 256ll << 20;
struct PagedPlan {
  int n_blocks, n_split, split_units, waves;
  size_t rows, part, part_ml, bytes;
};
static int wide_waves(const sv_paged_cache& c) {
  return c.head_dim <= 64 ? 8 : (c.head_dim <= 128 && c.dtype == SV_BF16 ? 6 : kPagedWaves);
}
static PagedPlan plan_paged(const sv_paged_cache& c, int n_q, int n_units) {
  PagedPlan p;
  p.n_blocks = ceil_div(n_q / c.n_kv_heads, 16);
  const int tasks = c.n_seqs * c.n_kv_heads * p.n_blocks;        // (2^23 at most)
  const int G = n_q / c.n_kv_heads, tile = c.dtype == SV_F32 ? 1 : 2, round = kPagedWaves * tile, wide = wide_waves(c) * tile;
  int few = kGroupsSmall / tasks;
  for (const int most : {ceil_div(n_units, wide), n_units / G}) few = most < few ? most : few;
  const int saved = few > 1 ? ceil_div(n_units, wide) - ceil_div(n_units, few * wide) : 0;
  p.n_split = saved >= (wide > round ? 3 : 2) ? few : 1;
  int cut = 1;
  if (ceil_div(n_units, p.n_split) > 10 * (p.n_split > 1 ? round : wide)) {
    const int most = ceil_div(c.n_seqs > 1 ? kGroupsRagged : kGroupsOne, tasks), fill = n_units / (G > 4 * round ? G : 4 * round);
    cut = fill < most ? fill : most;
  }
  for (const int n : {cut, ceil_div(n_units, kPagedWaves * kBatchUnits)}) p.n_split = n > p.n_split ? n : p.n_split;
  p.split_units = (ceil_div(n_units < 1 ? 1 : n_units, p.n_split) + 1) / 2 * 2;
  const int groups = tasks * p.n_split;
  const bool room = groups <= kGroupsSmall || (p.split_units > 6 * round && groups <= kGroupsWide);
  p.waves = room && ceil_div(p.split_units, wide) < ceil_div(p.split_units, round) ? wide_waves(c) : kPagedWaves;
  p.rows = (size_t)c.n_seqs * n_q;
  p.part = 0;
  p.part_ml = p.n_split > 1 ? align_up(p.rows * p.n_split * c.head_dim * 4, kAlign) : 0;
  p.bytes = p.n_split > 1 ? p.part_ml + align_up(p.rows * p.n_split * 8, kAlign) : kAlign;
  return p;
}

// Rows that are read once and fill the Infinity Cache (256 MB) go past the caches.
static bool past_caches(const sv_paged_cache& c, const PagedPlan& p, int n_units) {
  const long long row = 2ll * c.n_kv_heads * c.head_dim * (c.dtype == SV_F32 ? 4 : 2);
  return p.n_blocks == 1 && c.n_seqs * (n_units * 16ll) * row > kInfinityCache;
}

// Units that the visible rows of any sequence of up to max_len rows lie in, at most.
static int most_units(int max_len, int window, int n_sink) {
  const int all = ceil_div(max_len, 16);
  if (window == 0) return all;
  const long long some = (n_sink + 15ll) / 16 + (window + 15ll) / 16 + 1;      // (a window may begin inside a unit)
  return some < all ? (int)some : all;
}

static int launch_status() { return hipGetLastError() == hipSuccess ? SV_OK : SV_ERR_LAUNCH; }

}  // namespace sv

using namespace sv;

extern "C" {

int sv_paged_append(const sv_paged_cache* cache, int n_tokens, const int32_t* token_seq, const int32_t* token_pos,
                    const float* q, int n_q_heads, long long q_stride, const float* k, long long k_stride, const float* v,
                    long long v_stride, float rope_theta, float* q_out, int32_t* status, void* stream) {
  const int rc = check_paged(cache);
  if (rc != SV_OK) return rc;
  if (!token_seq || !token_pos || !k || !v || (q == nullptr) != (q_out == nullptr)) return SV_ERR_NULL;
  const long long d = cache->head_dim, kv = cache->n_kv_heads * d;
  if (n_tokens < 1 || n_tokens > (1 << 22) || n_q_heads < 0 || n_q_heads > (1 << 15) || (n_q_heads == 0) != (q == nullptr))
    return SV_ERR_SHAPE;
  if (k_stride < kv || v_stride < kv || k_stride % 4 || v_stride % 4 || (uintptr_t)k % 16 || (uintptr_t)v % 16) return SV_ERR_SHAPE;
  if (q && (q_stride < n_q_heads * d || q_stride % 4 || (uintptr_t)q % 16 || (uintptr_t)q_out % 16)) return SV_ERR_SHAPE;
  if (q == q_out && q && q_stride != n_q_heads * d) return SV_ERR_SHAPE;
  if (!(rope_theta > 0.f) || !std::isfinite(rope_theta)) return SV_ERR_SHAPE;
  AppendArgs a;
  a.c = view(*cache); a.seq = token_seq; a.pos = token_pos; a.q = q; a.k = k; a.v = v;
  a.q_stride = q ? q_stride : 0; a.k_stride = k_stride; a.v_stride = v_stride; a.n_q = n_q_heads;
  a.log2_theta = std::log2((double)rope_theta); a.q_out = q_out; a.status = status;
  if (cache->dtype == SV_F32) paged_append_kernel<float><<<n_tokens, 256, 0, (hipStream_t)stream>>>(a);
  else paged_append_kernel<bf16_t><<<n_tokens, 256, 0, (hipStream_t)stream>>>(a);
  return launch_status();
}

int sv_paged_workspace_bytes(const sv_paged_cache* cache, int n_q_heads, int max_len, size_t* bytes) {
  if (!bytes) return SV_ERR_NULL;
  int rc = check_paged(cache);
  if (rc == SV_OK) rc = check_heads(*cache, n_q_heads, max_len);
  if (rc != SV_OK) return rc;
  *bytes = plan_paged(*cache, n_q_heads, ceil_div(max_len, 16)).bytes;
  return SV_OK;
}

int sv_paged_attention(const sv_paged_cache* cache, const int32_t* seq_len, int max_len, const float* q, int n_q_heads,
                       float scale, int window, int n_sink, float* out, float* lse, int32_t* status, void* workspace,
                       size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int rc = sv_paged_workspace_bytes(cache, n_q_heads, max_len, &need);
  if (rc != SV_OK) return rc;
  if (!seq_len || !q || !out || !workspace) return SV_ERR_NULL;
  const float scale2 = scale * 1.4426950408889634f;
  if (window < 0 || n_sink < 0 || !std::isfinite(scale2) || (uintptr_t)q % 16 || (uintptr_t)out % 16) return SV_ERR_SHAPE;
  if ((uintptr_t)workspace % kAlign || ws_bytes < need) return SV_ERR_WORKSPACE;
  const int units = most_units(max_len, window, n_sink);
  const PagedPlan p = plan_paged(*cache, n_q_heads, units);
  PagedAttnArgs a;
  a.c = view(*cache); a.seq_len = seq_len; a.max_len = max_len; a.n_q = n_q_heads; a.window = window; a.n_sink = n_sink;
  a.n_blocks = p.n_blocks; a.n_split = p.n_split; a.split_units = p.split_units;
  a.scale = scale2; a.q = q; a.out = out; a.lse = lse; a.status = status;
  a.part = (float*)((char*)workspace + p.part); a.part_ml = (float*)((char*)workspace + p.part_ml);
  hipStream_t st = (hipStream_t)stream;
  const unsigned groups = (unsigned)(((size_t)cache->n_seqs * cache->n_kv_heads * p.n_split + 7) / 8 * 8 * p.n_blocks);
  auto run = [&](auto t, auto past) {
    using T = decltype(t);
    constexpr int NT = decltype(past)::value;
    auto launch = [&](auto dp, auto waves) {
      paged_attention_mfma<T, decltype(dp)::value, NT, decltype(waves)::value><<<groups, 64 * decltype(waves)::value, 0, st>>>(a);
    };
    auto by_waves = [&](auto dp, auto most) {
      if constexpr (NT == 0 && decltype(most)::value > kPagedWaves)
        if (p.waves > kPagedWaves) return launch(dp, most);
      launch(dp, std::integral_constant<int, kPagedWaves>{});
    };
    if (cache->head_dim <= 64) by_waves(std::integral_constant<int, 64>{}, std::integral_constant<int, 8>{});
    else if (cache->head_dim <= 128) by_waves(std::integral_constant<int, 128>{}, std::integral_constant<int, sizeof(T) == 2 ? 6 : kPagedWaves>{});
    else by_waves(std::integral_constant<int, 256>{}, std::integral_constant<int, kPagedWaves>{});
  };
  auto typed = [&](auto past) {
    if (cache->dtype == SV_F32) run(0.f, past);
    else run(bf16_t{}, past);
  };
  if (past_caches(*cache, p, units)) typed(std::integral_constant<int, 1>{});
  else typed(std::integral_constant<int, 0>{});
  if (p.n_split > 1) {
    const int joiners = p.n_split <= 16 ? 1 : 32;
    const unsigned n_join = (unsigned)((p.rows * (cache->head_dim / 4) * joiners + 255) / 256);
    auto join = p.n_split <= 8 ? paged_attention_join<1, 8> : (p.n_split <= 16 ? paged_attention_join<1, 16> : paged_attention_join<32, 0>);
    join<<<n_join + (status ? cache->n_seqs : 0), 256, 0, st>>>(a, n_join);
  }
  return launch_status();
}

}  // extern "C"
