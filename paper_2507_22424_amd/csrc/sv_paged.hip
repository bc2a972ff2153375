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
  return SV_OK;
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
  *bytes = kAlign;
  return SV_OK;
}

int sv_paged_attention(const sv_paged_cache* cache, const int32_t* seq_len, int max_len, const float* q, int n_q_heads,
                       float scale, int window, int n_sink, float* out, float* lse, int32_t* status, void* workspace,
                       size_t ws_bytes, void* stream) {
  size_t need = 0;
  const int rc = sv_paged_workspace_bytes(cache, n_q_heads, max_len, &need);
  if (rc != SV_OK) return rc;
  if (!seq_len || !q || !out || !workspace) return SV_ERR_NULL;
  if (window < 0 || n_sink < 0 || !std::isfinite(scale) || (uintptr_t)q % 16 || (uintptr_t)out % 16) return SV_ERR_SHAPE;
  if ((uintptr_t)workspace % kAlign || ws_bytes < need) return SV_ERR_WORKSPACE;
  PagedAttnArgs a;
  a.c = view(*cache); a.seq_len = seq_len; a.max_len = max_len; a.n_q = n_q_heads; a.window = window; a.n_sink = n_sink;
  a.scale = scale; a.q = q; a.out = out; a.lse = lse; a.status = status;
  const dim3 grid(n_q_heads, cache->n_seqs);
  if (cache->dtype == SV_F32) paged_attention_rows<float><<<grid, 256, 0, (hipStream_t)stream>>>(a);
  else paged_attention_rows<bf16_t><<<grid, 256, 0, (hipStream_t)stream>>>(a);
  return launch_status();
}

}  // extern "C"
