// C-ABI entry points of the sampled acceptance: argument checks and launches.
#include <cmath>

#include "sv_sample.h"

namespace sv {

static int token_probs(const float* logits, int n_rows, int n_vocab, float temperature, float* probs, hipStream_t st) {
  if (!logits || !probs) return SV_ERR_NULL;
  if (n_rows < 1 || n_rows >= (1 << 21) || n_vocab < 1 || n_vocab > SV_MAX_SAMPLED_VOCAB) return SV_ERR_SHAPE;
  const float inv_t = 1.f / temperature, c = (float)(1.4426950408889634 / (double)temperature);
  if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(inv_t) || !std::isfinite(c)) return SV_ERR_TOKEN;
  // Threads and columns a thread keeps, by the length of a row (us, 60 and 2000 or 960 rows: 256 columns 64 x 4 2.4, 3.0, 256 x 8
  // 2.6, 4.3; 2000 columns 256 x 8 2.8, 6.7, 1024 x 8 3.4, 13.8; 8000 columns 1024 x 8 3.7, 12.2, 1024 x 32 5.9, 22.7;
  // 32000 columns 1024 x 32 6.8, 42.7, two reads 9.0, 52.2).
  // (Below 2^100 a difference past the range of float32 is an exponent whose power is zero.)
  if (temperature > 0x1p100f)
    token_probs_kernel<1024, 0, true><<<n_rows, 1024, 0, st>>>(logits, n_vocab, (float)(1.4426950408889634 / ((double)temperature * kProbsUnit)), probs);
  else if (n_vocab <= 256) token_probs_kernel<64, 4><<<n_rows, 64, 0, st>>>(logits, n_vocab, c, probs);
  else if (n_vocab <= 2048) token_probs_kernel<256, 8><<<n_rows, 256, 0, st>>>(logits, n_vocab, c, probs);
  else if (n_vocab <= 8192) token_probs_kernel<1024, 8><<<n_rows, 1024, 0, st>>>(logits, n_vocab, c, probs);
  else if (n_vocab <= 32768) token_probs_kernel<1024, 32><<<n_rows, 1024, 0, st>>>(logits, n_vocab, c, probs);
  else {
    // shares of a row: as many as CUs that would be idle allow, eight at most (100 rows: 33.1 us by one workgroup each, 31.5 by two)
    const int shares = probs == logits || n_rows > 128 ? 1 : (n_rows <= 32 ? 8 : 256 / n_rows);
    token_probs_kernel<1024, 0><<<dim3(n_rows, shares), 1024, 0, st>>>(logits, n_vocab, c, probs);
  }
  return hipGetLastError() == hipSuccess ? SV_OK : SV_ERR_LAUNCH;
}

static int sampled_accept(const SampleArgs& a, int B, hipStream_t st) {
  // Threads by the length of a row (16 trees of 60 drawn tokens, about four children to a node, us with 64 / 128 / 256 / 512 /
  // 1024: 200 columns 6.1 / 6.9, 1000 - / 7.8 / 8.4, 2000 - / 9.1 / 7.7, 4000 - / - / 9.9 / 12.3, 8000 - / - / 14.4 / 12.3, 16000 - / - / - / 14.3 / 15.0; not held: 128 chains
  // of 128259 - / - / 56.0 / 32.9 / 32.1).  One wave takes 256 columns at most, see RowSearch::find.
  // Rows held take 128 KB of LDS for 1024 threads, so that one workgroup is on a CU instead of two: 400 trees of 32000
  // columns 57 us unheld, 42 held, but 1000 of 20000 78 and 86, 1000 chains 54 and 64.
  auto run = [&](auto drawn) {
    constexpr bool kDrawn = decltype(drawn)::value;
    if (a.n_vocab <= 256) sampled_accept_kernel<64, kDrawn, kDrawn><<<B, 64, 0, st>>>(a);
    else if (a.n_vocab <= 1024) sampled_accept_kernel<128, kDrawn, kDrawn><<<B, 128, 0, st>>>(a);
    else if (a.n_vocab <= 4096) sampled_accept_kernel<256, kDrawn, kDrawn><<<B, 256, 0, st>>>(a);
    else if (a.n_vocab <= 16384) sampled_accept_kernel<512, kDrawn, kDrawn><<<B, 512, 0, st>>>(a);
    else if (kDrawn && B <= 512 && a.n_vocab <= 1024 * HeldRow<1024>::kColumns)
      sampled_accept_kernel<1024, kDrawn, kDrawn><<<B, 1024, 0, st>>>(a);
    else sampled_accept_kernel<1024, kDrawn, false><<<B, 1024, 0, st>>>(a);
  };
  if (a.draft) run(std::true_type{});
  else run(std::false_type{});
  return hipGetLastError() == hipSuccess ? SV_OK : SV_ERR_LAUNCH;
}

}  // namespace sv

using namespace sv;

extern "C" {

int sv_token_probs(const float* logits, int n_rows, int n_vocab, float temperature, float* probs, void* stream) {
  return token_probs(logits, n_rows, n_vocab, temperature, probs, (hipStream_t)stream);
}

int sv_sampled_accept(const sv_tree* tree, const int32_t* draft_token, const float* target_prob, const float* draft_prob,
                      int n_vocab, int vocab_lo, const float* u_accept, const float* u_draw, int B, int d_cap,
                      uint8_t* accept_mask, int32_t* accepted_len, int32_t* best_node, int32_t* path, int32_t* out_tokens,
                      int32_t* status, void* stream) {
  if (!tree || !tree->parent || !draft_token || !target_prob || !u_accept || !u_draw || !accept_mask || !accepted_len ||
      !best_node || !path || !out_tokens || !status)
    return SV_ERR_NULL;
  const int T = tree->n_nodes;
  if (B < 1 || B > (1 << 15) || T < 1 || T > SV_MAX_TREE_NODES || d_cap < 0 || d_cap > SV_MAX_DEPTH || n_vocab < 1 ||
      n_vocab > SV_MAX_SAMPLED_VOCAB)
    return SV_ERR_SHAPE;
  if (vocab_lo < 0 || (long long)vocab_lo + n_vocab > 0x7fffffffll) return SV_ERR_TOKEN;
  SampleArgs a;
  a.parent = tree->parent; a.token = draft_token; a.target = target_prob; a.draft = draft_prob;
  a.u_accept = u_accept; a.u_draw = u_draw; a.T = T; a.n_vocab = n_vocab; a.lo = vocab_lo; a.d_cap = d_cap;
  a.accept_mask = accept_mask; a.accepted_len = accepted_len; a.best_node = best_node; a.path = path;
  a.out_tokens = out_tokens; a.status = status;
  return sampled_accept(a, B, (hipStream_t)stream);
}

}  // extern "C"
