// C-ABI of the operators around the logits (token log probabilities): argument
// checks on the host, workspace carve-up and launches, all on the caller's stream
// with no host synchronisation.

#include "turnkl_internal.h"

namespace turnkl {
namespace {

struct LogprobLayout {
  size_t part, cand, total;
  int n_chunks;
};

// Whether the arguments that size the workspace are in range.
bool logprob_sizes_ok(int64_t n_tokens, int64_t vocab, int32_t k) {
  return n_tokens >= 0 && n_tokens <= 0x7FFFFFFFll && vocab >= 1 && vocab <= kMaxLogprobVocab &&
         k >= 0 && k <= kMaxAlternatives && k <= vocab;
}

LogprobLayout logprob_layout(int64_t n_tokens, int64_t vocab, int32_t k) {
  LogprobLayout L{};
  L.n_chunks = logprob_chunks(n_tokens, vocab);
  const size_t tasks = L.n_chunks > 1 ? (size_t)n_tokens * (size_t)L.n_chunks : 0;
  L.part = align256(sizeof(Header));
  L.cand = align256(L.part + tasks * kLogprobPart * sizeof(float));
  L.total = align256(L.cand + tasks * (size_t)k * 8);
  return L;
}

bool misaligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

// Whether any of the outputs overlaps an input or another output.
bool any_overlap(std::initializer_list<Region> in, std::initializer_list<Region> out) {
  for (const Region* a = out.begin(); a != out.end(); ++a) {
    if (!a->p || !a->n) continue;
    if (overlaps_any(a->p, a->n, in)) return true;
    for (const Region* b = a + 1; b != out.end(); ++b)
      if (b->p && b->n && overlaps(a->p, a->n, b->p, b->n)) return true;
  }
  return false;
}

}  // namespace
}  // namespace turnkl

using namespace turnkl;

extern "C" {

size_t turnkl_token_logprobs_workspace_bytes(int64_t n_tokens, int64_t vocab, int32_t k) {
  if (!logprob_sizes_ok(n_tokens, vocab, k)) return 0;
  return logprob_layout(n_tokens, vocab, k).total;
}

int turnkl_token_logprobs(const void* logits, int64_t ld, int dtype, int64_t n_tokens,
                          int64_t vocab, const int32_t* token_ids, const uint8_t* mask, int32_t k,
                          float* logp_out, float* entropy_out, float* log_z_out,
                          int32_t* top_ids_out, float* top_logp_out, int64_t ld_top,
                          void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (dtype != TURNKL_BF16 && dtype != TURNKL_F32) return TURNKL_ERR_INVALID_ARG;
  if (!logprob_sizes_ok(n_tokens, vocab, k) || !workspace) return TURNKL_ERR_INVALID_ARG;
  const size_t es = dtype == TURNKL_BF16 ? 2 : 4;
  if (n_tokens > 0) {
    if (!logits || ld < vocab || ld > 0x7FFFFFFFll || misaligned(logits, es))
      return TURNKL_ERR_INVALID_ARG;
    if (logp_out && !token_ids) return TURNKL_ERR_INVALID_ARG;
    if (k > 0 && (!top_ids_out || !top_logp_out || ld_top < k || ld_top > 0x7FFFFFFFll))
      return TURNKL_ERR_INVALID_ARG;
    if (k == 0 && (top_ids_out || top_logp_out)) return TURNKL_ERR_INVALID_ARG;
  }
  for (const void* p : {(const void*)token_ids, (const void*)logp_out, (const void*)entropy_out,
                        (const void*)log_z_out, (const void*)top_ids_out, (const void*)top_logp_out})
    if (misaligned(p, 4)) return TURNKL_ERR_INVALID_ARG;
  if (misaligned(workspace, 256)) return TURNKL_ERR_WORKSPACE;
  const LogprobLayout L = logprob_layout(n_tokens, vocab, k);
  if (workspace_bytes < L.total) return TURNKL_ERR_WORKSPACE;
  if (n_tokens > 0) {
    const size_t n = (size_t)n_tokens, nt = matrix_bytes(n_tokens, ld_top, k, 4);
    if (any_overlap({{logits, matrix_bytes(n_tokens, ld, vocab, es)}, {token_ids, n * 4}, {mask, n}},
                    {{logp_out, n * 4}, {entropy_out, n * 4}, {log_z_out, n * 8},
                     {top_ids_out, k ? nt : 0}, {top_logp_out, k ? nt : 0},
                     {workspace, L.total}}))
      return TURNKL_ERR_ALIAS;
  }
  char* const ws = static_cast<char*>(workspace);
  LogprobParams p{};
  p.z = logits;
  p.ids = token_ids;
  p.mask = mask;
  p.logp = logp_out;
  p.entropy = entropy_out;
  p.log_z = log_z_out;
  p.top_ids = top_ids_out;
  p.top_logp = top_logp_out;
  p.hdr = reinterpret_cast<Header*>(ws);
  p.part = reinterpret_cast<float*>(ws + L.part);
  p.cand = reinterpret_cast<unsigned long long*>(ws + L.cand);
  p.ld = ld;
  p.ld_top = ld_top;
  p.n_rows = (int)n_tokens;
  p.vocab = (int)vocab;
  p.k = k;
  p.n_chunks = L.n_chunks;
  p.bf16 = dtype == TURNKL_BF16;
  p.ragged = misaligned(logits, 16) || (vocab * es) % 16 != 0 || (n_tokens > 1 && (ld * es) % 16 != 0);
  return launch_logprobs(p, stream) == hipSuccess ? TURNKL_OK : TURNKL_ERR_HIP;
}

}  // extern "C"
