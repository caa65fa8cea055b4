// C-ABI of the operators around the logits (token log probabilities and their
// gradient, row normalisation and its gradient): argument checks on the host,
// workspace carve-up and launches, all on the caller's stream with no host
// synchronisation.

#include <float.h>
#include <math.h>

#include "api_checks.h"

namespace turnkl {
namespace {

struct LogprobLayout {
  size_t rows, part, cand, total;
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
  const size_t tasks = (size_t)logprob_room(n_tokens, vocab);
  L.rows = align256(sizeof(Header));
  L.part = align256(L.rows + (size_t)n_tokens * sizeof(int));
  L.cand = align256(L.part + tasks * kLogprobPart * sizeof(float));
  L.total = align256(L.cand + tasks * (size_t)k * 8);
  return L;
}

// The arguments that both directions of the normalisation share.
bool norm_sizes_ok(int dtype, int param_dtype, int kind, int64_t n_rows, int64_t width) {
  return known_dtype(dtype) && known_dtype(param_dtype) &&
         (kind == TURNKL_NORM_LAYER || kind == TURNKL_NORM_RMS) && n_rows >= 0 &&
         n_rows <= 0x7FFFFFFFll && width >= 1 && width <= TURNKL_MAX_NORM_WIDTH;
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
  if (!known_dtype(dtype)) return TURNKL_ERR_INVALID_ARG;
  if (!logprob_sizes_ok(n_tokens, vocab, k) || !workspace) return TURNKL_ERR_INVALID_ARG;
  const size_t es = elem_size(dtype);
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
  p.rows = mask ? reinterpret_cast<int*>(ws + L.rows) : nullptr;
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

int turnkl_token_logprobs_bwd(const void* logits, int64_t ld, int dtype, int64_t n_tokens,
                              int64_t vocab, const int32_t* token_ids, const uint8_t* mask,
                              const float* log_z, const float* entropy, const float* grad_logp,
                              const float* grad_entropy, void* grad_out, int64_t ld_grad,
                              hipStream_t stream) {
  if (!known_dtype(dtype)) return TURNKL_ERR_INVALID_ARG;
  if (!logprob_sizes_ok(n_tokens, vocab, 0)) return TURNKL_ERR_INVALID_ARG;
  if (n_tokens == 0) return TURNKL_OK;
  const size_t es = elem_size(dtype);
  if (!logits || !log_z || !grad_out || (!grad_logp && !grad_entropy)) return TURNKL_ERR_INVALID_ARG;
  if ((grad_logp && !token_ids) || (grad_entropy && !entropy)) return TURNKL_ERR_INVALID_ARG;
  if (ld < vocab || ld > 0x7FFFFFFFll || ld_grad < vocab || ld_grad > 0x7FFFFFFFll)
    return TURNKL_ERR_INVALID_ARG;
  if (misaligned(logits, es) || misaligned(grad_out, es)) return TURNKL_ERR_INVALID_ARG;
  for (const void* p : {(const void*)token_ids, (const void*)log_z, (const void*)entropy,
                        (const void*)grad_logp, (const void*)grad_entropy})
    if (misaligned(p, 4)) return TURNKL_ERR_INVALID_ARG;
  const size_t n = (size_t)n_tokens, ng = matrix_bytes(n_tokens, ld_grad, vocab, es);
  const bool in_place = grad_out == logits && ld_grad == ld;
  if (overlaps_any(grad_out, ng,
                   {{in_place ? nullptr : logits, matrix_bytes(n_tokens, ld, vocab, es)},
                    {token_ids, n * 4}, {mask, n}, {log_z, n * 8}, {entropy, n * 4},
                    {grad_logp, n * 4}, {grad_entropy, n * 4}}))
    return TURNKL_ERR_ALIAS;
  LogprobGradParams p{};
  p.z = logits;
  p.ids = token_ids;
  p.mask = mask;
  p.log_z = log_z;
  p.entropy = grad_entropy ? entropy : nullptr;
  p.g_logp = grad_logp;
  p.g_entropy = grad_entropy;
  p.grad = grad_out;
  p.ld = ld;
  p.ld_g = ld_grad;
  p.n_rows = (int)n_tokens;
  p.vocab = (int)vocab;
  p.bf16 = dtype == TURNKL_BF16;
  p.ragged = misaligned(logits, 16) || misaligned(grad_out, 16) || (vocab * es) % 16 != 0 ||
             (n_tokens > 1 && ((ld * es) % 16 != 0 || (ld_grad * es) % 16 != 0));
  return launch_logprobs_bwd(p, stream) == hipSuccess ? TURNKL_OK : TURNKL_ERR_HIP;
}

int turnkl_norm_fwd(const void* x, int64_t ld_x, int dtype, int64_t n_rows, int64_t width,
                    const void* weight, const void* bias, int param_dtype, int kind, double eps,
                    void* y, int64_t ld_y, float* stats_out, hipStream_t stream) {
  if (!norm_sizes_ok(dtype, param_dtype, kind, n_rows, width)) return TURNKL_ERR_INVALID_ARG;
  if (!(eps >= 0.0) || eps > FLT_MAX) return TURNKL_ERR_INVALID_ARG;
  if (n_rows == 0) return TURNKL_OK;
  const size_t es = elem_size(dtype), ps = elem_size(param_dtype), w = (size_t)width;
  if (!rows_ok(x, ld_x, width, es) || !rows_ok(y, ld_y, width, es)) return TURNKL_ERR_INVALID_ARG;
  if (misaligned(weight, ps) || misaligned(bias, ps) || misaligned(stats_out, 4))
    return TURNKL_ERR_INVALID_ARG;
  const bool in_place = y == x && ld_y == ld_x;
  const size_t nx = matrix_bytes(n_rows, ld_x, width, es), ny = matrix_bytes(n_rows, ld_y, width, es);
  if (any_overlap({{weight, w * ps}, {bias, w * ps}, {in_place ? nullptr : x, nx}},
                  {{y, ny}, {stats_out, (size_t)n_rows * 8}}))
    return TURNKL_ERR_ALIAS;
  NormParams p{};
  p.x = x;
  p.weight = weight;
  p.bias = bias;
  p.out = y;
  p.stats = stats_out;
  p.ld_x = ld_x;
  p.ld_out = ld_y;
  p.n_rows = (int)n_rows;
  p.width = (int)width;
  // (rows without variance have an r for every eps but 0)
  p.eps = eps > 0.0 && (float)eps == 0.0f ? FLT_TRUE_MIN : (float)eps;
  p.bf16 = dtype == TURNKL_BF16;
  p.param_bf16 = param_dtype == TURNKL_BF16;
  p.rms = kind == TURNKL_NORM_RMS;
  p.ragged = !whole_packs(x, ld_x, n_rows, width, es) || !whole_packs(y, ld_y, n_rows, width, es);
  return launch_norm_fwd(p, stream) == hipSuccess ? TURNKL_OK : TURNKL_ERR_HIP;
}

size_t turnkl_norm_workspace_bytes(int64_t n_rows, int64_t width) {
  if (n_rows < 0 || n_rows > 0x7FFFFFFFll || width < 1 || width > TURNKL_MAX_NORM_WIDTH) return 0;
  const int b = norm_groups(n_rows, width, true), f = norm_groups(n_rows, width, false);
  return align256((size_t)(b > f ? b : f) * 2 * (size_t)width * sizeof(float));
}

int turnkl_norm_bwd(const void* grad_y, int64_t ld_gy, const void* x, int64_t ld_x, int dtype,
                    int64_t n_rows, int64_t width, const void* weight, int param_dtype, int kind,
                    const float* stats, void* grad_x, int64_t ld_gx, float* grad_weight,
                    float* grad_bias, int accumulate, void* workspace, size_t workspace_bytes,
                    hipStream_t stream) {
  if (!norm_sizes_ok(dtype, param_dtype, kind, n_rows, width)) return TURNKL_ERR_INVALID_ARG;
  if (!grad_x && !grad_weight && !grad_bias) return TURNKL_ERR_INVALID_ARG;
  const size_t es = elem_size(dtype), ps = elem_size(param_dtype), w = (size_t)width;
  if (n_rows > 0) {
    if (!rows_ok(grad_y, ld_gy, width, es) || !rows_ok(x, ld_x, width, es) || !stats)
      return TURNKL_ERR_INVALID_ARG;
    if (grad_x && !rows_ok(grad_x, ld_gx, width, es)) return TURNKL_ERR_INVALID_ARG;
  }
  if (misaligned(weight, ps)) return TURNKL_ERR_INVALID_ARG;
  for (const void* q : {(const void*)stats, (const void*)grad_weight, (const void*)grad_bias})
    if (misaligned(q, 4)) return TURNKL_ERR_INVALID_ARG;
  const bool sums = grad_weight || grad_bias;
  const size_t need = sums ? turnkl_norm_workspace_bytes(n_rows, width) : 0;
  if (sums) {
    if (!workspace) return TURNKL_ERR_INVALID_ARG;
    if (misaligned(workspace, 256) || workspace_bytes < need) return TURNKL_ERR_WORKSPACE;
  }
  const size_t ng = matrix_bytes(n_rows, ld_gy, width, es), nx = matrix_bytes(n_rows, ld_x, width, es);
  const bool over_g = grad_x && grad_x == grad_y && ld_gx == ld_gy;
  const bool over_x = grad_x && grad_x == x && ld_gx == ld_x;
  const Region out{n_rows > 0 ? grad_x : nullptr, matrix_bytes(n_rows, ld_gx, width, es)};
  if (overlaps_any(out.p, out.n, {{over_g ? nullptr : grad_y, ng}, {over_x ? nullptr : x, nx}}))
    return TURNKL_ERR_ALIAS;
  if (any_overlap({{weight, w * ps}, {stats, (size_t)n_rows * 8}},
                  {out, {grad_weight, w * 4}, {grad_bias, w * 4}, {workspace, need}}))
    return TURNKL_ERR_ALIAS;
  if (any_overlap({{grad_y, n_rows > 0 ? ng : 0}, {x, n_rows > 0 ? nx : 0}},
                  {{grad_weight, w * 4}, {grad_bias, w * 4}, {workspace, need}}))
    return TURNKL_ERR_ALIAS;
  NormParams p{};
  p.x = x;
  p.gy = grad_y;
  p.weight = weight;
  p.out = grad_x;
  p.stats = const_cast<float*>(stats);  // read only
  p.part = sums ? static_cast<float*>(workspace) : nullptr;
  p.gw = grad_weight;
  p.gb = grad_bias;
  p.ld_x = ld_x;
  p.ld_gy = ld_gy;
  p.ld_out = ld_gx;
  p.n_rows = (int)n_rows;
  p.width = (int)width;
  p.bf16 = dtype == TURNKL_BF16;
  p.n_groups = norm_groups(n_rows, width, p.bf16 != 0);
  p.param_bf16 = param_dtype == TURNKL_BF16;
  p.rms = kind == TURNKL_NORM_RMS;
  p.accumulate = accumulate != 0;
  p.ragged = !whole_packs(x, ld_x, n_rows, width, es) || !whole_packs(grad_y, ld_gy, n_rows, width, es) ||
             (grad_x && !whole_packs(grad_x, ld_gx, n_rows, width, es));
  return launch_norm_bwd(p, stream) == hipSuccess ? TURNKL_OK : TURNKL_ERR_HIP;
}

}  // extern "C"
