// C-ABI of the operators at the token boundary (embedding rows and the table's gradient,
// norms fused with a block's gate and residual, sampled tokens): argument checks on the
// host, workspace carve-up and launches, all on the caller's stream with no host
// synchronisation.

#include <float.h>
#include <math.h>

#include "api_checks.h"

namespace turnkl {
namespace {

bool embed_sizes_ok(int64_t n_tokens, int64_t vocab, int64_t width) {
  return n_tokens >= 0 && n_tokens <= 0x7FFFFFFFll && vocab >= 1 && vocab <= kMaxLogprobVocab &&
         width >= 1 && width <= TURNKL_MAX_EMBED_WIDTH;
}

struct EmbedLayout {
  size_t key[2], tok[2], count, part, total;
};

EmbedLayout embed_layout(int64_t n_tokens, const EmbedShape& s) {
  EmbedLayout L{};
  const size_t ints = align256((size_t)n_tokens * 4);
  const int64_t tiles = (n_tokens + 2047) / 2048;  // of the sort, at least as many as it takes
  L.key[0] = align256(sizeof(Header));
  L.key[1] = L.key[0] + ints;
  L.tok[0] = L.key[1] + ints;
  L.tok[1] = L.tok[0] + ints;
  L.count = L.tok[1] + ints;
  L.part = L.count + ((size_t)(tiles < 256 ? tiles : 256) << kEmbedDigitBits) * 4;
  L.total = align256(L.part + (size_t)s.room * 4);
  return L;
}

bool finite_float(double x) { return x == x && fabs(x) <= FLT_MAX; }

}  // namespace
}  // namespace turnkl

using namespace turnkl;

extern "C" {

int turnkl_embed_fwd(const void* table, int64_t ld_table, int table_dtype, int64_t vocab,
                     int64_t width, const int32_t* token_ids, const uint8_t* mask,
                     int64_t n_tokens, double scale, void* out, int64_t ld_out, int out_dtype,
                     hipStream_t stream) {
  if (!known_dtype(table_dtype) || !known_dtype(out_dtype) || !embed_sizes_ok(n_tokens, vocab, width) ||
      !finite_float(scale))
    return TURNKL_ERR_INVALID_ARG;
  if (n_tokens == 0) return TURNKL_OK;
  const size_t ts = elem_size(table_dtype), os = elem_size(out_dtype), n = (size_t)n_tokens;
  if (!rows_ok(table, ld_table, width, ts) || !rows_ok(out, ld_out, width, os) || !token_ids ||
      misaligned(token_ids, 4))
    return TURNKL_ERR_INVALID_ARG;
  if (overlaps_any(out, matrix_bytes(n_tokens, ld_out, width, os),
                   {{table, matrix_bytes(vocab, ld_table, width, ts)}, {token_ids, n * 4}, {mask, n}}))
    return TURNKL_ERR_ALIAS;
  EmbedParams p{};
  p.table = table;
  p.ids = token_ids;
  p.mask = mask;
  p.out = out;
  p.ld_table = ld_table;
  p.ld_out = ld_out;
  p.n_rows = (int)n_tokens;
  p.vocab = (int)vocab;
  p.width = (int)width;
  p.scale = (float)scale;
  p.table_bf16 = table_dtype == TURNKL_BF16;
  p.out_bf16 = out_dtype == TURNKL_BF16;
  return launch_embed(p, stream) == hipSuccess ? TURNKL_OK : TURNKL_ERR_HIP;
}

size_t turnkl_embed_workspace_bytes(int64_t n_tokens, int64_t vocab, int64_t width) {
  if (!embed_sizes_ok(n_tokens, vocab, width)) return 0;
  return embed_layout(n_tokens, embed_shape(n_tokens, vocab, width)).total;
}

int turnkl_embed_bwd(const void* grad_out, int64_t ld_grad, int grad_dtype, int64_t n_tokens,
                     int64_t width, const int32_t* token_ids, const uint8_t* mask, int64_t vocab,
                     double scale, void* grad_table, int64_t ld_table, int table_dtype,
                     int accumulate, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!known_dtype(grad_dtype) || !known_dtype(table_dtype) || !embed_sizes_ok(n_tokens, vocab, width) ||
      !finite_float(scale))
    return TURNKL_ERR_INVALID_ARG;
  const size_t gs = elem_size(grad_dtype), ts = elem_size(table_dtype), n = (size_t)n_tokens;
  if (!rows_ok(grad_table, ld_table, width, ts) || !workspace) return TURNKL_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!rows_ok(grad_out, ld_grad, width, gs) || !token_ids || misaligned(token_ids, 4)))
    return TURNKL_ERR_INVALID_ARG;
  const EmbedShape s = embed_shape(n_tokens, vocab, width);
  const EmbedLayout L = embed_layout(n_tokens, s);
  if (misaligned(workspace, 256) || workspace_bytes < L.total) return TURNKL_ERR_WORKSPACE;
  if (any_overlap({{grad_out, n ? matrix_bytes(n_tokens, ld_grad, width, gs) : 0},
                   {token_ids, n * 4}, {mask, n}},
                  {{grad_table, matrix_bytes(vocab, ld_table, width, ts)}, {workspace, L.total}}))
    return TURNKL_ERR_ALIAS;
  char* const ws = static_cast<char*>(workspace);
  EmbedGradParams p{};
  p.grad = grad_out;
  p.ids = token_ids;
  p.mask = mask;
  p.table = grad_table;
  p.hdr = reinterpret_cast<Header*>(ws);
  for (int i = 0; i < 2; ++i) {
    p.key[i] = reinterpret_cast<int*>(ws + L.key[i]);
    p.tok[i] = reinterpret_cast<int*>(ws + L.tok[i]);
  }
  p.count = reinterpret_cast<int*>(ws + L.count);
  p.part = reinterpret_cast<float*>(ws + L.part);
  p.ld_grad = ld_grad;
  p.ld_table = ld_table;
  p.part_ld = s.part_ld;
  p.tile = s.tile;
  p.n_rows = (int)n_tokens;
  p.vocab = (int)vocab;
  p.width = (int)width;
  p.run = s.run;
  p.n_runs = (int)s.n_runs;
  p.col_tiles = s.col_tiles;
  p.n_tiles = (int)s.n_tiles;
  p.key_bits = s.key_bits;
  p.scale = (float)scale;
  p.grad_bf16 = grad_dtype == TURNKL_BF16;
  p.table_bf16 = table_dtype == TURNKL_BF16;
  p.accumulate = accumulate != 0;
  return launch_embed_bwd(p, stream) == hipSuccess ? TURNKL_OK : TURNKL_ERR_HIP;
}

}  // extern "C"
