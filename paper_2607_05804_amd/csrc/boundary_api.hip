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

// What both directions of the block norm share, apart from their matrices.
bool block_sizes_ok(int dtype, int residual_dtype, int param_dtype, int kind, int gate_kind, int64_t n_rows,
                    int64_t width) {
  return known_dtype(dtype) && known_dtype(residual_dtype) && known_dtype(param_dtype) &&
         (residual_dtype == dtype || residual_dtype == TURNKL_F32) &&
         (kind == TURNKL_NORM_LAYER || kind == TURNKL_NORM_RMS) && gate_kind >= TURNKL_GATE_NONE &&
         gate_kind <= TURNKL_GATE_MATRIX && n_rows >= 0 && n_rows <= 0x7FFFFFFFll && width >= 1 &&
         width <= TURNKL_MAX_NORM_WIDTH;
}

bool block_gate_ok(const void* gate, int64_t ld_gate, int gate_kind, int64_t n_rows, int64_t width, size_t es,
                   size_t ps) {
  if (gate_kind == TURNKL_GATE_NONE) return !gate;
  if (gate_kind == TURNKL_GATE_VECTOR) return gate && !misaligned(gate, ps);
  return n_rows == 0 || rows_ok(gate, ld_gate, width, es);
}

void block_params(BlockNormParams& p, int dtype, int residual_dtype, int param_dtype, int kind, int gate_kind,
                  int post_norm, int64_t n_rows, int64_t width, bool bwd) {
  p.n_rows = (int)n_rows;
  p.width = (int)width;
  p.branch_bf16 = dtype == TURNKL_BF16;
  p.residual_bf16 = residual_dtype == TURNKL_BF16;
  p.param_bf16 = param_dtype == TURNKL_BF16;
  p.post = post_norm != 0;
  p.gate_matrix = gate_kind == TURNKL_GATE_MATRIX;
  p.rms = kind == TURNKL_NORM_RMS;
  const int el = p.branch_bf16 && p.residual_bf16 ? 8 : 4;
  p.ragged = width % el != 0;
  const BlockShape s = block_norm_shape(n_rows, width, el, bwd, p.post != 0);
  p.threads = s.threads;
  p.lanes = s.lanes;
  p.units = s.units;
  p.n_groups = s.groups;
}

struct SampleLayout {
  size_t mass, most, sum, unit, todo, total;
  int n_segs;
};

bool sample_sizes_ok(int64_t n_tokens, int64_t vocab) {
  return n_tokens >= 0 && n_tokens <= 0x7FFFFFFFll && vocab >= 1 && vocab <= kMaxLogprobVocab;
}

SampleLayout sample_layout(int64_t n_tokens, int64_t vocab) {
  SampleLayout L{};
  // (rows of any start lie up to 63 elements behind the line their first one is on)
  L.n_segs = (int)((vocab + 63 + kSampleSegment - 1) / kSampleSegment);
  const size_t segs = (size_t)n_tokens * L.n_segs;
  L.mass = align256(sizeof(Header));
  L.most = align256(L.mass + segs * sizeof(double));
  L.sum = align256(L.most + segs * sizeof(float));
  L.unit = align256(L.sum + segs * sizeof(double));
  L.todo = align256(L.unit + segs * 64 * sizeof(unsigned short));
  L.total = align256(L.todo + (size_t)n_tokens);
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

int turnkl_block_norm_fwd(const void* residual, int64_t ld_residual, int residual_dtype,
                          const void* branch, int64_t ld_branch, int dtype, int64_t n_rows,
                          int64_t width, const void* gate, int64_t ld_gate, int gate_kind,
                          int post_norm, const void* post_weight, const void* weight,
                          const void* bias, int param_dtype, int kind, double residual_scale,
                          double eps, void* residual_out, int64_t ld_residual_out, void* y,
                          int64_t ld_y, float* stats_out, float* post_stats_out,
                          hipStream_t stream) {
  if (!block_sizes_ok(dtype, residual_dtype, param_dtype, kind, gate_kind, n_rows, width) ||
      !finite_float(residual_scale) || !(eps >= 0.0) || eps > FLT_MAX)
    return TURNKL_ERR_INVALID_ARG;
  const size_t es = elem_size(dtype), rs = elem_size(residual_dtype), ps = elem_size(param_dtype);
  const size_t w = (size_t)width, n = (size_t)n_rows;
  if (!block_gate_ok(gate, ld_gate, gate_kind, n_rows, width, es, ps)) return TURNKL_ERR_INVALID_ARG;
  if (!post_norm && (post_weight || post_stats_out)) return TURNKL_ERR_INVALID_ARG;
  if (n_rows == 0) return TURNKL_OK;
  if (!rows_ok(residual, ld_residual, width, rs) || !rows_ok(branch, ld_branch, width, es) ||
      !rows_ok(residual_out, ld_residual_out, width, rs) || !rows_ok(y, ld_y, width, es))
    return TURNKL_ERR_INVALID_ARG;
  if (misaligned(weight, ps) || misaligned(bias, ps) || misaligned(post_weight, ps) ||
      misaligned(stats_out, 4) || misaligned(post_stats_out, 4))
    return TURNKL_ERR_INVALID_ARG;
  const bool over_h = residual_out == residual && ld_residual_out == ld_residual;
  const bool over_f = y == branch && ld_y == ld_branch;
  const Region h{residual, matrix_bytes(n_rows, ld_residual, width, rs)};
  const Region f{branch, matrix_bytes(n_rows, ld_branch, width, es)};
  const Region g{gate, gate_kind == TURNKL_GATE_MATRIX ? matrix_bytes(n_rows, ld_gate, width, es) : w * ps};
  const Region out{residual_out, matrix_bytes(n_rows, ld_residual_out, width, rs)};
  const Region norm{y, matrix_bytes(n_rows, ld_y, width, es)};
  if (overlaps_any(out.p, out.n, {over_h ? Region{} : h, f}) ||
      overlaps_any(norm.p, norm.n, {h, over_f ? Region{} : f}))
    return TURNKL_ERR_ALIAS;
  if (any_overlap({g, {weight, w * ps}, {bias, w * ps}, {post_weight, w * ps}},
                  {out, norm, {stats_out, n * 8}, {post_stats_out, n * 8}}) ||
      any_overlap({h, f}, {{stats_out, n * 8}, {post_stats_out, n * 8}}))
    return TURNKL_ERR_ALIAS;
  BlockNormParams p{};
  block_params(p, dtype, residual_dtype, param_dtype, kind, gate_kind, post_norm, n_rows, width, false);
  p.residual = residual;
  p.branch = branch;
  p.gate = gate;
  p.weight = weight;
  p.bias = bias;
  p.post_weight = post_weight;
  p.out = residual_out;
  p.y = y;
  p.stats = stats_out;
  p.post_stats = post_stats_out;
  p.ld_residual = ld_residual;
  p.ld_branch = ld_branch;
  p.ld_gate = ld_gate;
  p.ld_out = ld_residual_out;
  p.ld_y = ld_y;
  p.scale = (float)residual_scale;
  // (rows without variance have an r for every eps but 0)
  p.eps = eps > 0.0 && (float)eps == 0.0f ? FLT_TRUE_MIN : (float)eps;
  return launch_block_norm(p, false, stream) == hipSuccess ? TURNKL_OK : TURNKL_ERR_HIP;
}

size_t turnkl_block_norm_workspace_bytes(int64_t n_rows, int64_t width) {
  if (n_rows < 0 || n_rows > 0x7FFFFFFFll || width < 1 || width > TURNKL_MAX_NORM_WIDTH) return 0;
  int most = 0;
  for (int el : {4, 8})
    for (bool post : {false, true}) {
      const int g = block_norm_shape(n_rows, width, el, true, post).groups;
      most = g > most ? g : most;
    }
  return align256((size_t)most * 4 * (size_t)width * sizeof(float));
}

int turnkl_block_norm_bwd(const void* grad_y, int64_t ld_gy, const void* grad_residual,
                          int64_t ld_gr, const void* residual, int64_t ld_residual,
                          int residual_dtype, const float* stats, const void* branch,
                          int64_t ld_branch, int dtype, int64_t n_rows, int64_t width,
                          const void* gate, int64_t ld_gate, int gate_kind, int post_norm,
                          const void* post_weight, const float* post_stats, const void* weight,
                          int param_dtype, int kind, double residual_scale,
                          void* grad_residual_out, int64_t ld_gro, void* grad_branch_out,
                          int64_t ld_gbo, void* grad_gate_out, int64_t ld_ggo,
                          float* grad_weight, float* grad_bias, float* grad_post_weight,
                          int accumulate, void* workspace, size_t workspace_bytes,
                          hipStream_t stream) {
  if (!block_sizes_ok(dtype, residual_dtype, param_dtype, kind, gate_kind, n_rows, width) ||
      !finite_float(residual_scale))
    return TURNKL_ERR_INVALID_ARG;
  const size_t es = elem_size(dtype), rs = elem_size(residual_dtype), ps = elem_size(param_dtype);
  const size_t w = (size_t)width, n = (size_t)n_rows;
  const bool matrix = gate_kind == TURNKL_GATE_MATRIX, needs_f = post_norm || gate_kind != TURNKL_GATE_NONE;
  if (!block_gate_ok(gate, ld_gate, gate_kind, n_rows, width, es, ps)) return TURNKL_ERR_INVALID_ARG;
  if (!post_norm && (post_weight || grad_post_weight)) return TURNKL_ERR_INVALID_ARG;
  if (gate_kind == TURNKL_GATE_NONE && grad_gate_out) return TURNKL_ERR_INVALID_ARG;
  float* const gate_sums = matrix ? nullptr : static_cast<float*>(grad_gate_out);
  if (!grad_residual_out && !grad_branch_out && !grad_gate_out && !grad_weight && !grad_bias && !grad_post_weight)
    return TURNKL_ERR_INVALID_ARG;
  if (n_rows > 0) {
    if (!rows_ok(grad_y, ld_gy, width, es) || !rows_ok(residual, ld_residual, width, rs) || !stats ||
        (grad_residual && !rows_ok(grad_residual, ld_gr, width, rs)) ||
        (needs_f && !rows_ok(branch, ld_branch, width, es)) || (post_norm && !post_stats) ||
        (grad_residual_out && !rows_ok(grad_residual_out, ld_gro, width, rs)) ||
        (grad_branch_out && !rows_ok(grad_branch_out, ld_gbo, width, es)) ||
        (matrix && grad_gate_out && !rows_ok(grad_gate_out, ld_ggo, width, es)))
      return TURNKL_ERR_INVALID_ARG;
  }
  if (misaligned(weight, ps) || misaligned(post_weight, ps)) return TURNKL_ERR_INVALID_ARG;
  for (const void* q : {(const void*)stats, (const void*)post_stats, (const void*)gate_sums,
                        (const void*)grad_weight, (const void*)grad_bias, (const void*)grad_post_weight})
    if (misaligned(q, 4)) return TURNKL_ERR_INVALID_ARG;
  const int sums = (grad_weight ? 1 : 0) | (grad_bias ? 2 : 0) | (grad_post_weight ? 4 : 0) | (gate_sums ? 8 : 0);
  const size_t need = sums ? turnkl_block_norm_workspace_bytes(n_rows, width) : 0;
  if (sums) {
    if (!workspace) return TURNKL_ERR_INVALID_ARG;
    if (misaligned(workspace, 256) || workspace_bytes < need) return TURNKL_ERR_WORKSPACE;
  }
  const Region gy{n ? grad_y : nullptr, matrix_bytes(n_rows, ld_gy, width, es)};
  const Region gr{n ? grad_residual : nullptr, matrix_bytes(n_rows, ld_gr, width, rs)};
  const Region h{n ? residual : nullptr, matrix_bytes(n_rows, ld_residual, width, rs)};
  const Region f{n && needs_f ? branch : nullptr, matrix_bytes(n_rows, ld_branch, width, es)};
  const Region g{matrix && !n ? nullptr : gate, matrix ? matrix_bytes(n_rows, ld_gate, width, es) : w * ps};
  const Region gro{n ? grad_residual_out : nullptr, matrix_bytes(n_rows, ld_gro, width, rs)};
  const Region gbo{n ? grad_branch_out : nullptr, matrix_bytes(n_rows, ld_gbo, width, es)};
  const Region ggo{n && matrix ? grad_gate_out : nullptr, matrix_bytes(n_rows, ld_ggo, width, es)};
  const bool over_r = grad_residual_out && grad_residual_out == grad_residual && ld_gro == ld_gr;
  const bool over_y = grad_branch_out && grad_branch_out == grad_y && ld_gbo == ld_gy;
  const Region none{};
  if ((gro.p && overlaps_any(gro.p, gro.n, {gy, over_r ? none : gr, h, f, g})) ||
      (gbo.p && overlaps_any(gbo.p, gbo.n, {over_y ? none : gy, gr, h, f, g})) ||
      (ggo.p && overlaps_any(ggo.p, ggo.n, {gy, gr, h, f, g})))
    return TURNKL_ERR_ALIAS;
  if (any_overlap({{weight, w * ps}, {post_weight, w * ps}, {stats, n * 8}, {post_stats, post_norm ? n * 8 : 0}},
                  {gro, gbo, ggo, {grad_weight, w * 4}, {grad_bias, w * 4}, {grad_post_weight, w * 4},
                   {gate_sums, w * 4}, {workspace, need}}) ||
      any_overlap({gy, gr, h, f, g}, {{grad_weight, w * 4}, {grad_bias, w * 4}, {grad_post_weight, w * 4},
                                      {gate_sums, w * 4}, {workspace, need}}))
    return TURNKL_ERR_ALIAS;
  BlockNormParams p{};
  block_params(p, dtype, residual_dtype, param_dtype, kind, gate_kind, post_norm, n_rows, width, true);
  p.residual = residual;
  p.branch = needs_f ? branch : nullptr;
  p.gate = gate;
  p.weight = weight;
  p.post_weight = post_weight;
  p.grad_y = grad_y;
  p.grad_h = grad_residual;
  p.out = grad_residual_out;
  p.grad_branch = grad_branch_out;
  p.grad_gate = matrix ? grad_gate_out : nullptr;
  p.stats = const_cast<float*>(stats);  // read only
  p.post_stats = const_cast<float*>(post_stats);
  p.part = sums ? static_cast<float*>(workspace) : nullptr;
  p.gw = grad_weight;
  p.gbias = grad_bias;
  p.gpost = grad_post_weight;
  p.ggate = gate_sums;
  p.sums = sums;
  p.ld_residual = ld_residual;
  p.ld_branch = ld_branch;
  p.ld_gate = ld_gate;
  p.ld_gy = ld_gy;
  p.ld_gh = ld_gr;
  p.ld_out = ld_gro;
  p.ld_gb = ld_gbo;
  p.ld_gg = ld_ggo;
  p.scale = (float)residual_scale;
  p.accumulate = accumulate != 0;
  return launch_block_norm(p, true, stream) == hipSuccess ? TURNKL_OK : TURNKL_ERR_HIP;
}

size_t turnkl_sample_workspace_bytes(int64_t n_tokens, int64_t vocab) {
  if (!sample_sizes_ok(n_tokens, vocab)) return 0;
  return sample_layout(n_tokens, vocab).total;
}

int turnkl_sample_tokens(const void* logits, int64_t ld, int dtype, int64_t n_tokens,
                         int64_t vocab, const uint8_t* mask, const turnkl_sampling* sampling,
                         const double* uniforms, int32_t* token_ids_out, float* logq_out,
                         float* logp_out, void* workspace, size_t workspace_bytes,
                         hipStream_t stream) {
  if (!known_dtype(dtype) || !sample_sizes_ok(n_tokens, vocab) || !workspace) return TURNKL_ERR_INVALID_ARG;
  turnkl_sampling s{};
  s.temperature = 1.0;
  s.top_p = 1.0;
  if (sampling) s = *sampling;
  if (!s.row_temperature && (!finite_float(s.temperature) || s.temperature < 0.0)) return TURNKL_ERR_INVALID_ARG;
  if (!s.row_top_p && !(s.top_p >= 0.0)) return TURNKL_ERR_INVALID_ARG;
  if (!s.row_min_p && !(s.min_p >= 0.0)) return TURNKL_ERR_INVALID_ARG;
  const size_t es = elem_size(dtype), n = (size_t)n_tokens;
  if (n_tokens > 0 && (!rows_ok(logits, ld, vocab, es) || !uniforms || !token_ids_out))
    return TURNKL_ERR_INVALID_ARG;
  if (misaligned(uniforms, 8)) return TURNKL_ERR_INVALID_ARG;
  for (const void* q : {(const void*)s.row_temperature, (const void*)s.row_top_k, (const void*)s.row_top_p,
                        (const void*)s.row_min_p, (const void*)token_ids_out, (const void*)logq_out,
                        (const void*)logp_out})
    if (misaligned(q, 4)) return TURNKL_ERR_INVALID_ARG;
  const SampleLayout L = sample_layout(n_tokens, vocab);
  if (misaligned(workspace, 256) || workspace_bytes < L.total) return TURNKL_ERR_WORKSPACE;
  if (n_tokens > 0 &&
      any_overlap({{logits, matrix_bytes(n_tokens, ld, vocab, es)}, {mask, n}, {uniforms, n * 8},
                   {s.row_temperature, n * 4}, {s.row_top_k, n * 4}, {s.row_top_p, n * 4}, {s.row_min_p, n * 4}},
                  {{token_ids_out, n * 4}, {logq_out, n * 4}, {logp_out, n * 4}, {workspace, L.total}}))
    return TURNKL_ERR_ALIAS;
  char* const ws = static_cast<char*>(workspace);
  SampleParams p{};
  p.z = logits;
  p.mask = mask;
  p.u = uniforms;
  p.row_temperature = s.row_temperature;
  p.row_top_k = s.row_top_k;
  p.row_top_p = s.row_top_p;
  p.row_min_p = s.row_min_p;
  p.ids = token_ids_out;
  p.logq = logq_out;
  p.logp = logp_out;
  p.hdr = reinterpret_cast<Header*>(ws);
  p.seg_mass = reinterpret_cast<double*>(ws + L.mass);
  p.seg_max = reinterpret_cast<float*>(ws + L.most);
  p.seg_sum = reinterpret_cast<double*>(ws + L.sum);
  p.unit = reinterpret_cast<unsigned short*>(ws + L.unit);
  p.todo = reinterpret_cast<unsigned char*>(ws + L.todo);
  p.ld = ld;
  p.n_rows = (int)n_tokens;
  p.vocab = (int)vocab;
  p.n_segs = L.n_segs;
  p.top_k = s.top_k;
  p.temperature = (float)s.temperature;
  // (beyond a float's range they limit nothing, or everything but the likeliest)
  p.top_p = (float)(s.top_p < 2.0 ? s.top_p : 2.0);
  p.min_p = (float)(s.min_p < 2.0 ? s.min_p : 2.0);
  p.any_filter = s.row_temperature || s.row_top_k || s.row_top_p || s.row_min_p || p.top_k > 0 || p.top_p < 1.0f ||
                 p.min_p > 0.0f || p.temperature == 0.0f;
  p.bf16 = dtype == TURNKL_BF16;
  p.ragged = misaligned(logits, 16) || (vocab * es) % 16 != 0 || (n_tokens > 1 && (ld * es) % 16 != 0);
  return launch_sample(p, stream) == hipSuccess ? TURNKL_OK : TURNKL_ERR_HIP;
}

}  // extern "C"
