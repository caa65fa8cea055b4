// Gradient of token log probabilities and entropies with respect to the logits:
//   x = (z - M) - L = log p,  p = 2^(x log2 e),
//   G = gl ([v = t] - p) - gh p (x + H) = gl [v = t] - p (gl + gh (x + H)),
// element by element from the row's saved (M, L) and H; no row waits for another.
// x is held above kLogFloor in the product, so that a forbidden token (p = 0)
// gives 0 and not 0 * inf.

#include "row_span.h"

namespace turnkl {
namespace {

constexpr int kGradThreads = 256;
constexpr int kGradPacks = 4;            // packs of a thread
constexpr int kGradGrid = 1 << 22;       // workgroups; beyond, each takes several tasks
constexpr float kLogFloor = -200.0f;     // exp(-200) is zero

// One workgroup per run of 1,024 packs of a row, on the gradient's lines.
template <bool kBf16, bool kRagged>
__global__ __launch_bounds__(kGradThreads) void logprob_grad(LogprobGradParams p, int n_chunks) {
  using Span = RowSpan<kBf16, kRagged>;
  using P = typename Span::P;
  constexpr int kEpv = Span::kEpv;
  constexpr int kEs = Span::kEs;
  const int tid = threadIdx.x;
  const long long n_tasks = (long long)p.n_rows * n_chunks;
  for (long long task = blockIdx.x;;) {  // the grid holds no more workgroups than tasks
    const long long row = task / n_chunks;
    const int first = (int)(task - row * n_chunks) * (kGradThreads * kGradPacks);
    char* const out = static_cast<char*>(p.grad) + row * p.ld_g * kEs;
    const char* const in = static_cast<const char*>(p.z) + row * p.ld * kEs;
    const int pre = kRagged ? (int)(reinterpret_cast<uintptr_t>(out) & 127u) / kEs : 0;
    const int n_row = (int)(((long long)pre + p.vocab + kEpv - 1) / kEpv);
    // (a row that starts on a line may have no pack in the last run)
    const Span span{in, chunk_rsrc(in), p.vocab, first * kEpv - pre, n_row - first};
    const bool on = !p.mask || p.mask[row];
    const float m = on ? p.log_z[2 * row] : -INFINITY;
    const bool zero = m == -INFINITY && !(on && p.log_z[2 * row + 1] != p.log_z[2 * row + 1]);

    typename P::Data data[kGradPacks];
    int at[kGradPacks];
    unsigned bits[kGradPacks];
#pragma unroll
    for (int q = 0; q < kGradPacks; ++q) {
      at[q] = span.place(q * kGradThreads + tid, bits[q]);
      data[q] = P::zero();
    }
    if (!zero) {
      const float l = p.log_z[2 * row + 1];
      const float h = p.entropy ? p.entropy[row] : 0.0f;
      const float gl = p.g_logp ? p.g_logp[row] : 0.0f;
      const float gh = p.g_entropy ? p.g_entropy[row] : 0.0f;
      const int t = p.g_logp ? p.ids[row] : -1;
      P x[kGradPacks];
#pragma unroll
      for (int q = 0; q < kGradPacks; ++q) span.load(x[q], at[q]);
#pragma unroll
      for (int q = 0; q < kGradPacks; ++q) {
        float g[kEpv];
#pragma unroll
        for (int j = 0; j < kEpv; ++j) {
          const float y = (x[q].get(j) - m) - l;
          const float e = exp2_fast(y * kLog2e);
          g[j] = -e * fmaf(gh, fmaxf(y, kLogFloor) + h, gl);
          if (at[q] + j == t) g[j] += gl;
        }
        data[q] = P::encode(g, 0u);
      }
    }
    task += gridDim.x;
    const bool more = __builtin_amdgcn_readfirstlane(task < n_tasks);
    const Span dst{out, chunk_rsrc(out), p.vocab, span.col, span.n};
#pragma unroll
    for (int q = 0; q < kGradPacks; ++q) settle(data[q]);
#pragma unroll
    for (int q = 0; q < kGradPacks; ++q) dst.store_own(data[q], at[q], bits[q]);
#pragma unroll
    for (int q = 0; q < kGradPacks; ++q) dst.store_whole(data[q], at[q], bits[q]);
#pragma unroll
    for (int q = 0; q < kGradPacks; ++q) keep_alive(data[q]);
    if (!more) break;
    drain_stores();  // their data registers are free for the next task
  }
}

}  // namespace

hipError_t launch_logprobs_bwd(const LogprobGradParams& p, hipStream_t s) {
  const int epv = p.bf16 ? 8 : 4;
  const int packs = (p.vocab + (p.ragged ? 127 / (16 / epv) : 0) + epv - 1) / epv;
  const int n_chunks = (packs + kGradThreads * kGradPacks - 1) / (kGradThreads * kGradPacks);
  const long long tasks = (long long)p.n_rows * n_chunks;
  const int grid = (int)(tasks < kGradGrid ? tasks : kGradGrid);
  if (p.bf16 && p.ragged) logprob_grad<true, true><<<grid, kGradThreads, 0, s>>>(p, n_chunks);
  else if (p.bf16) logprob_grad<true, false><<<grid, kGradThreads, 0, s>>>(p, n_chunks);
  else if (p.ragged) logprob_grad<false, true><<<grid, kGradThreads, 0, s>>>(p, n_chunks);
  else logprob_grad<false, false><<<grid, kGradThreads, 0, s>>>(p, n_chunks);
  return hipGetLastError();
}

}  // namespace turnkl
