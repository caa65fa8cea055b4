// Gradient of token log probabilities and entropies with respect to the logits:
//   x = (z - M) - L = log p,  p = 2^(x log2 e),
//   G = gl ([v = t] - p) - gh p (x + H) = gl [v = t] - p (gl + gh (x + H)),
// element by element from the row's saved (M, L) and H; no row waits for another.
// x is held above kLogFloor in the product, so that a forbidden token (p = 0)
// gives 0 and not 0 * inf.  Bound: HBM (16,384 bf16 rows of 151,936, 60% asked for, the
// others written as zeros without being read: 1,426 us, 5.6 TB/s).

#include "row_span.h"

namespace turnkl {
namespace {

constexpr int kGradThreads = 256;        // (9,830 of 16,384 bf16 rows of 151,936: 1,417 us; 64: 1,410, 512: 1,467)
constexpr int kGradWaves = kGradThreads / kWave;
constexpr int kGradGrid = 1 << 22;       // workgroups; beyond, each takes several tasks (2,048: 1,699 us)
constexpr float kLogFloor = -200.0f;     // exp(-200) is zero

// A wave per run of 64 kPacks packs of a row, on the gradient's lines; the runs of a
// row, then those of the next, in the order of the waves.
template <bool kBf16, bool kRagged, int kPacks>
__global__ __launch_bounds__(kGradThreads) void logprob_grad(LogprobGradParams p, int n_runs) {
  using Span = RowSpan<kBf16, kRagged>;
  using P = typename Span::P;
  constexpr int kEpv = Span::kEpv;
  constexpr int kEs = Span::kEs;
  const int lane = threadIdx.x & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const long long n_tasks = (long long)p.n_rows * n_runs;
  const long long stride = (long long)gridDim.x * kGradWaves;
  for (long long task = (long long)blockIdx.x * kGradWaves + wid; task < n_tasks;) {
    const long long row = task / n_runs;
    const int first = (int)(task - row * n_runs) * (kWave * kPacks);
    char* const out = static_cast<char*>(p.grad) + row * p.ld_g * kEs;
    const char* const in = static_cast<const char*>(p.z) + row * p.ld * kEs;
    const int pre = kRagged ? (int)(reinterpret_cast<uintptr_t>(out) & 127u) / kEs : 0;
    const int n_row = (int)(((long long)pre + p.vocab + kEpv - 1) / kEpv);
    // (a row that starts on a line may have no pack in the last run)
    const Span span{in, chunk_rsrc(in), p.vocab, first * kEpv - pre, n_row - first};
    const bool on = !p.mask || p.mask[row];
    const float m = on ? p.log_z[2 * row] : -INFINITY;
    const float l = on ? p.log_z[2 * row + 1] : 0.0f;
    const bool zero = m == -INFINITY && l == l;  // not asked for, or empty

    typename P::Data data[kPacks];
    int at[kPacks];
    unsigned bits[kPacks];
#pragma unroll
    for (int q = 0; q < kPacks; ++q) {
      at[q] = span.place(q * kWave + lane, bits[q]);
      data[q] = P::zero();
    }
    if (!zero) {
      P x[kPacks];
#pragma unroll
      for (int q = 0; q < kPacks; ++q) span.load(x[q], at[q]);
      const float h = p.entropy ? p.entropy[row] : 0.0f;
      const float gl = p.g_logp ? p.g_logp[row] : 0.0f;
      const float gh = p.g_entropy ? p.g_entropy[row] : 0.0f;
      const int t = p.g_logp ? p.ids[row] : -1;
#pragma unroll
      for (int q = 0; q < kPacks; ++q) {
        float g[kEpv];
#pragma unroll
        for (int j = 0; j < kEpv; ++j) {
          const float y = (x[q].get(j) - m) - l;
          const float e = exp2_fast(y * kLog2e);
          g[j] = -e * fmaf(gh, fmaxf(y, kLogFloor) + h, gl);
        }
        if ((unsigned)(t - at[q]) < (unsigned)kEpv) {
#pragma unroll
          for (int j = 0; j < kEpv; ++j)
            if (at[q] + j == t) g[j] += gl;
        }
        data[q] = P::encode(g, 0u);
      }
    }
    task += stride;
    const bool more = __builtin_amdgcn_readfirstlane(task < n_tasks);
    const Span dst{out, chunk_rsrc(out), p.vocab, span.col, span.n};
#pragma unroll
    for (int q = 0; q < kPacks; ++q) settle(data[q]);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) dst.store_own(data[q], at[q], bits[q]);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) dst.store_whole(data[q], at[q], bits[q]);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) keep_alive(data[q]);
    if (!more) break;
    drain_stores();  // their data registers are free for the next task
  }
}

template <bool kBf16, bool kRagged, int kPacks>
void launch_packs(const LogprobGradParams& p, int packs, hipStream_t s) {
  const int n_runs = (packs + kWave * kPacks - 1) / (kWave * kPacks);
  const long long blocks = ((long long)p.n_rows * n_runs + kGradWaves - 1) / kGradWaves;
  const int grid = (int)(blocks < kGradGrid ? blocks : kGradGrid);
  logprob_grad<kBf16, kRagged, kPacks><<<grid, kGradThreads, 0, s>>>(p, n_runs);
}

// Two packs a lane of fp32 (5,000 rows of 151,936: 985 us, with four 1,093, with
// eight 1,078), four of bf16 (9,830 rows of 151,936, 60% asked for: 828 us, with two
// 872, with eight 890), as few as a short row needs.
template <bool kBf16, bool kRagged>
void launch_grad(const LogprobGradParams& p, hipStream_t s) {
  constexpr int kEpv = kBf16 ? 8 : 4;
  const int packs = (p.vocab + (kRagged ? 127 / (16 / kEpv) : 0) + kEpv - 1) / kEpv;
  if (packs <= kWave) launch_packs<kBf16, kRagged, 1>(p, packs, s);
  else if (packs <= 2 * kWave || !kBf16) launch_packs<kBf16, kRagged, 2>(p, packs, s);
  else if constexpr (kBf16) launch_packs<kBf16, kRagged, 4>(p, packs, s);
}

}  // namespace

hipError_t launch_logprobs_bwd(const LogprobGradParams& p, hipStream_t s) {
  if (p.bf16 && p.ragged) launch_grad<true, true>(p, s);
  else if (p.bf16) launch_grad<true, false>(p, s);
  else if (p.ragged) launch_grad<false, true>(p, s);
  else launch_grad<false, false>(p, s);
  return hipGetLastError();
}

}  // namespace turnkl
