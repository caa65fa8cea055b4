// Normalisation of rows (layer norm, or by the root mean square) and its gradient.
//
// A row is held in registers, kPacks 16-byte packs a thread, by the kThreads
// threads of one workgroup, so that it is read once and its mean and the sum of
// squared differences from it are taken one after the other.  Every workgroup goes
// from row to row and keeps its columns' weights (and, backward, the columns' sums
// over its rows) in registers; the next row is on its way while one is reduced.
// Backward a second kernel adds the workgroups' sums in their order.  Bound: HBM; small
// batches by latency.  65,536 bf16 rows of 4,096: 192 us forward (5.6 TB/s), 278
// backward (5.8 TB/s), where a copy of 2 GiB reaches 5.2; 64 rows of 2,048 forward 3 us.

#include "row_span.h"

namespace turnkl {
namespace {

constexpr int kNormThreads = 512;               // of a workgroup, at most
constexpr int kSumPacks = kNormThreads * 4;     // packs of a row whose columns' sums fit the registers

// Sums of kN values over the threads of a row, the same in each of them.  `lds`
// holds 2 x kMaxWaves x kN floats; `turn` alternates from call to call, so that one
// barrier serves: the other half is rewritten only after the next call's barrier.
constexpr int kMaxWaves = 8;
template <bool kOneWave, int kN>
__device__ inline void row_sums(float (&v)[kN], float* lds, int waves, int& turn) {
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = wave_sum(v[i]);
  if constexpr (!kOneWave) {
    float* const s = lds + turn * (kMaxWaves * kN);
    turn ^= 1;
    if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
      for (int i = 0; i < kN; ++i) s[(threadIdx.x / kWave) * kN + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = s[i];
    for (int w = 1; w < waves; ++w)
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] += s[w * kN + i];
  }
}

// Whether element j of a pack is its own (of rows of whole packs all are, or none).
template <bool kRagged>
__device__ inline bool own_element(unsigned bits, int j) {
  return kRagged ? ((bits >> j) & 1u) != 0 : bits != 0;
}

// A thread's packs of a vector of parameters: their own elements, `fill` for the others
// and where there is no vector.  All loads go out before one is waited for, here as for
// the rows: a branch around each makes every pack wait for the one before it (100 bf16
// rows of 2,048 backward took 12.0 us with such branches).
template <int kEpv, bool kRagged, int kPacks>
__device__ inline void load_params(const void* v, bool bf16, float fill, int width, const int* at,
                                   const unsigned* bits, float (&out)[kPacks][kEpv]) {
#pragma unroll
  for (int q = 0; q < kPacks; ++q)
#pragma unroll
    for (int j = 0; j < kEpv; ++j) out[q][j] = fill;
  if (!v) return;
  const auto r = chunk_rsrc(v);
  if (kRagged && width < kEpv) {  // a vector shorter than a pack: element by element
#pragma unroll
    for (int j = 0; j < kEpv; ++j)
      if ((bits[0] >> j) & 1u)
        out[0][j] = bf16 ? __uint_as_float((unsigned)__builtin_amdgcn_raw_buffer_load_b16(r, j * 2, 0, 0) << 16)
                         : __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, j * 4, 0, 0));
    return;
  }
  unsigned u[kPacks][kEpv];
  if (bf16) {
#pragma unroll
    for (int q = 0; q < kPacks; ++q) {
      if constexpr (kEpv == 8) {
        const auto x = __builtin_amdgcn_raw_buffer_load_b128(r, at[q] * 2, 0, 0);
        u[q][0] = x[0]; u[q][1] = x[1]; u[q][2] = x[2]; u[q][3] = x[3];
      } else {
        const auto x = __builtin_amdgcn_raw_buffer_load_b64(r, at[q] * 2, 0, 0);
        u[q][0] = x[0]; u[q][1] = x[1];
      }
    }
#pragma unroll
    for (int q = 0; q < kPacks; ++q)
#pragma unroll
      for (int j = kEpv - 1; j >= 0; --j)
        u[q][j] = j & 1 ? u[q][j >> 1] & 0xFFFF0000u : u[q][j >> 1] << 16;
  } else {
#pragma unroll
    for (int q = 0; q < kPacks; ++q)
#pragma unroll
      for (int k = 0; k < kEpv / 4; ++k) {
        const auto x = __builtin_amdgcn_raw_buffer_load_b128(r, at[q] * 4, 16 * k, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) u[q][4 * k + j] = x[j];
      }
  }
#pragma unroll
  for (int q = 0; q < kPacks; ++q)
#pragma unroll
    for (int j = 0; j < kEpv; ++j)
      if (own_element<kRagged>(bits[q], j)) out[q][j] = __uint_as_float(u[q][j]);
}

template <bool kBf16, bool kRagged>
__device__ inline RowSpan<kBf16, kRagged> row_of(const void* base, long long ld, long long row, int width,
                                                 int packs) {
  const char* const at = static_cast<const char*>(base) + row * ld * (kBf16 ? 2 : 4);
  return RowSpan<kBf16, kRagged>{at, chunk_rsrc(at), width, 0, packs};
}

template <bool kBf16, bool kRagged, bool kRms, bool kOneWave, int kPacks>
__global__ __launch_bounds__(kNormThreads) void norm_fwd_rows(NormParams p) {
  using Span = RowSpan<kBf16, kRagged>;
  using P = typename Span::P;
  constexpr int kEpv = Span::kEpv;
  __shared__ float s_sum[2 * kMaxWaves];
  const int waves = blockDim.x / kWave;
  const int threads = kOneWave ? kWave : blockDim.x;            // of a row
  const int tid = kOneWave ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const int slot = kOneWave ? __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) : 0;
  const long long stride = (long long)gridDim.x * (kOneWave ? waves : 1);
  const int packs = (p.width + kEpv - 1) / kEpv;
  const float width = (float)p.width;
  int at[kPacks], turn = 0;
  unsigned bits[kPacks];
  {
    const Span s = row_of<kBf16, kRagged>(p.x, 0, 0, p.width, packs);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) at[q] = s.place(q * threads + tid, bits[q]);
  }
  float w[kPacks][kEpv], b[kPacks][kEpv];
  load_params<kEpv, kRagged>(p.weight, p.param_bf16, 1.0f, p.width, at, bits, w);
  load_params<kEpv, kRagged>(p.bias, p.param_bf16, 0.0f, p.width, at, bits, b);
  P next[kPacks];
  auto fetch = [&](long long row) {
    const Span s = row_of<kBf16, kRagged>(p.x, p.ld_x, row, p.width, packs);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) s.load(next[q], at[q]);
  };
  // The stores of a row may read their data while the next row is summed: it stays
  // in registers of its own until then.
  typename P::Data data[kPacks];
#pragma unroll
  for (int q = 0; q < kPacks; ++q) data[q] = P::zero();
  long long row = kOneWave ? (long long)blockIdx.x * waves + slot : blockIdx.x;
  if (row < p.n_rows) fetch(row);
  for (; row < p.n_rows; row += stride) {
    P x[kPacks];
#pragma unroll
    for (int q = 0; q < kPacks; ++q) x[q] = next[q];
    if (row + stride < p.n_rows) fetch(row + stride);
    float mean = 0.0f;
    if constexpr (!kRms) {
      float v[1] = {0.0f};
#pragma unroll
      for (int q = 0; q < kPacks; ++q)
#pragma unroll
        for (int j = 0; j < kEpv; ++j) v[0] += own_element<kRagged>(bits[q], j) ? x[q].get(j) : 0.0f;
#pragma unroll
      for (int q = 0; q < kPacks; ++q) x[q].fence();  // unpacked again, rather than kept
      row_sums<kOneWave>(v, s_sum, waves, turn);
      mean = v[0] / width;
    }
    float v[1] = {0.0f};
#pragma unroll
    for (int q = 0; q < kPacks; ++q)
#pragma unroll
      for (int j = 0; j < kEpv; ++j) {
        const float d = own_element<kRagged>(bits[q], j) ? x[q].get(j) - mean : 0.0f;
        v[0] = fmaf(d, d, v[0]);
      }
#pragma unroll
    for (int q = 0; q < kPacks; ++q) x[q].fence();
    row_sums<kOneWave>(v, s_sum, waves, turn);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) keep_alive(data[q]);
    const float rstd = 1.0f / sqrtf(v[0] / width + p.eps);
    const Span out = row_of<kBf16, kRagged>(p.out, p.ld_out, row, p.width, packs);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) {
      float y[kEpv];
#pragma unroll
      for (int j = 0; j < kEpv; ++j) y[j] = fmaf((x[q].get(j) - mean) * rstd, w[q][j], b[q][j]);
      data[q] = P::encode(y, 0u);
    }
#pragma unroll
    for (int q = 0; q < kPacks; ++q) settle(data[q]);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) out.store_own(data[q], at[q], bits[q]);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) out.store_whole(data[q], at[q], bits[q]);
    if (p.stats && tid == 0) {
      p.stats[2 * row] = mean;
      p.stats[2 * row + 1] = rstd;
    }
  }
#pragma unroll
  for (int q = 0; q < kPacks; ++q) keep_alive(data[q]);
}

// Packs of a thread whose columns' sums go through LDS at a time: 32 KB at most.
constexpr int col_packs(bool one_wave, int packs) { return one_wave || packs < 2 ? packs : 2; }

template <bool kBf16, bool kRagged, bool kRms, bool kOneWave, int kPacks>
__global__ __launch_bounds__(kNormThreads) void norm_bwd_rows(NormParams p) {
  using Span = RowSpan<kBf16, kRagged>;
  using P = typename Span::P;
  constexpr int kEpv = Span::kEpv;
  // The widest rows fill the registers: there the weights are loaded for every row,
  // no row ahead, and the columns' sums are left to norm_bwd_columns.
  constexpr bool kLean = kPacks > 4;
  __shared__ float s_sum[2 * 2 * kMaxWaves];
  const int waves = blockDim.x / kWave;
  const int threads = kOneWave ? kWave : blockDim.x;            // of a row
  const int tid = kOneWave ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const int slot = kOneWave ? __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) : 0;
  const long long stride = (long long)gridDim.x * (kOneWave ? waves : 1);
  const int packs = (p.width + kEpv - 1) / kEpv;
  const float width = (float)p.width;
  int at[kPacks], turn = 0;
  unsigned bits[kPacks];
  {
    const Span s = row_of<kBf16, kRagged>(p.x, 0, 0, p.width, packs);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) at[q] = s.place(q * threads + tid, bits[q]);
  }
  float w[kLean ? 1 : kPacks][kEpv], gw[kLean ? 1 : kPacks][kEpv], gb[kLean ? 1 : kPacks][kEpv];
  if constexpr (!kLean) load_params<kEpv, kRagged>(p.weight, p.param_bf16, 1.0f, p.width, at, bits, w);
  auto weights = [&](int q) -> const float* {
    if constexpr (kLean)
      load_params<kEpv, kRagged>(p.weight, p.param_bf16, 1.0f, p.width, at + q, bits + q, w);
    return w[kLean ? 0 : q];
  };
#pragma unroll
  for (int q = 0; q < (kLean ? 1 : kPacks); ++q)
#pragma unroll
    for (int j = 0; j < kEpv; ++j) {
      gw[q][j] = 0.0f;
      gb[q][j] = 0.0f;
    }
  P next_x[kPacks], next_g[kPacks];
  float next_mean = 0.0f, next_rstd = 0.0f;
  auto fetch = [&](long long row) {
    const Span sx = row_of<kBf16, kRagged>(p.x, p.ld_x, row, p.width, packs);
    const Span sg = row_of<kBf16, kRagged>(p.gy, p.ld_gy, row, p.width, packs);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) {
      sx.load(next_x[q], at[q]);
      sg.load(next_g[q], at[q]);
    }
    if constexpr (!kRms) next_mean = p.stats[2 * row];
    next_rstd = p.stats[2 * row + 1];
  };
  typename P::Data data[kPacks];  // as in norm_fwd_rows
#pragma unroll
  for (int q = 0; q < kPacks; ++q) data[q] = P::zero();
  long long row = kOneWave ? (long long)blockIdx.x * waves + slot : blockIdx.x;
  if (!kLean && row < p.n_rows) fetch(row);
  for (; row < p.n_rows; row += stride) {
    if constexpr (kLean) fetch(row);
    P x[kPacks], g[kPacks];
#pragma unroll
    for (int q = 0; q < kPacks; ++q) {
      x[q] = next_x[q];
      g[q] = next_g[q];
    }
    const float mean = next_mean, rstd = next_rstd;
    if (!kLean && row + stride < p.n_rows) fetch(row + stride);
    float v[2] = {0.0f, 0.0f};  // sums of q xh and q
#pragma unroll
    for (int q = 0; q < kPacks; ++q) {
      const float* const wq = weights(q);
#pragma unroll
      for (int j = 0; j < kEpv; ++j) {
        const bool own = own_element<kRagged>(bits[q], j);
        const float gy = own ? g[q].get(j) : 0.0f;
        const float xh = own ? (x[q].get(j) - mean) * rstd : 0.0f;
        const float qq = gy * wq[j];
        v[0] = fmaf(qq, xh, v[0]);
        if constexpr (!kRms) v[1] += qq;
        if constexpr (!kLean) {
          gw[q][j] = fmaf(gy, xh, gw[q][j]);
          gb[q][j] += gy;
        }
      }
      if constexpr (!kLean)  // added here, and not at the end of the row
#pragma unroll
        for (int j = 0; j < kEpv; ++j) asm volatile("" : "+v"(gw[q][j]), "+v"(gb[q][j]));
      x[q].fence();                       // unpacked again, rather than kept
      g[q].fence();
    }
    row_sums<kOneWave>(v, s_sum, waves, turn);
#pragma unroll
    for (int q = 0; q < kPacks; ++q) keep_alive(data[q]);
    if (p.out) {
      const float c1 = v[0] / width, c0 = v[1] / width;
      const Span out = row_of<kBf16, kRagged>(p.out, p.ld_out, row, p.width, packs);
#pragma unroll
      for (int q = 0; q < kPacks; ++q) {
        float d[kEpv];
        const float* const wq = weights(q);
#pragma unroll
        for (int j = 0; j < kEpv; ++j) {
          const float xh = (x[q].get(j) - mean) * rstd;
          const float qq = g[q].get(j) * wq[j];
          d[j] = rstd * fmaf(-xh, c1, kRms ? qq : qq - c0);
        }
        data[q] = P::encode(d, 0u);
      }
#pragma unroll
      for (int q = 0; q < kPacks; ++q) settle(data[q]);
#pragma unroll
      for (int q = 0; q < kPacks; ++q) out.store_own(data[q], at[q], bits[q]);
#pragma unroll
      for (int q = 0; q < kPacks; ++q) out.store_whole(data[q], at[q], bits[q]);
    }
  }
#pragma unroll
  for (int q = 0; q < kPacks; ++q) keep_alive(data[q]);
  if constexpr (!kLean) {
    if (!p.part) return;
    // The rows' sums side by side through LDS, where columns lie in order, so that they
    // are stored in order: added over the waves that have rows of their own, one after
    // the other.
    extern __shared__ float s_col[];
    constexpr int kTurn = col_packs(kOneWave, kPacks);
    const int cols = threads * kTurn * kEpv;
    const int side = kOneWave ? waves : 1;
    float* const mine = s_col + slot * cols;
    float* const part = p.part + (long long)blockIdx.x * 2 * p.width;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      if (!(which ? p.gb : p.gw)) continue;
#pragma unroll
      for (int q0 = 0; q0 < kPacks; q0 += kTurn) {
#pragma unroll
        for (int q = 0; q < kTurn; ++q)
#pragma unroll
          for (int j = 0; j < kEpv; ++j)
            mine[(q * threads + tid) * kEpv + j] = which ? gb[q0 + q][j] : gw[q0 + q][j];
        __syncthreads();
        for (int i = threadIdx.x; i < cols; i += blockDim.x) {
          // element i % kEpv of the pack at e, which lies further left where it sticks out
          const int e = q0 * threads * kEpv + i / kEpv * kEpv;
          const int col = (kRagged ? inside_row(e, p.width > kEpv ? p.width - kEpv : 0) : e) + i % kEpv;
          if (e >= p.width || col < e || col >= p.width) continue;
          float v = s_col[i];
          for (int w = 1; w < side; ++w) v += s_col[w * cols + i];
          part[which * p.width + col] = v;
        }
        __syncthreads();
      }
    }
  }
}

// The column sums of the widest rows, which are read again: a thread per column, each
// of the n_groups runs of rows by workgroups of its own.
constexpr int kColumnThreads = 256;
__global__ __launch_bounds__(kColumnThreads) void norm_bwd_columns(NormParams p) {  // fp32 rows only
  const int col = blockIdx.x * kColumnThreads + threadIdx.x;
  if (col >= p.width) return;
  const float* const g = static_cast<const float*>(p.gy);
  const float* const x = static_cast<const float*>(p.x);
  float gw = 0.0f, gb = 0.0f;
#pragma unroll 4
  for (long long row = blockIdx.y; row < p.n_rows; row += p.n_groups) {
    const float gy = g[row * p.ld_gy + col];
    const float mean = p.rms ? 0.0f : p.stats[2 * row];
    gw = fmaf(gy, (x[row * p.ld_x + col] - mean) * p.stats[2 * row + 1], gw);
    gb += gy;
  }
  float* const part = p.part + (long long)blockIdx.y * 2 * p.width;
  if (p.gw) part[col] = gw;
  if (p.gb) part[p.width + col] = gb;
}

// Adds the workgroups' column sums in their order: 64 columns a workgroup, sixteen
// runs of partial rows side by side (blockIdx.y: the weight's sums or the bias's).
constexpr int kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void norm_bwd_join(NormParams p) {
  constexpr int kRuns = kJoinThreads / kWave;
  __shared__ float s_run[kRuns][kWave];
  const int lane = threadIdx.x & (kWave - 1);
  const int run = threadIdx.x / kWave;
  const int col = blockIdx.x * kWave + lane;
  float* const out = blockIdx.y ? p.gb : p.gw;
  if (!out) return;
  float s = 0.0f;
  if (col < p.width) {
    const float* at = p.part + (long long)blockIdx.y * p.width + col;
    const int lo = p.n_groups * run / kRuns, hi = p.n_groups * (run + 1) / kRuns;
#pragma unroll 8
    for (int i = lo; i < hi; ++i) s += at[(long long)i * 2 * p.width];
  }
  s_run[run][lane] = s;
  __syncthreads();
  if (run == 0 && col < p.width) {
    float t = s_run[0][lane];
#pragma unroll
    for (int r = 1; r < kRuns; ++r) t += s_run[r][lane];
    out[col] = p.accumulate ? out[col] + t : t;
  }
}

// How rows of a width are laid out over the threads, and how many workgroups go from
// row to row.
struct NormShape {
  bool one_wave;  // a wave per row, four or eight rows side by side in a workgroup
  int packs;      // of a thread
  int threads;    // of a workgroup
  int rows;       // side by side in a workgroup
  int groups;     // workgroups that fill the card
};

// Rows of up to 128 packs (backward 256) take one wave, which needs no barrier: backward,
// 12,000 bf16 rows of 2,048 (root mean square) take 33 us with four packs a lane and four
// rows a workgroup, 35 to 42 with two waves to a row (65,536 of them, layer form, 150
// against 145 to 162); 65,536 of 1,500, with the three packs that such a row fills, 122, with
// four 148, with two waves to a row 146.  Up to two packs a lane backward eight rows a
// workgroup: 65,536 of 512 take 40 us, with four rows 45, with two 70.  Wider rows take two
// packs a thread while 512 threads suffice (65,536 of 4,096 backward, layer form: 278 us,
// with four packs 329, with one 309), then four, and eight for fp32 rows past 8,192, whose
// column sums are a kernel of their own: it reads both matrices again (8,000 rows of 16,384
// 527 us, of 8,192 142).
// The workgroups go from row to row, so they are no more than the registers let the
// card hold at once, and backward fewer: what reads two streams and writes a third
// slows down with more of them in flight, and each leaves partial sums.  Forward 16
// waves a CU up to two packs (65,536 of 4,096: with 8 waves 231 us, with 24 213).
// Backward by measurement, us by workgroups a CU (1 / 2 / 3 / 4).
// A row to a workgroup and two packs a thread: two for eight waves of packs and more, fewer
// waves 24 in all.  65,536 bf16 rows of 4,096: 367 / 278 / 321 / 335, of 3,800: - / 280 / 314
// / 320; of 3,500 (seven waves): - / 364 / 304 / 305; of 2,500 (five): - / 339 / 268 / 228.
// 92 million fp32 elements in rows of 2,048: - / 188 / 201 / 215, of 1,537 (seven): - / 239 /
// 202 / 230, of 1,028 (five): - / 216 / 229 / 212; of whole packs two would do as well or
// better (of 1,792: - / 202 / 199 / 215, of 1,280: - / 186 / 199 / 193, of 1,536: - / 179 /
// 183 / 203).
// A wave to a row: two (65,536 of 512: 43 / 40 / 42; of 1,500: 176 / 122 / 153), but one where
// eight rows of more than 85 packs lie side by side, which is where the two cross: bf16 rows
// of 600: 62 / 54, of 680 (85 packs): 61.4 / 60.1, of 720: 62.7 / 63.2, of 1,000: 73 / 83;
// fp32 rows of 300: 51.2 / 50.6, of 340 (85): 56.5 / 56.8, of 400: 60.9 / 62.8.
// With a row to a workgroup and more packs a thread 8 waves.
NormShape norm_shape(long long width, int epv, bool bwd) {
  const int packs = (int)((width + epv - 1) / epv);
  NormShape s{};
  s.one_wave = packs <= (bwd ? 256 : 128);
  if (s.one_wave) {
    s.packs = (packs + 63) / 64;
    s.rows = bwd && s.packs <= 2 ? 8 : 4;
    s.threads = s.rows * kWave;
  } else {
    s.packs = packs <= 2 * kNormThreads ? 2 : packs <= kSumPacks ? 4 : 8;
    s.rows = 1;
    s.threads = ((packs + s.packs - 1) / s.packs + kWave - 1) / kWave * kWave;
  }
  const int waves = s.threads / kWave;
  int per_cu = (s.packs <= 2 ? 16 : 8) / waves;
  const int pieces = (packs + kWave - 1) / kWave;
  if (bwd && s.one_wave) per_cu = pieces == 2 && packs > 85 ? 1 : 2;
  else if (bwd && s.packs == 2) per_cu = pieces < 8 ? 24 / pieces : 2;
  s.groups = 256 * (per_cu < 1 ? 1 : per_cu);
  return s;
}

// Workgroups for a number of rows: backward every wave takes two rows at least, so
// that small batches leave fewer partial sums.
int groups_of(const NormShape& s, long long n_rows, bool bwd) {
  const long long per = (bwd ? 2 : 1) * s.rows;
  const long long g = (n_rows + per - 1) / per;
  return (int)(g < 1 ? 1 : g < s.groups ? g : s.groups);
}

template <bool kBwd, bool kBf16, bool kRagged, bool kRms, bool kOneWave, int kPacks>
void launch_one(const NormParams& p, const NormShape& n, hipStream_t s) {
  constexpr int kEpv = kBf16 ? 8 : 4;
  const size_t lds =
      kPacks <= 4 && p.part ? (size_t)n.threads * col_packs(kOneWave, kPacks) * kEpv * sizeof(float) : 0;
  if constexpr (kBwd)
    norm_bwd_rows<kBf16, kRagged, kRms, kOneWave, kPacks><<<p.n_groups, n.threads, lds, s>>>(p);
  else
    norm_fwd_rows<kBf16, kRagged, kRms, kOneWave, kPacks>
        <<<groups_of(n, p.n_rows, false), n.threads, 0, s>>>(p);
}

template <bool kBwd, bool kBf16, bool kRagged, bool kRms>
void launch_sized(const NormParams& p, hipStream_t s) {
  const NormShape n = norm_shape(p.width, kBf16 ? 8 : 4, kBwd);
  if (n.one_wave && n.packs == 1) launch_one<kBwd, kBf16, kRagged, kRms, true, 1>(p, n, s);
  else if (n.one_wave && n.packs == 2) launch_one<kBwd, kBf16, kRagged, kRms, true, 2>(p, n, s);
  else if (n.packs == 2) launch_one<kBwd, kBf16, kRagged, kRms, false, 2>(p, n, s);
  else if (!n.one_wave && n.packs == 4) launch_one<kBwd, kBf16, kRagged, kRms, false, 4>(p, n, s);
  else if constexpr (kBwd) {
    if (n.one_wave && n.packs == 3) launch_one<kBwd, kBf16, kRagged, kRms, true, 3>(p, n, s);
    else if (n.one_wave) launch_one<kBwd, kBf16, kRagged, kRms, true, 4>(p, n, s);
    else if constexpr (!kBf16) launch_one<kBwd, kBf16, kRagged, kRms, false, 8>(p, n, s);
  } else if constexpr (!kBf16) {
    launch_one<kBwd, kBf16, kRagged, kRms, false, 8>(p, n, s);
  }
}

template <bool kBwd>
void launch_norm(const NormParams& p, hipStream_t s) {
#define TURNKL_NORM(B, R, M)                                                      \
  if ((p.bf16 != 0) == B && (p.ragged != 0) == R && (p.rms != 0) == M)            \
    launch_sized<kBwd, B, R, M>(p, s);
  TURNKL_NORM(true, false, false) TURNKL_NORM(true, false, true) TURNKL_NORM(true, true, false)
  TURNKL_NORM(true, true, true) TURNKL_NORM(false, false, false) TURNKL_NORM(false, false, true)
  TURNKL_NORM(false, true, false) TURNKL_NORM(false, true, true)
#undef TURNKL_NORM
}

}  // namespace

int norm_groups(long long n_rows, long long width, bool bf16) {
  return groups_of(norm_shape(width, bf16 ? 8 : 4, true), n_rows, true);
}

hipError_t launch_norm_fwd(const NormParams& p, hipStream_t s) {
  if (p.n_rows == 0) return hipSuccess;
  launch_norm<false>(p, s);
  return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormParams& p, hipStream_t s) {
  const bool sums = p.gw || p.gb;
  const bool columns = !p.bf16 && (p.width + 3) / 4 > kSumPacks;  // whose rows leave no sums
  if (sums && columns) {  // before the rows: they may be in place
    const dim3 grid((p.width + kColumnThreads - 1) / kColumnThreads, p.n_groups);
    norm_bwd_columns<<<grid, kColumnThreads, 0, s>>>(p);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (p.out || !columns) launch_norm<true>(p, s);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (!sums) return hipSuccess;
  norm_bwd_join<<<dim3((p.width + kWave - 1) / kWave, p.gb ? 2 : 1), kJoinThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace turnkl
