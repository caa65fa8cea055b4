// The norms on either side of a block, fused with its gate and the residual sum, and
// their gradient.  For a row of the residual stream h and of a block's output f:
//   a  = (f - mu_f) r_f w_post  (or f itself),   h' = s h + gate a,
//   y  = (h' - mu) r w + b,
// and for the gradients gy of y and gh of h', with xh = (h' - mu) r, q = gy w:
//   t  = gh + r (q - mean q - xh mean(q xh)),    dh = s t,   dgate = t a,
//   df = the same for the first norm of q = gate t w_post, with fh = (f - mu_f) r_f
//        (or gate t itself),
//   dw = sum gy xh, db = sum gy, dw_post = sum gate t fh, and of a gate that is a
//   vector dgate = sum t a.
// A row is held in registers, a few units a thread, and read once; its sums are taken one
// after the other (layer: mean first, then squared differences).  Rows of up to 64 units
// share a wave, as many as fit; others take a workgroup each.  Workgroups go from row to
// row with the next row on its way, and keep parameters and, backward, their columns' sums
// in registers; a second kernel adds the workgroups' sums in their order.
//
// Bound: HBM.  65,536 bf16 rows of 4,096 with both norms and a vector's gate, forward: 428
// us, 5.0 TB/s over two streams in and two out, as a copy; backward 32,768 of them: 366 us,
// 4.4 TB/s over four streams in and two out, one workgroup of 162 VGPRs a CU and more of
// eight waves not fitting (at 128 VGPRs it spills: 1,033).  64 rows of 2,048: 4 us, two
// chains of sums.
#pragma once

#include "units.h"

namespace turnkl {
namespace {

constexpr int kBlockMaxWaves = 16;

// Sums of kN values over the threads of a row, the same in each: of `lanes` lanes side by
// side (kSub), or of a workgroup's waves, by LDS that alternates between two halves, so
// that one barrier serves.
template <bool kSub, int kN>
__device__ inline void block_row_sums(float (&v)[kN], float* lds, int lanes, int waves, int& turn) {
  if constexpr (kSub) {
#pragma unroll 1
    for (int o = lanes / 2; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] += __shfl_xor(v[i], o, kWave);
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = wave_sum_dpp(v[i]);
    float* const s = lds + turn * (kBlockMaxWaves * 2);
    turn ^= 1;
    if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
      for (int i = 0; i < kN; ++i) s[(threadIdx.x / kWave) * kN + i] = v[i];
    __syncthreads();
    // (a lane per wave: one load's latency, not one after the other)
    const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = lane < waves ? s[lane * kN + i] : 0.0f;
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = wave_sum_dpp(v[i]);
  }
}

template <bool kRagged, int kEl>
__device__ inline bool owns(const Place<kEl>& p, int j) {
  return kRagged ? ((p.bits >> j) & 1u) != 0 : p.bits != 0;
}

// A unit's parameters: `fill` where there is no vector, and for elements not its own.
template <bool kRagged, int kEl>
__device__ inline void load_vector(const void* v, bool bf16, float fill, const Place<kEl>& p, int width,
                                   float (&out)[kEl]) {
#pragma unroll
  for (int j = 0; j < kEl; ++j) out[j] = fill;
  if (!v) return;
  const char* const at = static_cast<const char*>(v);
  if (bf16) {
    Unit<true, kEl, true> x;
    load_unit(x, at, p, width);
#pragma unroll
    for (int j = 0; j < kEl; ++j)
      if (owns<kRagged>(p, j)) out[j] = x.get(j);
  } else {
    Unit<false, 4, true> x[kEl / 4];
#pragma unroll
    for (int i = 0; i < kEl / 4; ++i) {
      x[i].clear();
      if (width < kEl) x[i].load_some(at, p.at + 4 * i, (p.bits >> (4 * i)) & 15u);
      else if (p.bits) x[i].load(at, p.at + 4 * i);
    }
#pragma unroll
    for (int j = 0; j < kEl; ++j)
      if (owns<kRagged>(p, j)) out[j] = x[j / 4].get(j % 4);
  }
}

// Which rows a thread works on, and where its units of a row lie.
template <bool kSub, int kEl, int kUnits>
struct BlockRows {
  int lanes;        // threads of a row
  int tid;          // among them
  int waves;
  long long row, stride;
  Place<kEl> at[kUnits];

  __device__ explicit BlockRows(const BlockNormParams& p) {
    waves = blockDim.x / kWave;
    lanes = kSub ? p.lanes : (int)blockDim.x;
    tid = threadIdx.x & (lanes - 1);
    const int side = kSub ? (int)blockDim.x / lanes : 1;
    if (!kSub) tid = threadIdx.x;  // (not a power of two)
    row = (long long)blockIdx.x * side + (kSub ? threadIdx.x / lanes : 0);
    stride = (long long)gridDim.x * side;
    const int units = (p.width + kEl - 1) / kEl;
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      const int u = q * lanes + tid;
      at[q] = u < units ? place_unit<kEl>(u, p.width) : Place<kEl>{0, 0u};
    }
  }
  // whether any row of this wave (of this workgroup) is left
  __device__ bool left(const BlockNormParams& p) const {
    return kSub ? __any(row < p.n_rows) : row < p.n_rows;
  }
};

template <bool kBf16>
__device__ inline char* row_at(const void* base, long long ld, long long row) {
  return static_cast<char*>(const_cast<void*>(base)) + row * ld * (kBf16 ? 2 : 4);
}

// kF16: the branch, y and a gate per element; kR16: the residual stream.
template <bool kF16, bool kR16, bool kRagged, bool kSub, int kUnits, int kThreads>
__global__ __launch_bounds__(kThreads) void block_norm_rows(BlockNormParams p) {
  constexpr int kEl = unit_elements(kF16, kR16);
  __shared__ float s_sum[2 * 2 * kBlockMaxWaves];
  BlockRows<kSub, kEl, kUnits> r(p);
  const float width = (float)p.width;
  int turn = 0;
  float w[kUnits][kEl], b[kUnits][kEl], wp[kUnits][kEl], gv[kUnits][kEl];
#pragma unroll
  for (int q = 0; q < kUnits; ++q) {
    load_vector<kRagged>(p.weight, p.param_bf16, 1.0f, r.at[q], p.width, w[q]);
    load_vector<kRagged>(p.bias, p.param_bf16, 0.0f, r.at[q], p.width, b[q]);
    load_vector<kRagged>(p.post_weight, p.param_bf16, 1.0f, r.at[q], p.width, wp[q]);
    load_vector<kRagged>(p.gate_matrix ? nullptr : p.gate, p.param_bf16, 1.0f, r.at[q], p.width, gv[q]);
  }
  Unit<kF16, kEl> next_f[kUnits], next_g[kUnits];
  Unit<kR16, kEl> next_h[kUnits];
  auto fetch = [&](long long row) {
    const char* const f = row_at<kF16>(p.branch, p.ld_branch, row);
    const char* const h = row_at<kR16>(p.residual, p.ld_residual, row);
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      load_unit(next_f[q], f, r.at[q], p.width);
      load_unit(next_h[q], h, r.at[q], p.width);
    }
    if (p.gate_matrix) {
      const char* const g = row_at<kF16>(p.gate, p.ld_gate, row);
#pragma unroll
      for (int q = 0; q < kUnits; ++q) load_unit(next_g[q], g, r.at[q], p.width);
    }
  };
#pragma unroll
  for (int q = 0; q < kUnits; ++q) {
    next_f[q].clear();
    next_g[q].clear();
    next_h[q].clear();
  }
  // The data of a row's stores stay in registers of their own until the next row's.
  Unit<kF16, kEl> out_y[kUnits];
  Unit<kR16, kEl> out_h[kUnits];
#pragma unroll
  for (int q = 0; q < kUnits; ++q) {
    out_y[q].clear();
    out_h[q].clear();
  }
  if (r.row < p.n_rows) fetch(r.row);
  for (; r.left(p); r.row += r.stride) {
    const bool mine = r.row < p.n_rows;
    float x[kUnits][kEl], h[kUnits][kEl];
#pragma unroll
    for (int q = 0; q < kUnits; ++q)
#pragma unroll
      for (int j = 0; j < kEl; ++j) {
        x[q][j] = next_f[q].get(j);
        h[q][j] = next_h[q].get(j);
      }
    Unit<kF16, kEl> gate[kUnits];
#pragma unroll
    for (int q = 0; q < kUnits; ++q) gate[q] = next_g[q];
    if (r.row + r.stride < p.n_rows) fetch(r.row + r.stride);
    // mean and 1 / deviation of a row
    auto moments = [&](const float (&z)[kUnits][kEl], float& mean, float& rstd) {
      mean = 0.0f;
      if (!p.rms) {
        float v[1] = {0.0f};
#pragma unroll
        for (int q = 0; q < kUnits; ++q)
#pragma unroll
          for (int j = 0; j < kEl; ++j) v[0] += owns<kRagged>(r.at[q], j) ? z[q][j] : 0.0f;
        block_row_sums<kSub>(v, s_sum, r.lanes, r.waves, turn);
        mean = v[0] / width;
      }
      float v[1] = {0.0f};
#pragma unroll
      for (int q = 0; q < kUnits; ++q)
#pragma unroll
        for (int j = 0; j < kEl; ++j) {
          const float d = owns<kRagged>(r.at[q], j) ? z[q][j] - mean : 0.0f;
          v[0] = fmaf(d, d, v[0]);
        }
      block_row_sums<kSub>(v, s_sum, r.lanes, r.waves, turn);
      rstd = 1.0f / sqrtf(v[0] / width + p.eps);
    };
    float mean_f = 0.0f, rstd_f = 1.0f;
    if (p.post) {
      moments(x, mean_f, rstd_f);
      if (p.post_stats && r.tid == 0 && mine) {
        p.post_stats[2 * r.row] = mean_f;
        p.post_stats[2 * r.row + 1] = rstd_f;
      }
    }
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
#pragma unroll
      for (int j = 0; j < kEl; ++j) {
        const float g = p.gate_matrix ? gate[q].get(j) : gv[q][j];
        const float a = p.post ? (x[q][j] - mean_f) * rstd_f * wp[q][j] : x[q][j];
        h[q][j] = fmaf(h[q][j], p.scale, a * g);
      }
    }
    float mean, rstd;
    moments(h, mean, rstd);
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      out_y[q].keep();
      out_h[q].keep();
    }
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      float y[kEl];
#pragma unroll
      for (int j = 0; j < kEl; ++j) y[j] = fmaf((h[q][j] - mean) * rstd, w[q][j], b[q][j]);
      out_y[q].set(y);
      out_h[q].set(h[q]);
    }
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      out_y[q].fence();
      out_h[q].fence();
    }
    if (mine) {
      char* const to_y = row_at<kF16>(p.y, p.ld_y, r.row);
      char* const to_h = row_at<kR16>(p.out, p.ld_out, r.row);
      if constexpr (kRagged)
#pragma unroll
        for (int q = 0; q < kUnits; ++q) {
          store_edge(out_y[q], to_y, r.at[q]);
          store_edge(out_h[q], to_h, r.at[q]);
        }
#pragma unroll
      for (int q = 0; q < kUnits; ++q) {
        store_whole(out_y[q], to_y, r.at[q]);
        store_whole(out_h[q], to_h, r.at[q]);
      }
      if (p.stats && r.tid == 0) {
        p.stats[2 * r.row] = mean;
        p.stats[2 * r.row + 1] = rstd;
      }
    }
  }
#pragma unroll
  for (int q = 0; q < kUnits; ++q) {
    out_y[q].keep();
    out_h[q].keep();
  }
}

// The widest rows, forward: a workgroup a row, which is read from the caches again, and h'
// in LDS.  2^27 bf16 elements with both norms and a vector's gate, in rows of 12,288: 366 us
// (of 8,192, held in registers, 196).
constexpr int kWideThreads = 512;
template <bool kF16, bool kR16>
__global__ __launch_bounds__(kWideThreads) void block_norm_wide(BlockNormParams p) {
  constexpr int kEl = unit_elements(kF16, kR16);
  __shared__ float s_sum[2 * 2 * kBlockMaxWaves];
  extern __shared__ float s_row[];  // [units][kEl], unit by unit of a thread
  constexpr int kWaves = kWideThreads / kWave;
  const float width = (float)p.width;
  const int units = (p.width + kEl - 1) / kEl;
  int turn = 0;
  auto sum = [&](float v) {
    float one[1] = {v};
    block_row_sums<false>(one, s_sum, 0, kWaves, turn);
    return one[0];
  };
  // the mean and 1 / deviation of a row whose units' elements at() gives
  auto moments = [&](auto at, float& mean, float& rstd) {
    float v = 0.0f;
    mean = 0.0f;
    if (!p.rms) {
      for (int u = threadIdx.x; u < units; u += kWideThreads)
        at(u, [&](float z) { v += z; });
      mean = sum(v) / width;
      v = 0.0f;
    }
    for (int u = threadIdx.x; u < units; u += kWideThreads)
      at(u, [&](float z) { v = fmaf(z - mean, z - mean, v); });
    rstd = 1.0f / sqrtf(sum(v) / width + p.eps);
  };
  for (long long row = blockIdx.x; row < p.n_rows; row += gridDim.x) {
    Unit<kF16, kEl, true> f, g;
    Unit<kR16, kEl, true> h;
    float mean_f = 0.0f, rstd_f = 1.0f, mean, rstd;
    if (p.post) {
      moments([&](int u, auto use) {
        const Place<kEl> at = place_unit<kEl>(u, p.width);
        load_unit(f, row_at<kF16>(p.branch, p.ld_branch, row), at, p.width);
#pragma unroll
        for (int j = 0; j < kEl; ++j)
          if (owns<true>(at, j)) use(f.get(j));
      }, mean_f, rstd_f);
    }
    for (int u = threadIdx.x; u < units; u += kWideThreads) {
      const Place<kEl> at = place_unit<kEl>(u, p.width);
      load_unit(f, row_at<kF16>(p.branch, p.ld_branch, row), at, p.width);
      load_unit(h, row_at<kR16>(p.residual, p.ld_residual, row), at, p.width);
      float gv[kEl], wp[kEl], x[kEl];
      load_vector<true>(p.post_weight, p.param_bf16, 1.0f, at, p.width, wp);
      if (p.gate_matrix) {
        load_unit(g, row_at<kF16>(p.gate, p.ld_gate, row), at, p.width);
#pragma unroll
        for (int j = 0; j < kEl; ++j) gv[j] = g.get(j);
      } else {
        load_vector<true>(p.gate, p.param_bf16, 1.0f, at, p.width, gv);
      }
#pragma unroll
      for (int j = 0; j < kEl; ++j) {
        const float a = p.post ? (f.get(j) - mean_f) * rstd_f * wp[j] : f.get(j);
        x[j] = fmaf(h.get(j), p.scale, a * gv[j]);
        s_row[u * kEl + j] = x[j];
      }
      Unit<kR16, kEl> out;
      out.set(x);
      out.fence();
      char* const to = row_at<kR16>(p.out, p.ld_out, row);
      store_edge(out, to, at);
      store_whole(out, to, at);
      out.keep();
      store_gap();
    }
    moments([&](int u, auto use) {
      const Place<kEl> at = place_unit<kEl>(u, p.width);
#pragma unroll
      for (int j = 0; j < kEl; ++j)
        if (owns<true>(at, j)) use(s_row[u * kEl + j]);
    }, mean, rstd);
    for (int u = threadIdx.x; u < units; u += kWideThreads) {
      const Place<kEl> at = place_unit<kEl>(u, p.width);
      float w[kEl], b[kEl], y[kEl];
      load_vector<true>(p.weight, p.param_bf16, 1.0f, at, p.width, w);
      load_vector<true>(p.bias, p.param_bf16, 0.0f, at, p.width, b);
#pragma unroll
      for (int j = 0; j < kEl; ++j) y[j] = fmaf((s_row[u * kEl + j] - mean) * rstd, w[j], b[j]);
      Unit<kF16, kEl> out;
      out.set(y);
      out.fence();
      char* const to = row_at<kF16>(p.y, p.ld_y, row);
      store_edge(out, to, at);
      store_whole(out, to, at);
      out.keep();
      store_gap();
    }
    if (threadIdx.x == 0) {
      if (p.post_stats) {
        p.post_stats[2 * row] = mean_f;
        p.post_stats[2 * row + 1] = rstd_f;
      }
      if (p.stats) {
        p.stats[2 * row] = mean;
        p.stats[2 * row + 1] = rstd;
      }
    }
  }
}

// Backward.  What a thread holds of a row beyond eight elements leaves no room for the
// parameters, which are then loaded where they are used, nor, beyond two units, for a row
// ahead.
template <bool kF16, bool kR16, bool kRagged, bool kSub, bool kPost, bool kGateMatrix, int kUnits, int kThreads>
__global__ __launch_bounds__(kThreads) void block_norm_bwd_rows(BlockNormParams p) {
  constexpr int kEl = unit_elements(kF16, kR16);
  constexpr bool kHold = kUnits * kEl <= 8;
  constexpr bool kAhead = kUnits <= 2;
  constexpr int kHeld = kHold ? kUnits : 1;
  __shared__ float s_sum[2 * 2 * kBlockMaxWaves];
  BlockRows<kSub, kEl, kUnits> r(p);
  const float width = (float)p.width;
  int turn = 0;
  const bool branch = kPost || kGateMatrix || p.gate;  // whether f is needed
  float w[kHeld][kEl], wp[kHeld][kEl], gv[kHeld][kEl];
  float sw[kUnits][kEl], sb[kUnits][kEl], sp[kUnits][kEl], sg[kUnits][kEl];
  auto parameters = [&](int q) {
    const int i = kHold ? q : 0;
    Place<kEl> at = r.at[q];
    if constexpr (!kHold) asm volatile("" : "+v"(at.at));  // addresses made here, not held over the rows
    load_vector<kRagged>(p.weight, p.param_bf16, 1.0f, at, p.width, w[i]);
    if constexpr (kPost) load_vector<kRagged>(p.post_weight, p.param_bf16, 1.0f, at, p.width, wp[i]);
    if constexpr (!kGateMatrix) load_vector<kRagged>(p.gate, p.param_bf16, 1.0f, at, p.width, gv[i]);
  };
#pragma unroll
  for (int q = 0; q < kUnits; ++q) {
    if constexpr (kHold) parameters(q);
#pragma unroll
    for (int j = 0; j < kEl; ++j) sw[q][j] = sb[q][j] = sp[q][j] = sg[q][j] = 0.0f;
  }
  Unit<kF16, kEl> next_gy[kUnits], next_f[kUnits], next_g[kUnits];
  Unit<kR16, kEl> next_gh[kUnits], next_h[kUnits];
  float next_stat[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  auto fetch = [&](long long row) {
    const char* const gy = row_at<kF16>(p.grad_y, p.ld_gy, row);
    const char* const h = row_at<kR16>(p.residual, p.ld_residual, row);
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      load_unit(next_gy[q], gy, r.at[q], p.width);
      load_unit(next_h[q], h, r.at[q], p.width);
    }
    if (p.grad_h) {
      const char* const gh = row_at<kR16>(p.grad_h, p.ld_gh, row);
#pragma unroll
      for (int q = 0; q < kUnits; ++q) load_unit(next_gh[q], gh, r.at[q], p.width);
    }
    if (branch) {
      const char* const f = row_at<kF16>(p.branch, p.ld_branch, row);
#pragma unroll
      for (int q = 0; q < kUnits; ++q) load_unit(next_f[q], f, r.at[q], p.width);
    }
    if constexpr (kGateMatrix) {
      const char* const g = row_at<kF16>(p.gate, p.ld_gate, row);
#pragma unroll
      for (int q = 0; q < kUnits; ++q) load_unit(next_g[q], g, r.at[q], p.width);
    }
    if (!p.rms) next_stat[0] = p.stats[2 * row];
    next_stat[1] = p.stats[2 * row + 1];
    if constexpr (kPost) {
      if (!p.rms) next_stat[2] = p.post_stats[2 * row];
      next_stat[3] = p.post_stats[2 * row + 1];
    }
  };
#pragma unroll
  for (int q = 0; q < kUnits; ++q) {
    next_gy[q].clear();
    next_f[q].clear();
    next_g[q].clear();
    next_gh[q].clear();
    next_h[q].clear();
  }
  Unit<kR16, kEl> out_h[kUnits];  // as in block_norm_rows
  Unit<kF16, kEl> out_f[kUnits], out_g[kUnits];
#pragma unroll
  for (int q = 0; q < kUnits; ++q) {
    out_h[q].clear();
    out_f[q].clear();
    out_g[q].clear();
  }
  if (kAhead && r.row < p.n_rows) fetch(r.row);
  for (; r.left(p); r.row += r.stride) {
    const bool mine = r.row < p.n_rows;
    if (!kAhead && mine) fetch(r.row);
    Unit<kF16, kEl> gy[kUnits], f[kUnits], g[kUnits];
    Unit<kR16, kEl> gh[kUnits], h[kUnits];
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      gy[q] = next_gy[q];
      f[q] = next_f[q];
      g[q] = next_g[q];
      gh[q] = next_gh[q];
      h[q] = next_h[q];
    }
    // (a lane without a row has zeros throughout)
    const float mean = next_stat[0], rstd = mine ? next_stat[1] : 0.0f;
    const float mean_f = next_stat[2], rstd_f = mine ? next_stat[3] : 0.0f;
    if (kAhead && r.row + r.stride < p.n_rows) fetch(r.row + r.stride);
    float v[2] = {0.0f, 0.0f};  // sums of q xh and q
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      if constexpr (!kHold) parameters(q);
#pragma unroll
      for (int j = 0; j < kEl; ++j) {
        const bool own = mine && owns<kRagged>(r.at[q], j);
        const float d = own ? gy[q].get(j) : 0.0f;
        const float xh = own ? (h[q].get(j) - mean) * rstd : 0.0f;
        const float qq = d * w[kHold ? q : 0][j];
        v[0] = fmaf(qq, xh, v[0]);
        v[1] += qq;
        sw[q][j] = fmaf(d, xh, sw[q][j]);
        sb[q][j] += d;
      }
      gy[q].fence();
      h[q].fence();
    }
    block_row_sums<kSub>(v, s_sum, r.lanes, r.waves, turn);
    const float c1 = v[0] / width, c0 = p.rms ? 0.0f : v[1] / width;
    // t, as a value of an element that may be asked for again
    auto upstream = [&](int q, int j) {
      const float xh = (h[q].get(j) - mean) * rstd;
      const float qq = gy[q].get(j) * w[kHold ? q : 0][j];
      const float d = p.grad_h ? gh[q].get(j) : 0.0f;
      return fmaf(rstd, fmaf(-xh, c1, qq - c0), d);
    };
    float c1f = 0.0f, c0f = 0.0f;
    if constexpr (kPost) {
      float u[2] = {0.0f, 0.0f};
#pragma unroll
      for (int q = 0; q < kUnits; ++q) {
        if constexpr (!kHold) parameters(q);
#pragma unroll
        for (int j = 0; j < kEl; ++j) {
          const bool own = mine && owns<kRagged>(r.at[q], j);
          const float gate = kGateMatrix ? g[q].get(j) : gv[kHold ? q : 0][j];
          const float da = own ? upstream(q, j) * gate : 0.0f;
          const float fh = own ? (f[q].get(j) - mean_f) * rstd_f : 0.0f;
          const float qq = da * wp[kHold ? q : 0][j];
          u[0] = fmaf(qq, fh, u[0]);
          u[1] += qq;
          sp[q][j] = fmaf(da, fh, sp[q][j]);
        }
        gy[q].fence();
        gh[q].fence();
        h[q].fence();
        f[q].fence();
        g[q].fence();
      }
      block_row_sums<kSub>(u, s_sum, r.lanes, r.waves, turn);
      c1f = u[0] / width;
      c0f = p.rms ? 0.0f : u[1] / width;
    }
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      out_h[q].keep();
      out_f[q].keep();
      if constexpr (kGateMatrix) out_g[q].keep();
    }
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      if constexpr (!kHold) parameters(q);
      float dh[kEl], df[kEl], dg[kEl];
#pragma unroll
      for (int j = 0; j < kEl; ++j) {
        const bool own = mine && owns<kRagged>(r.at[q], j);
        const float t = own ? upstream(q, j) : 0.0f;
        const float gate = kGateMatrix ? g[q].get(j) : gv[kHold ? q : 0][j];
        dh[j] = t * p.scale;
        const float da = t * gate;
        if constexpr (kPost) {
          const float fh = own ? (f[q].get(j) - mean_f) * rstd_f : 0.0f;
          const float wj = wp[kHold ? q : 0][j];
          dg[j] = t * (fh * wj);
          df[j] = rstd_f * fmaf(-fh, c1f, da * wj - c0f);
        } else {
          dg[j] = branch && own ? t * f[q].get(j) : 0.0f;
          df[j] = da;
        }
      }
      if constexpr (!kGateMatrix)
#pragma unroll
        for (int j = 0; j < kEl; ++j) sg[q][j] += dg[j];
      out_h[q].set(dh);
      out_f[q].set(df);
      if constexpr (kGateMatrix) out_g[q].set(dg);
    }
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      out_h[q].fence();
      out_f[q].fence();
      if constexpr (kGateMatrix) out_g[q].fence();
    }
    if (mine) {
      char* const to_h = row_at<kR16>(p.out, p.ld_out, r.row);
      char* const to_f = row_at<kF16>(p.grad_branch, p.ld_gb, r.row);
      char* const to_g = row_at<kF16>(p.grad_gate, p.ld_gg, r.row);
      if constexpr (kRagged)
#pragma unroll
        for (int q = 0; q < kUnits; ++q) {
          if (p.out) store_edge(out_h[q], to_h, r.at[q]);
          if (p.grad_branch) store_edge(out_f[q], to_f, r.at[q]);
          if constexpr (kGateMatrix)
            if (p.grad_gate) store_edge(out_g[q], to_g, r.at[q]);
        }
#pragma unroll
      for (int q = 0; q < kUnits; ++q) {
        if (p.out) store_whole(out_h[q], to_h, r.at[q]);
        if (p.grad_branch) store_whole(out_f[q], to_f, r.at[q]);
        if constexpr (kGateMatrix)
          if (p.grad_gate) store_whole(out_g[q], to_g, r.at[q]);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < kUnits; ++q) {
    out_h[q].keep();
    out_f[q].keep();
    if constexpr (kGateMatrix) out_g[q].keep();
  }
  if (!p.part) return;
  // The sums of rows side by side, added in their order through LDS.
  extern __shared__ float s_col[];
  float* const part = p.part + (long long)blockIdx.x * 4 * p.width;
  const int side = kSub ? (int)blockDim.x / r.lanes : 1;
  const int cols = r.lanes * kEl;
  const int mine = kSub ? (int)threadIdx.x / r.lanes : 0;
#pragma unroll
  for (int which = 0; which < 4; ++which) {
    if (!((p.sums >> which) & 1)) continue;
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
      const float(&held)[kEl] = which == 0 ? sw[q] : which == 1 ? sb[q] : which == 2 ? sp[q] : sg[q];
#pragma unroll
      for (int j = 0; j < kEl; ++j) s_col[(mine * r.lanes + r.tid) * kEl + j] = held[j];
      __syncthreads();
      for (int i = threadIdx.x; i < cols; i += blockDim.x) {
        // element i % kEl of a unit, which lies further left where it sticks out
        const int e = (q * r.lanes + i / kEl) * kEl;
        const int col = inside_row(e, p.width > kEl ? p.width - kEl : 0) + i % kEl;
        if (e >= p.width || col < e || col >= p.width) continue;
        float v = s_col[i];
        for (int k = 1; k < side; ++k) v += s_col[k * cols + i];
        part[(long long)which * p.width + col] = v;
      }
      __syncthreads();
    }
  }
}

// Backward of the widest rows: a workgroup a row, which is read again for each of its sums
// (from the caches, then), and the columns' sums in the workspace, a row of the workgroup's
// own whose elements are always the same thread's.
//
// Bound: the columns' sums, which every row reads and writes, and the waits after each
// unit's stores: 2^27 bf16 elements with both norms and a vector's gate, in rows of 5,120
// 2,558 us, of 8,192 1,930, of 16,384 1,919 (of 4,096, held in registers, 366).
template <bool kF16, bool kR16>
__global__ __launch_bounds__(kWideThreads) void block_norm_bwd_wide(BlockNormParams p) {
  constexpr int kEl = unit_elements(kF16, kR16);
  __shared__ float s_sum[2 * 2 * kBlockMaxWaves];
  constexpr int kWaves = kWideThreads / kWave;
  const float width = (float)p.width;
  const int units = (p.width + kEl - 1) / kEl;
  const bool branch = p.post || p.gate;
  float* const part = p.part ? p.part + (long long)blockIdx.x * 4 * p.width : nullptr;
  int turn = 0;
  bool first = true;
  for (long long row = blockIdx.x; row < p.n_rows; row += gridDim.x) {
    const float mean = p.rms ? 0.0f : p.stats[2 * row], rstd = p.stats[2 * row + 1];
    const float mean_f = p.post && !p.rms ? p.post_stats[2 * row] : 0.0f;
    const float rstd_f = p.post ? p.post_stats[2 * row + 1] : 1.0f;
    Unit<kF16, kEl, true> gy, f, g;
    Unit<kR16, kEl, true> gh, h;
    float w[kEl], wp[kEl], gv[kEl];
    Place<kEl> at;
    auto load = [&](int u, bool all) {
      at = place_unit<kEl>(u, p.width);
      load_unit(gy, row_at<kF16>(p.grad_y, p.ld_gy, row), at, p.width);
      load_unit(h, row_at<kR16>(p.residual, p.ld_residual, row), at, p.width);
      load_vector<true>(p.weight, p.param_bf16, 1.0f, at, p.width, w);
      if (!all) return;
      gh.clear();
      f.clear();
      if (p.grad_h) load_unit(gh, row_at<kR16>(p.grad_h, p.ld_gh, row), at, p.width);
      if (branch) load_unit(f, row_at<kF16>(p.branch, p.ld_branch, row), at, p.width);
      load_vector<true>(p.post_weight, p.param_bf16, 1.0f, at, p.width, wp);
      if (p.gate_matrix) {
        load_unit(g, row_at<kF16>(p.gate, p.ld_gate, row), at, p.width);
#pragma unroll
        for (int j = 0; j < kEl; ++j) gv[j] = g.get(j);
      } else {
        load_vector<true>(p.gate, p.param_bf16, 1.0f, at, p.width, gv);
      }
    };
    auto add = [&](int which, const float (&v)[kEl]) {
      if (!part || !((p.sums >> which) & 1)) return;
      float* const to = part + (long long)which * p.width + at.at;
#pragma unroll
      for (int j = 0; j < kEl; ++j)
        if (owns<true>(at, j)) to[j] = first ? v[j] : to[j] + v[j];
    };
    float v[2] = {0.0f, 0.0f};
    for (int u = threadIdx.x; u < units; u += kWideThreads) {
      load(u, false);
      float dw[kEl], db[kEl];
#pragma unroll
      for (int j = 0; j < kEl; ++j) {
        const bool own = owns<true>(at, j);
        db[j] = own ? gy.get(j) : 0.0f;
        const float xh = own ? (h.get(j) - mean) * rstd : 0.0f;
        dw[j] = db[j] * xh;
        const float qq = db[j] * w[j];
        v[0] = fmaf(qq, xh, v[0]);
        v[1] += qq;
      }
      add(0, dw);
      add(1, db);
    }
    block_row_sums<false>(v, s_sum, 0, kWaves, turn);
    const float c1 = v[0] / width, c0 = p.rms ? 0.0f : v[1] / width;
    auto upstream = [&](int j) {
      const float xh = (h.get(j) - mean) * rstd;
      return fmaf(rstd, fmaf(-xh, c1, gy.get(j) * w[j] - c0), gh.get(j));
    };
    float c1f = 0.0f, c0f = 0.0f;
    if (p.post) {
      float s[2] = {0.0f, 0.0f};
      for (int u = threadIdx.x; u < units; u += kWideThreads) {
        load(u, true);
        float dp[kEl];
#pragma unroll
        for (int j = 0; j < kEl; ++j) {
          const bool own = owns<true>(at, j);
          const float da = own ? upstream(j) * gv[j] : 0.0f;
          const float fh = own ? (f.get(j) - mean_f) * rstd_f : 0.0f;
          dp[j] = da * fh;
          s[0] = fmaf(da * wp[j], fh, s[0]);
          s[1] += da * wp[j];
        }
        add(2, dp);
      }
      block_row_sums<false>(s, s_sum, 0, kWaves, turn);
      c1f = s[0] / width;
      c0f = p.rms ? 0.0f : s[1] / width;
    }
    for (int u = threadIdx.x; u < units; u += kWideThreads) {
      load(u, true);
      float dh[kEl], df[kEl], dg[kEl];
#pragma unroll
      for (int j = 0; j < kEl; ++j) {
        const float t = owns<true>(at, j) ? upstream(j) : 0.0f;
        const float fh = (f.get(j) - mean_f) * rstd_f;
        dh[j] = t * p.scale;
        df[j] = t * gv[j];
        dg[j] = t * (p.post ? fh * wp[j] : f.get(j));
        if (p.post) df[j] = rstd_f * fmaf(-fh, c1f, df[j] * wp[j] - c0f);
      }
      if (!p.gate_matrix && p.gate) add(3, dg);
      Unit<kR16, kEl> out_h;
      Unit<kF16, kEl> out_f, out_g;
      out_h.set(dh);
      out_f.set(df);
      out_g.set(dg);
      out_h.fence();
      out_f.fence();
      out_g.fence();
      char* const to_h = row_at<kR16>(p.out, p.ld_out, row);
      char* const to_f = row_at<kF16>(p.grad_branch, p.ld_gb, row);
      char* const to_g = row_at<kF16>(p.grad_gate, p.ld_gg, row);
      if (p.out) store_edge(out_h, to_h, at);
      if (p.grad_branch) store_edge(out_f, to_f, at);
      if (p.grad_gate) store_edge(out_g, to_g, at);
      if (p.out) store_whole(out_h, to_h, at);
      if (p.grad_branch) store_whole(out_f, to_f, at);
      if (p.grad_gate) store_whole(out_g, to_g, at);
      out_h.keep();
      out_f.keep();
      out_g.keep();
      store_gap();
    }
    first = false;
  }
}

template <bool kF16, bool kR16, bool kRagged, bool kSub, int kUnits>
void launch_block_bwd(const BlockNormParams& p, hipStream_t s) {
  constexpr int kThreads = kSub ? 256 : 512;
  const size_t lds = p.part ? (size_t)p.threads * unit_elements(kF16, kR16) * sizeof(float) : 0;
  constexpr bool kPosts = kUnits * unit_elements(kF16, kR16) <= 8;  // block_norm_shape's choice
#define TURNKL_BLOCK(P, G)                                                       \
  if constexpr (!P || kPosts)                                                    \
    if ((p.post != 0) == P && (p.gate_matrix != 0) == G)                         \
      block_norm_bwd_rows<kF16, kR16, kRagged, kSub, P, G, kUnits, kThreads>     \
          <<<p.n_groups, p.threads, lds, s>>>(p);
  TURNKL_BLOCK(false, false) TURNKL_BLOCK(false, true) TURNKL_BLOCK(true, false) TURNKL_BLOCK(true, true)
#undef TURNKL_BLOCK
}

template <bool kF16, bool kR16, bool kRagged>
hipError_t launch_block_typed(const BlockNormParams& p, bool bwd, hipStream_t s) {
  constexpr bool kWideUnit = unit_elements(kF16, kR16) == 8;
  if (!bwd) {
    if (p.lanes) block_norm_rows<kF16, kR16, kRagged, true, 1, 256><<<p.n_groups, p.threads, 0, s>>>(p);
    else if (p.units == 1) block_norm_rows<kF16, kR16, kRagged, false, 1, 512><<<p.n_groups, p.threads, 0, s>>>(p);
    else if (p.units == 2) block_norm_rows<kF16, kR16, kRagged, false, 2, 512><<<p.n_groups, p.threads, 0, s>>>(p);
    else if (p.units == 0)
      block_norm_wide<kF16, kR16>
          <<<p.n_groups, kWideThreads, ((size_t)p.width + 8) * sizeof(float), s>>>(p);
    else if constexpr (!kWideUnit)
      block_norm_rows<kF16, kR16, kRagged, false, 4, 512><<<p.n_groups, p.threads, 0, s>>>(p);
    return hipGetLastError();
  }
  if (p.lanes) launch_block_bwd<kF16, kR16, kRagged, true, 1>(p, s);
  else if (p.units == 1) launch_block_bwd<kF16, kR16, kRagged, false, 1>(p, s);
  else if (p.units == 2) launch_block_bwd<kF16, kR16, kRagged, false, 2>(p, s);
  else if (p.units == 0) block_norm_bwd_wide<kF16, kR16><<<p.n_groups, kWideThreads, 0, s>>>(p);
  else if constexpr (!kWideUnit) launch_block_bwd<kF16, kR16, kRagged, false, 4>(p, s);
  return hipGetLastError();
}

}  // namespace
}  // namespace turnkl
