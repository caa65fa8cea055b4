// Launch of the block norms (block_norm.h), and the join of their columns' sums.
#include "block_norm.h"

namespace turnkl {
namespace {

// Adds the workgroups' column sums in their order: 64 columns a workgroup, sixteen runs of
// partial rows side by side; blockIdx.y: which of the sums.
constexpr int kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void block_norm_join(BlockNormParams p) {
  constexpr int kRuns = kJoinThreads / kWave;
  __shared__ float s_run[kRuns][kWave];
  const int lane = threadIdx.x & (kWave - 1);
  const int run = threadIdx.x / kWave;
  const int col = blockIdx.x * kWave + lane;
  float* const out = blockIdx.y == 0 ? p.gw : blockIdx.y == 1 ? p.gbias : blockIdx.y == 2 ? p.gpost : p.ggate;
  if (!out) return;
  float s = 0.0f;
  if (col < p.width) {
    const float* at = p.part + (long long)blockIdx.y * p.width + col;
    const int lo = (int)((long long)p.n_groups * run / kRuns), hi = (int)((long long)p.n_groups * (run + 1) / kRuns);
#pragma unroll 8
    for (int i = lo; i < hi; ++i) s += at[(long long)i * 4 * p.width];
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

}  // namespace

// How rows are laid out over the threads: rows of up to 64 units a part of a wave, wider
// ones a workgroup with one unit a thread while that takes few waves, then two, then four.
// Rows past 8,192 elements, and backward past 4,096 where the branch is normalised, would
// not fit the registers (backward with both norms, 8 bf16 elements a thread take 162 of the
// 256 that two waves a SIMD leave each): they are not held (units 0).
//
// Measured with 4,096 bf16 columns, both norms and a vector's gate.  Forward, 512 units:
// two a thread 437 us (12 waves a CU; 8: 440, 16: 486), one a thread 449 (456 with 16
// waves, 511 with 8 or 12, 473 with 24, 481 with 32).  Backward, one a thread: 417 with 8
// or 12 waves a CU, 424 with 16, 431 with 24, 437 with 32.
BlockShape block_norm_shape(long long n_rows, long long width, int el, bool bwd, bool post) {
  const int units = (int)((width + el - 1) / el);
  BlockShape s{};
  s.units = 1;
  int side = 1;
  if (units <= kWave) {
    s.lanes = 1;
    while (s.lanes < units) s.lanes *= 2;
    s.threads = 256;
    side = s.threads / s.lanes;
  } else if (width > 8192 || (bwd && post && width > 4096)) {
    s.units = 0;
    s.threads = 512;
  } else {
    s.units = units <= (bwd ? 512 : 256) ? 1 : units <= 1024 ? 2 : 4;
    s.threads = ((units + s.units - 1) / s.units + kWave - 1) / kWave * kWave;
  }
  const int waves = s.threads / kWave;
  const int most = (bwd ? el == 8 && post : s.units == 2) ? 12 : 16;  // waves of a CU
  const int fill = 256 * (most / waves > 1 ? most / waves : 1);
  const long long per = (bwd ? 2 : 1) * (long long)side;
  const long long g = (n_rows + per - 1) / per;
  s.groups = (int)(g < 1 ? 1 : g < fill ? g : fill);
  return s;
}

hipError_t launch_block_norm(const BlockNormParams& given, bool bwd, hipStream_t s) {
  BlockNormParams p = given;
  if (p.n_rows == 0) {
    p.n_groups = 0;  // no row, no partial sums: the join's are zeros
  } else {
    const hipError_t e = p.branch_bf16 ? (p.residual_bf16 ? launch_block_norm_bf16(p, bwd, s)
                                                          : launch_block_norm_mixed(p, bwd, s))
                                       : launch_block_norm_f32(p, bwd, s);
    if (e != hipSuccess) return e;
  }
  if (!bwd || !p.sums) return hipSuccess;
  block_norm_join<<<dim3((p.width + kWave - 1) / kWave, 4), kJoinThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace turnkl
