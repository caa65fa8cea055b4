// A token sampled from each row of logits, with temperature, top-k, top-p and min-p, from
// given random numbers.
//
// Math.  w_v = exp((z_v - M) / T), M = max z.  In the order of descending logits, the lower
// id first among equal ones, the support is a prefix: the first k; of those the ones whose
// predecessors hold less than p of their mass; of those the ones with w >= min_p; the first
// one always.  The token is the first of the support, in the order of ids, whose running sum
// of w exceeds u times the support's.  Which token that is hangs on comparisons of sums, so
// weights and sums have 64 bits: with 32, where a row is flat, one row in a hundred would
// get a neighbour of its token.
//
// sample_scan goes over the logits once: a wave takes a segment of 2,048 elements and leaves
// its maximum and, where the row's filters need the mass of the whole row, its sum of
// weights; of rows with a filter also the largest of every lane's 32 elements (a unit), by
// its upper 16 bits.  sample_pick joins a row's segments, a workgroup a row.  Without a
// filter it looks for the segment where the running sum passes the bound and reads that one
// again.  With one it needs the elements at the top of the row only: the n-th largest unit
// maximum is a bound that at least n elements reach, units that reach it are read again, and
// up to 1,024 such elements are ranked against each other.  Where that is not enough (flat
// rows, long runs of equal logits) a histogram over the row shows between which logits the
// border lies, the mass above them is summed exactly, and the border is found bit by bit
// among the elements between them.

#include <type_traits>

#include "row_span.h"

namespace turnkl {
namespace {

constexpr int kScanThreads = 256;
constexpr int kScanWaves = kScanThreads / kWave;
constexpr int kSegElems = kSampleSegment;
constexpr int kPickThreads = 512;
constexpr int kPickWaves = kPickThreads / kWave;
constexpr int kRankEach = 2;                           // of a thread
constexpr int kRanked = kRankEach * kPickThreads;      // candidates that are sorted
constexpr int kUnitElems = kSegElems / kWave;
constexpr int kUnitsHeld = 2048;  // units that are read again, at most
constexpr int kUnitEach = 16;     // units of a thread that its registers hold
// Elements that are asked for where only top-p limits a row: 64 rows of 151,936 with settings
// of their own take 173, 164 and 166 us with 400, 600 and 800 (with 300 units 172), 512 rows
// of 32,000 at top-p 0.9 153, 126 and 133.  As many units would be more than a row of 5,752
// has, whose candidates would then be all its elements: 39 such rows 53 us, for 28.
constexpr double kWantByMass = 600;
constexpr int kBins = 2 * kPickThreads;                // of the histogram
constexpr int kBinEach = 8;                            // elements of a lane between two bins' edges
constexpr int kBinHeld = kBinEach * kWave;             // of a wave

// The logit's bits in an order of unsigned numbers (-0 and +0 alike, NaN as -inf).
__device__ inline unsigned order_of(float z) {
  const unsigned u = __float_as_uint((z == z ? z : -INFINITY) + 0.0f);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ inline float logit_of(unsigned o) {
  return __uint_as_float(o ^ ((unsigned)((int)~o >> 31) | 0x80000000u));
}
constexpr unsigned kNothing = 0x007FFFFFu;  // the order of -inf
constexpr double kLog2e64 = 1.4426950408889634074;
constexpr double kLn264 = 0.69314718055994530942;

// 2^r on [-1/2, 1/2]: a polynomial through 2^r at eleven Chebyshev points and 0, where it is
// exact; elsewhere it is off by 2e-17.
__device__ __forceinline__ double pow2_fraction(double r) {
  double s = 4.4549794711760616e-10;
  s = fma(s, r, 7.072621356539349e-09);
  s = fma(s, r, 1.0178062351388103e-07);
  s = fma(s, r, 1.3215442410711872e-06);
  s = fma(s, r, 1.525273382999124e-05);
  s = fma(s, r, 0.0001540353044202707);
  s = fma(s, r, 0.0013333558146416842);
  s = fma(s, r, 0.009618129107606715);
  s = fma(s, r, 0.0555041086648216);
  s = fma(s, r, 0.24022650695910097);
  s = fma(s, r, 0.6931471805599453);
  return fma(s, r, 1.0);
}
// 2^x for x <= 0
__device__ __forceinline__ double pow2(double x) {
  x = fmax(x, -1100.0);  // 0 from there on, -inf included
  const double n = rint(x);
  return ldexp(pow2_fraction(x - n), (int)n);
}
// the same for -1020 <= x <= 0: x's integer part comes out of an addition that leaves no
// bits for a fraction, in the sum's low word, and goes straight into the exponent
__device__ __forceinline__ double pow2_tame(double x) {
  const double kRound = 6755399441055744.0;  // 1.5 2^52
  const double t = x + kRound;
  const double f = pow2_fraction(x - (t - kRound));
  const int hi = __double2hiint(f) + (__double2loint(t) << 20);
  return __hiloint2double(hi, __double2loint(f));
}

// e^x for x <= 0: 2^t for t = x log2 e, and the part of t that its rounding lost in the
// slope of 2^t (an argument of -30 is rounded by up to 2^-20)
__device__ __forceinline__ float exp_fast(float x) {
  constexpr float kLow = (float)(kLog2e64 - (double)kLog2e);
  x = fmaxf(x, -1e4f);  // 0 from there on, -inf included
  const float t = x * kLog2e;
  const float lost = fmaf(x, kLow, fmaf(x, kLog2e, -t));
  const float e = exp2_fast(t);
  return fmaf(e, lost * (float)kLn264, e);
}

// What a row's parameters ask for.
struct Plan {
  double rate;      // log2 e / T
  int k;            // elements that count, 0: all
  float p, min_p;   // 1 and 0 where they do not limit
  bool bad;
  bool filtered;
  bool mass;        // the mass of the whole row is needed
};
__device__ inline Plan plan_of(const SampleParams& s, long long row) {
  const float t = s.row_temperature ? s.row_temperature[row] : s.temperature;
  const float p = s.row_top_p ? s.row_top_p[row] : s.top_p;
  const float m = s.row_min_p ? s.row_min_p[row] : s.min_p;
  const int k = s.row_top_k ? s.row_top_k[row] : s.top_k;
  Plan a;
  a.bad = !(t >= 0.0f && t < INFINITY) || !(p >= 0.0f) || !(m >= 0.0f);
  const bool first = t == 0.0f || p == 0.0f;  // the likeliest one alone
  a.rate = kLog2e64 / (t == 0.0f ? 1.0 : (double)t);
  a.k = first ? 1 : k <= 0 || k >= s.vocab ? 0 : k;
  a.p = first ? 1.0f : fminf(p, 1.0f);
  a.min_p = first ? 0.0f : fminf(m, 1.0f);
  a.filtered = a.k > 0 || a.p < 1.0f || a.min_p > 0.0f;
  a.mass = a.k == 0 && (a.p < 1.0f || a.min_p == 0.0f);
  return a;
}

// The segments of a row, on the grid of the 128-byte lines it lies on.
template <bool kBf16, bool kRagged>
struct Row {
  using Span = RowSpan<kBf16, kRagged>;
  using P = typename Span::P;
  static constexpr int kEpv = Span::kEpv;
  static constexpr int kPacks = kSegElems / (kWave * kEpv);  // of a lane
  Span span;
  int pre;

  __device__ __forceinline__ Row(const SampleParams& p, long long row) {
    const char* const at = static_cast<const char*>(p.z) + row * p.ld * Span::kEs;
    pre = kRagged ? (int)(reinterpret_cast<uintptr_t>(at) & 127u) / Span::kEs : 0;
    span = Span{at, chunk_rsrc(at), p.vocab, -pre, (pre + p.vocab + kEpv - 1) / kEpv};
  }
  // a lane's pack q of segment g: its first element, and which are its own
  __device__ __forceinline__ int place(int g, int q, unsigned& bits) const {
    return span.place((g * kPacks + q) * kWave + (threadIdx.x & (kWave - 1)), bits);
  }
  __device__ __forceinline__ void load(int g, P (&x)[kPacks], int (&at)[kPacks], unsigned (&bits)[kPacks]) const {
#pragma unroll
    for (int q = 0; q < kPacks; ++q) {
      at[q] = place(g, q, bits[q]);
      span.load(x[q], at[q]);
    }
  }
};

// The sum of a wave's lanes up to and with this one, by data-parallel moves between lanes
// (through LDS a step takes ten times as long), and of all lanes.
template <int kCtrl, int kRows>
__device__ __forceinline__ double lane_move64(double v) {
  return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), kCtrl, kRows, 0xF, false),
                          __builtin_amdgcn_update_dpp(0, __double2loint(v), kCtrl, kRows, 0xF, false));
}
__device__ __forceinline__ double wave_scan64(double v) {
  v += lane_move64<0x111, 0xF>(v);  // row_shr:1, 2, 4, 8
  v += lane_move64<0x112, 0xF>(v);
  v += lane_move64<0x114, 0xF>(v);
  v += lane_move64<0x118, 0xF>(v);
  v += lane_move64<0x142, 0xA>(v);  // row_bcast:15 into rows 1 and 3
  v += lane_move64<0x143, 0xC>(v);  // row_bcast:31 into rows 2 and 3
  return v;
}
__device__ __forceinline__ double last_lane64(double v) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), kWave - 1),
                          __builtin_amdgcn_readlane(__double2loint(v), kWave - 1));
}
__device__ __forceinline__ double wave_sum64(double v) { return last_lane64(wave_scan64(v)); }
template <int kCtrl, int kRows>
__device__ __forceinline__ int larger_of_lane(int v) {
  const int u = __builtin_amdgcn_update_dpp(v, v, kCtrl, kRows, 0xF, false);
  return u > v ? u : v;
}
__device__ __forceinline__ int wave_largest(int v) {
  v = larger_of_lane<0x111, 0xF>(v);
  v = larger_of_lane<0x112, 0xF>(v);
  v = larger_of_lane<0x114, 0xF>(v);
  v = larger_of_lane<0x118, 0xF>(v);
  v = larger_of_lane<0x142, 0xA>(v);
  v = larger_of_lane<0x143, 0xC>(v);
  return __builtin_amdgcn_readlane(v, kWave - 1);
}

// The largest of three, NaN where one is.
__device__ __forceinline__ float most3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// Bound: the 64-bit exponentials, some twenty operations an element (they run at the
// rate of 32-bit ones here): 1,024 rows of 151,936 in 136 us, of which HBM would need 48;
// of rows that only top-k or min-p limits log p's sum (300 fp32 rows of 50,257: 19 us).
// The next task's loads ahead of a wave's sums gave nothing: other waves fill their time.
template <bool kBf16, bool kRagged>
__global__ __launch_bounds__(kScanThreads) void sample_scan(SampleParams p) {
  using R = Row<kBf16, kRagged>;
  const int lane = threadIdx.x & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (p.first_row == 0 && blockIdx.x == 0 && threadIdx.x == 0) p.hdr->err_key = kNoError;
  // a segment a wave: task = row of this launch x segment
  const unsigned index = blockIdx.x * kScanWaves + wid;
  const unsigned of_launch = index / (unsigned)p.n_segs;
  const int g = (int)(index - of_launch * (unsigned)p.n_segs);
  const long long row = p.first_row + of_launch;
  if (row >= p.n_rows || (p.mask && !p.mask[row])) return;
  const long long task = row * p.n_segs + g;
  const Plan plan = plan_of(p, row);
  if (plan.bad) return;
  const R r(p, row);
  typename R::P x[R::kPacks];
  int at[R::kPacks];
  unsigned bits[R::kPacks];
  r.load(g, x, at, bits);
  auto sums = [&](auto edge) {
    constexpr bool kEdge = decltype(edge)::value;
    auto value = [&](int q, int j) {
      return !kEdge || ((bits[q] >> j) & 1u) ? x[q].get(j) : -INFINITY;
    };
    float best = -INFINITY;
#pragma unroll
    for (int q = 0; q < R::kPacks; ++q) {
#pragma unroll
      for (int j = 0; j < R::kEpv; j += 2) best = most3(best, value(q, j), value(q, j + 1));
      x[q].fence();
    }
    const bool none = __any(best != best);  // one is no number
    if (plan.filtered) p.unit[task * kWave + lane] = (unsigned short)(order_of(best) >> 16);
    const float m = none ? __builtin_nanf("") : wave_max_dpp(best);
    double mass = 0.0;
    double sum = 0.0;
    const bool numbers = fabsf(m) < INFINITY;
    if (plan.mass && numbers) {
      const double shift = -(double)m * plan.rate;
      // Nothing below 2^-1000 counts: -inf is taken for this number.  (Where temperatures
      // are so high that it has none, from 4.9e35, x would have to be -inf itself.)
      const float low = (float)((double)m - 1000.0 / plan.rate);
      if (plan.rate <= 0x1p20 && fabs(shift) <= 1024.0 && low > -INFINITY) {
        // x = z rate - m rate
#pragma unroll
        for (int q = 0; q < R::kPacks; ++q) {
#pragma unroll
          for (int j = 0; j < R::kEpv; ++j) {
            mass += pow2_tame(fma((double)fmaxf(value(q, j), low), plan.rate, shift));
            if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // not all 64-bit numbers at once
          }
          x[q].fence();
        }
        // What the maximum's product lost by its rounding (6e-14 at most) is a factor of the
        // whole segment: 2^-lost, of which its first two terms leave 1e-27.
        const double lost = fma((double)m, plan.rate, shift);
        mass = fma(mass, lost * -kLn264, mass);
      } else {
#pragma unroll
        for (int q = 0; q < R::kPacks; ++q)
#pragma unroll
          for (int j = 0; j < R::kEpv; ++j) {
            mass += pow2(((double)value(q, j) - (double)m) * plan.rate);
            __builtin_amdgcn_sched_barrier(0);
          }
      }
      mass = wave_sum64(mass);
    }
    if (p.logp && numbers && !(plan.mass && plan.rate == kLog2e64)) {
      // 32-bit exponentials of arguments with their rounding, added in 64 bits: where one
      // token has nearly all of a row, log p is what the others add to 1
#pragma unroll
      for (int q = 0; q < R::kPacks; ++q) {
#pragma unroll
        for (int j = 0; j < R::kEpv; ++j) {
          sum += (double)exp_fast(value(q, j) - m);
          if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
      }
      sum = wave_sum64(sum);
    }
    if (lane == 0) {
      p.seg_max[task] = m;
      p.seg_sum[task] = sum;
      p.seg_mass[task] = mass;
    }
  };
  const int first = g * kSegElems - r.pre;
  if (first >= 0 && first + kSegElems <= p.vocab) sums(std::false_type{});
  else sums(std::true_type{});
}

// ---------------------------------------------------------------------------
// picking

// A workgroup's sums and scans in a fixed order, through LDS that alternates between two
// halves: one barrier each.
struct Group {
  double (*lds)[kPickWaves * 3];  // LDS, two of them
  int (*ilds)[kPickWaves * 3];
  int turn = 0;

  template <int kN>
  __device__ __forceinline__ void sums(double (&v)[kN]) {
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = wave_sum64(v[i]);
    if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
      for (int i = 0; i < kN; ++i) lds[turn][threadIdx.x / kWave * kN + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      v[i] = lds[turn][i];
#pragma unroll
      for (int w = 1; w < kPickWaves; ++w) v[i] += lds[turn][w * kN + i];
    }
  }
  template <int kN>
  __device__ __forceinline__ void sums(int (&v)[kN]) {
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < kN; ++i) wave_exclusive_dpp(v[i], &v[i]);
    if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
      for (int i = 0; i < kN; ++i) ilds[turn][threadIdx.x / kWave * kN + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      v[i] = ilds[turn][i];
#pragma unroll
      for (int w = 1; w < kPickWaves; ++w) v[i] += ilds[turn][w * kN + i];
    }
  }
  template <typename V>
  __device__ __forceinline__ V sum(V v) {
    V one[1] = {v};
    sums(one);
    return one[0];
  }
  // the sum of the threads up to and with this one; *total: of all
  __device__ __forceinline__ double scan(double v, double* total) {
    turn ^= 1;
    const int lane = threadIdx.x & (kWave - 1), wid = threadIdx.x / kWave;
    v = wave_scan64(v);
    if (lane == kWave - 1) lds[turn][wid] = v;
    __syncthreads();
    double before = 0.0, all = 0.0;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) {
      const double s = lds[turn][w];
      before += w < wid ? s : 0.0;
      all += s;
    }
    *total = all;
    return before + v;
  }
  // the sum of the threads before this one
  __device__ __forceinline__ int scan(int v, int* total) {
    turn ^= 1;
    const int wid = threadIdx.x / kWave;
    int all_wave;
    const int mine = wave_exclusive_dpp(v, &all_wave);
    if ((threadIdx.x & (kWave - 1)) == 0) ilds[turn][wid] = all_wave;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) {
      const int s = ilds[turn][w];
      before += w < wid ? s : 0;
      all += s;
    }
    *total = all;
    return before + mine;
  }
  __device__ __forceinline__ int largest(int v) {
    turn ^= 1;
    v = wave_largest(v);
    if ((threadIdx.x & (kWave - 1)) == 0) ilds[turn][threadIdx.x / kWave] = v;
    __syncthreads();
    int m = ilds[turn][0];
#pragma unroll
    for (int w = 1; w < kPickWaves; ++w) m = ilds[turn][w] > m ? ilds[turn][w] : m;
    return m;
  }
};
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_wave_barrier();
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// Sorts the first `n` numbers of LDS, a power of two up to 2 kPickThreads, in descending
// order: bitonic, a pair a thread; pairs up to 64 apart stay within 128 numbers that are one
// wave's.
__device__ __forceinline__ void sort_down(unsigned long long* s, int n) {
  const int t = threadIdx.x;
  __syncthreads();
  for (int run = 2; run <= n; run *= 2) {
    for (int apart = run / 2; apart > 0; apart /= 2) {
      if (t < n / 2) {
        const int i = 2 * t - (t & (apart - 1)), j = i + apart;
        const unsigned long long a = s[i], b = s[j];
        const bool down = (i & run) == 0;
        if ((a < b) == down) {
          s[i] = b;
          s[j] = a;
        }
      }
      // (of the next pairs; the first of a longer run are half of it apart)
      const int next = apart > 1 ? apart / 2 : run;
      if (next > kWave || apart > kWave) __syncthreads();
      else wave_lds_order();
    }
  }
  __syncthreads();
}
// the least power of two that is n or more, 2 at least
__device__ __forceinline__ int power_of(int n) { return n <= 2 ? 2 : 1 << (32 - __clz(n - 1)); }

// orders as signed numbers of the same order
__device__ __forceinline__ int signed_order(unsigned o) { return (int)(o ^ 0x80000000u); }
__device__ __forceinline__ unsigned unsigned_order(int o) { return (unsigned)o ^ 0x80000000u; }

// Where a support ends: orders above `order`, and at it ids up to `id`.
struct Border {
  unsigned order;
  int id;
};

// A row being picked from.  All threads of the workgroup call every function.
template <bool kBf16, bool kRagged>
struct Pick {
  using R = Row<kBf16, kRagged>;
  const SampleParams& p;
  const R row;
  const Plan plan;
  Group& group;
  const long long first;  // segment
  float m;                // M
  int* found;             // LDS, 4
  double* held;           // LDS, 1 + kPickWaves

  __device__ __forceinline__ double weight(float z) const { return pow2(((double)z - (double)m) * plan.rate); }
  // the same of logits whose weight is 2^-1000 at least
  __device__ __forceinline__ double weight_tame(float z) const {
    return pow2_tame(((double)z - (double)m) * plan.rate);
  }

  // Goes through the row, a wave a segment in turn, the next one on its way: hands each
  // lane's packs to use(values, -inf for those that are not own ones, the id of the first),
  // and after a segment calls end(g).
  template <typename F, typename E>
  __device__ __forceinline__ void walk(F use, E end) const {
    typename R::P x[R::kPacks], next[R::kPacks];
    int at[R::kPacks];
    unsigned bits[R::kPacks];
    int g = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (g < p.n_segs) row.load(g, next, at, bits);
#pragma unroll 1
    for (; g < p.n_segs; g += kPickWaves) {
#pragma unroll
      for (int q = 0; q < R::kPacks; ++q) x[q] = next[q];
      if (g + kPickWaves < p.n_segs) row.load(g + kPickWaves, next, at, bits);
#pragma unroll
      for (int q = 0; q < R::kPacks; ++q) {
        at[q] = row.place(g, q, bits[q]);
        float z[R::kEpv];
#pragma unroll
        for (int j = 0; j < R::kEpv; ++j) z[j] = (bits[q] >> j) & 1u ? x[q].get(j) : -INFINITY;
        use(z, at[q]);
        __builtin_amdgcn_sched_barrier(0);  // not all packs' 64-bit numbers at once
      }
      end(g);
    }
  }
  // Hands the elements of segment g to use(value, id, whether it is an own one) in all lanes.
  template <typename F>
  __device__ __forceinline__ void each_of(int g, F use) const {
    typename R::P x[R::kPacks];
    int at[R::kPacks];
    unsigned bits[R::kPacks];
    row.load(g, x, at, bits);
#pragma unroll
    for (int q = 0; q < R::kPacks; ++q)
#pragma unroll
      for (int j = 0; j < R::kEpv; ++j) {
        use(x[q].get(j), at[q] + j, ((bits[q] >> j) & 1u) != 0);
        if (j % 2 == 1) __builtin_amdgcn_sched_barrier(0);  // not all elements' 64-bit numbers at once
      }
  }
  // The same for all segments whose maximum reaches `least`, a wave each in turn.
  template <typename F>
  __device__ __forceinline__ void each(unsigned least, F use) const {
    for (int g = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); g < p.n_segs; g += kPickWaves)
      if (order_of(p.seg_max[first + g]) >= least) each_of(g, use);
  }

  // The first id where the running sum of value(z, id) passes target_of(total), when a
  // segment's share of it is share(g); *total: of all shares.
  template <typename Target, typename Share, typename Value>
  __device__ __forceinline__ int by_segment(Target target_of, Share share, Value value, double* total) {
    // a run of segments a thread, so that the threads are in the order of ids
    const int run_of = (p.n_segs + kPickThreads - 1) / kPickThreads;
    const int lo = threadIdx.x * run_of;
    const int hi = lo + run_of < p.n_segs ? lo + run_of : p.n_segs;
    double mine = 0.0;
    int last = -1;  // the last one with a share
    for (int g = lo; g < hi; ++g) {
      const double s = share(g);
      mine += s;
      if (s > 0.0) last = g;
    }
    if (threadIdx.x == 0) *found = 0x7FFFFFFF;
    double all;
    const double upto = group.scan(mine, &all);
    *total = all;
    const double target = target_of(all);
    last = group.largest(last);
    // (A scan's sums are made in trees of their own: at a border the one of a thread without
    // a share may pass it by a rounding.  Such threads, and below such segments and lanes,
    // are never the place, so that a rounding leads to a border's other side at most.)
    int* const slot = found;
    if (mine > 0.0 && upto > target) atomicMin(slot, (int)threadIdx.x);
    __syncthreads();
    const int who = *found;
    if (who == 0x7FFFFFFF) {  // past the end by a rounding
      if (threadIdx.x == 0) {
        found[1] = last;
        held[0] = -1.0;
      }
    } else if ((int)threadIdx.x == who) {
      double run = upto - mine, before = run;
      int at = lo;
      for (int g = lo; g < hi; ++g) {
        const double s = share(g);
        if (!(s > 0.0)) continue;
        at = g;
        before = run;
        run += s;
        if (run > target) break;
      }
      found[1] = at;
      held[0] = fmax(target - before, 0.0);
    }
    __syncthreads();
    const int g = found[1];
    const double rest = held[0];
    // a wave for each lane's pack, in the order of ids
    const int lane = threadIdx.x & (kWave - 1);
    const int q = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    static_assert(R::kPacks <= kPickWaves, "a wave for each pack");
    double w[R::kEpv], s = 0.0, upto_lane = 0.0;
    int at = 0, end = -1;
    if (q < R::kPacks) {
      unsigned bits;
      typename R::P x;
      at = row.place(g, q, bits);
      row.span.load(x, at);
#pragma unroll
      for (int j = 0; j < R::kEpv; ++j) {
        w[j] = (bits >> j) & 1u ? value(x.get(j), at + j) : 0.0;
        s += w[j];
        if (w[j] > 0.0) end = at + j;
        if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
      upto_lane = wave_scan64(s);
      if (lane == kWave - 1) held[1 + q] = upto_lane;
    }
    if (threadIdx.x == 0) found[2] = 0x7FFFFFFF;
    end = group.largest(end);  // (has a barrier)
    if (q < R::kPacks) {
      double run = 0.0;
      for (int i = 0; i < q; ++i) run += held[1 + i];
      const unsigned long long past = __ballot(rest >= 0.0 && s > 0.0 && run + upto_lane > rest);
      if (past && lane == __ffsll((long long)past) - 1) {
        int got = -1;
        double t = run + (upto_lane - s);
#pragma unroll
        for (int j = 0; j < R::kEpv; ++j) {
          if (w[j] > 0.0 && (got < 0 || t <= rest)) got = at + j;
          t += w[j];
        }
        int* const slot = found + 2;
        if (got >= 0) atomicMin(slot, got);
      }
    }
    __syncthreads();
    return found[2] < 0x7FFFFFFF ? found[2] : end;
  }
};

// The support of a row at large.
template <bool kBf16, bool kRagged>
struct Wide {
  using R = Row<kBf16, kRagged>;
  Pick<kBf16, kRagged>& row;
  unsigned* bins;               // LDS, kBins + kWave
  unsigned long long* between;  // LDS, kPickWaves x kBinHeld

  // What locate() found last: its elements between two edges, in their lanes' hands (of a
  // wave's segments the wave's lanes), and whether seg_mass holds what lies above them.
  bool in_hand = false, by_segment = false;
  unsigned order[kBinEach];  // 0: none
  int id[kBinEach];
  double w[kBinEach];

  __device__ __forceinline__ int wave() const { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); }

  // The largest order that at least `target` elements (kCount) reach, or elements of at
  // least that mass; *above: how many, or what mass, lies above it.  kNothing where all
  // finite elements together are too few.
  //
  // A histogram of 1,024 bins gives the bin that holds the border (of the mass: nearly
  // always; what is above the bin is then summed exactly, and a neighbour is taken if need
  // be), and up to 512 elements a wave in the bin are put aside, in a fixed order.  If they
  // are more, the bin is cut into 1,024 again.
  template <bool kCount>
  __device__ __forceinline__ unsigned locate(double target, double* above) {
    Group& group = row.group;
    const SampleParams& p = row.p;
    const int tid = threadIdx.x;
    const int lane = tid & (kWave - 1);
    unsigned lo = kNothing + 1u, hi = order_of(row.m);  // orders that are looked at
    double over = 0.0;                                  // what lies above them
#pragma unroll 1
    for (int level = 0;; ++level) {
      // First by the logits' distance from the maximum, 1 / 16 of a power of two of weight
      // a bin and whatever is further down in the last one, then by their orders.
      constexpr float kWidth = 0.0625f;
      int shift = 0;
      while ((hi - lo) >> shift >= kBins) ++shift;
      const float per = (float)fmin(row.plan.rate * (1.0 / kWidth), 3e38);
      auto bin_of = [&](float z) {
        if (level > 0) return (int)((hi - order_of(z)) >> shift);
        const float x = (row.m - z) * per;
        return x < kBins - 1 ? (int)x : kBins - 1;
      };
      // the least order in bins up to b
      auto edge = [&](int b) {
        if (b < 0) return hi + 1u;
        unsigned t = lo, n = hi - lo;
        while (n > 0) {  // (the order hi is in bin 0)
          const unsigned half = n / 2;
          if (bin_of(logit_of(t + half)) <= b) {
            n = half;
          } else {
            t += half + 1u;
            n -= half + 1u;
          }
        }
        return t;
      };
      __syncthreads();
      for (int i = tid; i < kBins; i += kPickThreads) bins[i] = 0u;
      __syncthreads();
      // of masses in parts of the weight at the bin's edge, as many as all elements together
      // leave room for
      const float part = fminf(2147483648.0f / p.vocab, 65536.0f);
      // (what is not looked at goes to bins of the lanes' own, which takes no branch)
      const float from = logit_of(lo), to = logit_of(hi);
      auto fill = [&](auto first) {
        constexpr bool kFirst = decltype(first)::value;
        row.walk(
            [&](const float (&z)[R::kEpv], int) {
#pragma unroll
            for (int j = 0; j < R::kEpv; ++j) {
              unsigned n = 1;
              int b;
              if constexpr (kFirst) {
                // (2^-x within a bin by its chord)
                const float x = fminf((row.m - z[j]) * per, (float)(kBins - 1));
                b = (int)x;
                if constexpr (!kCount)
                  n = (unsigned)fmaf(x - truncf(x), part * -0.04239f, part + 0.5f);
                b = z[j] >= from ? b : kBins + lane;
              } else {
                b = z[j] >= from && z[j] <= to ? (int)((hi - order_of(z[j])) >> shift) : kBins + lane;
              }
              unsigned* const slot = bins + b;
              atomicAdd(slot, n);
            }
            },
            [](int) {});
      };
      if (level == 0) fill(std::true_type{});
      else fill(std::false_type{});
      __syncthreads();
      double v[2];
      int filled = -1;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int b = 2 * tid + i;
        const unsigned n = bins[b];
        if (n) filled = b;
        v[i] = n;
        if constexpr (!kCount) {
          if (n) v[i] *= level == 0 ? pow2(-(double)(b * kWidth)) / part
                                    : row.weight(logit_of(hi - ((unsigned)b << shift)));
        }
      }
      if (tid == 0) *row.found = 0x7FFFFFFF;
      double all;
      const double upto = over + group.scan(v[0] + v[1], &all);
      const int last = group.largest(filled);
      if (kCount && level == 0 && all < target) {
        *above = all;
        return kNothing;
      }
      int* const slot = row.found;
      if (upto >= target) atomicMin(slot, upto - v[1] >= target ? 2 * tid : 2 * tid + 1);
      __syncthreads();
      int bin = *row.found < last ? *row.found : last;
      int moved = 0;
#pragma unroll 1
      for (;;) {
        // what lies above the bin, segment by segment, and its elements
        const unsigned upper = edge(bin - 1), lower = edge(bin);
        const float upper_z = logit_of(upper), lower_z = logit_of(lower);
        const bool tame = ((double)row.m - (double)lower_z) * row.plan.rate < 1000.0;
        double sum[2] = {0.0, 0.0};
        int held = 0;  // of this wave
        int least = 0x7FFFFFFF, most = -0x7FFFFFFF - 1;
        double mine = 0.0;
        auto add = [&](auto tamed) {
          row.walk(
              [&](const float (&z)[R::kEpv], int i) {
                unsigned in = 0;
#pragma unroll
                for (int j = 0; j < R::kEpv; ++j) {
                  const bool above = z[j] >= upper_z, here = z[j] >= lower_z && !above;
                  double v = 1.0;
                  if constexpr (!kCount) {
                    const float near = fmaxf(z[j], lower_z);  // others' weights are not used
                    if constexpr (decltype(tamed)::value) v = row.weight_tame(near);
                    else v = row.weight(near);
                  }
                  mine += above ? v : 0.0;
                  sum[1] += here ? v : 0.0;
                  in |= here ? 1u << j : 0u;
                }
                if (!__any(in != 0u)) return;
                int all;
                int to = held + wave_exclusive_dpp(__popc(in), &all);
                held += all;
                for (; in; in &= in - 1, ++to) {
                  const int j = __ffs((int)in) - 1;
                  float one = z[0];
#pragma unroll
                  for (int k = 1; k < R::kEpv; ++k) one = k == j ? z[k] : one;
                  const unsigned o = order_of(one);
                  const int so = signed_order(o);
                  least = so < least ? so : least;
                  most = so > most ? so : most;
                  if (to < kBinHeld) between[wave() * kBinHeld + to] = ((unsigned long long)o << 32) | (unsigned)(i + j);
                }
              },
              [&](int g) {
                sum[0] += mine;
                if constexpr (!kCount) {
                  mine = wave_sum64(mine);
                  if (lane == 0) p.seg_mass[row.first + g] = mine;
                }
                mine = 0.0;
              });
        };
        if (tame) add(std::true_type{});
        else add(std::false_type{});
        group.sums(sum);
        const double before = sum[0];
        most = group.largest(most);
        least = ~group.largest(~least);
        // (A target between this bin's sums and the same elements' sum from the next bin on
        // would end a search between the two, where the bin may be empty: the direction is
        // kept until one is not, as the first and the last one are not.)
        const bool empty = least > most;
        if (moved <= 0 && bin > 0 && (before >= target || (empty && moved < 0))) {
          --bin;
          moved = -1;
          continue;
        }
        if (moved >= 0 && bin < last && (before + sum[1] < target || empty)) {
          ++bin;
          moved = 1;
          continue;
        }
        by_segment = !kCount;
        in_hand = group.largest(held) <= kBinHeld;
        if (!in_hand) {
          if (least == most) {  // equal, however many
            *above = before;
            return unsigned_order(least);
          }
          over = before;
          lo = unsigned_order(least);
          hi = unsigned_order(most);
          break;
        }
#pragma unroll
        for (int q = 0; q < kBinEach; ++q) {
          const int i = q * kWave + lane;
          const unsigned long long x = i < held ? between[wave() * kBinHeld + i] : 0ull;
          order[q] = (unsigned)(x >> 32);
          id[q] = (int)(unsigned)x;
          w[q] = i >= held ? 0.0 : kCount ? 1.0 : row.weight(logit_of(order[q]));
        }
        // the largest order bit by bit, two at a time
        unsigned t = 0;
#pragma unroll 1
        for (int b = 30; b >= (kBf16 ? 16 : 0); b -= 2) {
          double n[3] = {0.0, 0.0, 0.0};
#pragma unroll
          for (int q = 0; q < kBinEach; ++q)
#pragma unroll
            for (unsigned d = 0; d < 3; ++d) n[d] += order[q] >= (t | ((d + 1) << b)) ? w[q] : 0.0;
          group.sums(n);
          t |= (before + n[2] >= target ? 3u : before + n[1] >= target ? 2u : before + n[0] >= target ? 1u : 0u) << b;
        }
        // (of bf16 logits the lower half follows from the upper one: all ones below zero;
        // past an end by a rounding: the least or the largest one)
        t = !t ? unsigned_order(least) : kBf16 && !(t >> 31) ? t | 0xFFFFu : t;
        t = t < unsigned_order(most) ? t : unsigned_order(most);
        double n = 0.0;
#pragma unroll
        for (int q = 0; q < kBinEach; ++q) n += order[q] > t ? w[q] : 0.0;
        *above = before + group.sum(n);
        return t;
      }
    }
  }

  // The id of the n-th (from 1) element of that order in the order of ids, the largest
  // number where there are no more than n.
  __device__ __forceinline__ int nth_equal(unsigned o, double n, bool of_hand) {
    if (of_hand) {
      int equal = 0;
#pragma unroll
      for (int q = 0; q < kBinEach; ++q) equal += order[q] == o;
      if (row.group.sum(equal) <= n) return 0x7FFFFFFF;
      int x = 0;
#pragma unroll 1
      for (int b = 23; b >= 0; --b) {
        int below = 0;
#pragma unroll
        for (int q = 0; q < kBinEach; ++q) below += order[q] == o && id[q] < (x | (1 << b));
        if (row.group.sum(below) < n) x |= 1 << b;
      }
      return x;
    }
    const SampleParams& p = row.p;
    for (int g = wave(); g < p.n_segs; g += kPickWaves) {
      int equal = 0;
      if (order_of(p.seg_max[row.first + g]) >= o)
        row.each_of(g, [&](float z, int, bool own) { equal += own && order_of(z) == o; });
      wave_exclusive_dpp(equal, &equal);
      if ((threadIdx.x & (kWave - 1)) == 0) p.seg_sum[row.first + g] = (double)equal;
    }
    __syncthreads();
    double all;
    const int x = row.by_segment([&](double) { return n - 1.0; },
                                 [&](int g) { return p.seg_sum[row.first + g]; },
                                 [&](float z, int) { return order_of(z) == o ? 1.0 : 0.0; }, &all);
    return all <= n ? 0x7FFFFFFF : x;
  }

  // Where the support ends by top-k and top-p (`row_mass`: what top-p refers to without
  // top-k), and its mass segment by segment, in seg_mass.
  __device__ __forceinline__ Border support(double row_mass) {
    const Plan& plan = row.plan;
    const SampleParams& p = row.p;
    Border e{0u, 0x7FFFFFFF};
    double ties = 0x7FFFFFFF, whole = row_mass;
    bool last_ends = false;  // whether what locate() found last ends the support
    if (plan.k > 0) {
      double above;
      e.order = locate<true>((double)plan.k, &above);
      ties = (double)plan.k - above;
      last_ends = true;
      if (plan.p < 1.0f) {
        double mass = 0.0;
        row.each(e.order, [&](float z, int, bool own) {
          mass += own && order_of(z) > e.order ? row.weight(z) : 0.0;
        });
        whole = row.group.sum(mass);
        if (e.order != kNothing) whole += ties * row.weight(logit_of(e.order));
      }
    }
    if (plan.p < 1.0f) {
      const double least = (double)plan.p * whole;
      double above;
      const unsigned o = locate<false>(least, &above);
      // those of this order whose predecessors hold less
      const double v = row.weight(logit_of(o));
      const double n = v > 0.0 ? ceil((least - above) / v) : 1.0;
      const double some = n > 1.0 ? n : 1.0;
      last_ends = o >= e.order;
      if (o > e.order) {
        e.order = o;
        ties = some;
      } else if (o == e.order) {
        ties = some < ties ? some : ties;
      }
    }
    const bool of_hand = last_ends && in_hand;
    if (e.order > kNothing) e.id = nth_equal(e.order, ties, of_hand);
    const int lane = threadIdx.x & (kWave - 1);
    if (of_hand && by_segment && row.weight(logit_of(e.order)) >= (double)plan.min_p) {
      // what lies above the elements in hand is there: a wave adds those of its segments
      for (int g = wave(); g < p.n_segs; g += kPickWaves) {
        double s = 0.0;
#pragma unroll
        for (int q = 0; q < kBinEach; ++q)
          if (order[q] && (id[q] + row.row.pre) / kSegElems == g && inside(e, order[q], id[q])) s += w[q];
        s = wave_sum64(s);
        if (lane == 0 && s > 0.0) p.seg_mass[row.first + g] += s;
      }
    } else {
      for (int g = wave(); g < p.n_segs; g += kPickWaves) {
        double s = 0.0;
        if (order_of(p.seg_max[row.first + g]) >= e.order) {
          row.each_of(g, [&](float z, int i, bool own) {
            const double v = own && inside(e, order_of(z), i) ? row.weight(z) : 0.0;
            s += v >= (double)plan.min_p ? v : 0.0;
          });
          s = wave_sum64(s);
        }
        if (lane == 0) p.seg_mass[row.first + g] = s;
      }
    }
    __syncthreads();
    return e;
  }
  __device__ __forceinline__ static bool inside(const Border& e, unsigned o, int i) {
    return o > e.order || (o == e.order && i <= e.id);
  }
};

// kWide: rows that the ranked candidates do not settle are finished here; otherwise they are
// left to a second kernel, which (with p.todo) takes no others.
//
// Bound: the chain of its steps.  One row of 151,936, top 50: 14 us (a bound, its units read
// again, two sorts in LDS and five scans over the workgroup).  Rows at large: 64 with
// settings of their own 126 to 166 us, most of it the histogram's LDS atomics and the exact
// sum's 64-bit exponentials over a row by one compute unit; 1,024 threads a row took 168 for
// 150 then, and one row 28 for 24.
template <bool kBf16, bool kRagged, bool kWide>
__global__ __launch_bounds__(kPickThreads, kWide ? 2 : 4) void sample_pick(SampleParams p) {
  __shared__ double s_sum[2][kPickWaves * 3];
  __shared__ int s_scan[2][kPickWaves * 3];
  __shared__ int s_found[4];
  __shared__ double s_held[1 + kPickWaves];
  __shared__ unsigned long long s_key[kRanked];
  __shared__ unsigned long long s_ranked[kRanked];
  __shared__ double s_run[kRanked];
  __shared__ int s_unit[kUnitsHeld];
  __shared__ int s_far[kBins];
  const int tid = threadIdx.x;
  using R = Row<kBf16, kRagged>;
  Group group{s_sum, s_scan};
  const long long row = p.first_row + blockIdx.x;
  if (kWide && p.todo && !p.todo[row]) return;
  auto write = [&](int id, float logq, float logp) {
    if (tid != 0) return;
    p.ids[row] = id;
    if (p.logq) p.logq[row] = logq;
    if (p.logp) p.logp[row] = logp;
  };
  if (!kWide && tid == 0) p.todo[row] = 0;
  if (p.mask && !p.mask[row]) {
    write(-1, 0.0f, 0.0f);
    return;
  }
  const Plan plan = plan_of(p, row);
  const double u = p.u[row];
  const float nan = __builtin_nanf("");
  if (plan.bad || !(u >= 0.0 && u < 1.0)) {
    if (tid == 0) atomicMin(&p.hdr->err_key, err_key(row, kPrioSampling));
    write(-1, nan, nan);
    return;
  }
  const long long first = row * p.n_segs;
  const unsigned short* const unit = p.unit + first * kWave;
  const int units = p.n_segs * kWave;
  const bool few = units <= kUnitEach * kPickThreads;
  // what the row's segments left, and its units, on their way together
  const bool one_each = p.n_segs <= kPickThreads;
  float seg_max = -INFINITY;
  double seg_sum = 0.0, seg_mass = 0.0;
  if (one_each && tid < p.n_segs) {
    seg_max = p.seg_max[first + tid];
    seg_sum = p.seg_sum[first + tid];
    seg_mass = p.seg_mass[first + tid];
  }
  unsigned held[kUnitEach];
#pragma unroll
  for (int c = 0; c < kUnitEach; ++c)
    held[c] = plan.filtered && few && c * kPickThreads + tid < units ? unit[c * kPickThreads + tid] : 0u;
  auto each_segment = [&](auto use) {  // use(maximum, sum, mass)
    if (one_each) {
      use(seg_max, seg_sum, seg_mass);
    } else {
      for (int g = tid; g < p.n_segs; g += kPickThreads)
        use(p.seg_max[first + g], p.seg_sum[first + g], p.seg_mass[first + g]);
    }
  };
  // the row's maximum (above all numbers where one is none)
  int top = signed_order(kNothing);
  each_segment([&](float x, double, double) {
    const int o = x == x ? signed_order(order_of(x)) : 0x7FFFFFFF;
    top = o > top ? o : top;
  });
  top = group.largest(top);
  const float m = logit_of(unsigned_order(top));
  if (!(m < INFINITY)) {
    write(-1, nan, nan);
    return;
  }
  if (m == -INFINITY) {  // nothing is allowed
    write(-1, -INFINITY, -INFINITY);
    return;
  }
  Pick<kBf16, kRagged> pick{p, R(p, row), plan, group, first, m, s_found, s_held};
  const bool same = plan.mass && plan.rate == kLog2e64;
  double both[2] = {0.0, 0.0};  // sums at temperature 1 and at the row's
  each_segment([&](float x, double s, double w) {
    if (p.logp && !same) both[0] += s * pow2(((double)x - m) * kLog2e64);
    if (plan.mass) both[1] += w * pick.weight(x);
  });
  group.sums(both);
  const double row_mass = both[1], log_all = log(same ? both[1] : both[0]);
  auto finish = [&](int id, double total) {
    if (tid != 0) return;
    if (id < 0) {  // (no sum leads here; nothing before the row would be read if one did)
      write(-1, nan, nan);
      return;
    }
    const long long at = row * p.ld + id;
    const float z = kBf16 ? __uint_as_float((unsigned)static_cast<const unsigned short*>(p.z)[at] << 16)
                          : static_cast<const float*>(p.z)[at];
    const double x = (double)z - m;
    write(id, (float)(x * plan.rate * kLn264 - log(total)), (float)(x - log_all));
  };
  double total;
  if (!plan.filtered) {
    const int id = pick.by_segment([&](double all) { return u * all; },
                                   [&](int g) { return p.seg_mass[first + g] * pick.weight(p.seg_max[first + g]); },
                                   [&](float z, int) { return pick.weight(z); }, &total);
    finish(id, total);
    return;
  }
  const bool by_mass = plan.k == 0 && plan.p < 1.0f;
  int listed = kRanked + 1;
  if (!kWide || !p.todo) {
    auto each_unit = [&](auto use) {  // use(upper half of its order, index)
      if (few) {
#pragma unroll
        for (int c = 0; c < kUnitEach; ++c)
          if (c * kPickThreads < units) use(held[c], c * kPickThreads + tid);
      } else {
        for (int i = tid; i < units; i += kPickThreads) use((unsigned)unit[i], i);
      }
    };
    // the want-th largest unit maximum bounds the elements that are needed: by how far the
    // maxima lie below the row's (1,023 orders or more in the last bin)
    const int want = plan.k > 0 ? plan.k : by_mass ? p.units_by_mass : 0;
    unsigned bound = 0;
    if (want > 0 && want <= units) {
      const unsigned highest = order_of(m) >> 16;
      for (int i = tid; i < kBins; i += kPickThreads) s_far[i] = 0;
      __syncthreads();
      each_unit([&](unsigned o, int i) {
        const unsigned d = highest - o;
        if (i < units) atomicAdd(&s_far[d < kBins - 1 ? d : kBins - 1], 1);
      });
      if (tid == 0) s_found[0] = kBins;
      __syncthreads();
      const int n0 = s_far[2 * tid], n1 = s_far[2 * tid + 1];
      int all;
      const int upto = group.scan(n0 + n1, &all) + n0;
      if (upto < want && upto + n1 >= want) s_found[0] = 2 * tid + 1;
      else if (upto >= want && upto - n0 < want) s_found[0] = 2 * tid;
      __syncthreads();
      const int far = s_found[0];
      if (far < kBins - 1) {
        bound = highest - far;
      } else {
#pragma unroll 1
        for (int b = 14; b >= 0; b -= 2) {
          int n[3] = {0, 0, 0};
          each_unit([&](unsigned o, int) {
#pragma unroll
            for (unsigned d = 0; d < 3; ++d) n[d] += o >= (bound | ((d + 1) << b));
          });
          group.sums(n);
          bound |= (n[2] >= want ? 3u : n[1] >= want ? 2u : n[0] >= want ? 1u : 0u) << b;
        }
      }
    }
    unsigned least = bound << 16;
    if (least <= kNothing) least = kNothing + 1u;
    // By min-p alone: what lies clearly below its border is not needed.  (Weights are rounded:
    // by 4e-16 at most, which at high temperatures is a wide range of logits.)
    if (plan.p >= 1.0f && plan.min_p > 0.0f) {
      const double z = m + log2((double)plan.min_p) / plan.rate;
      const float low = (float)(z - 1e-5 * (fabs(z) + fabs((double)m)) - 1e-15 / plan.rate - 1e-30);
      if (order_of(low) > least) least = order_of(low);
    }
    // units that reach it
    int count = 0, all;
    each_unit([&](unsigned o, int i) { count += i < units && o >= (least >> 16); });
    int at = group.scan(count, &all);
    if (all <= kUnitsHeld) {
      each_unit([&](unsigned o, int i) {
        if (i < units && o >= (least >> 16)) s_unit[at++] = i;
      });
      __syncthreads();
      // and their elements that do, a pack a thread and turn, kPacks turns' loads together
      listed = 0;
      const int packs = all * R::kPacks;
      for (int base = 0; base < packs && listed <= kRanked; base += kPickThreads * R::kPacks) {
        typename R::P x[R::kPacks];
        int e[R::kPacks];
        unsigned in[R::kPacks];
#pragma unroll
        for (int q = 0; q < R::kPacks; ++q) {
          const int i = base + q * kPickThreads + tid;
          in[q] = 0;
          e[q] = 0;
          if (i < packs) {
            const int what = s_unit[i / R::kPacks];
            e[q] = pick.row.span.place((what / kWave * R::kPacks + i % R::kPacks) * kWave + what % kWave, in[q]);
            pick.row.span.load(x[q], e[q]);
          }
        }
#pragma unroll
        for (int q = 0; q < R::kPacks; ++q) {
          if (base + q * kPickThreads >= packs) break;
#pragma unroll
          for (int j = 0; j < R::kEpv; ++j)
            if (((in[q] >> j) & 1u) && order_of(x[q].get(j)) < least) in[q] &= ~(1u << j);
          x[q].fence();  // ordered again, rather than kept
          int some;
          int to = listed + group.scan(__popc(in[q]), &some);
          listed += some;
          for (; in[q]; in[q] &= in[q] - 1) {
            const int j = __ffs((int)in[q]) - 1;
            float z = x[q].get(0);
#pragma unroll
            for (int k = 1; k < R::kEpv; ++k) z = k == j ? x[q].get(k) : z;
            if (to < kRanked) s_key[to] = ((unsigned long long)order_of(z) << 32) | (unsigned)~(e[q] + j);
            ++to;
          }
        }
      }
      __syncthreads();
    }
  }
  if (listed <= kRanked) {
    // by logits, the lower id first (by min-p alone in any order)
    const bool ordered = plan.k > 0 || plan.p < 1.0f;
    const int full = power_of(listed);
    for (int i = listed + tid; i < full; i += kPickThreads) s_key[i] = 0ull;
    if (ordered) sort_down(s_key, full);
    else __syncthreads();
    // neighbours in that order a thread
    unsigned long long x[kRankEach];
    double w[kRankEach];
    bool in[kRankEach];
    double sum = 0.0, run_all;
#pragma unroll
    for (int c = 0; c < kRankEach; ++c) {
      const int i = kRankEach * tid + c;
      x[c] = i < listed ? s_key[i] : 0ull;
      w[c] = i < listed ? pick.weight(logit_of((unsigned)(x[c] >> 32))) : 0.0;
      in[c] = i < listed && (plan.k == 0 || i < plan.k);
      sum += in[c] ? w[c] : 0.0;
    }
    double before = group.scan(sum, &run_all) - sum;
    const double whole = by_mass ? row_mass : run_all;
    // (does the border by top-p lie among them?)
    if (!by_mass || run_all >= (double)plan.p * whole) {
      int n = 0;
#pragma unroll
      for (int c = 0; c < kRankEach; ++c) {
        const bool was = in[c];
        in[c] = was && (plan.p >= 1.0f || before < (double)plan.p * whole) &&
                (plan.min_p == 0.0f || w[c] >= (double)plan.min_p);
        // (the likeliest token always; its weight is 1, so that min-p keeps it by itself)
        in[c] = in[c] || (ordered && tid == 0 && c == 0);
        before += was ? w[c] : 0.0;
        n += in[c];
      }
      // the support in the order of ids (the complement of which the keys hold)
      int size;
      int place = group.scan(n, &size);
      const int ends = power_of(size);
#pragma unroll
      for (int c = 0; c < kRankEach; ++c)
        if (in[c]) {
          s_run[place] = w[c];
          s_ranked[place] = ((x[c] & 0xFFFFFFFFull) << 32) | (unsigned)place;
          ++place;
        }
      for (int i = size + tid; i < ends; i += kPickThreads) s_ranked[i] = 0ull;
      if (tid == 0) s_found[0] = 0x7FFFFFFF;
      sort_down(s_ranked, ends);
      double v[kRankEach];
      int last = -1;
      sum = 0.0;
#pragma unroll
      for (int c = 0; c < kRankEach; ++c) {
        const int i = kRankEach * tid + c;
        v[c] = i < size ? s_run[(unsigned)s_ranked[i]] : 0.0;
        sum += v[c];
        if (v[c] > 0.0) last = i;
      }
      double run = group.scan(sum, &total) - sum;
      last = group.largest(last);
      const double target = u * total;
#pragma unroll
      for (int c = 0; c < kRankEach; ++c) {
        run += v[c];
        if (v[c] > 0.0 && run > target) {
          atomicMin(&s_found[0], kRankEach * tid + c);
          break;
        }
      }
      __syncthreads();
      const int who = s_found[0] < last ? s_found[0] : last;
      finish((int)~(unsigned)(s_ranked[who] >> 32), total);
      return;
    }
  }
  if constexpr (!kWide) {
    if (tid == 0) p.todo[row] = 1;
  } else {
    __shared__ unsigned s_bins[kBins + kWave];
    __shared__ unsigned long long s_between[kPickWaves * kBinHeld];
    Wide<kBf16, kRagged> wide{pick, s_bins, s_between};
    const Border e = wide.support(row_mass);
    const int id = pick.by_segment(
        [&](double all) { return u * all; }, [&](int g) { return p.seg_mass[first + g]; },
        [&](float z, int i) {
          const double w = wide.inside(e, order_of(z), i) ? pick.weight(z) : 0.0;
          return w >= (double)plan.min_p ? w : 0.0;
        },
        &total);
    finish(id, total);
  }
}

constexpr int kPickGrid = 1 << 20;  // rows of a launch
// Rows: one for each compute unit.  Past it the rows at large are a kernel's of their own
// (1,024 unfiltered rows of 151,936: 149 us so, 164 with all in one; 300 fp32 rows of 50,257
// by min-p: 62 and 63).
constexpr int kPickApart = 256;

}  // namespace

hipError_t launch_sample(const SampleParams& given, hipStream_t s) {
  SampleParams p = given;
  // As many units as kWantByMass elements strewn among them would hit.
  const double units = (p.vocab + kUnitElems - 1) / kUnitElems;
  p.units_by_mass = (int)(units * -expm1(-kWantByMass / units));
  // Batches that fill the card more than once leave the rows that need it to a kernel of
  // their own, whose registers would leave room for few workgroups of all.
  const bool apart = p.n_rows > kPickApart;
  if (!apart) p.todo = nullptr;
  // rows of a launch, whose waves are fewer than 2^25
  const long long by_waves = (1 << 25) / p.n_segs;
  const long long most = by_waves < kPickGrid ? by_waves : kPickGrid;
#define TURNKL_SAMPLE(B, R)                                                         \
  if ((p.bf16 != 0) == B && (p.ragged != 0) == R) {                                 \
    for (p.first_row = 0; p.first_row == 0 || p.first_row < p.n_rows; p.first_row += most) { \
      const long long left = p.n_rows - p.first_row;                                \
      const long long rows = left < most ? left : most;                             \
      const long long waves = rows > 0 ? rows * p.n_segs : 1;                       \
      sample_scan<B, R><<<(int)((waves + kScanWaves - 1) / kScanWaves), kScanThreads, 0, s>>>(p); \
      if (hipError_t e = hipGetLastError(); e != hipSuccess || rows == 0) return e; \
      if (apart) sample_pick<B, R, false><<<(int)rows, kPickThreads, 0, s>>>(p);    \
      if (!apart || p.any_filter) sample_pick<B, R, true><<<(int)rows, kPickThreads, 0, s>>>(p); \
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;              \
    }                                                                               \
  }
  TURNKL_SAMPLE(true, false) TURNKL_SAMPLE(true, true) TURNKL_SAMPLE(false, false) TURNKL_SAMPLE(false, true)
#undef TURNKL_SAMPLE
  return hipGetLastError();
}

}  // namespace turnkl
