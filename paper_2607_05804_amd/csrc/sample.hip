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
// Two kernels.  sample_scan goes over the logits once: a wave takes a segment of 2,048
// elements and leaves its maximum and, where the row's filters need the mass of the whole
// row, its sum of weights; of rows with a filter also the largest of every lane's 32
// elements (a unit), by its upper 16 bits.  sample_pick joins a row's segments, a workgroup
// a row.  Without a filter it looks for the segment where the running sum passes the bound
// and reads that one again.  With one it needs the elements at the top of the row only: the
// n-th largest unit maximum is a bound that at least n elements reach, and only units that
// reach it are read again.  Up to 512 such elements are ranked against each other; up to
// 4,096 the borders of the support are found bit by bit; where more are needed (flat rows,
// long runs of equal logits) the same goes over the row itself.

#include "row_span.h"

namespace turnkl {
namespace {

constexpr int kScanThreads = 256;
constexpr int kScanWaves = kScanThreads / kWave;
constexpr int kSegElems = kSampleSegment;
constexpr int kPickThreads = 512;
constexpr int kPickWaves = kPickThreads / kWave;
constexpr int kRanked = 512;     // candidates that are ranked against each other
constexpr int kListed = 4096;    // candidates that LDS holds
constexpr int kUnitsHeld = 2048; // units that are read again
constexpr int kFirstWant = 200;  // elements that are asked for where only top-p limits a row,
constexpr int kMoreWant = 2400;  // and where those do not hold enough

// The logit's bits in an order of unsigned numbers (-0 and +0 alike, NaN as -inf).
__device__ inline unsigned order_of(float z) {
  const unsigned u = __float_as_uint((z == z ? z : -INFINITY) + 0.0f);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ inline float logit_of(unsigned o) {
  return __uint_as_float(o ^ ((unsigned)((int)~o >> 31) | 0x80000000u));
}
constexpr unsigned kNothing = 0x007FFFFFu;  // the order of -inf

// 2^x for x <= 0, from the series of exp around 0 in 64 bits: on [-1/2, 1/2] its remainder
// past the twelfth power is below 2e-16.
__device__ __forceinline__ double pow2(double x) {
  x = fmax(x, -1100.0);  // 0 from there on, -inf included
  const double n = rint(x);
  const double r = (x - n) * 0.69314718055994530942;
  double s = 1.0 / 479001600.0;
  s = fma(s, r, 1.0 / 39916800.0);
  s = fma(s, r, 1.0 / 3628800.0);
  s = fma(s, r, 1.0 / 362880.0);
  s = fma(s, r, 1.0 / 40320.0);
  s = fma(s, r, 1.0 / 5040.0);
  s = fma(s, r, 1.0 / 720.0);
  s = fma(s, r, 1.0 / 120.0);
  s = fma(s, r, 1.0 / 24.0);
  s = fma(s, r, 1.0 / 6.0);
  s = fma(s, r, 0.5);
  s = fma(s, r, 1.0);
  s = fma(s, r, 1.0);
  return ldexp(s, (int)n);
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
  a.rate = 1.4426950408889634074 / (t == 0.0f ? 1.0 : (double)t);
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

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

template <bool kBf16, bool kRagged>
__global__ __launch_bounds__(kScanThreads) void sample_scan(SampleParams p) {
  using R = Row<kBf16, kRagged>;
  const int lane = threadIdx.x & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (blockIdx.x == 0 && threadIdx.x == 0) p.hdr->err_key = kNoError;
  const long long tasks = (long long)p.n_rows * p.n_segs;
  for (long long task = (long long)blockIdx.x * kScanWaves + wid; task < tasks;
       task += (long long)gridDim.x * kScanWaves) {
    const long long row = task / p.n_segs;
    const int g = (int)(task - row * p.n_segs);
    if (p.mask && !p.mask[row]) continue;
    const Plan plan = plan_of(p, row);
    if (plan.bad) continue;
    const R r(p, row);
    typename R::P x[R::kPacks];
    int at[R::kPacks];
    unsigned bits[R::kPacks];
    r.load(g, x, at, bits);
    auto value = [&](int q, int j) { return (bits[q] >> j) & 1u ? x[q].get(j) : -INFINITY; };
    float best = -INFINITY;
    bool none = false;  // whether one is no number
#pragma unroll
    for (int q = 0; q < R::kPacks; ++q)
#pragma unroll
      for (int j = 0; j < R::kEpv; ++j) {
        const float z = value(q, j);
        none = none || z != z;
        best = fmaxf(best, z);
      }
    if (plan.filtered) p.unit[task * kWave + lane] = (unsigned short)(order_of(best) >> 16);
    const float m = __any(none) ? __builtin_nanf("") : wave_max_dpp(best);
    double mass = 0.0;
    float sum = 0.0f;
    const bool numbers = fabsf(m) < INFINITY;
    if (plan.mass && numbers) {
#pragma unroll
      for (int q = 0; q < R::kPacks; ++q)
#pragma unroll
        for (int j = 0; j < R::kEpv; ++j) mass += pow2(((double)value(q, j) - (double)m) * plan.rate);
      mass = wave_sum64(mass);
    }
    if (p.logp && numbers) {
#pragma unroll
      for (int q = 0; q < R::kPacks; ++q)
#pragma unroll
        for (int j = 0; j < R::kEpv; ++j) sum += exp2_fast((value(q, j) - m) * kLog2e);
      sum = wave_sum_dpp(sum);
    }
    if (lane == 0) {
      p.seg_max[task] = m;
      p.seg_sum[task] = sum;
      p.seg_mass[task] = mass;
    }
  }
}

// ---------------------------------------------------------------------------
// picking

// A workgroup's sums and scans in a fixed order; each has two barriers, after the second
// of which `lds` may be used again.
struct Group {
  double* lds;  // LDS, kPickWaves
  int* ilds;    // LDS, kPickWaves

  __device__ __forceinline__ double sum(double v) const {
    v = wave_sum64(v);
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    double s = lds[0];
#pragma unroll
    for (int w = 1; w < kPickWaves; ++w) s += lds[w];
    __syncthreads();
    return s;
  }
  // the sum of the threads before this one and itself; *total: of all
  __device__ __forceinline__ double scan(double v, double* total) const {
    const int lane = threadIdx.x & (kWave - 1), wid = threadIdx.x / kWave;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const double u = __shfl_up(v, o, kWave);
      if (lane >= o) v += u;
    }
    if (lane == kWave - 1) lds[wid] = v;
    __syncthreads();
    double before = 0.0, all = 0.0;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) {
      const double s = lds[w];
      before += w < wid ? s : 0.0;
      all += s;
    }
    __syncthreads();
    *total = all;
    return before + v;
  }
  __device__ __forceinline__ int scan(int v, int* total) const {  // of the threads before this one
    return block_exclusive_scan<kPickThreads>(v, ilds, total);
  }
  __device__ __forceinline__ int sum(int v) const {
    int all;
    block_exclusive_scan<kPickThreads>(v, ilds, &all);
    return all;
  }
  __device__ __forceinline__ int largest(int v) const {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) {
      const int u = __shfl_xor(v, o, kWave);
      v = u > v ? u : v;
    }
    if ((threadIdx.x & (kWave - 1)) == 0) ilds[threadIdx.x / kWave] = v;
    __syncthreads();
    int m = ilds[0];
#pragma unroll
    for (int w = 1; w < kPickWaves; ++w) m = ilds[w] > m ? ilds[w] : m;
    __syncthreads();
    return m;
  }
};

// The border of a support: orders above `order`, and at it ids up to `id`.
struct Border {
  unsigned order;
  int id;
};

// A row being picked from.
template <bool kBf16, bool kRagged>
struct Pick {
  using R = Row<kBf16, kRagged>;
  const SampleParams& p;
  const R row;
  const Plan plan;
  const Group group;
  const long long first;  // segment
  float m;                // M
  int* found;             // LDS
  double* held;           // LDS
  unsigned long long* list;  // LDS, kListed

  __device__ __forceinline__ double weight(float z) const { return pow2(((double)z - (double)m) * plan.rate); }

  // Hands every own element of segment g to use(value, id).
  template <typename F>
  __device__ __forceinline__ void each_of(int g, F use) const {
    typename R::P x[R::kPacks];
    int at[R::kPacks];
    unsigned bits[R::kPacks];
    row.load(g, x, at, bits);
#pragma unroll
    for (int q = 0; q < R::kPacks; ++q)
#pragma unroll
      for (int j = 0; j < R::kEpv; ++j)
        if ((bits[q] >> j) & 1u) use(x[q].get(j), at[q] + j);
  }
  // The same for all segments whose maximum reaches `least`, a wave each in turn.
  template <typename F>
  __device__ __forceinline__ void each(unsigned least, F use) const {
    for (int g = threadIdx.x / kWave; g < p.n_segs; g += kPickWaves)
      if (order_of(p.seg_max[first + g]) >= least) each_of(g, use);
  }

  // The first id where the running sum of weight(z) over kept elements passes target x
  // total, when a segment's share is share(g) (and each segment's elements are weighed
  // again); *total: of all shares.
  template <typename Share, typename Keep>
  __device__ __forceinline__ int by_segment(double u, Share share, Keep keep, double* total) const {
    // a run of segments a thread, so that the threads are in the order of ids
    const int each_run = (p.n_segs + kPickThreads - 1) / kPickThreads;
    const int lo = threadIdx.x * each_run;
    const int hi = lo + each_run < p.n_segs ? lo + each_run : p.n_segs;
    double mine = 0.0;
    int last = -1;  // the last one with a share
    for (int g = lo; g < hi; ++g) {
      const double s = share(g);
      mine += s;
      if (s > 0.0) last = g;
    }
    double all;
    const double upto = group.scan(mine, &all);
    *total = all;
    const double target = u * all;
    if (threadIdx.x == 0) *found = 0x7FFFFFFF;
    last = group.largest(last);  // (has the barriers)
    int* const slot = found;
    if (lo < hi && upto > target) atomicMin(slot, (int)threadIdx.x);
    __syncthreads();
    const int who = *found;
    if (who == 0x7FFFFFFF) {  // past the end by a rounding
      if (threadIdx.x == 0) {
        found[1] = last;
        *held = -1.0;
      }
    } else if ((int)threadIdx.x == who) {
      double run = upto - mine;
      int g = lo;
      for (; g < hi - 1; ++g) {
        const double s = share(g);
        if (run + s > target) break;
        run += s;
      }
      found[1] = g;
      *held = target - run;
    }
    __syncthreads();
    const int g = found[1];
    const double rest = *held;
    if (threadIdx.x < kWave) {
      const int lane = threadIdx.x;
      typename R::P x[R::kPacks];
      int at[R::kPacks];
      unsigned bits[R::kPacks];
      row.load(g, x, at, bits);
      int id = -1, end = -1;
      double run = 0.0;
#pragma unroll 1
      for (int q = 0; q < R::kPacks && id < 0; ++q) {
        typename R::P y;
        unsigned b;
        const int a = row.place(g, q, b);
        row.span.load(y, a);
        double s = 0.0;
#pragma unroll
        for (int j = 0; j < R::kEpv; ++j) {
          const float z = y.get(j);
          if (((b >> j) & 1u) && keep(z, a + j)) {
            const double w = weight(z);
            s += w;
            if (w > 0.0) end = a + j;
          }
        }
        double upto_lane = s;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
          const double t = __shfl_up(upto_lane, o, kWave);
          if (lane >= o) upto_lane += t;
        }
        const unsigned long long past = __ballot(rest >= 0.0 && run + upto_lane > rest);
        if (past) {
          const int who_lane = __ffsll((long long)past) - 1;
          int got = -1;
          if (lane == who_lane) {
            double t = run + (upto_lane - s);
#pragma unroll
            for (int j = 0; j < R::kEpv; ++j) {
              const float z = y.get(j);
              if (((b >> j) & 1u) && keep(z, a + j)) {
                const double w = weight(z);
                if (w > 0.0 && (got < 0 || t <= rest)) got = a + j;
                t += w;
              }
            }
          }
          id = __shfl(got, who_lane, kWave);
        }
        run += __shfl(upto_lane, kWave - 1, kWave);
      }
#pragma unroll
      for (int o = kWave / 2; o > 0; o >>= 1) {
        const int t = __shfl_xor(end, o, kWave);
        end = t > end ? t : end;
      }
      if (lane == 0) found[2] = id >= 0 ? id : end;
    }
    __syncthreads();
    return found[2];
  }

  // The largest t whose number of elements >= t is at least k (kCount), or whose mass is at
  // least `least`, two bits at a time; `over` hands elements of at least an order to its
  // argument.
  template <bool kCount, typename Over>
  __device__ __forceinline__ unsigned border_order(int k, double least, Over over) const {
    unsigned t = 0;
#pragma unroll 1
    for (int b = 30; b >= (kBf16 ? 16 : 0); b -= 2) {
      int n[3] = {0, 0, 0};
      double w[3] = {0.0, 0.0, 0.0};
      over(t | (1u << b), [&](unsigned o, int, double weight_of) {
#pragma unroll
        for (unsigned d = 0; d < 3; ++d)
          if (o >= (t | ((d + 1) << b))) {
            if constexpr (kCount) ++n[d];
            else w[d] += weight_of;
          }
      });
      unsigned digit = 0;
#pragma unroll
      for (unsigned d = 0; d < 3; ++d) {
        bool enough;
        if constexpr (kCount) enough = group.sum(n[d]) >= k;
        else enough = group.sum(w[d]) >= least;
        if (enough) digit = d + 1;
      }
      t |= digit << b;
    }
    // (of bf16 logits the lower half follows from the upper one: all ones below zero)
    return kBf16 && t && !(t >> 31) ? t | 0xFFFFu : t;
  }
  // The id of the n-th (from 1) element of that order, in the order of ids.
  template <typename Over>
  __device__ __forceinline__ int nth_equal(unsigned order, int n, Over over) const {
    int x = 0;
#pragma unroll 1
    for (int b = 23; b >= 0; --b) {
      int below = 0;
      over(order, [&](unsigned o, int id, double) { below += o == order && id < (x | (1 << b)); });
      if (group.sum(below) < n) x |= 1 << b;
    }
    return x;
  }
  // Where the support ends by top-k and top-p.  (*whole: the mass that top-p refers to.)
  template <typename Over>
  __device__ __forceinline__ Border border(double row_mass, Over over) const {
    Border e{0u, 0x7FFFFFFF};
    int ties = 0x7FFFFFFF;
    double whole = row_mass;
    if (plan.k > 0) {
      e.order = border_order<true>(plan.k, 0.0, over);
      int above = 0;
      double mass = 0.0;
      over(e.order, [&](unsigned o, int, double w) {
        if (o > e.order) {
          ++above;
          mass += w;
        }
      });
      ties = plan.k - group.sum(above);
      whole = group.sum(mass) + ties * weight(logit_of(e.order));
    }
    if (plan.p < 1.0f) {
      const double least = (double)plan.p * whole;
      const unsigned order = border_order<false>(0, least, over);
      double mass = 0.0;
      over(order, [&](unsigned o, int, double w) { mass += o > order ? w : 0.0; });
      mass = group.sum(mass);
      // those of this order whose predecessors hold less
      const double w = weight(logit_of(order));
      const double n = w > 0.0 ? ceil((least - mass) / w) : 0.0;
      const int some = n < 1.0 ? 1 : n < 1e9 ? (int)n : 1000000000;
      if (order > e.order || plan.k == 0) {
        e.order = order;
        ties = some;
      } else if (order == e.order) {
        ties = some < ties ? some : ties;
      }
    }
    if (e.order) {
      int equal = 0;
      over(e.order, [&](unsigned o, int, double) { equal += o == e.order; });
      if (group.sum(equal) > ties) e.id = nth_equal(e.order, ties, over);
    }
    return e;
  }
};

template <bool kBf16, bool kRagged>
__global__ __launch_bounds__(kPickThreads) void sample_pick(SampleParams p) {
  __shared__ double s_sum[kPickWaves];
  __shared__ int s_scan[kPickWaves];
  __shared__ int s_found[4];
  __shared__ double s_held;
  __shared__ unsigned long long s_list[kListed];
  __shared__ int s_unit[kUnitsHeld];
  __shared__ double s_run[kRanked];
  __shared__ int s_id[kRanked];
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
  using R = Row<kBf16, kRagged>;
  const Group group{s_sum, s_scan};
  for (long long row = blockIdx.x; row < p.n_rows; row += gridDim.x) {
    auto write = [&](int id, float logq, float logp) {
      if (tid != 0) return;
      p.ids[row] = id;
      if (p.logq) p.logq[row] = logq;
      if (p.logp) p.logp[row] = logp;
    };
    if (p.mask && !p.mask[row]) {
      write(-1, 0.0f, 0.0f);
      continue;
    }
    const Plan plan = plan_of(p, row);
    const double u = p.u[row];
    const float nan = __builtin_nanf("");
    if (plan.bad || !(u >= 0.0 && u < 1.0)) {
      if (tid == 0) atomicMin(&p.hdr->err_key, err_key(row, kPrioSampling));
      write(-1, nan, nan);
      continue;
    }
    const long long first = row * p.n_segs;
    // the row's maximum (no number where one is none)
    float m = -INFINITY;
    bool none = false;
    for (int g = tid; g < p.n_segs; g += kPickThreads) {
      const float x = p.seg_max[first + g];
      none = none || x != x;
      m = fmaxf(m, x);
    }
    m = logit_of((unsigned)group.largest((int)(order_of(m) ^ 0x80000000u)) ^ 0x80000000u);
    if (group.sum(none ? 1 : 0) || m == INFINITY) {
      write(-1, nan, nan);
      continue;
    }
    if (m == -INFINITY) {  // nothing is allowed
      write(-1, -INFINITY, -INFINITY);
      continue;
    }
    double log_all = 0.0;
    if (p.logp) {
      double s = 0.0;
      for (int g = tid; g < p.n_segs; g += kPickThreads)
        s += p.seg_sum[first + g] * pow2(((double)p.seg_max[first + g] - m) * 1.4426950408889634074);
      log_all = log(group.sum(s));
    }
    const Pick<kBf16, kRagged> pick{p, R(p, row), plan, group, first, m, s_found, &s_held, s_list};
    auto segment = [&](int g) {
      const double s = p.seg_mass[first + g];
      return s > 0.0 ? s * pick.weight(p.seg_max[first + g]) : 0.0;
    };
    auto finish = [&](int id, double total) {
      if (tid != 0) return;
      const long long at = row * p.ld + id;
      const float z = kBf16 ? __uint_as_float((unsigned)static_cast<const unsigned short*>(p.z)[at] << 16)
                            : static_cast<const float*>(p.z)[at];
      const double x = (double)z - m;
      write(id, (float)(x * plan.rate * 0.69314718055994530942 - log(total)), (float)(x - log_all));
    };
    double total;
    if (!plan.filtered) {
      const int id = pick.by_segment(u, segment, [](float, int) { return true; }, &total);
      finish(id, total);
      __syncthreads();
      continue;
    }
    double row_mass = 0.0;
    if (plan.mass) {
      double s = 0.0;
      for (int g = tid; g < p.n_segs; g += kPickThreads) s += segment(g);
      row_mass = group.sum(s);
    }
    const unsigned short* const unit = p.unit + first * kWave;
    const int units = p.n_segs * kWave;
    // by min-p alone: what lies clearly below its border is not needed
    unsigned floor = kNothing + 1u;
    if (plan.p >= 1.0f && plan.min_p > 0.0f) {
      const double z = m + log((double)plan.min_p) * 1.4426950408889634074 / plan.rate;
      const float low = (float)(z - 1e-5 * (fabs(z) + fabs((double)m)) - 1e-30);
      if (order_of(low) > floor) floor = order_of(low);
    }
    const bool by_mass = plan.k == 0 && plan.p < 1.0f;
    int want = plan.k > 0 ? plan.k : by_mass ? kFirstWant : 0;
    int listed = kListed + 1;
    bool ended = false;
    for (int turn = 0; turn < 2 && !ended; ++turn) {
      // the want-th largest unit maximum
      unsigned bound = 0;
      if (want > 0 && want <= units) {
#pragma unroll 1
        for (int b = 15; b >= 0; --b) {
          int n = 0;
          for (int i = tid; i < units; i += kPickThreads) n += unit[i] >= (bound | (1u << b));
          if (group.sum(n) >= want) bound |= 1u << b;
        }
      }
      unsigned least = bound << 16;
      least = least > floor ? least : floor;
      // units that reach it
      int count = 0, all;
      for (int i = tid; i < units; i += kPickThreads) count += unit[i] >= (least >> 16);
      int at = group.scan(count, &all);
      listed = kListed + 1;
      if (all <= kUnitsHeld) {
        for (int i = tid; i < units; i += kPickThreads)
          if (unit[i] >= (least >> 16)) s_unit[at++] = i;
        __syncthreads();
        // and their elements that do
        listed = 0;
        const int packs = all * R::kPacks;
        for (int base = 0; base < packs; base += kPickThreads) {
          const int i = base + tid;
          typename R::P x;
          unsigned in = 0;
          int e = 0;
          if (i < packs) {
            const int what = s_unit[i / R::kPacks];
            unsigned bits;
            e = pick.row.span.place((what / kWave * R::kPacks + i % R::kPacks) * kWave + what % kWave, bits);
            pick.row.span.load(x, e);
#pragma unroll
            for (int j = 0; j < R::kEpv; ++j)
              if (((bits >> j) & 1u) && order_of(x.get(j)) >= least) in |= 1u << j;
          }
          int some;
          int to = listed + group.scan(__popc(in), &some);
#pragma unroll
          for (int j = 0; j < R::kEpv; ++j)
            if ((in >> j) & 1u) {
              if (to < kListed) s_list[to] = ((unsigned long long)order_of(x.get(j)) << 32) | (unsigned)(e + j);
              ++to;
            }
          listed += some;
        }
        __syncthreads();
      }
      ended = true;
      if (by_mass && listed <= kListed) {
        double s = 0.0;
        for (int i = tid; i < listed; i += kPickThreads) s += pick.weight(logit_of((unsigned)(s_list[i] >> 32)));
        if (group.sum(s) < (double)plan.p * row_mass) {  // the border lies further down
          ended = turn > 0 || want >= kMoreWant;
          want = kMoreWant;
          listed = kListed + 1;
        }
      }
    }
    if (listed <= kRanked) {
      // ranked against each other: by logits, then ids
      unsigned long long mine = 0;
      int rank = 0;
      if (tid < listed) {
        mine = s_list[tid] ^ 0xFFFFFFFFull;  // the lower id first
        for (int j = 0; j < listed; ++j) rank += (s_list[j] ^ 0xFFFFFFFFull) > mine;
      }
      __syncthreads();
      if (tid < listed) s_list[kRanked + rank] = mine ^ 0xFFFFFFFFull;
      __syncthreads();
      const unsigned long long x = tid < listed ? s_list[kRanked + tid] : 0ull;
      const double w = tid < listed ? pick.weight(logit_of((unsigned)(x >> 32))) : 0.0;
      bool in = tid < listed && (plan.k == 0 || tid < plan.k);
      double all;
      const double upto = group.scan(in ? w : 0.0, &all);
      if (plan.p < 1.0f) in = in && upto - w < (double)plan.p * (by_mass ? row_mass : all);
      in = in && (plan.min_p == 0.0f || w >= (double)plan.min_p);
      in = in || tid == 0;
      // the support in the order of ids
      int size;
      const int place = group.scan(in ? 1 : 0, &size);
      if (in) s_id[place] = (int)(unsigned)x;
      __syncthreads();
      int before = 0;
      if (in)
        for (int j = 0; j < size; ++j) before += s_id[j] < (int)(unsigned)x;
      if (in) {
        s_run[before] = w;
        s_list[before] = x;
      }
      __syncthreads();
      const double mine_w = tid < size ? s_run[tid] : 0.0;
      const double run = group.scan(mine_w, &total);
      if (tid == 0) {
        s_found[0] = 0x7FFFFFFF;
      }
      const int last = group.largest(mine_w > 0.0 ? tid : -1);
      if (tid < size && mine_w > 0.0 && run > u * total) atomicMin(&s_found[0], tid);
      __syncthreads();
      const int who = s_found[0] < last ? s_found[0] : last;
      finish((int)(unsigned)s_list[who], total);
    } else {
      Border e;
      double mass = 0.0;
      auto keep = [&](unsigned o, int id, double w) {
        return (o > e.order || (o == e.order && id <= e.id)) && w >= (double)plan.min_p;
      };
      if (listed <= kListed) {
        constexpr int kEach = kListed / kPickThreads;
        unsigned order[kEach];
        int id[kEach];
        double w[kEach];
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
          const int i = q * kPickThreads + tid;
          const unsigned long long x = i < listed ? s_list[i] : 0ull;
          order[q] = (unsigned)(x >> 32);
          id[q] = (int)(unsigned)x;
          w[q] = i < listed ? pick.weight(logit_of(order[q])) : 0.0;
        }
        auto over = [&](unsigned least, auto use) {
#pragma unroll
          for (int q = 0; q < kEach; ++q)
            if (order[q] != 0u && order[q] >= least) use(order[q], id[q], w[q]);
        };
        e = pick.border(row_mass, over);
        over(0u, [&](unsigned o, int i, double v) { mass += keep(o, i, v) ? v : 0.0; });
        total = group.sum(mass);
        // the largest x with no more than the target before it
        const double target = u * total;
        int x = 0, last = -1;
#pragma unroll 1
        for (int b = 23; b >= 0; --b) {
          double below = 0.0;
          over(0u, [&](unsigned o, int i, double v) { below += i < (x | (1 << b)) && keep(o, i, v) ? v : 0.0; });
          if (group.sum(below) <= target) x |= 1 << b;
        }
        over(0u, [&](unsigned o, int i, double v) {
          if (v > 0.0 && i > last && keep(o, i, v)) last = i;
        });
        last = group.largest(last);
        finish(x < last ? x : last, total);
      } else {
        auto over = [&](unsigned least, auto use) {
          pick.each(least, [&](float z, int i) {
            const unsigned o = order_of(z);
            if (o >= least) use(o, i, pick.weight(z));
          });
        };
        e = pick.border(row_mass, over);
        // the support's mass segment by segment, in place of the whole one's
        for (int g = wid; g < p.n_segs; g += kPickWaves) {
          double s = 0.0;
          pick.each_of(g, [&](float z, int i) {
            const double w = pick.weight(z);
            s += keep(order_of(z), i, w) ? w : 0.0;
          });
          s = wave_sum64(s);
          if (lane == 0) p.seg_mass[first + g] = s;
        }
        __syncthreads();
        const int id = pick.by_segment(
            u, [&](int g) { return p.seg_mass[first + g]; },
            [&](float z, int i) { return keep(order_of(z), i, pick.weight(z)); }, &total);
        finish(id, total);
      }
    }
    __syncthreads();
  }
}

constexpr int kPickGrid = 1 << 20;

}  // namespace

hipError_t launch_sample(const SampleParams& p, hipStream_t s) {
  const long long tasks = (long long)p.n_rows * p.n_segs;
  const long long blocks = (tasks + kScanWaves - 1) / kScanWaves;
  const int grid = (int)(blocks < 1 ? 1 : blocks < 2048 ? blocks : 2048);
  const int rows = p.n_rows < kPickGrid ? p.n_rows : kPickGrid;
#define TURNKL_SAMPLE(B, R)                                                     \
  if ((p.bf16 != 0) == B && (p.ragged != 0) == R) {                             \
    sample_scan<B, R><<<grid, kScanThreads, 0, s>>>(p);                         \
    if (hipError_t e = hipGetLastError(); e != hipSuccess || rows == 0) return e; \
    sample_pick<B, R><<<rows, kPickThreads, 0, s>>>(p);                         \
  }
  TURNKL_SAMPLE(true, false) TURNKL_SAMPLE(true, true) TURNKL_SAMPLE(false, false) TURNKL_SAMPLE(false, true)
#undef TURNKL_SAMPLE
  return hipGetLastError();
}

}  // namespace turnkl
