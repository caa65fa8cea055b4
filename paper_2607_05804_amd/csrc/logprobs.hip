// Token log probabilities: per row of logits the log-partition function, the
// entropy, the log probability of a given token and the K largest logits.
//
// Math.  With M = max z, S = sum 2^x, A = sum 2^x x over x = (z - M) log2 e:
//   L = ln S,  H = L - ln2 A / S,  log p_v = (z_v - M) - L.
// A wave sums against a reference r of its own that follows the maximum, with
// x = fma(z, log2 e, -r): r is any float, the product is not rounded, and r is set
// against M log2 e in the same way when the waves are joined, so that no error of
// r enters.  The reference moves (and the sums with it) when a lane meets a logit
// more than kSlack above it, so that no sum overflows and no second pass is needed;
// A / S then cancels a few units at most.  A forbidden token (-inf) makes A NaN: its
// group is summed again, and all that follow, over max(x, kFloor), which gives
// 0 * kFloor, not 0 * -inf.  Rows beyond the reach of that (|M| > kHuge, NaN, +inf)
// are summed again against their exact maximum.
//
// Alternatives.  Ranking works on 64-bit numbers that order logits and ids at
// once: the logit's bits, made monotone, above the complement of its id.  While
// the row streams by, each thread keeps its largest logit, and the upper 16 bits
// of the largest of every sixteen elements (a unit) go to LDS.  The k-th largest of
// the threads' maxima is a bound that at least k elements reach, and few more do
// (about 56 for k = 50 and 256 threads when the large ones are spread evenly).
// Only the units that reach it are read again, and the elements that do are
// ranked against each other.  Where more do than the lists hold (equal logits,
// or a run of large ones), the row is read again in steps, and the list is cut
// to its best k, with a higher bound, whenever the next step might not fit.

#include <type_traits>

#include "candidate_walk.h"
#include "row_span.h"

namespace turnkl {
namespace {

constexpr int kLpThreads = 256;
constexpr int kLpWaves = kLpThreads / kWave;
constexpr int kGroupElems = 32 * kLpThreads;  // elements of a group: 32 a lane
__host__ __device__ constexpr int group_packs(bool bf16) { return bf16 ? 4 : 8; }  // a lane's packs of it
constexpr float kSlack = 8.0f;           // logit units
constexpr float kFloor = -256.0f;        // log2 units: 2^kFloor is zero
// Rows with a larger |M| are summed again: log2 e times the reference is rounded, here by
// up to eight, which x then carries until the waves are joined, and A's sum with it; from
// 1.5e9 on the rounding alone takes every 2^x out of a float's range.
constexpr float kHuge = 1e8f;
constexpr int kCand = 896;        // elements held for ranking: k and a step's, at least
constexpr int kList = 384;         // units held for a second look

// The logit's bits in an order of unsigned numbers (-0 and +0 alike, NaN as -inf).
__device__ inline unsigned order_of(float z) {
  const unsigned u = __float_as_uint((z == z ? z : -INFINITY) + 0.0f);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ inline float logit_of(unsigned o) {
  return __uint_as_float(o ^ ((unsigned)((int)~o >> 31) | 0x80000000u));
}
__device__ inline unsigned long long ranked(unsigned order, int id) {
  return ((unsigned long long)order << 32) | (unsigned)~id;
}

// Maxima in one instruction each (the compiler's would quiet signalling NaNs with
// one more per operand; here a number beside one may be lost, which a row with NaN
// never uses).
__device__ inline float max2(float a, float b) {
  float r;
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// The largest t with at least k of a wave's kPer numbers per lane >= t (0 if
// there are fewer), its kLow lowest bits zero: the k-th largest, two bits at a time.
template <int kLow, int kPer>
__device__ inline unsigned kth_largest(const unsigned (&v)[kPer], int k) {
  unsigned t = 0;
#pragma unroll 1
  for (int b = 30; b >= kLow; b -= 2) {
    int n[3] = {0, 0, 0};
#pragma unroll
    for (int q = 0; q < kPer; ++q)
#pragma unroll
      for (unsigned d = 0; d < 3; ++d) n[d] += __popcll(__ballot(v[q] >= (t | ((d + 1) << b))));
    t |= (n[2] >= k ? 3u : n[1] >= k ? 2u : n[0] >= k ? 1u : 0u) << b;
  }
  return t;
}

// The workgroup's list of candidates.  All threads call every function, with the
// list complete.
constexpr int kRankers = 4;   // lanes that rank one candidate
constexpr int kRankTurn = 8;  // numbers a lane compares with at a time
constexpr int kRankPad = kRankers * kRankTurn;
struct Best {
  unsigned long long* cand;   // LDS, kCand + kRankPad
  unsigned long long* kept;   // LDS, kMaxAlternatives
  int* n;                     // LDS
  unsigned long long* floor;  // LDS: numbers below it are out

  // Hands every candidate's number and rank among `count` to use(), in one thread
  // each: four lanes compare it with a quarter of the list each.  One barrier.
  template <typename F>
  __device__ void ranks(int count, F use) const {
    if (threadIdx.x < kRankPad) cand[count + threadIdx.x] = 0ull;
    __syncthreads();
    const int part = threadIdx.x % kRankers;
    for (int i = threadIdx.x / kRankers; i < count; i += kLpThreads / kRankers) {
      const unsigned long long x = cand[i];
      int r = 0;
      for (int j = part; j < count; j += kRankPad) {
        unsigned long long c[kRankTurn];
#pragma unroll
        for (int q = 0; q < kRankTurn; ++q) c[q] = cand[j + q * kRankers];
#pragma unroll
        for (int q = 0; q < kRankTurn; ++q) r += c[q] > x;
      }
      r += __shfl_xor(r, 1, kWave);
      r += __shfl_xor(r, 2, kWave);
      if (part == 0) use(x, r);
    }
  }
  // Keeps the k best of `count` and raises the floor above the k-th.
  __device__ void cut(int count, int k) {
    ranks(count, [&](unsigned long long x, int r) {
      if (r >= k) return;
      kept[r] = x;
      if (r == k - 1) *floor = x + 1ull;
    });
    __syncthreads();
    for (int i = threadIdx.x; i < k && i < count; i += kLpThreads) cand[i] = kept[i];
    if (threadIdx.x == 0) *n = count < k ? count : k;
    __syncthreads();
  }
};

// Whether a wave's row has a given token, and its logit, read while the row streams by.
struct Given {
  bool in;
  float z;
};
__device__ inline Given given_of(const LogprobParams& p, long long row) {
  Given g{false, __builtin_nanf("")};
  if (!p.ids) return g;
  const int id = __builtin_amdgcn_readfirstlane(p.ids[row]);
  g.in = id >= 0 && id < p.vocab;
  if (g.in && p.logp) {
    const long long at = row * p.ld + id;
    g.z = p.bf16 ? __uint_as_float((unsigned)static_cast<const unsigned short*>(p.z)[at] << 16)
                 : static_cast<const float*>(p.z)[at];
  }
  return g;
}

// L of a row: 0 for one of nothing but -inf.
__device__ inline float log_sum(float m, float s) {
  return m == -INFINITY && s == 0.0f ? 0.0f : kLn2 * log2f(s);
}

// One thread writes a row's outputs but the alternatives.
__device__ inline void write_row(const LogprobParams& p, long long row, float m, float s, float a,
                                 const Given& g) {
  const bool empty = m == -INFINITY && s == 0.0f;
  const float l = log_sum(m, s);
  if (p.entropy) p.entropy[row] = empty ? 0.0f : l - kLn2 * (a / s);
  if (p.log_z) {
    p.log_z[2 * row] = m;
    p.log_z[2 * row + 1] = l;
  }
  if (p.ids && !g.in) atomicMin(&p.hdr->err_key, err_key(row, kPrioTokenId));
  if (p.logp) p.logp[row] = empty && g.in ? -INFINITY : (g.z - m) - l;
}

__device__ inline void write_alternative(const LogprobParams& p, long long row, int rank,
                                         unsigned long long x, float m, float l) {
  const float z = logit_of((unsigned)(x >> 32));
  p.top_ids[row * p.ld_top + rank] = (int)~(unsigned)x;
  // -inf - -inf is -inf here, but rows of NaN say so everywhere
  p.top_logp[row * p.ld_top + rank] = z == -INFINITY && l == l ? -INFINITY : (z - m) - l;
}

// A row that is not asked for, by the `n` threads that call with i = 0 .. n - 1.
__device__ inline void write_masked_row(const LogprobParams& p, long long row, int i, int n) {
  if (i == 0) {
    if (p.logp) p.logp[row] = 0.0f;
    if (p.entropy) p.entropy[row] = 0.0f;
    if (p.log_z) {
      p.log_z[2 * row] = __builtin_nanf("");
      p.log_z[2 * row + 1] = __builtin_nanf("");
    }
  }
  for (int j = i; j < p.k; j += n) {
    p.top_ids[row * p.ld_top + j] = -1;
    p.top_logp[row * p.ld_top + j] = -INFINITY;
  }
}

// Chunks' sums, each against its own maximum, joined against the row's.
struct Sums {
  float m, s, a;
};
__device__ inline void add_part(Sums& t, float m, float s, float a) {
  if (m == -INFINITY) {  // nothing but -inf and NaN: sums of 0 or NaN
    t.s += s;
    t.a += s;
    return;
  }
  const float d = (m - t.m) * kLog2e;
  const float f = exp2f(d);
  t.s = fmaf(f, s, t.s);
  t.a = fmaf(f, fmaf(s, f == 0.0f ? 0.0f : d, a), t.a);
}

// Clears the status; with a mask, lists the rows that are asked for, in order.
constexpr int kBeginThreads = 1024;
__global__ __launch_bounds__(kBeginThreads) void logprob_begin(LogprobParams p) {
  if (threadIdx.x == 0) p.hdr->err_key = kNoError;
  if (!p.rows) return;
  __shared__ int s_scan[kBeginThreads / kWave];
  constexpr int kEach = 16;  // rows of a thread and turn
  int done = 0;
  for (long long base = 0; base < p.n_rows; base += kBeginThreads * kEach) {
    const long long first = base + (long long)threadIdx.x * kEach;
    unsigned on = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (first + j < p.n_rows && p.mask[first + j]) on |= 1u << j;
    int total;
    int at = done + block_exclusive_scan<kBeginThreads>(__popc(on), s_scan, &total);
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if ((on >> j) & 1u) p.rows[at++] = (int)(first + j);
    done += total;
  }
  if (threadIdx.x == 0) p.hdr->n_sup = done;
}

// One chunk of a row after the other (task = row of the list x chunk), by workgroups
// that fill the card.  Bound: HBM; the arithmetic (a fused multiply-add, an exponential,
// two sums and half a maximum an element) keeps the vector units busy for three quarters
// of that time, so nothing may be added to it, and what a row's end takes is hidden by
// the other workgroups' loads only in part.  9,830 bf16 rows of 151,936 out of 16,384:
// 463 us without alternatives (6.5 TB/s), 492 with 5, 523 to 529 with 50 (side by side 444,
// 462 and 490); 3,000 fp32 rows of 50,257 94 us (6.4 TB/s), 104 with 20; 4,900 of 151,936
// 441 (6.8 TB/s), 480 with 50.  Two groups ahead instead of one, in four workgroups a CU
// instead of five, or as few workgroups as take no more turns gave nothing or 2% less.
// Workgroups of a variant that a CU has registers for.  (The one of bf16 rows on packs
// with alternatives has five without being held to it; held to it, it spills.)
__host__ __device__ constexpr int rows_a_cu(bool bf16, bool ragged, bool top) {
  return bf16 ? (top ? 5 : 6) : (ragged && top ? 3 : 4);
}

template <bool kBf16, bool kRagged, bool kTop>
__global__ __launch_bounds__(kLpThreads, kBf16 && kTop && !kRagged ? 4 : rows_a_cu(kBf16, kRagged, kTop))
    void logprob_rows(LogprobParams p) {
  constexpr int kLpPacks = group_packs(kBf16);
  using Span = RowSpan<kBf16, kRagged>;
  using P = typename Span::P;
  constexpr int kEpv = Span::kEpv;
  constexpr int kEs = Span::kEs;
  constexpr int kUnitPacks = kLpPacks / 2;  // packs of a unit: a group is two, in one LDS word
  constexpr int kGroup = kLpThreads * kLpPacks;        // packs of a group
  extern __shared__ unsigned s_unit[];
  __shared__ float s_wave[kLpWaves][4];
  __shared__ unsigned s_max[kLpThreads];
  __shared__ unsigned long long s_cand[kCand + kRankPad];
  __shared__ unsigned long long s_kept[kMaxAlternatives];
  __shared__ unsigned long long s_floor;
  __shared__ int s_list[kList];
  __shared__ int s_n, s_units;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
  const long long count = p.rows ? p.hdr->n_sup : p.n_rows;
  // (the status of a call without logprob_begin: only the join reports to it)
  if (p.clear && blockIdx.x == 0 && tid == 0) p.hdr->err_key = kNoError;

  if (p.mask)  // the rows that are not asked for
    for (long long base = blockIdx.x; base < p.n_rows; base += (long long)gridDim.x * kWave) {
      const long long row = base + (long long)lane * gridDim.x;
      unsigned long long off = __ballot(row < p.n_rows && !p.mask[row < p.n_rows ? row : 0]);
      for (; off; off &= off - 1)
        write_masked_row(p, base + (long long)(__ffsll((long long)off) - 1) * gridDim.x, tid, kLpThreads);
    }

  const long long n_tasks = count * p.n_chunks;
  // A task: a chunk of a row, packs [lo, lo + n) of it (of ragged rows on the grid of
  // 128-byte lines); g0 to g1: its groups of whole packs that lie in the row, all but
  // the last, and of ragged rows all but the first.
  struct Task {
    Span span;
    int groups, g0, g1;
  };
  auto task_of = [&](long long row, int c) {
    const char* const at = static_cast<const char*>(p.z) + row * p.ld * kEs;
    const int pre = kRagged ? (int)(reinterpret_cast<uintptr_t>(at) & 127u) / kEs : 0;
    const int n_row = (int)(((long long)pre + p.vocab + kEpv - 1) / kEpv);
    const int lo = (int)chunk_start(n_row, p.n_chunks, 8, c);
    const int n = (int)chunk_start(n_row, p.n_chunks, 8, c + 1) - lo;
    const int groups = (n + kGroup - 1) / kGroup;
    return Task{Span{at, chunk_rsrc(at), p.vocab, lo * kEpv - pre, n}, groups, kRagged ? 1 : 0,
                kRagged ? groups - 1 : n / kGroup};
  };
  auto row_of = [&](long long task) -> long long {
    return p.rows ? p.rows[task / p.n_chunks] : task / p.n_chunks;
  };
  // The next task of this workgroup from `task` on (without the list, rows that are
  // not asked for are passed over here), n_tasks or more if there is none.
  auto next_of = [&](long long task) {
    if (p.mask && !p.rows)
      while (task < n_tasks && !p.mask[task / p.n_chunks]) task += gridDim.x;
    return task;
  };
  // Whether this wave has met a forbidden token: from then on A is summed over
  // max(x, kFloor), which changes no bit of rows without one.
  bool floored = false;
  P next[kLpPacks];  // the group that comes next, of this task or the next one
  auto fetch = [&](const Task& of, int g) {
    if (g >= of.g1) return;
#pragma unroll
    for (int q = 0; q < kLpPacks; ++q)
      next[q].load(of.span.rsrc, tid * 16, of.span.col * kEs + (g * kLpPacks + q) * (kLpThreads * 16));
  };
  long long task = next_of(blockIdx.x);
  if (task >= n_tasks) return;
  long long row = row_of(task);
  Task now = task_of(row, (int)(task % p.n_chunks));
  fetch(now, now.g0);
  for (;;) {
    const int c = (int)(task % p.n_chunks);
    const long long next_task = next_of(task + gridDim.x);
    const bool more = next_task < n_tasks;
    const long long next_row = more ? row_of(next_task) : 0;
    const Given given = p.n_chunks == 1 ? given_of(p, row) : Given{};
    const Span& span = now.span;
    const int n = span.n, groups = now.groups;

    float ref = -kHuge, ref2 = ref * kLog2e;           // the wave's reference, in log2 units too
    float ss = 0.0f, aa = 0.0f;                        // the lane's sums
    float best = -INFINITY;                            // the lane's largest logit
    auto sums = [&](int g, const P (&x)[kLpPacks], const unsigned (&bits)[kLpPacks], auto edge) {
      constexpr bool kEdge = decltype(edge)::value;
      // (of an edge a wave passes over the packs beyond the chunk)
      auto live = [&](int q) { return !kEdge || (g * kLpPacks + q) * kLpThreads + wid * kWave < span.n; };
      float z[kLpPacks][kEpv], most[kLpPacks];
#pragma unroll
      for (int q = 0; q < kLpPacks; ++q) {
        most[q] = -INFINITY;
        if (!live(q)) continue;
#pragma unroll
        for (int j = 0; j < kEpv; ++j) {
          z[q][j] = x[q].get(j);
          if constexpr (kEdge)
            if (!((bits[q] >> j) & 1u)) z[q][j] = -INFINITY;
        }
        most[q] = max3(z[q][0], z[q][1], z[q][2]);
#pragma unroll
        for (int j = 3; j + 1 < kEpv; j += 2) most[q] = max3(most[q], z[q][j], z[q][j + 1]);
        most[q] = max2(most[q], z[q][kEpv - 1]);
      }
      float top[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int q = u * kUnitPacks;
        if constexpr (kUnitPacks == 2) top[u] = max2(most[q], most[q + 1]);
        else top[u] = max2(max3(most[q], most[q + 1], most[q + 2]), most[q + 3]);
      }
      best = max3(best, top[0], top[1]);
      if constexpr (kTop) {
        // the upper halves of both
        s_unit[g * kLpThreads + tid] =
            __builtin_amdgcn_perm(__float_as_uint(top[1]), __float_as_uint(top[0]), 0x07060302u);
      }
      if (__any(best > ref + kSlack)) {
        ref = wave_max_dpp(best);
        const float to = ref * kLog2e, d = ref2 - to;
        const float f = exp2f(d);
        aa = f == 0.0f ? 0.0f : fmaf(ss, d, aa) * f;
        ss *= f;
        ref2 = to;
      }
      float gs = 0.0f, ga = 0.0f;
      auto add = [&](auto floored) {
        gs = 0.0f;
        ga = 0.0f;
#pragma unroll
        for (int q = 0; q < kLpPacks; ++q) {
          if (!live(q)) continue;
          float ps = 0.0f, pa = 0.0f;
#pragma unroll
          for (int j = 0; j < kEpv; ++j) {
            const float y = fmaf(z[q][j], kLog2e, -ref2);
            const float e = exp2_fast(y);
            const float x = decltype(floored)::value ? fmaxf(y, kFloor) : y;
            ps = j ? ps + e : e;
            pa = j ? fmaf(e, x, pa) : e * x;
          }
          gs += ps;
          ga += pa;
        }
      };
      if constexpr (!kEdge) {
        if (!floored) {
          add(std::false_type{});
          floored = __any(ga != ga);
        }
      }
      if (kEdge || floored) add(std::true_type{});
      ss += gs;
      aa += ga;
    };
    auto edge_group = [&](int g) {
      P x[kLpPacks];
      unsigned bits[kLpPacks];
#pragma unroll
      for (int q = 0; q < kLpPacks; ++q)
        span.load(x[q], span.place((g * kLpPacks + q) * kLpThreads + tid, bits[q]));
      sums(g, x, bits, std::true_type{});
    };
    if (kRagged) edge_group(0);
#pragma unroll 1
    for (int g = now.g0; g < now.g1; ++g) {
      P x[kLpPacks];
      const unsigned all[kLpPacks] = {};
#pragma unroll
      for (int q = 0; q < kLpPacks; ++q) x[q] = next[q];
      fetch(now, g + 1);
      sums(g, x, all, std::false_type{});
    }
    if (now.g1 < groups && now.g1 >= now.g0) edge_group(groups - 1);
    Task then = now;
    if (more) {  // its first loads are on their way while this row is finished
      then = task_of(next_row, (int)(next_task % p.n_chunks));
      fetch(then, then.g0);
    }

    const float wm = wave_max_dpp(best);
    ss = wave_sum_dpp(ss);
    aa = wave_sum_dpp(aa);
    if (lane == 0) {
      s_wave[wid][0] = wm;
      s_wave[wid][1] = ref2;
      s_wave[wid][2] = ss;
      s_wave[wid][3] = aa;
    }
    if (kTop) s_max[tid] = order_of(best);
    if (tid == 0) {
      s_n = 0;
      s_units = 0;
    }
    __syncthreads();
    Sums t{-INFINITY, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kLpWaves; ++w) {
      t.m = fmaxf(t.m, s_wave[w][0]);
      t.s += s_wave[w][2];
    }
    // (every thread comes to the same answer)
    const bool odd = (fabsf(t.m) > kHuge && t.m != -INFINITY) || !(t.s < INFINITY);
    t.s = 0.0f;
    if (!odd && t.m != -INFINITY) {
#pragma unroll
      for (int w = 0; w < kLpWaves; ++w) {
        const float d = -fmaf(t.m, kLog2e, -s_wave[w][1]);
        const float f = exp2f(d);
        t.s = fmaf(f, s_wave[w][2], t.s);
        t.a = fmaf(f, fmaf(s_wave[w][2], f == 0.0f ? 0.0f : d, s_wave[w][3]), t.a);
      }
    }
    if (odd) {
      // against the exact maximum of what are numbers, with differences that
      // cannot overflow into each other
      auto each = [&](auto use) {
#pragma unroll 1
        for (int i = tid; i < n; i += kLpThreads) {
          unsigned bits;
          const int at = span.place(i, bits);
          P x;
          span.load(x, at);
#pragma unroll
          for (int j = 0; j < kEpv; ++j)
            if ((bits >> j) & 1u) use(x.get(j));
        }
      };
      best = -INFINITY;
      each([&](float z) { best = z > best ? z : best; });
      const float m = wave_max_dpp(best);
      __syncthreads();
      if (lane == 0) s_wave[wid][0] = m;
      if (kTop) s_max[tid] = order_of(best);
      __syncthreads();
      t.m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kLpWaves; ++w) t.m = fmaxf(t.m, s_wave[w][0]);
      const float u = t.m == -INFINITY ? 0.0f : t.m;
      ss = 0.0f;
      aa = 0.0f;
      each([&](float z) {
        const float y = (z - u) * kLog2e;
        const float e = exp2_fast(y);
        ss += e;
        aa = fmaf(e, fmaxf(y, kFloor), aa);
      });
      ss = wave_sum_dpp(ss);
      aa = wave_sum_dpp(aa);
      if (lane == 0) {
        s_wave[wid][2] = ss;
        s_wave[wid][3] = aa;
      }
      __syncthreads();
      t.s = 0.0f;
      t.a = 0.0f;
#pragma unroll
      for (int w = 0; w < kLpWaves; ++w) {
        t.s += s_wave[w][2];
        t.a += s_wave[w][3];
      }
    }
    if (tid == 0) {
      if (p.n_chunks == 1) {
        write_row(p, row, t.m, t.s, t.a, given);
      } else {
        float* const out = p.part + (row * p.n_chunks + c) * kLogprobPart;
        out[0] = t.m;
        out[1] = t.s;
        out[2] = t.a;
        drain_stores();  // their data registers are free
      }
    }
    if constexpr (kTop) {
      if (wid == kLpWaves - 1) {
        unsigned v[kLpWaves];
#pragma unroll
        for (int q = 0; q < kLpWaves; ++q) v[q] = s_max[q * kWave + lane];
        // (a bf16's order is in its upper half)
        const unsigned k_th = kth_largest<kBf16 ? 16 : 8>(v, p.k);
        if (lane == 0) s_floor = (unsigned long long)k_th << 32;
      }
      __syncthreads();
      // units whose largest reaches the bound (by its upper half, which orders
      // halves as it orders floats)
      const float bound = __uint_as_float(__float_as_uint(logit_of((unsigned)(s_floor >> 32))) & 0xFFFF0000u);
      if (!odd) {
        unsigned long long reach = 0;  // bit 2 g + h: unit h of group g
#pragma unroll 4
        for (int g = 0; g < groups; ++g) {
          const unsigned x = s_unit[g * kLpThreads + tid];
          const unsigned two = (__uint_as_float(x << 16) >= bound ? 1u : 0u) |
                               (__uint_as_float(x & 0xFFFF0000u) >= bound ? 2u : 0u);
          reach |= (unsigned long long)two << (2 * g);
        }
        // (one atomic a wave: of lanes with numbers of their own it takes a turn for each)
        int wave_units;
        int i = wave_exclusive_dpp(__popcll(reach), &wave_units);
        if (wave_units) {
          int first = 0;
          if (lane == 0) first = atomicAdd(&s_units, wave_units);
          i += __builtin_amdgcn_readfirstlane(first);
          for (; reach && i < kList; reach &= reach - 1, ++i)  // the unit's first pack
            s_list[i] = (__ffsll((long long)reach) - 1) * (kUnitPacks * kLpThreads) + tid;
        }
      }
      __syncthreads();
      // Elements of pack i that reach the floor join the candidates where there is room
      // (i < 0: no pack).  All threads call it.
      auto gather = [&](int i, unsigned long long least) {
        unsigned bits = 0, in = 0;
        int at = 0;
        P x;
        if (i >= 0) {
          at = span.place(i, bits);
          span.load(x, at);
#pragma unroll
          for (int q = 0; q < kEpv; ++q)
            if (ranked(order_of(x.get(q)), at + q) >= least) in |= 1u << q;
          in &= bits;
        }
        int wave_in;
        int to = wave_exclusive_dpp(__popc(in), &wave_in);
        if (!wave_in) return;
        int first = 0;
        if (lane == 0) first = atomicAdd(&s_n, wave_in);
        to += __builtin_amdgcn_readfirstlane(first);
        if (!in) return;
#pragma unroll
        for (int q = 0; q < kEpv; ++q)
          if (((in >> q) & 1u) && to < kCand) s_cand[to++] = ranked(order_of(x.get(q)), at + q);
      };
      Best list{s_cand, s_kept, &s_n, &s_floor};
      int held = kCand + 1;
      if (!odd && s_units <= kList) {
        const int total = s_units * kUnitPacks;
        const unsigned long long least = s_floor;
        for (int base = 0; base < total; base += kLpThreads) {
          const int j = base + tid;
          gather(j < total ? s_list[j / kUnitPacks] + j % kUnitPacks * kLpThreads : -1, least);
        }
        __syncthreads();
        held = s_n;
      }
      if (held > kCand) {
        // More than the lists hold: all packs of the chunk in steps.  (Every thread
        // has read s_n before it is cleared.)
        __syncthreads();
        if (tid == 0) s_n = 0;
        __syncthreads();
        held = walk_candidates(
            n, kEpv, 16 * kEpv, kLpThreads, kCand, p.k, [&](int all) { list.cut(all, p.k); },
            [&](int base, int step) { gather(tid < step && base + tid < n ? base + tid : -1, s_floor); },
            [&] { return s_n; }, [] { __syncthreads(); });
      }
      if (p.n_chunks == 1) {
        const float l = log_sum(t.m, t.s);
        list.ranks(held, [&](unsigned long long x, int r) {
          if (r < p.k) write_alternative(p, row, r, x, t.m, l);
        });
      } else {
        unsigned long long* const out = p.cand + (row * p.n_chunks + c) * p.k;
        list.ranks(held, [&](unsigned long long x, int r) {
          if (r < p.k) out[r] = x;
        });
        for (int j = held + tid; j < p.k; j += kLpThreads) out[j] = 0ull;  // a chunk shorter than k
      }
    }
    if (!more) break;
    __syncthreads();  // LDS is reused by the next task
    task = next_task;
    row = next_row;
    now = then;
  }
}

// Joins the chunks of a row: one workgroup per row.  The first candidates are loaded
// before anything is waited for, and one wave adds the sums while another looks for the
// bound: few rows wait for nothing but this chain (64 bf16 rows of 151,936, k = 5: 4.5 us).
constexpr int kJoinEach = 3;  // candidates that a thread keeps
__global__ __launch_bounds__(kLpThreads) void logprob_join(LogprobParams p) {
  __shared__ float s_row[2];
  __shared__ unsigned s_max[kLpThreads];
  __shared__ unsigned long long s_cand[kCand + kRankPad];
  __shared__ unsigned long long s_kept[kMaxAlternatives];
  __shared__ unsigned long long s_floor;
  __shared__ int s_n;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int total = p.n_chunks * p.k;
  for (long long row = blockIdx.x; row < p.n_rows; row += gridDim.x) {
    if (p.mask && !p.mask[row]) continue;  // written by the row kernel
    const unsigned long long* const in = p.cand + row * total;
    unsigned long long got[kJoinEach];
#pragma unroll
    for (int q = 0; q < kJoinEach; ++q) got[q] = q * kLpThreads + tid < total ? in[q * kLpThreads + tid] : 0ull;
    // a chunk per lane and turn, joined in a fixed tree
    const float* const part = p.part + row * p.n_chunks * kLogprobPart;
    Given given{};
    float m = -INFINITY, s = 0.0f, a = 0.0f;
    if (wid == 0) {
      given = given_of(p, row);
      if (lane < p.n_chunks) {
        m = part[lane * kLogprobPart];
        s = part[lane * kLogprobPart + 1];
        a = part[lane * kLogprobPart + 2];
      }
    }
    if (tid == 0) s_n = 0;
    if (p.k > 0) {
      // The chunks' lists are sorted: the first of each, by as many threads as there are
      // (by chunk, then rank), bound the k-th largest of all closely.
      const int rank = tid / p.n_chunks, c0 = tid - rank * p.n_chunks;
      unsigned long long best = 0;
      if (rank < p.k)
        for (int c = c0; c < p.n_chunks; c += kLpThreads) {
          const unsigned long long x = in[(long long)c * p.k + rank];
          best = x > best ? x : best;
        }
      s_max[tid] = (unsigned)(best >> 32);
    }
    __syncthreads();
    if (wid == 0) {
      Sums t{m, 0.0f, 0.0f};
      for (int c = lane + kWave; c < p.n_chunks; c += kWave) t.m = fmaxf(t.m, part[c * kLogprobPart]);
      t.m = wave_max_dpp(t.m);
      if (lane < p.n_chunks) add_part(t, m, s, a);
      for (int c = lane + kWave; c < p.n_chunks; c += kWave)
        add_part(t, part[c * kLogprobPart], part[c * kLogprobPart + 1], part[c * kLogprobPart + 2]);
      t.s = wave_sum_dpp(t.s);
      t.a = wave_sum_dpp(t.a);
      if (lane == 0) {
        write_row(p, row, t.m, t.s, t.a, given);
        s_row[0] = t.m;
        s_row[1] = log_sum(t.m, t.s);
      }
    } else if (wid == 1 && p.k > 0) {
      unsigned v[kLpWaves];
#pragma unroll
      for (int q = 0; q < kLpWaves; ++q) v[q] = s_max[q * kWave + lane];
      const unsigned t = p.bf16 ? kth_largest<16>(v, p.k) : kth_largest<8>(v, p.k);
      // numbers of 0 stand for no element
      if (lane == 0) s_floor = t ? (unsigned long long)t << 32 : 1ull;
    }
    __syncthreads();
    if (p.k > 0) {
      Best list{s_cand, s_kept, &s_n, &s_floor};
      auto add = [&](unsigned long long y, unsigned long long least) {
        const bool reaches = y >= least;
        const unsigned long long who = __ballot(reaches);
        int first = 0;
        if (lane == 0 && who) first = atomicAdd(&s_n, __popcll(who));
        first = __builtin_amdgcn_readfirstlane(first);
        const int to = first + __popcll(who & ((1ull << lane) - 1ull));
        if (reaches && to < kCand) s_cand[to] = y;
      };
      const unsigned long long least = s_floor;
#pragma unroll
      for (int q = 0; q < kJoinEach; ++q) add(got[q], least);
      for (int base = kJoinEach * kLpThreads; base < total; base += kLpThreads)
        add(base + tid < total ? in[base + tid] : 0ull, least);
      __syncthreads();
      int held = s_n;
      if (held > kCand) {  // in steps, as in the row kernel
        __syncthreads();
        if (tid == 0) s_n = 0;
        __syncthreads();
        held = walk_candidates(
            total, 1, kLpThreads, kLpThreads, kCand, p.k, [&](int all) { list.cut(all, p.k); },
            [&](int base, int) { add(base + tid < total ? in[base + tid] : 0ull, s_floor); },
            [&] { return s_n; }, [] { __syncthreads(); });
      }
      list.ranks(held, [&](unsigned long long x, int r) {
        if (r < p.k) write_alternative(p, row, r, x, s_row[0], s_row[1]);
      });
    }
    __syncthreads();
  }
}

// Short rows: a wave each, the row in registers (kPacks packs a lane), four rows a
// workgroup and no barriers.  Bound: the arithmetic and, with alternatives, the chain of
// steps that finds them (20,000 bf16 rows of 8,192: 60 us, 5.5 TB/s, with 20 alternatives
// 89; of 4,000 32 and 50 us; 65,536 of 1,000 37 us, with 50 alternatives 118).  The bound of
// the alternatives is the k-th largest of the packs' maxima; where more elements reach it
// than the list holds, the k-th largest element and, among its equals, the largest id that
// counts are found bit by bit (20,000 rows of 4,000 with ten allowed tokens, k = 20: 1.2 ms).
constexpr int kShortPacks = 16;   // of a lane, at most
constexpr int kShortCand = 256;   // elements held for ranking
constexpr int kShortList = 256;   // packs held for a second look
constexpr int kShortGrid = 1 << 20;
__device__ inline void wave_lds_order() {
  __builtin_amdgcn_wave_barrier();
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

template <bool kBf16, bool kRagged, int kPacks, bool kTop>
__global__ __launch_bounds__(kLpThreads, kPacks > 8 ? 3 : 4) void logprob_short(LogprobParams p) {
  using Span = RowSpan<kBf16, kRagged>;
  using P = typename Span::P;
  constexpr int kEpv = Span::kEpv;
  constexpr int kEs = Span::kEs;
  __shared__ unsigned long long s_cand[kLpWaves][kShortCand + kRankTurn];
  __shared__ int s_pack[kLpWaves][kShortList];
  const int lane = threadIdx.x & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const long long stride = (long long)gridDim.x * kLpWaves;
  for (long long row = (long long)blockIdx.x * kLpWaves + wid; row < p.n_rows; row += stride) {
    if (p.mask && !p.mask[row]) {
      write_masked_row(p, row, lane, kWave);
      continue;
    }
    const Given given = given_of(p, row);
    const char* const at_row = static_cast<const char*>(p.z) + row * p.ld * kEs;
    const int pre = kRagged ? (int)(reinterpret_cast<uintptr_t>(at_row) & 15u) / kEs : 0;
    const Span span{at_row, chunk_rsrc(at_row), p.vocab, -pre, (pre + p.vocab + kEpv - 1) / kEpv};
    P x[kPacks];
    int at[kPacks];
    unsigned bits[kPacks];
#pragma unroll
    for (int q = 0; q < kPacks; ++q) {
      at[q] = span.place(q * kWave + lane, bits[q]);
      span.load(x[q], at[q]);
    }
    // Others' elements count as -inf.  Of rows of any start whole packs are passed over
    // and only the packs at the ends are made so (4,500 rows of 2,136, k = 26: 23 to 18
    // us); of rows of whole packs, whose loops then spill, every lane's pack is asked.
    auto live = [&](int q) { return !kRagged || q * kWave < span.n; };
    auto value = [&](int q, int j) { return kRagged || bits[q] ? x[q].get(j) : -INFINITY; };
    float top[kPacks], best = -INFINITY;
#pragma unroll
    for (int q = 0; q < kPacks; ++q) {
      top[q] = -INFINITY;
      if (!live(q)) continue;
      if (kRagged && __any(bits[q] != (1u << kEpv) - 1u)) forbid(x[q], bits[q]);
#pragma unroll
      for (int j = 0; j < kEpv; ++j) top[q] = fmaxf(top[q], value(q, j));
      best = fmaxf(best, top[q]);
      x[q].fence();  // unpacked again, rather than kept
    }
    const float m = wave_max_dpp(best);
    const float u = m == -INFINITY ? 0.0f : m;
    float s = 0.0f, a = 0.0f;
#pragma unroll
    for (int q = 0; q < kPacks; ++q) {
      if (!live(q)) continue;
#pragma unroll
      for (int j = 0; j < kEpv; ++j) {
        const float y = (value(q, j) - u) * kLog2e;
        const float e = exp2_fast(y);
        s += e;
        a = fmaf(e, fmaxf(y, kFloor), a);
      }
      x[q].fence();
    }
    s = wave_sum_dpp(s);
    a = wave_sum_dpp(a);
    if (lane == 0) write_row(p, row, m, s, a, given);
    if constexpr (kTop) {
      const float l = log_sum(m, s);
      unsigned v[kPacks];
#pragma unroll
      for (int q = 0; q < kPacks; ++q) v[q] = bits[q] ? order_of(top[q]) : 0u;
      // (of up to 32 the lanes' maxima bound them nearly as well as the packs')
      constexpr int kLow = kBf16 ? 16 : 8;
      const unsigned lane_best[1] = {order_of(best)};
      const unsigned bound = 2 * p.k <= kWave ? kth_largest<kLow>(lane_best, p.k) : kth_largest<kLow>(v, p.k);
      unsigned long long* const cand = s_cand[wid];
      int held = 0;
      // Adds the elements of a pack (`mine`: which of them are the lane's) to the list,
      // where there is room, that keep(order, id) says yes to.
      auto add = [&](const P& y, int first, unsigned mine, auto keep) {
        unsigned in = 0;
#pragma unroll
        for (int j = 0; j < kEpv; ++j)
          if (keep(order_of(y.get(j)), first + j)) in |= 1u << j;
        in &= mine;
        int wave_in;
        int to = held + wave_exclusive_dpp(__popc(in), &wave_in);
        held += wave_in;
        if (!in) return;
#pragma unroll
        for (int j = 0; j < kEpv; ++j)
          if (((in >> j) & 1u) && to < kShortCand) cand[to++] = ranked(order_of(y.get(j)), first + j);
      };
      if constexpr (kPacks <= 2) {
#pragma unroll
        for (int q = 0; q < kPacks; ++q)
          add(x[q], at[q], bits[q], [&](unsigned o, int) { return o >= bound; });
      } else {
        // the packs whose largest reaches the bound, loaded again by a lane each
        int packs = 0;
#pragma unroll
        for (int q = 0; q < kPacks; ++q) {
          const bool in = v[q] >= bound && v[q] != 0u;
          const unsigned long long who = __ballot(in);
          const int i = packs + __popcll(who & ((1ull << lane) - 1ull));
          if (in && i < kShortList) s_pack[wid][i] = q * kWave + lane;
          packs += __popcll(who);
        }
        if (packs <= kShortList) {
          wave_lds_order();
          for (int base = 0; base < packs; base += kWave) {
            P y;
            unsigned mine = 0;
            int first = 0;
            if (base + lane < packs) {
              first = span.place(s_pack[wid][base + lane], mine);
              span.load(y, first);
            }
            add(y, first, mine, [&](unsigned o, int) { return o >= bound; });
          }
        } else {
          held = kShortCand + 1;
        }
      }
      if (held > kShortCand) {
        // Hands every pack to use(pack, its first element, its own elements): up to two a
        // lane from the registers, more (whose orders would fill them) from memory.
        auto each = [&](auto use) {
          if constexpr (kPacks <= 2) {
#pragma unroll
            for (int q = 0; q < kPacks; ++q) use(x[q], at[q], bits[q]);
          } else {
#pragma unroll 1
            for (int q = 0; q < kPacks; ++q) {
              P y;
              unsigned mine;
              const int first = span.place(q * kWave + lane, mine);
              span.load(y, first);
              use(y, first, mine);
            }
          }
        };
        // how many elements `which` says yes to
        auto number = [&](auto which) {
          int n = 0;
          each([&](const P& y, int first, unsigned mine) {
#pragma unroll
            for (int j = 0; j < kEpv; ++j)
              n += __popcll(__ballot(((mine >> j) & 1u) && which(order_of(y.get(j)), first + j)));
          });
          return n;
        };
        constexpr int kCut = kBf16 ? 16 : 0;  // a bf16's order is in its upper half
        unsigned k_th = 0;
#pragma unroll 1
        for (int b = 31; b >= kCut; --b) {
          const unsigned t = k_th | (1u << b);
          if (number([&](unsigned o, int) { return o >= t; }) >= p.k) k_th = t;
        }
        k_th >>= kCut;
        const int equal = p.k - number([&](unsigned o, int) { return o >> kCut > k_th; });
        int last = 0;  // the largest id with fewer than `equal` equals below it
#pragma unroll 1
        for (int b = 13; b >= 0; --b) {
          const int t = last | (1 << b);
          if (number([&](unsigned o, int id) { return o >> kCut == k_th && id < t; }) < equal) last = t;
        }
        held = 0;
        each([&](const P& y, int first, unsigned mine) {
          add(y, first, mine, [&](unsigned o, int id) {
            return o >> kCut > k_th || (o >> kCut == k_th && id <= last);
          });
        });
      }
      if (lane < kRankTurn) cand[held + lane] = 0ull;
      wave_lds_order();
      for (int i = lane; i < held; i += kWave) {
        const unsigned long long mine = cand[i];
        int r = 0;
        for (int j = 0; j < held; j += kRankTurn) {
          unsigned long long c[kRankTurn];
#pragma unroll
          for (int q = 0; q < kRankTurn; ++q) c[q] = cand[j + q];
#pragma unroll
          for (int q = 0; q < kRankTurn; ++q) r += c[q] > mine;
        }
        if (r < p.k) write_alternative(p, row, r, mine, m, l);
      }
      wave_lds_order();  // the list is rewritten for the next row
    }
  }
}

constexpr int kMaxChunkElems = 24 * kGroupElems;  // and one group more for rows of any start: 50 units a lane
constexpr int kMinChunkElems = 4096;
constexpr int kFillTasks = 768;  // three workgroups a CU, which every variant has room for
constexpr int kJoinGrid = 1 << 20;  // workgroups; beyond, each takes several rows

}  // namespace

// Chunks of a row: as many as its units' LDS asks for, and for few rows so many that
// they fill the card, of 4,096 elements at least (a depth that depends on sizes only, so
// that the workspace can be sized for it; with 1,280 tasks 173 fp32 rows of 45,230, k = 3,
// took 25 us instead of 20, 64 bf16 rows of 151,936, k = 128, 29 instead of 25, but k = 0
// a microsecond less).  From 385 rows on a row is one chunk: bf16 rows of 151,936
// without alternatives take, whole, in two chunks and in three, 200 of them 19.1, 16.6 and
// 17.4 us, 300 22.6, 22.5 and 22.2, 384 23.9, 24.8 and 27.0, 512 28.7, 31.2 and 30.3, 1,280
// 62.4, 65.6 and 66.2; with 20 alternatives whole rows win from 256 on (23.7, 24.4, 24.7).
static int chunks_by_size(long long vocab) {
  // ragged rows hold up to 64 elements more, and boundaries move by eight packs
  return (int)((vocab + 192 + kMaxChunkElems - 1) / kMaxChunkElems);
}
int logprob_chunks(long long n_rows, long long vocab) {
  const int by_size = chunks_by_size(vocab);
  if (n_rows < 1) return by_size;
  const long long fill = kFillTasks / n_rows, most = vocab / kMinChunkElems;
  const int by_rows = (int)(fill < most ? fill : most);
  return by_rows > by_size ? by_rows : by_size;
}

// Chunks of all rows together of any batch up to n_rows rows, where they are joined:
// the workspace has room for as many, so that one for n_rows rows serves fewer too, of
// which each is split into more.
long long logprob_room(long long n_rows, long long vocab) {
  const long long by_size = chunks_by_size(vocab), most = vocab / kMinChunkElems;
  const long long split = most > 1 ? (n_rows * most < kFillTasks ? n_rows * most : kFillTasks) : 0;
  const long long whole = by_size > 1 ? n_rows * by_size : 0;
  return split > whole ? split : whole;
}

template <bool kBf16, bool kRagged, bool kTop>
void launch_short(const LogprobParams& p, int packs, hipStream_t s) {
  const long long blocks = ((long long)p.n_rows + kLpWaves - 1) / kLpWaves;
  const int grid = (int)(blocks < kShortGrid ? blocks : kShortGrid);
  if (packs <= kWave) logprob_short<kBf16, kRagged, 1, kTop><<<grid, kLpThreads, 0, s>>>(p);
  else if (packs <= 2 * kWave) logprob_short<kBf16, kRagged, 2, kTop><<<grid, kLpThreads, 0, s>>>(p);
  else if (packs <= 4 * kWave) logprob_short<kBf16, kRagged, 4, kTop><<<grid, kLpThreads, 0, s>>>(p);
  else if (packs <= 8 * kWave) logprob_short<kBf16, kRagged, 8, kTop><<<grid, kLpThreads, 0, s>>>(p);
  else logprob_short<kBf16, kRagged, 16, kTop><<<grid, kLpThreads, 0, s>>>(p);
}

hipError_t launch_logprobs(const LogprobParams& p, hipStream_t s) {
  const int epv = p.bf16 ? 8 : 4;
  // packs of a row of any start, on 16-byte boundaries
  const int short_packs = (p.vocab + (p.ragged ? epv - 1 : 0) + epv - 1) / epv;
  const bool is_short = short_packs <= kShortPacks * kWave;
  LogprobParams q = p;
  // Many rows with a mask are listed, so that every workgroup gets as many of them;
  // where few are split only the join reports a bad id, and the row kernel can clear
  // the status itself.
  if (is_short || p.n_rows < kFillTasks) q.rows = nullptr;
  q.clear = !is_short && p.n_chunks > 1 && !q.rows;
  if (!q.clear || p.n_rows == 0)
    logprob_begin<<<1, q.rows ? kBeginThreads : kWave, 0, s>>>(q);
  if (p.n_rows == 0) return hipGetLastError();
#define TURNKL_LP(B, R, K) \
  if ((p.bf16 != 0) == B && (p.ragged != 0) == R && (p.k > 0) == K) launch_short<B, R, K>(p, short_packs, s);
  if (is_short) {
    TURNKL_LP(true, false, false) TURNKL_LP(true, false, true) TURNKL_LP(true, true, false)
    TURNKL_LP(true, true, true) TURNKL_LP(false, false, false) TURNKL_LP(false, false, true)
    TURNKL_LP(false, true, false) TURNKL_LP(false, true, true)
    return hipGetLastError();
  }
#undef TURNKL_LP
  const long long tasks = (long long)p.n_rows * p.n_chunks;
  // packs of the widest chunk: chunk_start's boundaries lie within eight packs
  const long long packs = ((long long)p.vocab + 127 / (16 / epv) + epv - 1) / epv;
  const long long widest = p.n_chunks == 1 ? packs : packs / p.n_chunks + 9;
  const int group = kLpThreads * group_packs(p.bf16 != 0);
  const int words = (int)((widest + group - 1) / group) * kLpThreads;
  const size_t lds = p.k > 0 ? (size_t)words * 4 : 0;
  // as many workgroups as the card holds at once
  const size_t each = lds + (p.k > 0 ? 11 * 1024 : 0);
  const int regs = rows_a_cu(p.bf16 != 0, p.ragged != 0, p.k > 0);
  const int per_cu = each * regs > 160 * 1024 ? (int)(160 * 1024 / each) : regs;
  const int grid = (int)(tasks < 256 * per_cu ? tasks : 256 * per_cu);
#define TURNKL_LP(B, R, K)                                                       \
  if ((p.bf16 != 0) == B && (p.ragged != 0) == R && (p.k > 0) == K)              \
    logprob_rows<B, R, K><<<grid, kLpThreads, lds, s>>>(q);
  TURNKL_LP(true, false, false) TURNKL_LP(true, false, true) TURNKL_LP(true, true, false)
  TURNKL_LP(true, true, true) TURNKL_LP(false, false, false) TURNKL_LP(false, false, true)
  TURNKL_LP(false, true, false) TURNKL_LP(false, true, true)
#undef TURNKL_LP
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (p.n_chunks > 1) {
    logprob_join<<<(int)(p.n_rows < kJoinGrid ? p.n_rows : kJoinGrid), kLpThreads, 0, s>>>(p);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace turnkl
