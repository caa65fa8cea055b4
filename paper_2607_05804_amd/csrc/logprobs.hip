// Token log probabilities: per row of logits the log-partition function, the
// entropy, the log probability of a given token and the K largest logits.
//
// Math.  With M = max z, S = sum 2^x, A = sum 2^x x over x = (z - M) log2 e:
//   L = ln S,  H = L - ln2 A / S,  log p_v = (z_v - M) - L.
// A wave sums against a reference of its own that follows the maximum: it moves
// (and the sums with it) when a group of packs holds a logit more than kSlack
// above it, so that no sum overflows and no second pass is needed; A / S then
// cancels a few units at most.  A is summed over max(x, kFloor): a forbidden
// token (-inf) gives 0 * kFloor, not 0 * -inf.
//
// Alternatives.  Ranking works on 64-bit numbers that order logits and ids at
// once: the logit's bits, made monotone, above the complement of its id.  While
// the row streams by, each thread keeps its largest logit, and the upper 16 bits
// of the largest of every eight elements (a unit) go to LDS.  The k-th largest of
// the threads' maxima is a bound that at least k elements reach, and few more do
// (about 56 for k = 50 and 256 threads when the large ones are spread evenly).
// Only the units that reach it are read again, and the elements that do are
// ranked against each other.  Where more do than the lists hold (equal logits,
// or a run of large ones), the row is read again in steps, and the list is cut
// to its best k, with a higher bound, whenever the next step might not fit.

#include <type_traits>

#include "row_span.h"

namespace turnkl {
namespace {

constexpr int kLpThreads = 256;
constexpr int kLpWaves = kLpThreads / kWave;
constexpr int kLpPacks = 4;        // packs in flight per lane
constexpr int kLpGrid = 1 << 22;   // workgroups; beyond, each takes several tasks
constexpr float kSlack = 8.0f;     // logit units
constexpr float kFloor = -256.0f;  // log2 units: 2^kFloor is zero
constexpr int kStep = 128;                            // packs looked at again at a time
constexpr int kCand = kMaxAlternatives + kStep * 8;   // elements held for ranking
constexpr int kList = 512;                            // units held for a second look

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

// The largest t with at least k of a wave's kPer numbers per lane >= t (0 if
// there are fewer): the k-th largest, bit by bit.
template <int kPer>
__device__ inline unsigned kth_largest(const unsigned (&v)[kPer], int k) {
  unsigned t = 0;
#pragma unroll 1
  for (int b = 31; b >= 0; --b) {
    const unsigned c = t | (1u << b);
    int n = 0;
#pragma unroll
    for (int q = 0; q < kPer; ++q) n += __popcll(__ballot(v[q] >= c));
    if (n >= k) t = c;
  }
  return t;
}

// The workgroup's list of candidates.  All threads call every function.
struct Best {
  unsigned long long* cand;  // LDS, kCand
  int* n;                    // LDS
  unsigned long long* floor;  // LDS: numbers below it are out

  // the rank of each of this thread's candidates tid, tid + 256, ...
  static constexpr int kMine = (kCand + kLpThreads - 1) / kLpThreads;
  __device__ void ranks(int count, unsigned long long (&x)[kMine], int (&r)[kMine]) const {
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      const int i = threadIdx.x + q * kLpThreads;
      x[q] = i < count ? cand[i] : 0ull;
      r[q] = 0;
    }
    const int mine = (count + kLpThreads - 1) / kLpThreads;
#pragma unroll 4
    for (int j = 0; j < count; ++j) {
      const unsigned long long c = cand[j];
      r[0] += c > x[0];
#pragma unroll
      for (int q = 1; q < kMine; ++q)
        if (q < mine) r[q] += c > x[q];
    }
  }
  // keeps the k best and raises the floor above the k-th
  __device__ void cut(int k) {
    unsigned long long x[kMine];
    int r[kMine];
    const int count = *n;
    ranks(count, x, r);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      if (x[q] == 0ull || r[q] >= k) continue;
      cand[r[q]] = x[q];
      if (r[q] == k - 1) *floor = x[q] + 1ull;
    }
    if (threadIdx.x == 0) *n = count < k ? count : k;
    __syncthreads();
  }
};

// What a row's outputs need once its maximum and sums are known.
__device__ inline void write_row(const LogprobParams& p, long long row, float m, float s, float a,
                                 float* s_row) {
  const bool empty = m == -INFINITY && s == 0.0f;
  const float l = empty ? 0.0f : kLn2 * log2f(s);
  s_row[0] = m;
  s_row[1] = l;
  if (p.entropy) p.entropy[row] = empty ? 0.0f : l - kLn2 * (a / s);
  if (p.log_z) {
    p.log_z[2 * row] = m;
    p.log_z[2 * row + 1] = l;
  }
  if (p.ids) {
    const int t = p.ids[row];
    const bool in = t >= 0 && t < p.vocab;
    if (!in) atomicMin(&p.hdr->err_key, err_key(row, kPrioTokenId));
    if (p.logp) {
      float z = __builtin_nanf("");
      if (in) {
        const long long at = row * p.ld + t;
        z = p.bf16 ? __uint_as_float((unsigned)static_cast<const unsigned short*>(p.z)[at] << 16)
                   : static_cast<const float*>(p.z)[at];
      }
      p.logp[row] = empty && in ? -INFINITY : (z - m) - l;
    }
  }
}

__device__ inline void write_masked_row(const LogprobParams& p, long long row) {
  if (threadIdx.x == 0) {
    if (p.logp) p.logp[row] = 0.0f;
    if (p.entropy) p.entropy[row] = 0.0f;
    if (p.log_z) {
      p.log_z[2 * row] = __builtin_nanf("");
      p.log_z[2 * row + 1] = __builtin_nanf("");
    }
  }
  for (int j = threadIdx.x; j < p.k; j += kLpThreads) {
    p.top_ids[row * p.ld_top + j] = -1;
    p.top_logp[row * p.ld_top + j] = -INFINITY;
  }
}

// Ranks the candidates and writes the row's alternatives.
__device__ inline void write_top(const LogprobParams& p, long long row, const Best& best, float m,
                                 float l) {
  unsigned long long x[Best::kMine];
  int r[Best::kMine];
  best.ranks(*best.n, x, r);
#pragma unroll
  for (int q = 0; q < Best::kMine; ++q) {
    if (x[q] == 0ull || r[q] >= p.k) continue;
    const float z = logit_of((unsigned)(x[q] >> 32));
    p.top_ids[row * p.ld_top + r[q]] = (int)~(unsigned)x[q];
    // NaN rows say so everywhere; -inf - -inf is -inf here
    p.top_logp[row * p.ld_top + r[q]] = z == -INFINITY && l == l ? -INFINITY : (z - m) - l;
  }
}

// The join of waves' or chunks' sums against their own references.
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

__global__ void logprob_begin(Header* hdr) { hdr->err_key = kNoError; }

// One workgroup per chunk of a row.
template <bool kBf16, bool kRagged, bool kTop>
__global__ __launch_bounds__(kLpThreads) void logprob_rows(LogprobParams p) {
  constexpr int kEpv = kBf16 ? 8 : 4;
  constexpr int kEs = kBf16 ? 2 : 4;
  constexpr int kUnitPacks = 8 / kEpv;                      // packs of a unit
  constexpr int kWords = kLpPacks / (2 * kUnitPacks);       // LDS words of a group: two units each
  constexpr int kStepBytes = kLpThreads * 16;
  using P = Pack<kBf16, kEpv>;
  extern __shared__ unsigned s_unit[];
  __shared__ float s_wave[kLpWaves][4];
  __shared__ float s_row[2];
  __shared__ unsigned s_max[kLpThreads];
  __shared__ unsigned long long s_cand[kCand];
  __shared__ unsigned long long s_floor;
  __shared__ int s_list[kList];
  __shared__ int s_n, s_units;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
  const long long n_tasks = (long long)p.n_rows * p.n_chunks;
  for (long long task = blockIdx.x; task < n_tasks; task += gridDim.x) {
    const long long row = task / p.n_chunks;
    const int c = (int)(task - row * p.n_chunks);
    if (p.mask && !p.mask[row]) {
      if (c == 0) write_masked_row(p, row);
      continue;
    }
    // packs [lo, hi) of the row; ragged rows: on the grid of 128-byte lines
    const char* const at_row = static_cast<const char*>(p.z) + row * p.ld * kEs;
    const int pre = kRagged ? (int)(reinterpret_cast<uintptr_t>(at_row) & 127u) / kEs : 0;
    const int n_row = (int)(((long long)pre + p.vocab + kEpv - 1) / kEpv);
    const int lo = (int)chunk_start(n_row, p.n_chunks, 8, c);
    const int n = (int)chunk_start(n_row, p.n_chunks, 8, c + 1) - lo;
    const int col = lo * kEpv - pre;  // first element of the chunk
    const RowSpan<kBf16, kRagged> span{at_row, chunk_rsrc(at_row), p.vocab, col, n};
    const int groups = (n + kLpThreads * kLpPacks - 1) / (kLpThreads * kLpPacks);

    float ref = -INFINITY, ss = 0.0f, aa = 0.0f;  // the wave's reference and lane sums
    float best = -INFINITY;                       // the lane's largest logit
    auto group = [&](int g, auto edge) {
      constexpr bool kEdge = decltype(edge)::value;
      P x[kLpPacks];
      unsigned bits[kLpPacks];
#pragma unroll
      for (int q = 0; q < kLpPacks; ++q) {
        const int v = g * kLpPacks + q;
        if constexpr (kEdge) {
          const int at = span.place(v * kLpThreads + tid, bits[q]);
          span.load(x[q], at);
        } else {
          x[q].load(span.rsrc, tid * 16, col * kEs + v * kStepBytes);
        }
      }
      float top[kLpPacks / kUnitPacks];
      float gm = -INFINITY;
#pragma unroll
      for (int q = 0; q < kLpPacks; ++q) {
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < kEpv; ++j) {
          const float z = x[q].get(j);
          m = fmaxf(m, kEdge && !((bits[q] >> j) & 1u) ? -INFINITY : z);
        }
        top[q / kUnitPacks] = q % kUnitPacks ? fmaxf(top[q / kUnitPacks], m) : m;
        gm = fmaxf(gm, m);
      }
      best = fmaxf(best, gm);
      if constexpr (kTop) {
#pragma unroll
        for (int w = 0; w < kWords; ++w)
          s_unit[(g * kWords + w) * kLpThreads + tid] =
              (order_of(top[2 * w]) >> 16) | (order_of(top[2 * w + 1]) & 0xFFFF0000u);
      }
      if (__any(gm > ref + kSlack)) {
        const float to = fmaxf(ref, wave_max(gm));
        const float d = ref == -INFINITY ? 0.0f : (ref - to) * kLog2e;
        const float f = exp2f(d);
        aa = f == 0.0f ? 0.0f : fmaf(ss, d, aa) * f;
        ss *= f;
        ref = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(to)));
      }
      const float u = ref == -INFINITY ? 0.0f : ref;
#pragma unroll
      for (int q = 0; q < kLpPacks; ++q) {
        x[q].fence();  // unpacked again, rather than kept
        float ps = 0.0f, pa = 0.0f;
#pragma unroll
        for (int j = 0; j < kEpv; ++j) {
          float y = (x[q].get(j) - u) * kLog2e;
          if (kEdge && !((bits[q] >> j) & 1u)) y = kFloor;
          const float e = exp2_fast(y);
          ps += e;
          pa = fmaf(e, fmaxf(y, kFloor), pa);
        }
        ss += ps;
        aa += pa;
      }
    };
    group(0, std::true_type{});
#pragma unroll 1
    for (int g = 1; g + 1 < groups; ++g) group(g, std::false_type{});
    if (groups > 1) group(groups - 1, std::true_type{});

    const float wm = wave_max(best);
    ss = wave_sum(ss);
    aa = wave_sum(aa);
    if (lane == 0) {
      s_wave[wid][0] = wm;
      s_wave[wid][1] = ref;
      s_wave[wid][2] = ss;
      s_wave[wid][3] = aa;
    }
    if (kTop) s_max[tid] = order_of(best);
    if (tid == 0) {
      s_n = 0;
      s_units = 0;
    }
    __syncthreads();
    if (tid == 0) {
      Sums t{-INFINITY, 0.0f, 0.0f};
      for (int w = 0; w < kLpWaves; ++w) t.m = fmaxf(t.m, s_wave[w][0]);
      for (int w = 0; w < kLpWaves; ++w) add_part(t, s_wave[w][1], s_wave[w][2], s_wave[w][3]);
      if (p.n_chunks == 1) {
        write_row(p, row, t.m, t.s, t.a, s_row);
      } else {
        float* const out = p.part + task * kLogprobPart;
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
        const unsigned t = kth_largest(v, p.k);
        if (lane == 0) s_floor = (unsigned long long)t << 32;
      }
      __syncthreads();
      Best list{s_cand, &s_n, &s_floor};
      const unsigned bound = (unsigned)(s_floor >> 32) & 0xFFFF0000u;
      for (int w = 0; w < groups * kWords; ++w) {
        const unsigned x = s_unit[w * kLpThreads + tid];
        const int first = w * 2 * kUnitPacks * kLpThreads + tid;  // the unit's first pack
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if ((h ? x & 0xFFFF0000u : x << 16) < bound) continue;
          const int i = atomicAdd(&s_units, 1);
          if (i < kList) s_list[i] = first + h * kUnitPacks * kLpThreads;
        }
      }
      __syncthreads();
      // the units' packs, or all of the chunk's where there are too many
      const bool listed = s_units <= kList;
      const int total = listed ? s_units * kUnitPacks : n;
      for (int base = 0; base < total; base += kStep) {
        const int j = base + tid;
        if (tid < kStep && j < total) {
          const int i = listed ? s_list[j / kUnitPacks] + j % kUnitPacks * kLpThreads : j;
          unsigned bits;
          const int at = span.place(i, bits);
          P x;
          span.load(x, at);
          const unsigned long long least = s_floor;
#pragma unroll
          for (int q = 0; q < kEpv; ++q) {
            const unsigned long long y = ranked(order_of(x.get(q)), at + q);
            if (((bits >> q) & 1u) && y >= least) s_cand[atomicAdd(&s_n, 1)] = y;
          }
        }
        __syncthreads();
        if (base + kStep < total) {
          const int held = s_n;
          __syncthreads();  // every thread has read it before the next step adds to it
          if (held > kMaxAlternatives) list.cut(p.k);
        }
      }
      if (p.n_chunks == 1) {
        write_top(p, row, list, s_row[0], s_row[1]);
      } else {
        unsigned long long x[Best::kMine];
        int r[Best::kMine];
        list.ranks(s_n, x, r);
        unsigned long long* const out = p.cand + task * p.k;
#pragma unroll
        for (int q = 0; q < Best::kMine; ++q)
          if (x[q] != 0ull && r[q] < p.k) out[r[q]] = x[q];
        for (int j = s_n + tid; j < p.k; j += kLpThreads) out[j] = 0ull;  // a chunk shorter than k
      }
    }
    __syncthreads();  // LDS is reused by the next task
  }
}

// Joins the chunks of a row: one workgroup per row.
__global__ __launch_bounds__(kLpThreads) void logprob_join(LogprobParams p) {
  __shared__ float s_row[2];
  __shared__ unsigned s_max[kLpThreads];
  __shared__ unsigned long long s_cand[kCand];
  __shared__ unsigned long long s_floor;
  __shared__ int s_n;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  for (long long row = blockIdx.x; row < p.n_rows; row += gridDim.x) {
    if (p.mask && !p.mask[row]) continue;  // written by the row kernel
    if (tid == 0) {
      const float* const part = p.part + row * p.n_chunks * kLogprobPart;
      Sums t{-INFINITY, 0.0f, 0.0f};
      for (int c = 0; c < p.n_chunks; ++c) t.m = fmaxf(t.m, part[c * kLogprobPart]);
      for (int c = 0; c < p.n_chunks; ++c)
        add_part(t, part[c * kLogprobPart], part[c * kLogprobPart + 1], part[c * kLogprobPart + 2]);
      write_row(p, row, t.m, t.s, t.a, s_row);
      s_n = 0;
    }
    if (p.k > 0) {
      const unsigned long long* const in = p.cand + row * p.n_chunks * p.k;
      const int total = p.n_chunks * p.k;
      unsigned long long best = 0;
      for (int j = tid; j < total; j += kLpThreads) best = in[j] > best ? in[j] : best;
      s_max[tid] = (unsigned)(best >> 32);
      __syncthreads();
      if (tid < kWave) {
        unsigned v[kLpWaves];
#pragma unroll
        for (int q = 0; q < kLpWaves; ++q) v[q] = s_max[q * kWave + lane];
        const unsigned t = kth_largest(v, p.k);
        // numbers of 0 stand for no element
        if (lane == 0) s_floor = t ? (unsigned long long)t << 32 : 1ull;
      }
      __syncthreads();
      Best list{s_cand, &s_n, &s_floor};
      constexpr int kEach = kStep * 8 / kLpThreads;
      for (int base = 0; base < total; base += kStep * 8) {
        const unsigned long long least = s_floor;
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
          const int j = base + q * kLpThreads + tid;
          const unsigned long long y = j < total ? in[j] : 0ull;
          if (y >= least) s_cand[atomicAdd(&s_n, 1)] = y;
        }
        __syncthreads();
        if (base + kStep * 8 < total) {
          const int held = s_n;
          __syncthreads();  // every thread has read it before the next step adds to it
          if (held > kMaxAlternatives) list.cut(p.k);
        }
      }
      write_top(p, row, list, s_row[0], s_row[1]);
    }
    __syncthreads();
  }
}

constexpr int kMaxChunkElems = 24 * kLpPacks * kLpThreads * 8;  // 48 KiB of units

}  // namespace

// Chunks of a row: as many as its units' LDS asks for.
int logprob_chunks(long long n_rows, long long vocab) {
  (void)n_rows;
  // ragged rows hold up to 64 elements more, and boundaries move by eight packs
  return (int)((vocab + 192 + kMaxChunkElems - 1) / kMaxChunkElems);
}

hipError_t launch_logprobs(const LogprobParams& p, hipStream_t s) {
  logprob_begin<<<1, 1, 0, s>>>(p.hdr);
  if (p.n_rows == 0) return hipGetLastError();
  const int epv = p.bf16 ? 8 : 4;
  const long long tasks = (long long)p.n_rows * p.n_chunks;
  const int grid = (int)(tasks < kLpGrid ? tasks : kLpGrid);
  // packs of the widest chunk: chunk_start's boundaries lie within eight packs
  const long long packs = ((long long)p.vocab + 127 / (16 / epv) + epv - 1) / epv;
  const long long widest = p.n_chunks == 1 ? packs : packs / p.n_chunks + 9;
  const int groups = (int)((widest + kLpThreads * kLpPacks - 1) / (kLpThreads * kLpPacks));
  const int words = groups * kLpPacks / (2 * (8 / epv)) * kLpThreads;
  const size_t lds = p.k > 0 ? (size_t)words * 4 : 0;
#define TURNKL_LP(B, R, K)                                                       \
  if ((p.bf16 != 0) == B && (p.ragged != 0) == R && (p.k > 0) == K)              \
    logprob_rows<B, R, K><<<grid, kLpThreads, lds, s>>>(p);
  TURNKL_LP(true, false, false) TURNKL_LP(true, false, true) TURNKL_LP(true, true, false)
  TURNKL_LP(true, true, true) TURNKL_LP(false, false, false) TURNKL_LP(false, false, true)
  TURNKL_LP(false, true, false) TURNKL_LP(false, true, true)
#undef TURNKL_LP
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (p.n_chunks > 1) {
    logprob_join<<<(int)(p.n_rows < kLpGrid ? p.n_rows : kLpGrid), kLpThreads, 0, s>>>(p);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace turnkl
