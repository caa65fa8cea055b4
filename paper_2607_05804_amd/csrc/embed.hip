// Rows of an embedding table for tokens, and the table's gradient.
//
// Forward: y_i = s E[t_i], one pass.  Bound: HBM, at the rate of a copy (65,536 bf16 rows
// of 4,096 out of 151,936: 141 us, 5.0 TB/s); 64 rows of 2,048: 4 us, a chain of three loads.
//
// Backward: dE[v] = s sum over the tokens i with t_i = v of g_i.  The
// tokens are sorted by id first (a stable radix sort of (id, token) pairs: in LDS by one
// workgroup for short batches, else two kernels a digit), so that every table row is one
// segment of the sorted order and no atomic decides in which order a row is summed.  The
// order is cut into runs of equal length whatever the segments: a token that fills a tenth
// of a batch then takes no longer than others.  A wave sums a run for 512 columns; a
// segment inside one run is written to the table, pieces of segments that cross from run
// to run go to the workspace, and a second kernel adds them, a fixed share a wave.
//
// The table's zeros are most of what is written.  Where the batch is small beside a large
// table all of it is zeroed beside the sort, which leaves the card idle (151,936 x 4,096
// in fp32: 362 to 395 us, 6.3 to 6.9 TB/s with the sort in it; the sums then 189 us at the
// rate of a copy, the join 11 to 12); else further workgroups of the summing kernel zero the rows
// that do not occur in the sorted order.  Bound: HBM, mostly those writes; of a small
// table three dependent kernels (1,500 tokens: 10, 10 and 4 us).

#include "units.h"

namespace turnkl {
namespace {

constexpr int kEmbThreads = 256;
constexpr int kEmbUnits = 4;    // of a lane, whose loads go out together
constexpr int kEmbGrid = 1 << 20;

template <bool kTab16, bool kOut16>
__global__ __launch_bounds__(kEmbThreads) void embed_rows(EmbedParams p) {
  const int lane = threadIdx.x & (p.lanes - 1);
  const int slot = threadIdx.x / p.lanes;
  const int side = kEmbThreads / p.lanes;  // rows side by side in a workgroup
  constexpr int kEl = unit_elements(kTab16, kOut16);
  const int units = (p.width + kEl - 1) / kEl;
  for (long long block = blockIdx.x; block < p.n_blocks; block += gridDim.x) {
    const long long row = block / p.parts * side + slot;
    const int first = (int)(block % p.parts) * (p.lanes * kEmbUnits) + lane;
    if (row >= p.n_rows) continue;
    const bool on = !p.mask || p.mask[row];
    const int id = on ? p.ids[row] : -1;
    const bool in = id >= 0 && id < p.vocab;
    const char* const from = static_cast<const char*>(p.table) + (in ? (long long)id * p.ld_table : 0) * (kTab16 ? 2 : 4);
    char* const to = static_cast<char*>(p.out) + row * p.ld_out * (kOut16 ? 2 : 4);
    Place<kEl> at[kEmbUnits];
    Unit<kTab16, kEl, true> x[kEmbUnits];
    Unit<kOut16, kEl> y[kEmbUnits];
#pragma unroll
    for (int q = 0; q < kEmbUnits; ++q) {
      const int u = first + q * p.lanes;
      at[q] = u < units ? place_unit<kEl>(u, p.width) : Place<kEl>{0, 0u};
      x[q].clear();
      if (in) load_unit(x[q], from, at[q], p.width);
    }
    // an id outside the table has no row: NaN, which cannot be taken for one
    const float none = on ? __builtin_nanf("") : 0.0f;
#pragma unroll
    for (int q = 0; q < kEmbUnits; ++q) {
      float v[kEl];
#pragma unroll
      for (int j = 0; j < kEl; ++j) v[j] = in ? x[q].get(j) * p.scale : none;
      y[q].set(v);
    }
#pragma unroll
    for (int q = 0; q < kEmbUnits; ++q) y[q].fence();
#pragma unroll
    for (int q = 0; q < kEmbUnits; ++q) store_edge(y[q], to, at[q]);
#pragma unroll
    for (int q = 0; q < kEmbUnits; ++q) store_whole(y[q], to, at[q]);
#pragma unroll
    for (int q = 0; q < kEmbUnits; ++q) y[q].keep();
    if (block + gridDim.x < p.n_blocks) drain_stores();  // before their data is rewritten
  }
}

// ---------------------------------------------------------------------------
// zeroing the table beside the sort

constexpr int kSortThreads = 512;
constexpr int kFillLine = 128;  // bytes

// 16 bytes of zeros at `from` of a run of `size` bytes, or as many of them as are its own.
template <int kEs, typename Vec>
__device__ __forceinline__ void zero_pack(char* run, long long size, long long from, bool stream) {
  const Vec z = {0u, 0u, 0u, 0u};
  if (from >= 0 && from + 16 <= size) {
    if (stream) __builtin_nontemporal_store(z, reinterpret_cast<Vec*>(run + from));
    else *reinterpret_cast<Vec*>(run + from) = z;
  } else {
    const long long end = from + 16 < size ? from + 16 : size;
    for (long long b = from > 0 ? from : 0; b < end; b += kEs) {
      if constexpr (kEs == 2) *reinterpret_cast<unsigned short*>(run + b) = 0;
      else *reinterpret_cast<unsigned*>(run + b) = 0u;
    }
  }
}

// The share of one of the sort's launches in zeroing the whole table, by the workgroups
// behind the p.n_tiles that sort: 16 bytes a thread, in address order, and nothing loaded
// before (2.5 GB: 6.9 TB/s; longer-lived workgroups write 5.7).  A table without padding is
// one run.  With it a row's packs are counted from the line that it starts in, so that waves
// write whole lines wherever rows start (93,051 bf16 rows of 6,688 at a stride of 6,782, with
// 798 tokens: 287 us, 324 from the rows' starts; of one run the arithmetic would cost more
// than it gives: 2.5 GB, with its sums, 650 us for 598).
template <int kEs>
__device__ inline void zero_share(const EmbedGradParams& p) {
  const unsigned per_row = p.fill_per_row;
  char* const table = static_cast<char*>(p.table);
  const long long stride = (long long)(gridDim.x - p.n_tiles) * kSortThreads;
  for (long long i = p.fill_from + (long long)(blockIdx.x - p.n_tiles) * kSortThreads; i < p.fill_to; i += stride) {
    if (i + threadIdx.x >= p.fill_to) continue;
    if (!per_row) {
      zero_pack<kEs, u32x4_any>(table, p.fill_elems * kEs, (i + threadIdx.x) * 16, p.fill_stream);
      continue;
    }
    const long long row0 = i / per_row;
    const unsigned q = (unsigned)(i - row0 * per_row) + threadIdx.x;
    char* const row = table + (row0 + q / per_row) * p.ld_table * kEs;
    const int skew = (int)(reinterpret_cast<uintptr_t>(row) & (kFillLine - 1));
    zero_pack<kEs, u32x4>(row, (long long)p.width * kEs, (long long)(q % per_row) * 16 - skew, p.fill_stream);
  }
}
__device__ inline bool zeroes_instead(const EmbedGradParams& p) {
  if ((int)blockIdx.x < p.n_tiles) return false;
  if (p.table_bf16) zero_share<2>(p);
  else zero_share<4>(p);
  return true;
}

// ---------------------------------------------------------------------------
// sorting by id

__device__ inline void wave_lds_order() {
  __builtin_amdgcn_wave_barrier();
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// The key of a token: its id, or the vocabulary's size where it takes no part (masked, or
// an id outside the table, which is recorded): such tokens come last.
__device__ inline int key_of(const EmbedGradParams& p, int i, bool record) {
  if (i >= p.n_rows || (p.mask && !p.mask[i])) return p.vocab;
  const int id = p.ids[i];
  if (id >= 0 && id < p.vocab) return id;
  if (record) atomicMin(&p.hdr->err_key, err_key(i, kPrioTokenId));
  return p.vocab;
}

// The lanes whose digit (of kBits bits) is this lane's.
template <int kBits>
__device__ inline unsigned long long same_digit(int d) {
  unsigned long long m = ~0ull;
#pragma unroll
  for (int b = 0; b < kBits; ++b) {
    const unsigned long long one = __ballot((d >> b) & 1);
    m &= (d >> b) & 1 ? one : ~one;
  }
  return m;
}

constexpr int kSortWaves = kSortThreads / kWave;
constexpr int kSmallSort = kEmbedSmallSort;
constexpr int kSmallSteps = kSmallSort / kSortThreads;

// A batch of up to kSmallSort tokens: one workgroup, eight bits a turn.
__global__ __launch_bounds__(kSortThreads) void embed_sort_small(EmbedGradParams p) {
  constexpr int kDigits = 256;
  __shared__ int s_key[2][kSmallSort];
  __shared__ unsigned short s_tok[2][kSmallSort];
  __shared__ int s_hist[kSortWaves][kDigits];
  __shared__ int s_scan[kSortWaves];
  if (zeroes_instead(p)) return;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
  if (tid == 0) {
    p.hdr->err_key = kNoError;
    drain_stores();  // complete before any token reports to it
  }
  __syncthreads();
  const int steps = (p.n_rows + kSortThreads - 1) / kSortThreads;
  for (int s = 0; s < steps; ++s) {
    const int i = s * kSortThreads + tid;
    s_key[0][i] = key_of(p, i, true);
    s_tok[0][i] = (unsigned short)i;
  }
  int cur = 0;
  for (int shift = 0; shift < p.key_bits; shift += 8) {
    for (int d = lane; d < kDigits; d += kWave) s_hist[wid][d] = 0;
    __syncthreads();
    int key[kSmallSteps], tok[kSmallSteps], rank[kSmallSteps];
    const int first = wid * steps * kWave;
#pragma unroll
    for (int s = 0; s < kSmallSteps; ++s) {
      if (s >= steps) break;
      key[s] = s_key[cur][first + s * kWave + lane];
      tok[s] = s_tok[cur][first + s * kWave + lane];
      const int d = (key[s] >> shift) & (kDigits - 1);
      const unsigned long long same = same_digit<8>(d);
      const int before = __popcll(same & ((1ull << lane) - 1ull));
      const int seen = s_hist[wid][d];
      rank[s] = seen + before;
      wave_lds_order();
      if (before == 0) s_hist[wid][d] = seen + __popcll(same);
      wave_lds_order();
    }
    __syncthreads();
    int total = 0;
    if (tid < kDigits)
      for (int w = 0; w < kSortWaves; ++w) {
        const int c = s_hist[w][tid];
        s_hist[w][tid] = total;
        total += c;
      }
    int all;
    const int base = block_exclusive_scan<kSortThreads>(total, s_scan, &all);
    if (tid < kDigits)
      for (int w = 0; w < kSortWaves; ++w) s_hist[w][tid] += base;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kSmallSteps; ++s) {
      if (s >= steps) break;
      const int to = s_hist[wid][(key[s] >> shift) & (kDigits - 1)] + rank[s];
      s_key[cur ^ 1][to] = key[s];
      s_tok[cur ^ 1][to] = (unsigned short)tok[s];
    }
    cur ^= 1;
    __syncthreads();
  }
  for (int i = tid; i < p.n_rows; i += kSortThreads) {
    p.key_out[i] = s_key[cur][i];
    p.tok_out[i] = s_tok[cur][i];
  }
}

// Longer batches, kEmbedDigitBits bits a turn: how often each digit occurs in each of
// p.n_tiles tiles of consecutive tokens ...
constexpr int kDigits = 1 << kEmbedDigitBits;
static_assert(kDigits == kSortThreads, "a thread per digit");
__global__ __launch_bounds__(kSortThreads) void embed_count(EmbedGradParams p) {
  __shared__ int s_count[kDigits];
  if (zeroes_instead(p)) return;
  s_count[threadIdx.x] = 0;
  if (p.turn == 0 && blockIdx.x == 0 && threadIdx.x == 0) p.hdr->err_key = kNoError;
  __syncthreads();
  const long long lo = (long long)blockIdx.x * p.tile;
  const long long hi = lo + p.tile < p.n_rows ? lo + p.tile : p.n_rows;
  for (long long i = lo + threadIdx.x; i < hi; i += kSortThreads) {
    const int key = p.turn == 0 ? key_of(p, (int)i, false) : p.key_in[i];
    atomicAdd(&s_count[(key >> (p.turn * kEmbedDigitBits)) & (kDigits - 1)], 1);
  }
  __syncthreads();
  p.count[(long long)blockIdx.x * kDigits + threadIdx.x] = s_count[threadIdx.x];
}

// ... and each tile's tokens to where they belong: behind those of lower digits and of
// earlier tiles, in their order.
constexpr int kScatterSteps = 4;  // of a wave between two barriers
__global__ __launch_bounds__(kSortThreads) void embed_scatter(EmbedGradParams p) {
  __shared__ int s_hist[kSortWaves][kDigits];
  __shared__ int s_base[kDigits];
  __shared__ int s_scan[kSortWaves];
  if (zeroes_instead(p)) return;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int shift = p.turn * kEmbedDigitBits;
  {
    int before = 0, total = 0;
#pragma unroll 8
    for (int b = 0; b < p.n_tiles; ++b) {
      const int c = p.count[(long long)b * kDigits + tid];
      before += b < (int)blockIdx.x ? c : 0;
      total += c;
    }
    int all;
    s_base[tid] = block_exclusive_scan<kSortThreads>(total, s_scan, &all) + before;
  }
  const long long lo = (long long)blockIdx.x * p.tile;
  const long long hi = lo + p.tile < p.n_rows ? lo + p.tile : p.n_rows;
  for (long long at = lo; at < hi; at += kSortThreads * kScatterSteps) {
    for (int d = lane; d < kDigits; d += kWave) s_hist[wid][d] = 0;
    __syncthreads();
    const long long first = at + wid * (kScatterSteps * kWave) + lane;
    int key[kScatterSteps], tok[kScatterSteps], rank[kScatterSteps];
#pragma unroll
    for (int s = 0; s < kScatterSteps; ++s) {
      const long long i = first + s * kWave;
      const bool in = i < hi;
      key[s] = !in ? 0 : p.turn == 0 ? key_of(p, (int)i, true) : p.key_in[i];
      tok[s] = !in ? 0 : p.turn == 0 ? (int)i : p.tok_in[i];
    }
#pragma unroll
    for (int s = 0; s < kScatterSteps; ++s) {
      const bool in = first + s * kWave < hi;
      const int d = (key[s] >> shift) & (kDigits - 1);
      const unsigned long long same = same_digit<kEmbedDigitBits>(d) & __ballot(in);
      const int before = __popcll(same & ((1ull << lane) - 1ull));
      const int seen = s_hist[wid][d];
      rank[s] = seen + before;
      wave_lds_order();
      if (in && before == 0) s_hist[wid][d] = seen + __popcll(same);
      wave_lds_order();
    }
    __syncthreads();
    {
      int next = s_base[tid];
      for (int w = 0; w < kSortWaves; ++w) {
        const int c = s_hist[w][tid];
        s_hist[w][tid] = next;
        next += c;
      }
      s_base[tid] = next;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kScatterSteps; ++s) {
      if (first + s * kWave >= hi) continue;
      const int to = s_hist[wid][(key[s] >> shift) & (kDigits - 1)] + rank[s];
      p.key_out[to] = key[s];
      p.tok_out[to] = tok[s];
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// summing

constexpr int kSumCols = kEmbedTileCols;  // columns of a wave
constexpr int kSumBatch = 4;              // rows whose loads are under way together

// A lane's columns of a run of 512: two units of four, 256 columns apart.
constexpr int kSumEl = 4;
constexpr int kSumUnits = 2;
using SumPlace = Place<kSumEl>;
__device__ inline void sum_places(int tile, int lane, int width, SumPlace (&at)[kSumUnits]) {
#pragma unroll
  for (int q = 0; q < kSumUnits; ++q)
    at[q] = place_unit<kSumEl>(tile * (kSumCols / kSumEl) + q * kWave + lane, width);
}

// They are stored, or added to what is there.
template <bool kTab16>
__device__ inline void write_table(const EmbedGradParams& p, int id, const SumPlace (&at)[kSumUnits],
                                   const float (&sum)[kSumUnits][kSumEl]) {
  char* const row = static_cast<char*>(p.table) + (long long)id * p.ld_table * (kTab16 ? 2 : 4);
  Unit<kTab16, kSumEl> old[kSumUnits], out[kSumUnits];
  if (p.accumulate) {
#pragma unroll
    for (int q = 0; q < kSumUnits; ++q) load_unit(old[q], row, at[q], p.width);
  }
#pragma unroll
  for (int q = 0; q < kSumUnits; ++q) {
    float v[kSumEl];
#pragma unroll
    for (int j = 0; j < kSumEl; ++j) {
      v[j] = sum[q][j] * p.scale;
      if (p.accumulate) v[j] += old[q].get(j);
    }
    out[q].set(v);
  }
#pragma unroll
  for (int q = 0; q < kSumUnits; ++q) out[q].fence();
#pragma unroll
  for (int q = 0; q < kSumUnits; ++q) store_edge(out[q], row, at[q]);
#pragma unroll
  for (int q = 0; q < kSumUnits; ++q) store_whole(out[q], row, at[q]);
#pragma unroll
  for (int q = 0; q < kSumUnits; ++q) out[q].keep();
  store_gap();
}

// The first position of the sorted keys whose key is at least v, by all lanes of a wave:
// 64 places are looked at at a time.
__device__ inline int first_at_least(const int* key, int n, int v) {
  const int lane = threadIdx.x & (kWave - 1);
  long long lo = 0, hi = n;  // the answer lies in [lo, hi]
  while (hi > lo) {
    const long long step = (hi - lo + kWave - 1) / kWave;
    const long long i = lo + step * lane;
    const unsigned long long less = __ballot(i < hi && key[i < hi ? i : lo] < v);
    if (!less) break;  // the first one is not less
    const int last = 63 - __clzll((long long)less);  // the keys are sorted: the lanes up to it
    const long long at = lo + step * last;
    hi = at + step < hi ? at + step : hi;
    lo = at + 1;
  }
  return (int)lo;
}

// Zeroes those of fill_rows table rows that no token has.
template <bool kTab16>
__device__ inline void zero_absent(const EmbedGradParams& p, int block) {
  __shared__ unsigned s_seen[kEmbedFillRows / 32];
  const int tid = threadIdx.x;
  const long long first = (long long)block * p.fill_rows;
  const int rows = (int)(p.vocab - first < p.fill_rows ? p.vocab - first : p.fill_rows);
  for (int i = tid; i < kEmbedFillRows / 32; i += kEmbThreads) s_seen[i] = 0u;
  __syncthreads();
  const int* const key = p.key_in;
  const int lo = first_at_least(key, p.n_rows, (int)first);  // every wave finds it
  for (long long base = lo; base < p.n_rows; base += kEmbThreads) {
    const long long i = base + tid;
    const int k = i < p.n_rows ? key[i] : p.vocab;
    const bool in = k < first + rows;
    if (in) atomicOr(&s_seen[(k - first) >> 5], 1u << ((k - first) & 31));
    if (!__syncthreads_or(in)) break;  // sorted: none of those that follow either
  }
  __syncthreads();
  // 16 bytes a thread side by side (32 as two stores leave gaps in every line that a wave
  // writes), as many threads to a row as it has such packs
  constexpr int kEs = kTab16 ? 2 : 4, kPack = 16 / kEs;
  const int packs = p.width / kPack, rest = p.width - packs * kPack;
  int lanes = kEmbThreads;
  while (lanes > 1 && lanes / 2 >= packs + (rest > 0)) lanes /= 2;
  u32x4 none{0u, 0u, 0u, 0u};
  settle_words(none);
  for (int r = tid / lanes; r < rows; r += kEmbThreads / lanes) {
    if ((s_seen[r >> 5] >> (r & 31)) & 1u) continue;
    char* const row = static_cast<char*>(p.table) + (first + r) * p.ld_table * kEs;
    for (int u = tid % lanes; u < packs + (rest > 0); u += lanes) {
      if (u < packs) {
        u32x4_any* const at = reinterpret_cast<u32x4_any*>(row + 16 * u);
        if (p.fill_stream) __builtin_nontemporal_store(u32x4_any(none), at);
        else *at = none;
      } else {
        for (int j = packs * kPack; j < p.width; ++j) {
          if constexpr (kTab16) reinterpret_cast<unsigned short*>(row)[j] = 0;
          else reinterpret_cast<unsigned*>(row)[j] = 0u;
        }
      }
    }
  }
  keep_alive(none);
}

template <bool kGrad16, bool kTab16>
__global__ __launch_bounds__(kEmbThreads) void embed_sum(EmbedGradParams p) {
  if ((int)blockIdx.x >= p.sum_blocks) {
    zero_absent<kTab16>(p, (int)blockIdx.x - p.sum_blocks);
    return;
  }
  const int lane = threadIdx.x & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const long long task = (long long)blockIdx.x * (kEmbThreads / kWave) + wid;
  const int run = (int)(task / p.col_tiles), tile = (int)(task % p.col_tiles);
  if (run >= p.n_runs) return;
  const int* const keys = p.key_in;
  const int* const toks = p.tok_in;
  const long long start = (long long)run * p.run;
  const long long mine = start + lane;
  const bool held = lane < p.run && mine < p.n_rows;
  const int key = held ? keys[mine] : p.vocab;
  const int tok = held ? toks[mine] : 0;
  const int key_before = start > 0 ? keys[start - 1] : -1;
  const int key_after = start + p.run < p.n_rows ? keys[start + p.run] : p.vocab;
  const int count = __popcll(__ballot(key < p.vocab));  // sorted: the first ones
  SumPlace at[kSumUnits];
  sum_places(tile, lane, p.width, at);
  const long long ld = p.ld_grad * (kGrad16 ? 2 : 4);
  float sum[kSumUnits][kSumEl];
  auto restart = [&] {
#pragma unroll
    for (int q = 0; q < kSumUnits; ++q)
#pragma unroll
      for (int j = 0; j < kSumEl; ++j) sum[q][j] = 0.0f;
  };
  restart();
  float* const part = p.part + (long long)run * 2 * p.part_ld + tile * kSumCols + lane * kSumEl;
  int begun = 0;  // position where the segment at hand begins in the run
  // A batch's rows are asked for before the one ahead is summed: loads behind a store are
  // not seen until it has been acknowledged.
  using Batch = Unit<kGrad16, kSumEl>[kSumBatch][kSumUnits];
  auto fetch = [&](Batch& g, int i0) {
#pragma unroll
    for (int b = 0; b < kSumBatch; ++b)
#pragma unroll
      for (int q = 0; q < kSumUnits; ++q) {
        g[b][q].clear();
        if (i0 + b < count)
          load_unit(g[b][q], static_cast<const char*>(p.grad) + __builtin_amdgcn_readlane(tok, i0 + b) * ld, at[q],
                    p.width);
      }
  };
  auto add = [&](const Batch& g, int i0) {
#pragma unroll
    for (int b = 0; b < kSumBatch; ++b) {
      const int i = i0 + b;
      if (i >= count) break;
#pragma unroll
      for (int q = 0; q < kSumUnits; ++q)
#pragma unroll
        for (int j = 0; j < kSumEl; ++j) sum[q][j] += g[b][q].get(j);
      const int id = __builtin_amdgcn_readlane(key, i);
      const bool run_ends = i + 1 == p.run;
      const int next = run_ends ? key_after : i + 1 < count ? __builtin_amdgcn_readlane(key, i + 1) : p.vocab;
      if (!run_ends && next == id) continue;
      const bool whole_front = begun > 0 || key_before != id;
      if (whole_front && next != id) {
        write_table<kTab16>(p, id, at, sum);
      } else {
        // a piece: behind [1] where the segment begins here, else in front [0]
        char* const to = reinterpret_cast<char*>(part + (whole_front ? p.part_ld : 0));
        Unit<false, kSumEl> piece[kSumUnits];
#pragma unroll
        for (int q = 0; q < kSumUnits; ++q) {
          piece[q].set(sum[q]);
          piece[q].fence();
        }
#pragma unroll
        for (int q = 0; q < kSumUnits; ++q) piece[q].store(to, q * kWave * kSumEl);
#pragma unroll
        for (int q = 0; q < kSumUnits; ++q) piece[q].keep();
        store_gap();
      }
      begun = i + 1;
      restart();
    }
  };
  Batch even, odd;
  fetch(even, 0);
#pragma unroll 1
  for (int i0 = 0; i0 < count; i0 += 2 * kSumBatch) {
    fetch(odd, i0 + kSumBatch);
    add(even, i0);
    fetch(even, i0 + 2 * kSumBatch);
    add(odd, i0 + kSumBatch);
  }
}

// Adds the pieces of the segment that begins in a run and goes on in the next ones: a
// workgroup per run and 512 columns, whose waves take the pieces in turn.  They are added in
// 64 bits: a token may have thousands of them (1,024 in sequence a wave in floats: a sum of
// 32,768 equal numbers off by 255 2^-24).
template <bool kTab16>
__global__ __launch_bounds__(kEmbThreads) void embed_join(EmbedGradParams p) {
  constexpr int kWaves = kEmbThreads / kWave;
  __shared__ double s_sum[kWaves][kSumCols];
  const int lane = threadIdx.x & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int run = p.first_join + blockIdx.x / p.col_tiles, tile = blockIdx.x % p.col_tiles;
  const int* const keys = p.key_in;
  const long long end = (long long)(run + 1) * p.run;  // of the run, the next one's start
  if (end >= p.n_rows) return;
  const int id = keys[end];
  if (id >= p.vocab || keys[end - 1] != id) return;  // nothing goes on
  const long long start = end - p.run;
  if (start > 0 && keys[start] == id && keys[start - 1] == id) return;  // it began earlier
  // the runs that start with it
  int last = run;
  for (;;) {
    const long long r = (long long)last + 1 + lane;
    const unsigned long long go = __ballot(r < p.n_runs && keys[r < p.n_runs ? r * p.run : 0] == id);
    const int n = go == ~0ull ? kWave : __ffsll((long long)~go) - 1;
    last += n;
    if (n < kWave) break;
  }
  const float* const part = p.part + tile * kSumCols + lane * kSumEl;
  SumPlace at[kSumUnits];
  sum_places(tile, lane, p.width, at);
  double sum[kSumUnits][kSumEl] = {};
#pragma unroll 4
  for (int r = run + wid; r <= last; r += kWaves) {
    const char* const from = reinterpret_cast<const char*>(part + ((long long)r * 2 + (r == run ? 1 : 0)) * p.part_ld);
#pragma unroll
    for (int q = 0; q < kSumUnits; ++q) {
      Unit<false, kSumEl> x;
      x.load(from, q * kWave * kSumEl);
#pragma unroll
      for (int j = 0; j < kSumEl; ++j) sum[q][j] += x.get(j);
    }
  }
#pragma unroll
  for (int q = 0; q < kSumUnits; ++q)
#pragma unroll
    for (int j = 0; j < kSumEl; ++j) s_sum[wid][(q * kSumEl + j) * kWave + lane] = sum[q][j];
  __syncthreads();
  if (wid != 0) return;
  // (one wave's at a time: with all of them in registers the kernel takes 14 us for 11)
#pragma unroll 1
  for (int w = 1; w < kWaves; ++w)
#pragma unroll
    for (int q = 0; q < kSumUnits; ++q)
#pragma unroll
      for (int j = 0; j < kSumEl; ++j) sum[q][j] += s_sum[w][(q * kSumEl + j) * kWave + lane];
  float joined[kSumUnits][kSumEl];
#pragma unroll
  for (int q = 0; q < kSumUnits; ++q)
#pragma unroll
    for (int j = 0; j < kSumEl; ++j) joined[q][j] = (float)sum[q][j];
  write_table<kTab16>(p, id, at, joined);
}

}  // namespace

// Tokens of a run: as many as leave every compute unit sixteen waves, 8 to 64.
EmbedShape embed_shape(long long n, long long vocab, long long width) {
  EmbedShape s{};
  s.col_tiles = (int)((width + kEmbedTileCols - 1) / kEmbedTileCols);
  s.part_ld = (long long)s.col_tiles * kEmbedTileCols;
  s.run = 64;
  while (s.run > 8 && (n + s.run - 1) / s.run * s.col_tiles < kEmbedWaves) s.run /= 2;
  s.n_runs = (n + s.run - 1) / s.run;
  // Room for the pieces of any smaller batch of narrower rows too: of runs of 64 no more
  // than here, of shorter ones (which twice as long would be fewer than kEmbedWaves) less
  // than 2 kEmbedWaves times the columns of a wave, and one for eight tokens.
  const long long few = 2ll * kEmbedWaves * kEmbedTileCols, eighth = (n + 7) / 8 * s.part_ld;
  const long long full = (n + 63) / 64 * s.part_ld, least = few < eighth ? few : eighth;
  s.room = 2 * (full > least ? full : least);
  s.tile = 2048;
  if (n > 256 * s.tile) s.tile = ((n + 255) / 256 + 2047) / 2048 * 2048;
  s.n_tiles = (n + s.tile - 1) / s.tile;
  s.key_bits = 1;
  while ((vocab >> s.key_bits) != 0) ++s.key_bits;
  return s;
}

hipError_t launch_embed(const EmbedParams& given, hipStream_t s) {
  EmbedParams p = given;
  if (p.n_rows == 0) return hipSuccess;
  const int el = unit_elements(p.table_bf16, p.out_bf16);
  const int units = (p.width + el - 1) / el;
  p.lanes = 1;
  while (p.lanes < kWave && p.lanes < units) p.lanes *= 2;
  p.parts = (units + p.lanes * kEmbUnits - 1) / (p.lanes * kEmbUnits);
  const int side = kEmbThreads / p.lanes;
  p.n_blocks = ((long long)p.n_rows + side - 1) / side * p.parts;
  const int grid = (int)(p.n_blocks < kEmbGrid ? p.n_blocks : kEmbGrid);
  if (p.table_bf16 && p.out_bf16) embed_rows<true, true><<<grid, kEmbThreads, 0, s>>>(p);
  else if (p.table_bf16) embed_rows<true, false><<<grid, kEmbThreads, 0, s>>>(p);
  else if (p.out_bf16) embed_rows<false, true><<<grid, kEmbThreads, 0, s>>>(p);
  else embed_rows<false, false><<<grid, kEmbThreads, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_embed_bwd(const EmbedGradParams& given, hipStream_t s) {
  EmbedGradParams p = given;
  const int es = p.table_bf16 ? 2 : 4;
  // A table is zeroed whole, beside the sort, where the tokens touch little of it and its
  // zeros are worth hiding (whole against only the absent rows: 32,000 x 2,048 fp32, 1,500
  // tokens, 57 against 63 us; 32,000 x 1,024 bf16, 4,000 tokens, 41 against 37, 15,000 of
  // 1,000 columns 49 against 45, where the sort's launches get in each other's way; with the
  // sort of one launch, 1 token of 45,386 x 544 bf16, 13.6 against 16.8, 131 of 1,371 x
  // 10,730 18.7 against 21.6, which this border by bytes gives away); else where it has no
  // token, beside the sums.  Past 192 MB, which the last cache holds
  // beside the gradient, its zeros go past the caches.
  const double bytes = (double)p.vocab * p.width * es;
  p.fill_stream = bytes > kEmbedCachedFill;
  const bool whole = !p.accumulate && p.n_rows <= p.vocab / 2 && bytes >= kEmbedWholeFill;
  const bool small = p.n_rows <= kEmbedSmallSort;
  const int turns = small ? 1 : (p.key_bits + kEmbedDigitBits - 1) / kEmbedDigitBits;
  const int launches = small ? 1 : 2 * turns;
  long long packs = 0, fills = 0;  // of the table, and workgroups of a launch for them
  if (whole) {
    const long long row = ((long long)p.width * es + 2 * kFillLine - 2) / kFillLine * (kFillLine / 16);
    p.fill_per_row = p.ld_table == p.width ? 0 : (unsigned)row;
    p.fill_elems = (long long)p.vocab * p.width;
    packs = p.fill_per_row ? row * p.vocab : (p.fill_elems * es + 15) / 16;
    fills = (packs / launches + kSortThreads) / kSortThreads;
    fills = fills < kEmbedFillBlocks ? fills : kEmbedFillBlocks;
  }
  auto share = [&](int launch) {
    p.fill_from = packs * launch / launches;
    p.fill_to = packs * (launch + 1) / launches;
  };
  if (small) {
    p.key_out = p.key[0];
    p.tok_out = p.tok[0];
    p.n_tiles = 1;
    share(0);
    embed_sort_small<<<1 + (int)fills, kSortThreads, 0, s>>>(p);
    p.key_in = p.key_out;
    p.tok_in = p.tok_out;
  }
  for (p.turn = 0; !small && p.turn < turns; ++p.turn) {
    p.key_out = p.key[p.turn & 1];
    p.tok_out = p.tok[p.turn & 1];
    share(2 * p.turn);
    embed_count<<<p.n_tiles + (int)fills, kSortThreads, 0, s>>>(p);
    share(2 * p.turn + 1);
    embed_scatter<<<p.n_tiles + (int)fills, kSortThreads, 0, s>>>(p);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    p.key_in = p.key_out;
    p.tok_in = p.tok_out;
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const long long tasks = (long long)p.n_runs * p.col_tiles;
  p.sum_blocks = (int)((tasks + kEmbThreads / kWave - 1) / (kEmbThreads / kWave));
  p.fill_rows = kEmbedFillRows;
  while (p.fill_rows > 2 && (long long)p.fill_rows * p.width > kEmbedFillElems) p.fill_rows /= 2;
  const int absent = p.accumulate || whole ? 0 : (int)(((long long)p.vocab + p.fill_rows - 1) / p.fill_rows);
  if (p.sum_blocks + absent == 0) return hipSuccess;
  const int grid = p.sum_blocks + absent;
  if (p.grad_bf16 && p.table_bf16) embed_sum<true, true><<<grid, kEmbThreads, 0, s>>>(p);
  else if (p.grad_bf16) embed_sum<true, false><<<grid, kEmbThreads, 0, s>>>(p);
  else if (p.table_bf16) embed_sum<false, true><<<grid, kEmbThreads, 0, s>>>(p);
  else embed_sum<false, false><<<grid, kEmbThreads, 0, s>>>(p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (p.n_runs > 1) {
    // (a workgroup for each of 2^24 runs would be more threads than a launch can hold)
    const int most = kEmbedJoinBlocks / p.col_tiles;
    for (p.first_join = 0; p.first_join < p.n_runs - 1; p.first_join += most) {
      const int left = p.n_runs - 1 - p.first_join;
      const int grid = (left < most ? left : most) * p.col_tiles;
      if (p.table_bf16) embed_join<true><<<grid, kEmbThreads, 0, s>>>(p);
      else embed_join<false><<<grid, kEmbThreads, 0, s>>>(p);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
  }
  return hipGetLastError();
}

}  // namespace turnkl
