// Rows of an embedding table for tokens, and the table's gradient.
//
// Forward: y_i = s E[t_i], one pass; bound: HBM.
//
// Backward: dE[v] = s sum over the tokens i with t_i = v, in the order of i, of g_i.  The
// tokens are sorted by id first (a stable radix sort of (id, token) pairs: in LDS by one
// workgroup for short batches, else two kernels a digit), so that every table row is one
// segment of the sorted order and no atomic decides in which order a row is summed.  The
// order is cut into runs of equal length whatever the segments: a token that fills a tenth
// of a batch then takes no longer than others.  A wave sums a run for 512 columns; a
// segment inside one run is written to the table, pieces of segments that cross from run
// to run go to the workspace, and a second kernel adds them in the order of the runs.  The
// table's other rows are zeroed by further workgroups of the summing kernel, which find
// the rows that occur in the sorted order.  Bound: HBM, mostly the writes of the table.

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
  const int units = (p.width + kUnit - 1) / kUnit;
  for (long long block = blockIdx.x; block < p.n_blocks; block += gridDim.x) {
    const long long row = block / p.parts * side + slot;
    const int first = (int)(block % p.parts) * (p.lanes * kEmbUnits) + lane;
    if (row >= p.n_rows) continue;
    const bool on = !p.mask || p.mask[row];
    const int id = on ? p.ids[row] : -1;
    const bool in = id >= 0 && id < p.vocab;
    const char* const from = static_cast<const char*>(p.table) + (in ? (long long)id * p.ld_table : 0) * (kTab16 ? 2 : 4);
    char* const to = static_cast<char*>(p.out) + row * p.ld_out * (kOut16 ? 2 : 4);
    Place at[kEmbUnits];
    Unit<kTab16, true> x[kEmbUnits];
    Unit<kOut16> y[kEmbUnits];
#pragma unroll
    for (int q = 0; q < kEmbUnits; ++q) {
      const int u = first + q * p.lanes;
      at[q] = u < units ? place_unit(u, p.width) : Place{0, 0u};
      x[q].clear();
      if (in) load_unit(x[q], from, at[q], p.width);
    }
    // an id outside the table has no row: NaN, which cannot be taken for one
    const float none = on ? __builtin_nanf("") : 0.0f;
#pragma unroll
    for (int q = 0; q < kEmbUnits; ++q) {
      float v[kUnit];
#pragma unroll
      for (int j = 0; j < kUnit; ++j) v[j] = in ? x[q].get(j) * p.scale : none;
      y[q].set(v);
    }
#pragma unroll
    for (int q = 0; q < kEmbUnits; ++q) y[q].settle();
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

constexpr int kSortThreads = 512;
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
constexpr int kSumBatch = 8;              // rows whose loads are under way together

// A lane's eight columns of a table row: stored, or added to what is there.
template <bool kTab16>
__device__ inline void write_table(const EmbedGradParams& p, int id, const Place& at, const float (&sum)[kUnit]) {
  char* const row = static_cast<char*>(p.table) + (long long)id * p.ld_table * (kTab16 ? 2 : 4);
  float v[kUnit];
#pragma unroll
  for (int j = 0; j < kUnit; ++j) v[j] = sum[j] * p.scale;
  if (p.accumulate) {
    Unit<kTab16> old;
    load_unit(old, row, at, p.width);
#pragma unroll
    for (int j = 0; j < kUnit; ++j) v[j] += old.get(j);
  }
  Unit<kTab16> out;
  out.set(v);
  out.settle();
  store_unit(out, row, at);
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

// The table's rows [first, first + rows) that occur nowhere are zeroed.
template <bool kTab16>
__device__ inline void zero_absent(const EmbedGradParams& p, long long block) {
  __shared__ unsigned s_seen[kEmbedFillRows / 32];
  const int tid = threadIdx.x;
  const long long first = block * p.fill_rows;
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
  const int units = (p.width + kUnit - 1) / kUnit;
  Unit<kTab16> none;
  none.clear();
  none.settle();
  for (int r = 0; r < rows; ++r) {
    if ((s_seen[r >> 5] >> (r & 31)) & 1u) continue;
    char* const row = static_cast<char*>(p.table) + (first + r) * p.ld_table * (kTab16 ? 2 : 4);
    for (int u = tid; u < units; u += kEmbThreads) store_unit(none, row, place_unit(u, p.width));
  }
  none.keep();
}

template <bool kGrad16, bool kTab16>
__global__ __launch_bounds__(kEmbThreads) void embed_sum(EmbedGradParams p) {
  if ((int)blockIdx.x >= p.sum_blocks) {
    zero_absent<kTab16>(p, blockIdx.x - p.sum_blocks);
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
  const Place at = place_unit(tile * (kSumCols / kUnit) + lane, p.width);
  const long long ld = p.ld_grad * (kGrad16 ? 2 : 4);
  float sum[kUnit];
#pragma unroll
  for (int j = 0; j < kUnit; ++j) sum[j] = 0.0f;
  float* const part = p.part + (long long)run * 2 * p.part_ld + tile * kSumCols + lane * kUnit;
  int begun = 0;  // position where the segment at hand begins in the run
  for (int i0 = 0; i0 < count; i0 += kSumBatch) {
    Unit<kGrad16> g[kSumBatch];
#pragma unroll
    for (int b = 0; b < kSumBatch; ++b) {
      g[b].clear();
      if (i0 + b < count)
        load_unit(g[b], static_cast<const char*>(p.grad) + __builtin_amdgcn_readlane(tok, i0 + b) * ld, at, p.width);
    }
#pragma unroll
    for (int b = 0; b < kSumBatch; ++b) {
      const int i = i0 + b;
      if (i >= count) break;
#pragma unroll
      for (int j = 0; j < kUnit; ++j) sum[j] += g[b].get(j);
      const int id = __builtin_amdgcn_readlane(key, i);
      const bool run_ends = i + 1 == p.run;
      const int next = run_ends ? key_after : i + 1 < count ? __builtin_amdgcn_readlane(key, i + 1) : p.vocab;
      if (!run_ends && next == id) continue;
      const bool whole_front = begun > 0 || key_before != id;
      if (whole_front && next != id) {
        write_table<kTab16>(p, id, at, sum);
      } else {
        // a piece: behind [1] where the segment begins here, else in front [0]
        Unit<false> piece;
        piece.set(sum);
        piece.settle();
        piece.store(reinterpret_cast<char*>(part + (whole_front ? p.part_ld : 0)), 0);
        store_gap();
      }
      begun = i + 1;
#pragma unroll
      for (int j = 0; j < kUnit; ++j) sum[j] = 0.0f;
    }
  }
}

// Adds the pieces of the segment that begins in a run and goes on in the next ones: a
// workgroup per run and 512 columns, whose waves take the pieces in turn.
template <bool kTab16>
__global__ __launch_bounds__(kEmbThreads) void embed_join(EmbedGradParams p) {
  constexpr int kWaves = kEmbThreads / kWave;
  __shared__ float s_sum[kWaves][kSumCols];
  const int lane = threadIdx.x & (kWave - 1);
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int run = blockIdx.x / p.col_tiles, tile = blockIdx.x % p.col_tiles;
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
  const long long col = tile * kSumCols + lane * kUnit;
  const Place at = place_unit(tile * (kSumCols / kUnit) + lane, p.width);
  float sum[kUnit];
#pragma unroll
  for (int j = 0; j < kUnit; ++j) sum[j] = 0.0f;
#pragma unroll 4
  for (int r = run + wid; r <= last; r += kWaves) {
    const float* const from = p.part + ((long long)r * 2 + (r == run ? 1 : 0)) * p.part_ld + col;
    Unit<false> x;
    x.load(reinterpret_cast<const char*>(from), 0);
#pragma unroll
    for (int j = 0; j < kUnit; ++j) sum[j] += x.get(j);
  }
#pragma unroll
  for (int j = 0; j < kUnit; ++j) s_sum[wid][lane * kUnit + j] = sum[j];
  __syncthreads();
  if (wid != 0) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w)
#pragma unroll
    for (int j = 0; j < kUnit; ++j) sum[j] += s_sum[w][lane * kUnit + j];
  write_table<kTab16>(p, id, at, sum);
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
  const int units = (p.width + kUnit - 1) / kUnit;
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
  if (p.n_rows <= kEmbedSmallSort) {
    p.key_out = p.key[0];
    p.tok_out = p.tok[0];
    embed_sort_small<<<1, kSortThreads, 0, s>>>(p);
    p.key_in = p.key[0];
    p.tok_in = p.tok[0];
  } else {
    const int turns = (p.key_bits + kEmbedDigitBits - 1) / kEmbedDigitBits;
    for (p.turn = 0; p.turn < turns; ++p.turn) {
      p.key_out = p.key[p.turn & 1];
      p.tok_out = p.tok[p.turn & 1];
      embed_count<<<p.n_tiles, kSortThreads, 0, s>>>(p);
      embed_scatter<<<p.n_tiles, kSortThreads, 0, s>>>(p);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      p.key_in = p.key_out;
      p.tok_in = p.tok_out;
    }
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const long long tasks = (long long)p.n_runs * p.col_tiles;
  p.sum_blocks = (int)((tasks + kEmbThreads / kWave - 1) / (kEmbThreads / kWave));
  p.fill_rows = kEmbedFillRows;
  while (p.fill_rows > 64 && (long long)p.fill_rows * p.width > (1 << 18)) p.fill_rows /= 2;
  const int fills = p.accumulate ? 0 : (int)(((long long)p.vocab + p.fill_rows - 1) / p.fill_rows);
  if (p.sum_blocks + fills == 0) return hipSuccess;
  const int grid = p.sum_blocks + fills;
  if (p.grad_bf16 && p.table_bf16) embed_sum<true, true><<<grid, kEmbThreads, 0, s>>>(p);
  else if (p.grad_bf16) embed_sum<true, false><<<grid, kEmbThreads, 0, s>>>(p);
  else if (p.table_bf16) embed_sum<false, true><<<grid, kEmbThreads, 0, s>>>(p);
  else embed_sum<false, false><<<grid, kEmbThreads, 0, s>>>(p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (p.n_runs > 1) {
    const int join = (p.n_runs - 1) * p.col_tiles;
    if (p.table_bf16) embed_join<true><<<join, kEmbThreads, 0, s>>>(p);
    else embed_join<false><<<join, kEmbThreads, 0, s>>>(p);
  }
  return hipGetLastError();
}

}  // namespace turnkl
