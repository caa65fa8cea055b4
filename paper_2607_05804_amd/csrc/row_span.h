// A run of 16-byte packs of a row of any start and length, for the kernels over
// token rows: where a pack lies, which of its elements are its own, and its load.
#pragma once

#include "row_ops.h"

namespace turnkl {
namespace {

// A pack with -inf in place of the elements outside `bits`.
__device__ inline void forbid(Pack<true, 8>& x, unsigned bits) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const unsigned keep = ((bits >> (2 * k)) & 1u ? 0xFFFFu : 0u) | ((bits >> (2 * k + 1)) & 1u ? 0xFFFF0000u : 0u);
    x.w[k] = (x.w[k] & keep) | (0xFF80FF80u & ~keep);
  }
}
__device__ inline void forbid(Pack<false, 4>& x, unsigned bits) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x.f[j] = (bits >> j) & 1u ? x.f[j] : -INFINITY;
}

// Computes the data of a store here, before any of the stores (whose own data must
// not be rewritten closely behind them), and not where it is stored.
__device__ inline void settle(u32x4& x) { asm volatile("" : "+v"(x)); }

template <bool kBf16, bool kRagged>
struct RowSpan {
  static constexpr int kEpv = kBf16 ? 8 : 4;
  static constexpr int kEs = kBf16 ? 2 : 4;
  using P = Pack<kBf16, kEpv>;

  const char* row;               // first element of the row
  __amdgpu_buffer_rsrc_t rsrc;   // based there
  int vocab;
  int col;                       // first element of the span
  int n;                         // packs

  // Pack i of the span: the element its load starts at, moved inside the row where
  // the pack sticks out, and which of the loaded elements are its own.
  __device__ int place(int i, unsigned& bits) const {
    const int e = col + i * kEpv;
    if constexpr (kRagged) {
      const int at = inside_row(e, vocab > kEpv ? vocab - kEpv : 0);
      bits = i < n ? own_bits<kEpv>(e - at) : 0u;
      if (vocab < kEpv) bits &= (1u << vocab) - 1u;
      return at;
    } else {
      bits = i < n ? (1u << kEpv) - 1u : 0u;
      return i < n ? e : 0;
    }
  }
  // Load at an element that place() gave.
  __device__ void load(P& x, int at) const {
    if constexpr (kRagged) {
      if (vocab < kEpv) {  // a row shorter than a pack: element by element
        if constexpr (kBf16) {
#pragma unroll
          for (int j = 0; j < 4; ++j) x.w[j] = 0u;
#pragma unroll
          for (int j = 0; j < kEpv; ++j) {
            const unsigned w = j < vocab ? reinterpret_cast<const unsigned short*>(row)[j] : 0u;
            x.w[j >> 1] |= w << (16 * (j & 1));
          }
        } else {
#pragma unroll
          for (int j = 0; j < kEpv; ++j)
            x.f[j] = j < vocab ? reinterpret_cast<const float*>(row)[j] : 0.0f;
        }
        return;
      }
    }
    x.load(rsrc, at * kEs, 0);
  }
  // Stores at an element that place() gave: of packs that are their thread's
  // entirely, and of the own elements of the others, at the ends of a row.  Partial
  // packs are stored first: their code shifts the data, which must not follow the
  // wide stores closely.
  __device__ void store_own(const typename P::Data& d, int at, unsigned bits) const {
    if constexpr (kRagged) {
      if (bits == (1u << kEpv) - 1u || !bits) return;
#pragma unroll
      for (int j = 0; j < kEpv; ++j) {
        if (!((bits >> j) & 1u)) continue;
        if constexpr (kBf16)
          __builtin_amdgcn_raw_buffer_store_b16((unsigned short)(d[j >> 1] >> (16 * (j & 1))), rsrc,
                                                (at + j) * kEs, 0, kStream);
        else
          __builtin_amdgcn_raw_buffer_store_b32(d[j], rsrc, (at + j) * kEs, 0, kStream);
      }
    }
  }
  __device__ void store_whole(const typename P::Data& d, int at, unsigned bits) const {
    if (bits == (1u << kEpv) - 1u) P::store(rsrc, at * kEs, 0, d);
  }
};

}  // namespace
}  // namespace turnkl
